// What the row-wise kernels share: elements of bf16 or fp32 rows as fp32 values, `W` of them at a time
// (16 bytes where rows are aligned, one element where they are not), and sums over a workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rov {

// nearest bf16, ties to even; a NaN stays one
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 v = {lo, hi};
    const b2 h = __builtin_convertvector(v, b2);
    return __builtin_bit_cast(uint32_t, h);
}

// T: uint16_t (bf16 bits) or float.  A Piece holds W elements as they lie in memory; its load and store are one
// instruction each, which the hardware takes at any address.
template <typename T, int W>
struct Piece;
template <>
struct Piece<uint16_t, 8> {
    uint4 raw;
    __device__ __forceinline__ void load(const uint16_t* p) { __builtin_memcpy(&raw, p, 16); }
    __device__ __forceinline__ void store(uint16_t* p) const { __builtin_memcpy(p, &raw, 16); }
    __device__ __forceinline__ void zero() { raw = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ float at(int i) const {   // (i known at compile time)
        const uint32_t w = i < 2 ? raw.x : i < 4 ? raw.y : i < 6 ? raw.z : raw.w;
        return __uint_as_float(i % 2 ? w & 0xFFFF0000u : w << 16);
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        raw = make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
    }
};
template <>
struct Piece<uint16_t, 1> {
    uint16_t raw;
    __device__ __forceinline__ void load(const uint16_t* p) { raw = *p; }
    __device__ __forceinline__ void store(uint16_t* p) const { *p = raw; }
    __device__ __forceinline__ void zero() { raw = 0; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = __uint_as_float((uint32_t)raw << 16); }
    __device__ __forceinline__ float at(int) const { return __uint_as_float((uint32_t)raw << 16); }
    __device__ __forceinline__ void set(const float (&f)[1]) { raw = (uint16_t)bf16_pair(f[0], 0.0f); }
};
template <>
struct Piece<float, 4> {
    float4 raw;
    __device__ __forceinline__ void load(const float* p) { __builtin_memcpy(&raw, p, 16); }
    __device__ __forceinline__ void store(float* p) const { __builtin_memcpy(p, &raw, 16); }
    __device__ __forceinline__ void zero() { raw = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = raw.x; f[1] = raw.y; f[2] = raw.z; f[3] = raw.w; }
    __device__ __forceinline__ float at(int i) const { return i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w; }
    __device__ __forceinline__ void set(const float (&f)[4]) { raw = make_float4(f[0], f[1], f[2], f[3]); }
};
template <>
struct Piece<float, 1> {
    float raw;
    __device__ __forceinline__ void load(const float* p) { raw = *p; }
    __device__ __forceinline__ void store(float* p) const { *p = raw; }
    __device__ __forceinline__ void zero() { raw = 0.0f; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = raw; }
    __device__ __forceinline__ float at(int) const { return raw; }
    __device__ __forceinline__ void set(const float (&f)[1]) { raw = f[0]; }
};

// Elements e .. e + W of a row of n > e (e a multiple of W; nothing beyond the row).  !RAGGED: n is a multiple of W; RAGGED: n > W.  A row's last, shorter piece is
// loaded as the row's last W elements, by the same instruction as the whole ones, and `settle` moves it down where it is used: what would wait
// for the load must not stand beside it.  (8192 x 4095 in fp32, backward: 205 us with the last piece's elements loaded one by one.)
template <bool RAGGED, typename T, int W>
__device__ __forceinline__ void fetch_piece(Piece<T, W>& v, const T* row, int e, int n) {
    v.load(row + (RAGGED && e + W > n ? n - W : e));
}
template <bool RAGGED, typename T, int W>
__device__ __forceinline__ void settle(Piece<T, W>& v, int e, int n) {
    if constexpr (!RAGGED) return;
    if (e >= n || e + W <= n) return;
    uint32_t w[4];
    __builtin_memcpy(w, &v.raw, sizeof(v.raw));
    const int by = (e + W - n) * (int)sizeof(T);
    if (by & 8) { w[0] = w[2]; w[1] = w[3]; w[2] = w[3] = 0u; }
    if (by & 4) { w[0] = w[1]; w[1] = w[2]; w[2] = w[3]; w[3] = 0u; }
    if (by & 2) {
        w[0] = w[0] >> 16 | w[1] << 16;
        w[1] = w[1] >> 16 | w[2] << 16;
        w[2] = w[2] >> 16 | w[3] << 16;
        w[3] >>= 16;
    }
    __builtin_memcpy(&v.raw, w, sizeof(v.raw));
}
template <bool RAGGED, typename T, int W>
__device__ __forceinline__ void put_piece(const Piece<T, W>& v, T* row, int e, int n) {
    if (!RAGGED || e + W <= n) {
        v.store(row + e);
        return;
    }
    uint32_t w[4];
    __builtin_memcpy(w, &v.raw, sizeof(v.raw));
    const int bytes = (n - e) * (int)sizeof(T);
    char* at = (char*)(row + e);
    if (bytes & 8) { __builtin_memcpy(at, w, 8); at += 8; w[0] = w[2]; w[1] = w[3]; }
    if (bytes & 4) { __builtin_memcpy(at, w, 4); at += 4; w[0] = w[1]; }
    if (bytes & 2) __builtin_memcpy(at, w, 2);
}

// Sums by data-parallel moves between lanes (vector instructions; a shuffle would go through the LDS unit).  `mask`: rows of 16
// lanes that add; what a lane has no partner for counts as zero.
template <int CTRL, int MASK = 0xF>
__device__ __forceinline__ float add_moved(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, MASK, 0xF, false));
}
// Lane 15 of each row of 16 lanes: the row's sum.
__device__ __forceinline__ float row16_sum(float v) {
    v = add_moved<0x111>(v);   // from one lane below
    v = add_moved<0x112>(v);   // two
    v = add_moved<0x114>(v);   // four
    return add_moved<0x118>(v);   // eight
}
// Lane 63: the wave's sum.
__device__ __forceinline__ float wave_sum(float v) {
    v = row16_sum(v);
    v = add_moved<0x142, 0xA>(v);      // rows 1 and 3 take the row below
    return add_moved<0x143, 0xC>(v);   // rows 2 and 3 take the half below
}
__device__ __forceinline__ float from_lane(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// N <= 8 sums over the workgroup's NT threads, the same bits in every thread and run.  `red` holds 16 * N floats (one wave
// needs none) that nobody else uses between this call and the next barrier behind it.
template <int NT, int N>
__device__ __forceinline__ void workgroup_sums(float (&v)[N], float* red) {
    constexpr int WAVES = NT / 64;
    static_assert(WAVES <= 16 && N <= 8, "sixteen waves, eight sums");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = from_lane(v[i], 63);
    } else {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (lane == 63)
#pragma unroll
            for (int i = 0; i < N; ++i) red[16 * i + wave] = v[i];
        __syncthreads();
        // lane 16 * i + w takes sum i of wave w: a row of lanes adds the waves up
#pragma unroll
        for (int half = 0; half < (N + 3) / 4; ++half) {
            const int at = 64 * half + lane;
            const float s = row16_sum(at < 16 * N && (lane & 15) < WAVES ? red[at] : 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (4 * half + i < N) v[4 * half + i] = from_lane(s, 16 * i + 15);
        }
    }
}
template <int NT>
__device__ __forceinline__ float workgroup_sum(float v, float* red) {
    float s[1] = {v};
    workgroup_sums<NT, 1>(s, red);
    return s[0];
}

}  // namespace rov
