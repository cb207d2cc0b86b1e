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

// T: uint16_t (bf16 bits) or float.  A Piece holds W elements as they lie in memory.
template <typename T, int W>
struct Piece;
template <>
struct Piece<uint16_t, 8> {
    uint4 raw;
    __device__ __forceinline__ void load(const uint16_t* p) { raw = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = raw; }
    __device__ __forceinline__ void zero() { raw = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
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
    __device__ __forceinline__ void set(const float (&f)[1]) { raw = (uint16_t)bf16_pair(f[0], 0.0f); }
};
template <>
struct Piece<float, 4> {
    float4 raw;
    __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = raw; }
    __device__ __forceinline__ void zero() { raw = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = raw.x; f[1] = raw.y; f[2] = raw.z; f[3] = raw.w; }
    __device__ __forceinline__ void set(const float (&f)[4]) { raw = make_float4(f[0], f[1], f[2], f[3]); }
};
template <>
struct Piece<float, 1> {
    float raw;
    __device__ __forceinline__ void load(const float* p) { raw = *p; }
    __device__ __forceinline__ void store(float* p) const { *p = raw; }
    __device__ __forceinline__ void zero() { raw = 0.0f; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = raw; }
    __device__ __forceinline__ void set(const float (&f)[1]) { raw = f[0]; }
};

// Sum over the workgroup's NT threads, the same bits in every thread and run.  `red` holds NT / 64
// floats that nobody else uses between this call and the next barrier behind it.
template <int NT>
__device__ __forceinline__ float workgroup_sum(float v, float* red) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) v += red[i];
    }
    return v;
}

}  // namespace rov
