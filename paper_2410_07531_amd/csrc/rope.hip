// Rotary positions for queries and keys (the embedding inside the paper's Fig. 2 block in its Llama form), as
// an operator of its own: adjacent or split pairs, the whole head or its first `rot` elements, the frequencies of
// long-context scalings, any positions, any strides, forward and backward (the rotation by the negated angle).
//
// Pair p of a head, (a, b), at position s becomes m * (a cos t - b sin t, a sin t + b cos t), t = s * f_p.
// What bounds it: memory, every element read and written once.  The sines of a token serve all its heads, so a
// workgroup owns a few tokens, forms their rot / 2 sines once into LDS and then walks over the heads, 16 bytes
// a thread.  16384 x (32 + 8) heads x 128 in bf16: 69 us, 4.9 TB/s, the rate of a large copy; 16 tokens of it 4.5 us, the chain of position, sines
// and store.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rov_internal.h"
#include "row_device.h"

namespace rov {
namespace {

constexpr int kMaxHead = 512;

struct RopeParams {
    const void* src[2];          // Q, K
    void* dst[2];
    int64_t sb[2], ss[2], sh[2]; // strides of src: batch, token, head (elements)
    int64_t db[2], ds[2], dh[2]; // of dst
    const int64_t* positions;
    int64_t positions_stride;
    int64_t tokens;
    int S, H, heads;             // heads = H + Hkv
    int rot, copy, tpb;          // copy: elements behind `rot` that go along (0 in place); tpb: tokens a workgroup
    uint32_t units, token_units, inv_units, inv_token_units;   // of a head, of a token
    double power[8];             // theta^(-2 * 2^k / rot)
    double inv_factor, low, inv_width, turns;   // turns: trained_len / (2 pi)
    int scaling;
    float magnitude, sign;
};

// Sine and cosine of position * frequency(p).  The angle is formed and reduced modulo 2 pi in double, so that
// positions of a million keep fp32-accurate sines.  The frequency is a product of powers theta^(-2 * 2^k / rot), one
// per bit of the pair's number, that the host worked out: at most eight products in place of an exponential in double.
__device__ __forceinline__ void rope_sincos(const RopeParams& p, int64_t pos, int pair, float* sn, float* cs) {
    double f = 1.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) f *= (pair >> k) & 1 ? p.power[k] : 1.0;
    if (p.scaling == ROV_ROPE_SCALE_LINEAR) f *= p.inv_factor;
    if (p.scaling == ROV_ROPE_SCALE_PARTS) {
        double keep = (p.turns * f - p.low) * p.inv_width;
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        f *= keep + (1.0 - keep) * p.inv_factor;
    }
    double ang = (double)pos * f;
    ang -= 6.283185307179586476925 * rint(ang * 0.15915494309189533577);
    float s, c;
    sincosf((float)ang, &s, &c);
    *sn = s * p.magnitude * p.sign;
    *cs = c * p.magnitude;
}

// n / d by a multiplication where that is exact (inv = 2^32 / d rounded up, n * d < 2^32), else inv == 0
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t d, uint32_t inv) { return inv != 0 ? __umulhi(n, inv) : n / d; }

// W: elements a thread moves at once (16 bytes, from any address), or 1 where heads or `rot` are no whole pieces.
// A unit of a head is W pairs (split layout: W elements of each half), max(1, W / 2) pairs (adjacent), or W elements to copy; a
// workgroup's units are those of all heads of its tokens.  A thread loads two units before it waits for anything, the first two
// before the sines are formed.
template <typename T, int W, bool HALVES>
__global__ __launch_bounds__(256) void rope_kernel(const RopeParams p) {
    extern __shared__ __attribute__((aligned(16))) float lds[];   // [tokens][rot / 2] sines, then cosines
    constexpr int AHEAD = 2;
    constexpr bool TWO = HALVES || W == 1;                 // a unit's pairs lie in two pieces
    constexpr int P = HALVES ? W : (W > 1 ? W / 2 : 1);    // pairs of a unit
    const int half = p.rot / 2, turn_units = half / P;
    float* const sines = lds;
    float* const cosines = lds + p.tpb * half;
    // beside a co-resident RNG grid the waves would wait for issue slots behind its long integer multiplies
    __builtin_amdgcn_s_setprio(3);
    const int64_t token0 = (int64_t)blockIdx.x * p.tpb;
    const int here = p.tokens - token0 < p.tpb ? (int)(p.tokens - token0) : p.tpb;
    const uint32_t total = (uint32_t)here * p.token_units;
    const int64_t b0 = token0 / p.S;
    const uint32_t s0 = (uint32_t)(token0 - b0 * p.S);
    const bool one_row = s0 + (uint32_t)here <= (uint32_t)p.S;   // (one sequence holds the workgroup's tokens)
    for (uint32_t base = 0; base < total; base += 256 * AHEAD) {
        Piece<T, W> va[AHEAD], vb[AHEAD];
        T* dst[AHEAD];
        int unit[AHEAD], at[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            const uint32_t i = base + q * 256 + threadIdx.x;
            unit[q] = -1;
            if (i >= total) continue;
            const uint32_t tk = quotient(i, p.token_units, p.inv_token_units), in_token = i - tk * p.token_units;
            const uint32_t head = quotient(in_token, p.units, p.inv_units);
            unit[q] = (int)(in_token - head * p.units);
            at[q] = (int)tk * half + unit[q] * P;
            const uint32_t over = one_row ? 0 : (s0 + tk) / (uint32_t)p.S;
            const int64_t b = b0 + over, s = s0 + tk - over * (uint32_t)p.S;
            const int k = (int)head >= p.H, hh = k ? (int)head - p.H : (int)head;
            const T* const src = (const T*)p.src[k] + b * p.sb[k] + s * p.ss[k] + (int64_t)hh * p.sh[k];
            dst[q] = (T*)p.dst[k] + b * p.db[k] + s * p.ds[k] + (int64_t)hh * p.dh[k];
            if (unit[q] >= turn_units) {
                va[q].load(src + p.rot + (unit[q] - turn_units) * W);
            } else if constexpr (TWO) {
                va[q].load(src + (HALVES ? unit[q] * W : 2 * unit[q]));
                vb[q].load(src + (HALVES ? half + unit[q] * W : 2 * unit[q] + 1));
            } else {
                va[q].load(src + unit[q] * W);
            }
        }
        if (base == 0) {
            for (int i = threadIdx.x; i < here * half; i += 256) {
                const int tk = i / half;
                const uint32_t over = one_row ? 0 : (s0 + (uint32_t)tk) / (uint32_t)p.S;
                const int64_t b = b0 + over, s = s0 + (uint32_t)tk - over * (uint32_t)p.S;
                const int64_t pos = p.positions != nullptr ? p.positions[b * p.positions_stride + s] : s;
                rope_sincos(p, pos, i - tk * half, &sines[i], &cosines[i]);
            }
            __syncthreads();
        }
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            if (unit[q] < 0) continue;
            if (unit[q] >= turn_units) {
                va[q].store(dst[q] + p.rot + (unit[q] - turn_units) * W);
                continue;
            }
            const float* const sn = sines + at[q];
            const float* const cs = cosines + at[q];
            float a[W];
            va[q].get(a);
            if constexpr (TWO) {
                float c[W];
                vb[q].get(c);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float x = a[j], y = c[j];
                    a[j] = x * cs[j] - y * sn[j];
                    c[j] = x * sn[j] + y * cs[j];
                }
                va[q].set(a);
                vb[q].set(c);
                va[q].store(dst[q] + (HALVES ? unit[q] * W : 2 * unit[q]));
                vb[q].store(dst[q] + (HALVES ? half + unit[q] * W : 2 * unit[q] + 1));
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float x = a[2 * j], y = a[2 * j + 1];
                    a[2 * j] = x * cs[j] - y * sn[j];
                    a[2 * j + 1] = x * sn[j] + y * cs[j];
                }
                va[q].set(a);
                va[q].store(dst[q] + unit[q] * W);
            }
        }
    }
}

template <typename T, int W, bool HALVES>
int launch_form(RopeParams& p, hipStream_t stream) {
    const int pairs = HALVES ? W : (W > 1 ? W / 2 : 1);
    const int64_t units = p.rot / 2 / pairs + p.copy / W, token_units = units * p.heads;
    if (token_units > 0x0FFFFFFF) return ROV_ERR_UNSUPPORTED;
    p.units = (uint32_t)units;
    p.token_units = (uint32_t)token_units;
    // tokens a workgroup: a sine for every thread, as long as three workgroups a compute unit are left
    int tpb = 1;
    while (tpb * p.rot <= 256 && p.tokens >= (int64_t)device_cu_count() * 6 * tpb) tpb *= 2;
    p.tpb = tpb;
    auto inverse = [&](int64_t n, int64_t d) { return n * d < ((int64_t)1 << 32) && d > 1 ? (uint32_t)((((uint64_t)1 << 32) + d - 1) / d) : 0u; };
    p.inv_token_units = inverse(tpb * token_units, token_units);
    p.inv_units = inverse(token_units, units);
    const int64_t blocks = (p.tokens + tpb - 1) / tpb;
    if (!grid_fits(blocks, 256)) return ROV_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((rope_kernel<T, W, HALVES>), dim3((unsigned)blocks), dim3(256), (size_t)tpb * p.rot * sizeof(float), stream, p);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}

}  // namespace

int check_rope_cfg(const rov_rope_cfg* c, int d) {
    if (c == nullptr || d <= 0) return ROV_ERR_INVALID;
    if (c->layout != ROV_ROPE_INTERLEAVED && c->layout != ROV_ROPE_HALVES) return ROV_ERR_INVALID;
    if (c->rot <= 0 || c->rot % 2 != 0 || c->rot > d || !(c->theta > 0.0f) || !isfinite(c->theta) || !isfinite(c->magnitude))
        return ROV_ERR_INVALID;
    if (c->scaling != ROV_ROPE_SCALE_NONE && c->scaling != ROV_ROPE_SCALE_LINEAR && c->scaling != ROV_ROPE_SCALE_PARTS)
        return ROV_ERR_INVALID;
    if (c->scaling != ROV_ROPE_SCALE_NONE && (!(c->factor > 0.0f) || !isfinite(c->factor))) return ROV_ERR_INVALID;
    if (c->scaling == ROV_ROPE_SCALE_PARTS &&
        (c->trained_len <= 0 || !(c->turns_low >= 0.0f) || !(c->turns_high > c->turns_low) || !isfinite(c->turns_high)))
        return ROV_ERR_INVALID;
    return d > kMaxHead ? ROV_ERR_UNSUPPORTED : ROV_OK;
}

int check_rope(const rov_rope_cfg* c, const void* Q, const void* Qo, const void* K, const void* Ko, int B, int S, int H, int Hkv,
               int d, const int64_t strides[12], int dtype, const int64_t* positions) {
    const int rc = check_rope_cfg(c, d);
    if (rc != ROV_OK && rc != ROV_ERR_UNSUPPORTED) return rc;
    if (Q == nullptr || Qo == nullptr || strides == nullptr || B <= 0 || S <= 0 || H <= 0 || Hkv < 0) return ROV_ERR_INVALID;
    if (Hkv > 0 && (K == nullptr || Ko == nullptr)) return ROV_ERR_INVALID;
    if (dtype != ROV_F32 && dtype != ROV_BF16) return dtype == ROV_FP8_E4M3 ? ROV_ERR_UNSUPPORTED : ROV_ERR_INVALID;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    if (!aligned(positions, 8)) return ROV_ERR_INVALID;
    if (!aligned(Q, esz) || !aligned(Qo, esz) || (Hkv > 0 && (!aligned(K, esz) || !aligned(Ko, esz)))) return ROV_ERR_INVALID;
    // a buffer turned in place is its own result, stride for stride
    for (int t = 0; t < (Hkv > 0 ? 2 : 1); ++t)
        if ((t ? K : Q) == (t ? Ko : Qo))
            for (int i = 0; i < 3; ++i)
                if (strides[6 * t + i] != strides[6 * t + 3 + i]) return ROV_ERR_INVALID;
    if (Hkv > 0 && (Qo == Ko || Qo == K || Ko == Q)) return ROV_ERR_INVALID;   // (turned by two threads, or by one before the other has read it)
    if ((int64_t)H + Hkv > 0x7FFFFFFF / kMaxHead) return ROV_ERR_UNSUPPORTED;
    return rc;
}

int launch_rope_cfg(const rov_rope_cfg* c, const void* Q, void* Qo, const void* K, void* Ko, int B, int S, int H, int Hkv, int d,
                    const int64_t strides[12], int dtype, const int64_t* positions, int64_t positions_stride, int backward,
                    hipStream_t stream) {
    {
        const int rc = check_rope(c, Q, Qo, K, Ko, B, S, H, Hkv, d, strides, dtype, positions);
        if (rc != ROV_OK) return rc;
    }
    RopeParams p{};
    p.src[0] = Q; p.src[1] = K; p.dst[0] = Qo; p.dst[1] = Ko;
    const int64_t esz = dtype == ROV_F32 ? 4 : 2, w = 16 / esz;
    const bool vec = d % w == 0 && c->rot % (c->layout == ROV_ROPE_HALVES ? 2 * w : w) == 0;
    bool copy = false;
    for (int t = 0; t < 2; ++t) {
        p.sb[t] = strides[6 * t]; p.ss[t] = strides[6 * t + 1]; p.sh[t] = strides[6 * t + 2];
        p.db[t] = strides[6 * t + 3]; p.ds[t] = strides[6 * t + 4]; p.dh[t] = strides[6 * t + 5];
        if (t == 1 && Hkv == 0) break;
        copy = copy || p.src[t] != p.dst[t];
    }
    p.positions = positions; p.positions_stride = positions_stride;
    p.tokens = (int64_t)B * S;
    p.S = S; p.H = H; p.heads = H + Hkv;
    p.rot = c->rot; p.copy = copy ? d - c->rot : 0;
    p.power[0] = exp2(-2.0 / (double)c->rot * log2((double)c->theta));
    for (int k = 1; k < 8; ++k) p.power[k] = p.power[k - 1] * p.power[k - 1];
    p.scaling = c->scaling;
    p.inv_factor = c->scaling == ROV_ROPE_SCALE_NONE ? 1.0 : 1.0 / (double)c->factor;
    if (c->scaling == ROV_ROPE_SCALE_PARTS) {
        p.low = c->turns_low;
        p.inv_width = 1.0 / ((double)c->turns_high - (double)c->turns_low);
        p.turns = (double)c->trained_len / 6.283185307179586476925;
    }
    p.magnitude = c->magnitude;
    p.sign = backward ? -1.0f : 1.0f;
    const bool halves = c->layout == ROV_ROPE_HALVES;
    if (dtype == ROV_BF16)
        return vec ? (halves ? launch_form<uint16_t, 8, true>(p, stream) : launch_form<uint16_t, 8, false>(p, stream))
                   : (halves ? launch_form<uint16_t, 1, true>(p, stream) : launch_form<uint16_t, 1, false>(p, stream));
    return vec ? (halves ? launch_form<float, 4, true>(p, stream) : launch_form<float, 4, false>(p, stream))
               : (halves ? launch_form<float, 1, true>(p, stream) : launch_form<float, 1, false>(p, stream));
}

}  // namespace rov

extern "C" int rov_rope(const rov_rope_cfg* cfg, const void* Q, void* Qo, const void* K, void* Ko, int B, int S, int H, int Hkv,
                        int d, const int64_t strides[12], int dtype, const int64_t* positions, int64_t positions_stride,
                        int backward, void* stream) {
    return rov::launch_rope_cfg(cfg, Q, Qo, K, Ko, B, S, H, Hkv, d, strides, dtype, positions, positions_stride, backward,
                                (hipStream_t)stream);
}
