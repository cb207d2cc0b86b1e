// Softmax cross entropy of logits z = scale * X W^T over a large vocabulary, and its gradients, without keeping z:
//     lse_m = log sum_v exp z_mv,   loss_m = lse_m - z_m,target(m)
//     G_mv = scale * (exp(z_mv - lse_m) * (dloss_m + dlse_m) - [v == target(m)] * dloss_m),   dX = G W,   dW = G^T X.
// 2 M V K operations forward and 6 backward, which makes the logits again: matrix cores bound both, but for few rows, where
// W's bytes do.
//
// bf16: the 256-row tile of gemm_head.hip.  Forward, a tile's logits are reduced in the accumulators to a
// maximum and a sum of exponentials per row and 128 columns, which a second kernel joins; nothing else leaves the tile.  Backward
// walks the vocabulary in pieces: the accumulators of a piece's logits become G, stored in bf16 (the tile's columns are dealt to the lanes so
// that G leaves in 16-byte stores), and the products for dX and dW read G, W and X as they lie, k across the rows, through transposing LDS
// loads.  dX is summed over the pieces, and either over shares of k where its tiles alone would leave compute units idle, in fp32.
// G is rounded to bf16 without its row's factor dloss: with the factor in it, the entries of the targets, which are the bulk of it and
// nearly the same number -dloss in every row of a mean, would all be off by the same part of up to 2^-9, and so would dX and dW (0.0033 of
// their norm at 8192 x 131072 x 4096, 0.0017 without).  dX is multiplied by its row's factor in fp32; for dW the rows of X are multiplied by theirs over the largest,
// which changes nothing where they are all the same and rounds X once more where they differ, and dW by the largest.  Errors of the norm, where a result rounded once is
// off by 0.0017 (1000 x 8000 x 512, dX / dW): a mean 0.0017 / 0.0017 with targets far below a probability of 2^-9, up to 0.0024 / 0.0023 with likely ones, whose
// entries are no longer -1; factors that differ from row to row 0.0017 / 0.0023 and up to 0.0023 / 0.0028.
// fp32: the fp32 products of gemm_ring.hip; a piece's logits live in the workspace while they are reduced, or turned into G in place.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "rov_internal.h"
#include "row_device.h"

namespace rov {
namespace {

struct RowState { float top, sum, picked, pad; };   // running maximum, sum of exp(z - top), logit of the target

// A row counts if its target is not the ignored index; a target outside the vocabulary shows as NaN.
__device__ __forceinline__ bool in_vocab(int64_t t, int V) { return t >= 0 && t < V; }

// ------------------------------------------------------------------ fp32
// dst [rows][cols] = src, row strides ldd and lds; rows of ignored targets (targets may be NULL) zero.
__global__ __launch_bounds__(256) void xent_copy_kernel(const float* __restrict__ src, int64_t lds, float* __restrict__ dst, int64_t ldd, int64_t rows,
                                                        int cols, const int64_t* __restrict__ targets, int64_t ignore) {
    const int64_t total = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / cols;
        const int c = (int)(i - r * cols);
        dst[r * ldd + c] = targets != nullptr && targets[r] == ignore ? 0.0f : src[r * lds + c];
    }
}

__global__ __launch_bounds__(256) void xent_add_kernel(const float* __restrict__ src, float* __restrict__ dst, int64_t total) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) dst[i] += src[i];
}

// Statistics of one piece's logits z [M][cols] (vocabulary v0 ..), joined with those of the pieces before it; the last
// piece's launch writes the results.  One workgroup a row.
__global__ __launch_bounds__(256) void xent_stats_kernel(const float* __restrict__ z, int cols, int v0, int V, float scale,
                                                         const int64_t* __restrict__ targets, int64_t ignore,
                                                         RowState* __restrict__ state, float* __restrict__ loss,
                                                         float* __restrict__ lse) {
    __shared__ float red[4 + 16];
    const int64_t row = blockIdx.x;
    const float* const zr = z + row * cols;
    // four logits of the row at a time (16 bytes from any address), the last ones one by one
    auto each = [&](auto take) {
        const int whole = cols / 4 * 4;
        for (int c = 4 * threadIdx.x; c < whole; c += 1024) {
            Piece<float, 4> v;
            v.load(zr + c);
#pragma unroll
            for (int j = 0; j < 4; ++j) take(scale * v.at(j));
        }
        if (whole + (int)threadIdx.x < cols) take(scale * zr[whole + threadIdx.x]);
    };
    float top = -INFINITY;
    each([&](float z) { top = fmaxf(top, z); });
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    RowState st = {-INFINITY, 0.0f, NAN, 0.0f};
    if (v0 > 0) st = state[row];
    top = fmaxf(top, st.top);
    const float base = top > -INFINITY ? top : 0.0f;   // (every logit minus infinity: the sum is 0, not NaN)
    float sum = 0.0f;
    each([&](float z) { sum += __expf(z - base); });
    sum = workgroup_sum<256>(sum, red + 4);
    sum += st.sum * __expf(st.top - base);
    if (threadIdx.x != 0) return;
    const int64_t t = targets[row];
    if (t >= v0 && t < (int64_t)v0 + cols) st.picked = scale * zr[t - v0];
    if (v0 + cols < V) {
        state[row] = RowState{top, sum, st.picked, 0.0f};
        return;
    }
    const float l = base + logf(sum);
    lse[row] = l;
    loss[row] = t == ignore ? 0.0f : in_vocab(t, V) ? l - st.picked : NAN;
}

// G of one piece in place of its logits z [M][cols], and its transpose gt [cols][M].
__global__ __launch_bounds__(256) void xent_grad_kernel(float* __restrict__ z, float* __restrict__ gt, int M, int cols, int v0, int V,
                                                        float scale, const int64_t* __restrict__ targets, int64_t ignore,
                                                        const float* __restrict__ lse, const float* __restrict__ dloss,
                                                        const float* __restrict__ dlse) {
    __shared__ float tile[64][65];
    const int c0 = blockIdx.x * 64, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    for (int64_t m0 = (int64_t)blockIdx.y * 64; m0 < M; m0 += (int64_t)gridDim.y * 64) {
        for (int i = ty; i < 64; i += 4) {
            const int64_t m = m0 + i;
            const int c = c0 + tx;
            float g = 0.0f;
            if (m < M && c < cols) {
                const int64_t t = targets[m];
                if (t != ignore) {
                    const float a = in_vocab(t, V) ? dloss[m] : NAN, b = dlse != nullptr ? dlse[m] : 0.0f;
                    g = __expf(scale * z[m * cols + c] - lse[m]) * (a + b);
                    if (t - v0 == c) g -= a;
                    g *= scale;
                }
                z[m * cols + c] = g;
            }
            tile[i][tx] = g;
        }
        __syncthreads();
        for (int i = ty; i < 64; i += 4) {
            const int64_t m = m0 + tx;
            const int c = c0 + i;
            if (m < M && c < cols) gt[(int64_t)c * M + m] = tile[tx][i];
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ bf16
// factor[m]: dloss, or dloss + dlse where dloss is next to nothing beside it; 0 for rows of ignored targets, NaN for targets outside the
// vocabulary.  factor[M]: the largest of their magnitudes.  rows: what the epilogue for G needs of a row.  One workgroup.
__global__ __launch_bounds__(1024) void xent_factor_kernel(const int64_t* __restrict__ targets, int64_t ignore, int V, const float* __restrict__ dloss,
                                                           const float* __restrict__ dlse, const float* __restrict__ lse,
                                                           float* __restrict__ factor, float4* __restrict__ rows, int M) {
    __shared__ float red[16];
    float most = 0.0f;
    for (int m = threadIdx.x; m < M; m += 1024) {
        const int64_t t = targets[m];
        const float a = dloss[m], s = dlse != nullptr ? a + dlse[m] : a;
        const float f = t == ignore ? 0.0f : !in_vocab(t, V) ? NAN : fabsf(a) * 1048576.0f >= fabsf(s) ? a : s;
        factor[m] = f;
        const bool keep = t != ignore && f != 0.0f;
        rows[m] = make_float4(keep ? lse[m] * 1.44269504088896341f : 0.0f, keep ? s / f : 0.0f, keep ? a / f : 0.0f,
                              __int_as_float(!keep ? INT_MIN : in_vocab(t, V) ? (int)t : -1));
        most = fmaxf(most, fabsf(f));
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) most = fmaxf(most, red[i]);
    factor[M] = most;
}

// dst [rows][kp] = src, columns K .. kp zero; times factor[r] / factor[rows] where it is given, rows with factor 0 zero whatever they
// hold.  Eight values a thread.
__global__ __launch_bounds__(256) void xent_pack_kernel(const uint16_t* __restrict__ src, int64_t ld, uint16_t* __restrict__ dst, int64_t rows, int K, int kp,
                                                        const float* __restrict__ factor) {
    const int chunks = kp / 8;
    const int64_t total = rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int c = (int)(i - r * chunks) * 8;
        float f = factor != nullptr ? factor[r] : 1.0f;
        Piece<uint16_t, 8> v;
        v.zero();
        if (f != 0.0f) {
            const uint16_t* const at = src + r * ld + c;
            if (c + 7 < K) {
                __builtin_memcpy(&v.raw, at, 16);   // (one load, whatever the rows' alignment)
            } else {
                uint32_t h[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = c + e < K ? at[e] : 0u;
                v.raw = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
            }
            if (factor != nullptr) f /= factor[rows];
            if (f != 1.0f) {
                float x[8];
                v.get(x);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= f;
                v.set(x);
            }
        }
        v.store(dst + r * kp + c);
    }
}

// Joins the statistics part[count][M] of M rows (units of log 2) and writes the results: R rows a workgroup, 256 / R threads a row.
template <int R>
__global__ __launch_bounds__(256) void xent_join_kernel(const float2* __restrict__ part, int count, const float* __restrict__ picked, int M, int V,
                                                        const int64_t* __restrict__ targets, int64_t ignore, float* __restrict__ loss,
                                                        float* __restrict__ lse) {
    constexpr int SLICES = 256 / R;
    __shared__ float2 red[SLICES][R];
    const int r = threadIdx.x % R, slice = threadIdx.x / R;
    const int64_t m = (int64_t)blockIdx.x * R + r;
    float top = -INFINITY, sum = 0.0f;
    auto join = [&](float2 v) {
        const float t = fmaxf(top, v.x), base = t > -INFINITY ? t : 0.0f;
        sum = sum * __builtin_amdgcn_exp2f(top - base) + v.y * __builtin_amdgcn_exp2f(v.x - base);
        top = t;
    };
    if (m < M)
#pragma unroll 8
        for (int c = slice; c < count; c += SLICES) join(part[(int64_t)c * M + m]);
    red[slice][r] = make_float2(top, sum);
    __syncthreads();
    if (slice < 8) {
        for (int i = slice + 8; i < SLICES; i += 8) join(red[i][r]);
        red[slice][r] = make_float2(top, sum);
    }
    __syncthreads();
    if (slice != 0 || m >= M) return;
    for (int i = 1; i < 8; ++i) join(red[i][r]);
    constexpr double ln2 = 0.69314718055994530942;
    const float base = top > -INFINITY ? top : 0.0f;
    // (units of log 2 -> of e in double: the loss is a difference of two such values)
    const double l = ((double)base + (double)log2f(sum)) * ln2;
    const int64_t t = targets[m];
    lse[m] = (float)l;
    loss[m] = t == ignore ? 0.0f : in_vocab(t, V) ? (float)(l - (double)picked[m] * ln2) : NAN;
}

// dW [V][K] (rows of ldo) = factor[0] * scale * G^T X over at most 64 * SLOTS rows: G [M][ldg], X [M][ldx], both with rows of whole 16-byte chunks.
// What bounds it: dW's bytes.  A 256 x 256 tile of gemm_head.hip has one or two slots of 64 rows to walk here, and with one workgroup a compute unit
// nothing runs while its operands travel and its results leave.  Here a workgroup keeps 128 columns of X in registers, walks over
// tiles of 128 columns of G, the next of which is on its way, and three (two) workgroups share a compute unit.  131072 x 4096, us, 256 x 256
// tiles / this: 16 rows 425 / 259 (4.1 TB/s), 64 rows 462 / 288, 128 rows 515 / 360.
// Four waves, 64 x 64 each; tiles lie in LDS as 64 rows of 128 columns (256 bytes, the chunk swizzle of gemm_ring.hip's [K, N] tiles), fragments
// come by the transposing LDS load; X's columns are dealt so that a lane ends up with eight neighbours and stores 16 bytes.
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4* lds_i16x4_ptr;

template <int SLOTS>
__global__ __launch_bounds__(256, SLOTS == 1 ? 3 : 2) void xent_outer_kernel(const uint16_t* __restrict__ G, int64_t ldg, const uint16_t* __restrict__ X, int64_t ldx,
                                                           uint16_t* __restrict__ out, int64_t ldo, int V, int K, int M, int tiles_v,
                                                           const float* __restrict__ factor, float scale) {
    constexpr int kTile = SLOTS * 64 * 256;
    __shared__ __attribute__((aligned(16))) char lds[2][kTile];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wv = wave >> 1, wk = wave & 1;
    const int k0 = blockIdx.x * 128;
    auto swz = [](int row) { return ((row & 3) | (((row >> 3) & 1) << 2)) << 1; };
    // thread t moves chunk t % 16 of rows t / 16 + 16 * i
    const int chunk = threadIdx.x & 15, row0 = threadIdx.x >> 4;
    uint4 next[4 * SLOTS];
    auto fetch = [&](const uint16_t* from, int64_t ld, int col) {
        const bool in = col + chunk * 8 < ld;
#pragma unroll
        for (int i = 0; i < 4 * SLOTS; ++i) {
            const int m = row0 + 16 * i;
            next[i] = make_uint4(0u, 0u, 0u, 0u);
            if (m < M && in) next[i] = *reinterpret_cast<const uint4*>(from + (int64_t)m * ld + col + chunk * 8);
        }
    };
    auto put = [&](char* to) {
#pragma unroll
        for (int i = 0; i < 4 * SLOTS; ++i) {
            const int row = row0 + 16 * i;
            *reinterpret_cast<uint4*>(to + row * 256 + ((chunk ^ swz(row)) << 4)) = next[i];
        }
    };
    // lane 16q + 4r + s supplies rows 32h + 8q (+4) + r, four columns of a block, and receives its own column's values
    const int r = (lane >> 2) & 3, q = lane >> 4, s = lane & 3, f = (r | ((q & 1) << 2)) << 1;
    auto fragment = [&](const char* from, int h, int byte) {
        char* const at = const_cast<char*>(from) + (32 * h + 8 * q + r) * 256 + ((((byte >> 4) ^ f) << 4) | (byte & 8));
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)at);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(at + 4 * 256));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    fetch(X, ldx, k0);
    put(lds[1]);
    int tile = blockIdx.y;   // (the grid has no more rows than tiles)
    fetch(G, ldg, tile * 128);
    __syncthreads();
    // block j holds columns 32 * (j / 2) + 8 * (c / 4) + 4 * (j % 2) + c % 4, c = 0 .. 15
    bf16x8 b[2 * SLOTS][4];
#pragma unroll
    for (int h = 0; h < 2 * SLOTS; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) b[h][j] = fragment(lds[1], h, wk * 128 + (j >> 1) * 64 + s * 16 + (j & 1) * 8);
    put(lds[0]);
    __syncthreads();
    const int steps = (M + 31) / 32;
    const float times = factor[0] * scale;
    for (int buf = 0; tile < tiles_v; buf ^= 1) {
        const int here = tile;
        tile += gridDim.y;
        if (tile < tiles_v) fetch(G, ldg, tile * 128);
        f32x4 acc[4][4];   // [16 columns of X][16 columns of G]
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][i][e] = 0.0f;
#pragma unroll
        for (int h = 0; h < 2 * SLOTS; ++h) {
            if (h >= steps) break;
            bf16x8 a[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = fragment(lds[buf], h, wv * 128 + i * 32 + s * 8);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[h][j], a[i], acc[j][i], 0, 0, 0);
        }
        if (tile < tiles_v) put(lds[buf ^ 1]);   // (last read two tiles ago, a barrier between)
        // a lane holds column lane % 16 of G's block and eight columns of X's two blocks
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int v = here * 128 + wv * 64 + i * 16 + (lane & 15);
            if (v >= V) continue;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int k = k0 + wk * 64 + t * 32 + q * 8;
                uint16_t* const to = out + (int64_t)v * ldo + k;
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = bf16_pair(times * acc[2 * t + (e >> 1)][i][2 * (e & 1)], times * acc[2 * t + (e >> 1)][i][2 * (e & 1) + 1]);
                if (k + 7 < K) {
                    __builtin_memcpy(to, w, 16);   // (one store, whatever the rows' alignment)
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (k + e < K) to[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
        __syncthreads();
    }
}

// out [rows][K] (bf16, rows of ldo) = sum over shares of sums[share][rows][lds], times factor[step * r] * scale.
__global__ __launch_bounds__(256) void xent_fold_kernel(const float* __restrict__ sums, int shares, int64_t lds, uint16_t* __restrict__ out, int64_t ldo,
                                                        int64_t rows, int K, const float* __restrict__ factor, int64_t step, float scale) {
    const int64_t quads = lds / 4, total = rows * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / quads;
        const int c = (int)(i - r * quads) * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
        for (int k = 0; k < shares; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(sums + ((int64_t)k * rows + r) * lds + c);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const float f = factor[step * r] * scale;
        const uint32_t lo = bf16_pair(f * s.x, f * s.y), hi = bf16_pair(f * s.z, f * s.w);
        const uint32_t h[2] = {lo, hi};
        uint16_t* const to = out + r * ldo + c;
        if (c + 3 < K) {
            __builtin_memcpy(to, h, 8);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < K) to[e] = (uint16_t)(h[e >> 1] >> (16 * (e & 1)));
        }
    }
}

constexpr size_t kAlign = 256;
int64_t up_to(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
size_t up(size_t bytes) { return (bytes + kAlign - 1) / kAlign * kAlign; }

// Columns of a piece: at most 256 MiB of fp32 logits, in whole tiles.
int piece_cols(int M, int V, int asked) {
    int64_t p = asked > 0 ? asked : ((int64_t)64 << 20) / M;
    p = (p + 255) / 256 * 256;
    return p > V ? V : (int)p;
}

struct XentLayout {
    int piece;
    size_t x, w, z, gt, part, sum, state, total;
};
XentLayout layout(int M, int V, int K, int asked, bool backward) {
    XentLayout l{};
    l.piece = piece_cols(M, V, asked);
    size_t at = 0;
    auto take = [&](size_t values) { const size_t here = at; at += up(values * 4); return here; };
    l.x = take((size_t)M * K);
    l.w = take((size_t)l.piece * K);
    l.z = take((size_t)M * l.piece);
    if (backward) {
        l.gt = take((size_t)M * l.piece);
        l.part = take((size_t)(M > l.piece ? M : l.piece) * K);
        l.sum = take((size_t)M * K);
    } else {
        l.state = take((size_t)M * 4);
    }
    l.total = at;
    return l;
}

constexpr int64_t kPanel = ((int64_t)1 << 32) - (1 << 20);   // bytes that an operand's 32-bit offsets reach, with room for a slot

// Columns of a piece of the bf16 backward pass: G takes at most 256 MiB, and W's rows stay within reach.  Columns of W packed at a time, where it has to be: 128 MiB.
int piece_cols_bf16(int M, int V, int64_t kp, int asked) {
    int64_t p = asked > 0 ? up_to(asked, 256) : ((int64_t)128 << 20) / M / 256 * 256;
    if (asked <= 0 && p < 1024) p = 1024;
    const int64_t reach = kPanel / (2 * kp) / 256 * 256;
    if (p > reach && reach > 0) p = reach;
    return p > V ? V : (int)p;
}
int pack_cols(int V, int64_t kp) {
    int64_t p = ((int64_t)64 << 20) / kp / 256 * 256;
    if (p < 1024) p = 1024;
    return p > V ? V : (int)p;
}

// Workgroups that share a 256 x 256 tile's k in the products for dX and dW: enough to cover the compute units, at
// least eight slots (512 values of k) each.
int shares_of(int M, int N, int64_t K) {
    const int64_t tiles = up_to(M, 256) / 256 * (up_to(N, 256) / 256), ncu = device_cu_count();
    int64_t s = ncu / tiles;
    if (s > K / 512) s = K / 512;
    return s < 1 ? 1 : (int)s;
}

struct HeadLayout {
    int piece, packed, shares_x, shares_w;   // columns of a piece, of a piece of W that is packed
    int64_t kp, ks;                          // K as rows of packed operands, of sums
    size_t x, w, part, picked, factor, rows, xs, g, sum_x, sum_w, total;   // xs: X times its rows' factors
};
HeadLayout head_layout(int M, int V, int K, int asked, bool backward) {
    HeadLayout l{};
    l.kp = up_to(K, 8);
    l.ks = up_to(K, 4);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += up(bytes); return here; };
    l.packed = pack_cols(V, l.kp);
    if (backward) {
        l.piece = piece_cols_bf16(M, V, l.kp, asked);
        if (l.packed > l.piece) l.packed = l.piece;
    }
    l.x = take((size_t)M * l.kp * 2);
    l.w = take((size_t)l.packed * l.kp * 2);
    if (!backward) {
        // (whole, or in packed pieces: as many partial statistics, up to the narrower tiles of each)
        const int64_t whole = gemm_head_parts(M, V), by_piece = (int64_t)(V / l.packed) * gemm_head_parts(M, l.packed) +
                                                               (V % l.packed != 0 ? gemm_head_parts(M, V % l.packed) : 0);
        l.part = take((size_t)(whole > by_piece ? whole : by_piece) * M * sizeof(float2));
        l.picked = take((size_t)M * 4);
    } else {
        l.shares_x = shares_of(M, K, l.packed);
        l.shares_w = shares_of(l.packed, K, M);
        l.factor = take(((size_t)M + 1) * 4);
        l.rows = take((size_t)M * sizeof(float4));
        l.xs = take((size_t)M * l.kp * 2);
        l.g = take((size_t)M * up_to(l.piece, 64) * 2);
        l.sum_x = take(l.shares_x > 1 || l.packed < V ? (size_t)l.shares_x * M * l.ks * 4 : 0);
        l.sum_w = take(l.shares_w > 1 ? (size_t)l.shares_w * l.piece * l.ks * 4 : 0);
    }
    l.total = at;
    return l;
}

unsigned sweep_grid(int64_t total) {
    const int64_t g = (total + 255) / 256, most = (int64_t)device_cu_count() * 32;
    return (unsigned)(g < most ? g : most);
}

int check_xent(const void* X, const void* W, const int64_t* targets, int M, int V, int K, int64_t ldx, int64_t ldw, int dtype, float scale,
               int64_t ignore, int vocab_piece) {
    if (X == nullptr || W == nullptr || targets == nullptr || M <= 0 || V <= 0 || K <= 0 || ldx < K || ldw < K || vocab_piece < 0)
        return ROV_ERR_INVALID;
    if (!(scale > 0.0f) || !isfinite(scale) || (ignore >= 0 && ignore < V)) return ROV_ERR_INVALID;
    if (dtype != ROV_F32 && dtype != ROV_BF16) return dtype == ROV_FP8_E4M3 ? ROV_ERR_UNSUPPORTED : ROV_ERR_INVALID;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    if (!aligned(X, esz) || !aligned(W, esz) || !aligned(targets, 8)) return ROV_ERR_INVALID;
    // (fp32: a workgroup a row; bf16: tiles are counted below)
    if (V > (1 << 30) || M > (1 << 27) || (dtype == ROV_F32 && !grid_fits(M, 256))) return ROV_ERR_UNSUPPORTED;
    return ROV_OK;
}

int pack(const void* src, int64_t ld, void* dst, int64_t rows, int K, int64_t kp, const float* factor, hipStream_t st) {
    hipLaunchKernelGGL(xent_pack_kernel, dim3(sweep_grid(rows * kp / 8)), dim3(256), 0, st, (const uint16_t*)src, ld, (uint16_t*)dst, rows, K, (int)kp, factor);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
int fold(const float* sums, int shares, int64_t lds, void* out, int64_t ldo, int rows, int K, const float* factor, int64_t step, float scale, hipStream_t st) {
    hipLaunchKernelGGL(xent_fold_kernel, dim3(sweep_grid((int64_t)rows * lds / 4)), dim3(256), 0, st, sums, shares, lds, (uint16_t*)out, ldo, (int64_t)rows, K,
                       factor, step, scale);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
// out [M][N] (rows of ldo) = A W or A^T W summed over `shares` of k; sum == NULL (one share): at once, else through sum, to which it is added
// (`add`), and from there to out if `last`, times factor[step * m] * scale.  Strides in elements.
int product(int kind, const void* A, int64_t lda, const void* W, int64_t ldw, void* out, int64_t ldo, int M, int N, int K, int shares, float* sum,
            int64_t lds, bool add, bool last, const float* factor, int64_t step, float scale, hipStream_t st) {
    HeadArgs h;
    h.factor = factor;
    h.factor_step = step;
    h.scale = scale;
    h.ld_a = (size_t)lda * 2;
    h.ld_w = (size_t)ldw * 2;
    h.sum = sum;
    h.ld_sum = lds;
    h.add = add;
    h.ld_out = ldo;
    const int rc = launch_gemm_head(kind, A, W, out, M, N, K, 1.0f, shares, h, st);
    if (rc != ROV_OK || sum == nullptr || !last) return rc;
    return fold(sum, shares, lds, out, ldo, M, N, factor, step, scale, st);
}
int outer(const void* G, int64_t ldg, const void* X, int64_t ldx, uint16_t* out, int64_t ldo, int V, int K, int M, const float* factor, float scale,
          hipStream_t st) {
    const int64_t tiles_k = up_to(K, 128) / 128, tiles_v = up_to(V, 128) / 128;
    int64_t rows = 3 * device_cu_count() / tiles_k;   // as many workgroups as run at once
    if (rows > tiles_v) rows = tiles_v;
    if (rows < 1) rows = 1;
    const dim3 grid((unsigned)tiles_k, (unsigned)rows);
    if (M <= 64)
        hipLaunchKernelGGL(xent_outer_kernel<1>, grid, dim3(256), 0, st, (const uint16_t*)G, ldg, (const uint16_t*)X, ldx, out, ldo, V, K, M, (int)tiles_v,
                           factor, scale);
    else
        hipLaunchKernelGGL(xent_outer_kernel<2>, grid, dim3(256), 0, st, (const uint16_t*)G, ldg, (const uint16_t*)X, ldx, out, ldo, V, K, M, (int)tiles_v,
                           factor, scale);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
bool rows_fit(const void* p, int64_t ld, int K) { return K % 8 == 0 && ld % 8 == 0 && aligned(p, 16); }
constexpr float kLog2e = 1.44269504088896341f;

// Operands are addressed with 32-bit byte offsets: 256 rows, or all rows of k of the products for dX (a piece of W, packed where its
// own rows reach too far) and dW (X times its factors, G).
int check_head(int M, int V, int64_t ldx, int64_t ldw, const HeadLayout& l, bool backward) {
    const int64_t ld = ldx > ldw ? ldx : ldw;
    if (512 * up_to(ld, 8) > kPanel || 512 * l.kp > kPanel) return ROV_ERR_UNSUPPORTED;
    const int64_t widest = V > l.kp ? V : l.kp, longest = M > V ? M : V;
    if (!grid_fits(up_to(longest, 256) / 256 * (up_to(widest, 128) / 128), 256)) return ROV_ERR_UNSUPPORTED;   // tiles of any of the products
    if (backward && (up_to(l.packed, 64) * 2 * l.kp > kPanel || up_to(M, 64) * 2 * l.kp > kPanel || up_to(M, 64) * 2 * up_to(l.piece, 64) > kPanel))
        return ROV_ERR_UNSUPPORTED;
    return ROV_OK;
}

int head_forward(const void* X, const void* W, const int64_t* targets, int M, int V, int K, int64_t ldx, int64_t ldw, float scale, int64_t ignore,
                 float* loss, float* lse, char* ws, const HeadLayout& l, hipStream_t st) {
    HeadArgs h;
    h.targets = targets;
    h.picked = (float*)(ws + l.picked);
    h.part = (float2*)(ws + l.part);
    const void* x = X;
    h.ld_a = (size_t)ldx * 2;
    int kx = K;
    const bool fit_w = rows_fit(W, ldw, K);
    if (!fit_w || !rows_fit(X, ldx, K)) {
        x = ws + l.x;
        h.ld_a = (size_t)l.kp * 2;
        kx = (int)l.kp;
        const int rc = pack(X, ldx, ws + l.x, M, K, l.kp, nullptr, st);
        if (rc != ROV_OK) return rc;
    }
    int count = 0;
    if (fit_w) {
        count = gemm_head_parts(M, V);
        h.ld_w = (size_t)ldw * 2;
        const int rc = launch_gemm_head(HEAD_STATS, x, W, nullptr, M, V, kx, scale * kLog2e, 1, h, st);
        if (rc != ROV_OK) return rc;
    } else {
        h.ld_w = (size_t)l.kp * 2;
        for (int v0 = 0; v0 < V; v0 += l.packed) {
            const int cols = V - v0 < l.packed ? V - v0 : l.packed;
            int rc = pack((const char*)W + (size_t)v0 * ldw * 2, ldw, ws + l.w, cols, K, l.kp, nullptr, st);
            if (rc != ROV_OK) return rc;
            h.v0 = v0;
            h.part = (float2*)(ws + l.part) + (size_t)count * M;
            count += gemm_head_parts(M, cols);
            rc = launch_gemm_head(HEAD_STATS, x, ws + l.w, nullptr, M, cols, kx, scale * kLog2e, 1, h, st);
            if (rc != ROV_OK) return rc;
        }
    }
    // (few rows: more threads a row, 16 x 131072 12 -> 5 us)
    if (M < 1024)
        hipLaunchKernelGGL(xent_join_kernel<4>, dim3((unsigned)((M + 3) / 4)), dim3(256), 0, st, (const float2*)(ws + l.part), count,
                           h.picked, M, V, targets, ignore, loss, lse);
    else
        hipLaunchKernelGGL(xent_join_kernel<16>, dim3((unsigned)((M + 15) / 16)), dim3(256), 0, st, (const float2*)(ws + l.part),
                           count, h.picked, M, V, targets, ignore, loss, lse);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}

int head_backward(const void* X, const void* W, const int64_t* targets, const float* lse, const float* dloss, const float* dlse, int M, int V, int K,
                  int64_t ldx, int64_t ldw, float scale, int64_t ignore, void* dX, void* dW, int64_t lddx, int64_t lddw, char* ws, const HeadLayout& l,
                  hipStream_t st) {
    HeadArgs h;
    h.rows = (const float4*)(ws + l.rows);
    h.factor = (const float*)(ws + l.factor);
    hipLaunchKernelGGL(xent_factor_kernel, dim3(1), dim3(1024), 0, st, targets, ignore, V, dloss, dlse, lse,
                       (float*)(ws + l.factor), (float4*)(ws + l.rows), M);
    ROV_LAUNCH_CHECK();
    const bool fit_w = rows_fit(W, ldw, K) && up_to(l.piece, 64) * 2 * ldw <= kPanel;
    const char* x = (const char*)X;
    h.ld_a = (size_t)ldx * 2;
    int rc = ROV_OK;
    if (!fit_w || !rows_fit(X, ldx, K)) {
        x = ws + l.x;
        h.ld_a = (size_t)l.kp * 2;
        rc = pack(X, ldx, ws + l.x, M, K, l.kp, nullptr, st);
        if (rc != ROV_OK) return rc;
    }
    if (dW != nullptr) {
        rc = pack(X, ldx, ws + l.xs, M, K, l.kp, h.factor, st);
        if (rc != ROV_OK) return rc;
    }
    const int kx = (int)l.kp, piece = fit_w ? l.piece : l.packed;   // (operands that fit have K = kp)
    float* const sum_x = l.shares_x > 1 || piece < V ? (float*)(ws + l.sum_x) : nullptr;
    float* const sum_w = l.shares_w > 1 ? (float*)(ws + l.sum_w) : nullptr;
    for (int v0 = 0; v0 < V; v0 += piece) {
        const int cols = V - v0 < piece ? V - v0 : piece;
        const int64_t ldg = up_to(cols, 64);
        const char* w = (const char*)W + (size_t)v0 * ldw * 2;
        int64_t ld = ldw;
        if (!fit_w) {
            rc = pack(w, ldw, ws + l.w, cols, K, l.kp, nullptr, st);
            if (rc != ROV_OK) return rc;
            w = ws + l.w;
            ld = l.kp;
        }
        h.ld_w = (size_t)ld * 2;
        h.v0 = v0;
        h.g = (uint16_t*)(ws + l.g);
        h.ld_g = h.g_cols = ldg;
        rc = launch_gemm_head(HEAD_GRAD, x, w, nullptr, M, cols, kx, scale * kLog2e, 1, h, st);
        if (rc != ROV_OK) return rc;
        if (dX != nullptr) {
            // (the last, shorter piece may have fewer slots of k than shares: the sums of the shares left out stay)
            const int shares = l.shares_x > ldg / 64 ? (int)(ldg / 64) : l.shares_x;
            rc = product(HEAD_DX, ws + l.g, ldg, w, ld, dX, lddx, M, K, cols, shares, sum_x, l.ks, v0 > 0, false, h.factor, 1, scale, st);
            if (rc != ROV_OK) return rc;
        }
        if (dW != nullptr) {
            if (M <= 128) {
                rc = outer(ws + l.g, ldg, ws + l.xs, l.kp, (uint16_t*)dW + (size_t)v0 * lddw, lddw, cols, K, M, h.factor + M, scale, st);
                if (rc != ROV_OK) return rc;
                continue;
            }
            rc = product(HEAD_DW, ws + l.g, ldg, ws + l.xs, l.kp, (char*)dW + (size_t)v0 * lddw * 2, lddw, cols, K, M, l.shares_w, sum_w, l.ks, false, true,
                         h.factor + M, 0, scale, st);
            if (rc != ROV_OK) return rc;
        }
    }
    return dX != nullptr && sum_x != nullptr ? fold(sum_x, l.shares_x, l.ks, dX, lddx, M, K, h.factor, 1, scale, st) : ROV_OK;
}

// The products of head_forward and head_backward whose workgroups take several tiles, for operands that lie as the kernels take them.
int head_walks(int M, int V, int K, const HeadLayout& l, bool backward) {
    const int kx = (int)l.kp, piece = K % 8 != 0 ? l.packed : backward ? l.piece : V;
    int found = 0;
    for (int v0 = 0; v0 < V; v0 += piece) {
        const int cols = V - v0 < piece ? V - v0 : piece;
        if (!backward) {
            found |= gemm_head_walks(HEAD_STATS, M, cols, kx, 1) ? 1 : 0;
            continue;
        }
        const int64_t slots = up_to(cols, 64) / 64;
        found |= gemm_head_walks(HEAD_GRAD, M, cols, kx, 1) ? 2 : 0;
        found |= gemm_head_walks(HEAD_DX, M, K, cols, l.shares_x > slots ? (int)slots : l.shares_x) ? 4 : 0;
        found |= M > 128 && gemm_head_walks(HEAD_DW, cols, K, M, l.shares_w) ? 8 : 0;
    }
    return found;
}

int copy(const void* src, int64_t lds, void* dst, int64_t ldd, int64_t rows, int cols, const int64_t* targets, int64_t ignore, hipStream_t st) {
    hipLaunchKernelGGL(xent_copy_kernel, dim3(sweep_grid(rows * cols)), dim3(256), 0, st, (const float*)src, lds, (float*)dst, ldd, rows, cols, targets,
                       ignore);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
// rows that the fp32 products take, and leave, where they lie
bool dense(const void* p, int64_t ld, int K) { return ld == K && aligned(p, 16); }

#define ROV_STEP(expr)               \
    do {                             \
        const int rc_ = (expr);      \
        if (rc_ != ROV_OK) return rc_; \
    } while (0)

}  // namespace
}  // namespace rov

extern "C" size_t rov_linear_xent_workspace_bytes(int M, int V, int K, int dtype, int backward, int vocab_piece) {
    if (M <= 0 || V <= 0 || K <= 0 || vocab_piece < 0 || (dtype != ROV_F32 && dtype != ROV_BF16)) return 0;
    return dtype == ROV_BF16 ? rov::head_layout(M, V, K, vocab_piece, backward != 0).total : rov::layout(M, V, K, vocab_piece, backward != 0).total;
}

extern "C" int rov_linear_xent_walks(int M, int V, int K, int backward, int vocab_piece) {
    if (M <= 0 || V <= 0 || K <= 0 || vocab_piece < 0) return ROV_ERR_INVALID;
    using namespace rov;
    const HeadLayout l = head_layout(M, V, K, vocab_piece, backward != 0);
    ROV_STEP(check_head(M, V, K, K, l, backward != 0));
    return head_walks(M, V, K, l, backward != 0);
}

extern "C" int rov_linear_xent(const void* X, const void* W, const int64_t* targets, int M, int V, int K, int64_t ldx, int64_t ldw, int dtype,
                               float scale, int64_t ignore_index, float* loss, float* lse, int vocab_piece, void* workspace,
                               size_t workspace_bytes, void* stream) {
    using namespace rov;
    ROV_STEP(check_xent(X, W, targets, M, V, K, ldx, ldw, dtype, scale, ignore_index, vocab_piece));
    if (loss == nullptr || lse == nullptr || loss == lse || !aligned(loss, 4) || !aligned(lse, 4)) return ROV_ERR_INVALID;
    if (workspace == nullptr || !aligned(workspace, kAlign)) return ROV_ERR_INVALID;
    if (dtype == ROV_BF16) {
        const HeadLayout hl = head_layout(M, V, K, vocab_piece, false);
        ROV_STEP(check_head(M, V, ldx, ldw, hl, false));
        if (workspace_bytes < hl.total) return ROV_ERR_WORKSPACE;
        return head_forward(X, W, targets, M, V, K, ldx, ldw, scale, ignore_index, loss, lse, (char*)workspace, hl, (hipStream_t)stream);
    }
    const XentLayout l = layout(M, V, K, vocab_piece, false);
    if (workspace_bytes < l.total) return ROV_ERR_WORKSPACE;
    char* const ws = (char*)workspace;
    float* const z = (float*)(ws + l.z);
    hipStream_t st = (hipStream_t)stream;
    const void* const x = dense(X, ldx, K) ? X : ws + l.x;
    ROV_STEP(check_gemm(x, ws + l.w, z, nullptr, EPI_ADD, M, l.piece, K, ROV_F32, 1));
    if (x != X) ROV_STEP(copy(X, ldx, ws + l.x, K, M, K, nullptr, 0, st));
    for (int v0 = 0; v0 < V; v0 += l.piece) {
        const int cols = V - v0 < l.piece ? V - v0 : l.piece;
        const void* w = (const char*)W + (size_t)v0 * ldw * 4;
        if (!dense(W, ldw, K)) {
            ROV_STEP(copy(w, ldw, ws + l.w, K, cols, K, nullptr, 0, st));
            w = ws + l.w;
        }
        ROV_STEP(launch_gemm(x, w, z, M, cols, K, ROV_F32, 1, 1.0f, 1.0f, st));
        hipLaunchKernelGGL(xent_stats_kernel, dim3((unsigned)M), dim3(256), 0, st, z, cols, v0, V, scale, targets, ignore_index,
                           (RowState*)(ws + l.state), loss, lse);
        ROV_LAUNCH_CHECK();
    }
    return ROV_OK;
}

extern "C" int rov_linear_xent_bwd(const void* X, const void* W, const int64_t* targets, const float* lse, const float* dloss,
                                   const float* dlse, int M, int V, int K, int64_t ldx, int64_t ldw, int dtype, float scale,
                                   int64_t ignore_index, void* dX, void* dW, int64_t lddx, int64_t lddw, int vocab_piece, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    using namespace rov;
    ROV_STEP(check_xent(X, W, targets, M, V, K, ldx, ldw, dtype, scale, ignore_index, vocab_piece));
    if (lse == nullptr || dloss == nullptr || dX == dW) return ROV_ERR_INVALID;
    if ((dX != nullptr && dX == W) || (dW != nullptr && dW == X)) return ROV_ERR_INVALID;   // (the next piece of the vocabulary reads both operands)
    if (!aligned(lse, 4) || !aligned(dloss, 4) || !aligned(dlse, 4)) return ROV_ERR_INVALID;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    if ((dX != nullptr && (lddx < K || !aligned(dX, esz))) || (dW != nullptr && (lddw < K || !aligned(dW, esz)))) return ROV_ERR_INVALID;
    if (workspace == nullptr || !aligned(workspace, kAlign)) return ROV_ERR_INVALID;
    if (dtype == ROV_BF16) {
        const HeadLayout hl = head_layout(M, V, K, vocab_piece, true);
        ROV_STEP(check_head(M, V, ldx, ldw, hl, true));
        if (workspace_bytes < hl.total) return ROV_ERR_WORKSPACE;
        return head_backward(X, W, targets, lse, dloss, dlse, M, V, K, ldx, ldw, scale, ignore_index, dX, dW, lddx, lddw, (char*)workspace, hl,
                             (hipStream_t)stream);
    }
    const XentLayout l = layout(M, V, K, vocab_piece, true);
    if (workspace_bytes < l.total) return ROV_ERR_WORKSPACE;
    char* const ws = (char*)workspace;
    float *z = (float*)(ws + l.z), *gt = (float*)(ws + l.gt), *part = (float*)(ws + l.part);
    hipStream_t st = (hipStream_t)stream;
    // (rows of ignored targets zero: what they hold must not reach dW)
    float* const x = (float*)(ws + l.x);
    ROV_STEP(check_gemm(x, ws + l.w, z, nullptr, EPI_ADD, M, l.piece, K, ROV_F32, 1));
    ROV_STEP(check_gemm(z, ws + l.w, part, nullptr, EPI_ADD, M, K, l.piece, ROV_F32, 0));
    ROV_STEP(check_gemm(gt, x, part, nullptr, EPI_ADD, l.piece, K, M, ROV_F32, 0));
    ROV_STEP(copy(X, ldx, x, K, M, K, targets, ignore_index, st));
    float* const sum = dense(dX, lddx, K) ? (float*)dX : (float*)(ws + l.sum);
    for (int v0 = 0; v0 < V; v0 += l.piece) {
        const int cols = V - v0 < l.piece ? V - v0 : l.piece;
        const void* w = (const char*)W + (size_t)v0 * ldw * 4;
        if (!dense(W, ldw, K)) {
            ROV_STEP(copy(w, ldw, ws + l.w, K, cols, K, nullptr, 0, st));
            w = ws + l.w;
        }
        ROV_STEP(launch_gemm(x, w, z, M, cols, K, ROV_F32, 1, 1.0f, 1.0f, st));
        const int ytiles = (M + 63) / 64;
        hipLaunchKernelGGL(xent_grad_kernel, dim3((unsigned)((cols + 63) / 64), (unsigned)(ytiles < 65535 ? ytiles : 65535)), dim3(256), 0, st, z, gt, M,
                           cols, v0, V, scale, targets, ignore_index, lse, dloss, dlse);
        ROV_LAUNCH_CHECK();
        if (dX != nullptr) {
            ROV_STEP(launch_gemm(z, w, v0 == 0 ? sum : part, M, K, cols, ROV_F32, 0, 1.0f, 1.0f, st));
            if (v0 > 0) {
                hipLaunchKernelGGL(xent_add_kernel, dim3(sweep_grid((int64_t)M * K)), dim3(256), 0, st, part, sum, (int64_t)M * K);
                ROV_LAUNCH_CHECK();
            }
        }
        if (dW != nullptr) {
            char* const out = (char*)dW + (size_t)v0 * lddw * 4;
            const bool at_once = dense(dW, lddw, K);
            ROV_STEP(launch_gemm(gt, x, at_once ? (void*)out : part, cols, K, M, ROV_F32, 0, 1.0f, 1.0f, st));
            if (!at_once) ROV_STEP(copy(part, K, out, lddw, cols, K, nullptr, 0, st));
        }
    }
    return dX != nullptr && sum != dX ? copy(sum, K, dX, lddx, M, K, nullptr, 0, st) : ROV_OK;
}
