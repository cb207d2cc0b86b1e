// Softmax cross entropy of logits z = scale * X W^T over a large vocabulary, and its gradients, without keeping z:
//     lse_m = log sum_v exp z_mv,   loss_m = lse_m - z_m,target(m)
//     G_mv = scale * (exp(z_mv - lse_m) * (dloss_m + dlse_m) - [v == target(m)] * dloss_m),   dX = G W,   dW = G^T X.
// 2 M V K operations forward and 6 backward, which makes the logits again: matrix cores bound both, but for few rows, where
// W's bytes do.
//
// bf16: the 256-row kernel of gemm.hip with its own epilogues.  Forward, a tile's logits are reduced in the accumulators to a
// maximum and a sum of exponentials per row and 128 columns, which a second kernel joins; nothing else leaves the tile.  Backward
// walks the vocabulary in pieces: the accumulators of a piece's logits become G, stored in bf16 with k contiguous for either of the next
// products (G for dX, its transpose for dW; the tile's rows and columns are dealt to the lanes so that both leave in 16-byte stores), and
// X and the piece of W are transposed once for them.  dX is summed over the pieces, and over shares of the vocabulary where its tiles alone
// would leave compute units idle, in fp32.
// fp32: the fp32 products of gemm_ring.hip; a piece's logits live in the workspace while they are reduced, or turned into G in place.
#include <hip/hip_runtime.h>
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
    float top = -INFINITY;
    for (int c = threadIdx.x; c < cols; c += 256) top = fmaxf(top, scale * zr[c]);
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
    for (int c = threadIdx.x; c < cols; c += 256) sum += __expf(scale * zr[c] - base);
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
// dst [rows][kp] = src, columns K .. kp zero.
__global__ __launch_bounds__(256) void xent_pack_kernel(const uint16_t* __restrict__ src, int64_t ld, uint16_t* __restrict__ dst, int64_t rows, int K, int kp) {
    const int64_t total = rows * kp;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / kp;
        const int c = (int)(i - r * kp);
        dst[i] = c < K ? src[r * ld + c] : (uint16_t)0;
    }
}

// dst [K][ldt] = src [rows][ld] transposed; rows of ignored targets (targets may be NULL) and columns rows .. ldt are zero.
// 64 x 64 values a workgroup through LDS, 128 bytes of a row at a time on either side; VEC: src rows on 16 bytes.
template <bool VEC>
__global__ __launch_bounds__(256) void xent_transpose_kernel(const uint16_t* __restrict__ src, int64_t ld, uint16_t* __restrict__ dst, int64_t ldt, int rows,
                                                            int K, const int64_t* __restrict__ targets, int64_t ignore) {
    __shared__ uint16_t tile[64][66];
    const int r0 = blockIdx.x * 64, k0 = blockIdx.y * 64;
    for (int i = threadIdx.x; i < 512; i += 256) {
        const int r = i >> 3, c = (i & 7) * 8;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        const bool in = r0 + r < rows && !(targets != nullptr && targets[r0 + r] == ignore);
        const uint16_t* const at = src + (int64_t)(r0 + r) * ld + k0 + c;
        if (in) {
            if (VEC && k0 + c + 8 <= K) {
                v = *reinterpret_cast<const uint4*>(at);
            } else {
                uint32_t h[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = k0 + c + e < K ? at[e] : 0u;
                v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
            }
        }
        uint32_t* const to = reinterpret_cast<uint32_t*>(&tile[r][c]);
        to[0] = v.x; to[1] = v.y; to[2] = v.z; to[3] = v.w;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 512; i += 256) {
        const int k = i >> 3, r = (i & 7) * 8;
        if (k0 + k >= K || r0 + r >= ldt) continue;
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = tile[r + e][k];
        *reinterpret_cast<uint4*>(dst + (int64_t)(k0 + k) * ldt + r0 + r) =
            make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
}

// Joins the statistics part[count][M] of M rows (units of log 2) and writes the results: 16 rows a workgroup, 16 threads a row.
__global__ __launch_bounds__(256) void xent_join_kernel(const float2* __restrict__ part, int count, const float* __restrict__ picked, int M, int V,
                                                        const int64_t* __restrict__ targets, int64_t ignore, float* __restrict__ loss,
                                                        float* __restrict__ lse) {
    __shared__ float2 red[16][16];
    const int r = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int64_t m = (int64_t)blockIdx.x * 16 + r;
    float top = -INFINITY, sum = 0.0f;
    auto join = [&](float2 v) {
        const float t = fmaxf(top, v.x), base = t > -INFINITY ? t : 0.0f;
        sum = sum * __builtin_amdgcn_exp2f(top - base) + v.y * __builtin_amdgcn_exp2f(v.x - base);
        top = t;
    };
    if (m < M)
#pragma unroll 4
        for (int c = slice; c < count; c += 16) join(part[(int64_t)c * M + m]);
    red[slice][r] = make_float2(top, sum);
    __syncthreads();
    if (slice != 0 || m >= M) return;
    for (int i = 1; i < 16; ++i) join(red[i][r]);
    constexpr double ln2 = 0.69314718055994530942;
    const float base = top > -INFINITY ? top : 0.0f;
    // (units of log 2 -> of e in double: the loss is a difference of two such values)
    const double l = ((double)base + (double)log2f(sum)) * ln2;
    const int64_t t = targets[m];
    lse[m] = (float)l;
    loss[m] = t == ignore ? 0.0f : in_vocab(t, V) ? (float)(l - (double)picked[m] * ln2) : NAN;
}

// out [rows][K] (bf16, rows of ldo) = sum over shares of sums[share][rows][lds].
__global__ __launch_bounds__(256) void xent_fold_kernel(const float* __restrict__ sums, int shares, int64_t lds, uint16_t* __restrict__ out, int64_t ldo,
                                                        int64_t rows, int K) {
    const int64_t quads = lds / 4, total = rows * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / quads;
        const int c = (int)(i - r * quads) * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k = 0; k < shares; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(sums + ((int64_t)k * rows + r) * lds + c);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const uint32_t lo = bf16_pair(s.x, s.y), hi = bf16_pair(s.z, s.w);
        const uint16_t h[4] = {(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
        uint16_t* const to = out + r * ldo + c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < K) to[e] = h[e];
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

// Columns of a piece of the bf16 backward pass: G, its transpose and the piece of W transposed take at most 128 MiB each (8192 x
// 131072 x 4096: 16 pieces).
int piece_cols_bf16(int M, int V, int K, int asked) {
    const int64_t wide = M > K ? M : K;
    int64_t p = asked > 0 ? up_to(asked, 256) : ((int64_t)64 << 20) / wide / 256 * 256;
    if (asked <= 0 && p < 1024) p = 1024;
    return p > V ? V : (int)p;
}
constexpr int kPackCols = 4096;   // columns of W that the forward pass packs at a time, where it has to

// Workgroups that share a 256 x 256 tile's k in the products for dX and dW: enough to cover the compute units, at
// least eight slots (512 values of k) each.
int shares_of(int M, int N, int64_t K) {
    const int64_t tiles = up_to(M, 256) / 256 * (up_to(N, 256) / 256), ncu = device_cu_count();
    int64_t s = ncu / tiles;
    if (s > K / 512) s = K / 512;
    return s < 1 ? 1 : (int)s;
}

struct HeadLayout {
    int piece, shares_x, shares_w;
    int64_t kp, mp, ks;    // K and M as rows of products, K as rows of sums
    size_t x, w, part, picked, xt, g, gt, sum_x, sum_w, total;
};
HeadLayout head_layout(int M, int V, int K, int asked, bool backward) {
    HeadLayout l{};
    l.kp = up_to(K, 8);
    l.mp = up_to(M, 64);
    l.ks = up_to(K, 4);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += up(bytes); return here; };
    l.x = take((size_t)M * l.kp * 2);
    if (!backward) {
        l.piece = V < kPackCols ? V : kPackCols;
        l.w = take((size_t)l.piece * l.kp * 2);
        l.part = take((size_t)(2 * gemm_head_tiles_n(V) + 2) * M * sizeof(float2));
        l.picked = take((size_t)M * 4);
    } else {
        l.piece = piece_cols_bf16(M, V, K, asked);
        const int64_t pp = up_to(l.piece, 64);
        l.shares_x = shares_of(M, K, pp);
        l.shares_w = shares_of(l.piece, K, l.mp);
        const size_t packed = (size_t)l.piece * l.kp * 2, turned = (size_t)K * pp * 2;
        l.w = take(packed > turned ? packed : turned);   // the piece of W: packed for the logits, then transposed
        l.xt = take((size_t)K * l.mp * 2);
        l.g = take((size_t)M * pp * 2);
        l.gt = take((size_t)l.piece * l.mp * 2);
        l.sum_x = take(l.shares_x > 1 || l.piece < V ? (size_t)l.shares_x * M * l.ks * 4 : 0);
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
    if (M > (1 << 30) || V > (1 << 30)) return ROV_ERR_UNSUPPORTED;
    return ROV_OK;
}

int pack(const void* src, int64_t ld, void* dst, int64_t rows, int K, int64_t kp, hipStream_t st) {
    hipLaunchKernelGGL(xent_pack_kernel, dim3(sweep_grid(rows * kp)), dim3(256), 0, st, (const uint16_t*)src, ld, (uint16_t*)dst, rows, K, (int)kp);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
int transpose(const void* src, int64_t ld, void* dst, int64_t ldt, int rows, int K, const int64_t* targets, int64_t ignore, hipStream_t st) {
    const dim3 grid((unsigned)(up_to(rows, 64) / 64), (unsigned)(up_to(K, 64) / 64));
    if (grid.y > 65535u) return ROV_ERR_UNSUPPORTED;
    if (aligned(src, 16) && ld % 8 == 0)
        hipLaunchKernelGGL((xent_transpose_kernel<true>), grid, dim3(256), 0, st, (const uint16_t*)src, ld, (uint16_t*)dst, ldt, rows, K, targets, ignore);
    else
        hipLaunchKernelGGL((xent_transpose_kernel<false>), grid, dim3(256), 0, st, (const uint16_t*)src, ld, (uint16_t*)dst, ldt, rows, K, targets, ignore);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
// out [M][N] = A W^T summed over `shares` of k; sum == NULL (one share): at once, else through sum, to which it is added (`add`), and
// from there to out if `last`.
int product(const void* A, int64_t lda, const void* W, int64_t ldw, void* out, int64_t ldo, int M, int N, int64_t K, int shares, float* sum, int64_t lds,
            bool add, bool last, hipStream_t st) {
    HeadArgs h;
    h.ld_a = (size_t)lda * 2;
    h.ld_w = (size_t)ldw * 2;
    h.sum = sum;
    h.ld_sum = lds;
    h.add = add;
    h.ld_out = ldo;
    h.out_wide = aligned(out, 8) && ldo % 4 == 0;
    const int rc = launch_gemm_head(HEAD_SUM, A, W, out, M, N, (int)K, 1.0f, shares, h, st);
    if (rc != ROV_OK || sum == nullptr || !last) return rc;
    hipLaunchKernelGGL(xent_fold_kernel, dim3(sweep_grid((int64_t)M * lds / 4)), dim3(256), 0, st, sum, shares, lds, (uint16_t*)out, ldo, (int64_t)M, N);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
bool rows_fit(const void* p, int64_t ld, int K) { return K % 8 == 0 && ld % 8 == 0 && aligned(p, 16); }
constexpr float kLog2e = 1.44269504088896341f;

int check_head(int M, int V, int K, int64_t ldx, int64_t ldw) {
    // 256-row panels of every operand are addressed with 32-bit byte offsets, sizes are products' ints
    const int64_t most = ((int64_t)1 << 32) / 512 - 64;
    if (K > most || ldx > most || ldw > most || M > most) return ROV_ERR_UNSUPPORTED;
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
        int rc = pack(X, ldx, ws + l.x, M, K, l.kp, st);
        if (rc != ROV_OK) return rc;
    }
    if (fit_w) {
        h.ld_w = (size_t)ldw * 2;
        const int rc = launch_gemm_head(HEAD_STATS, x, W, nullptr, M, V, kx, scale * kLog2e, 1, h, st);
        if (rc != ROV_OK) return rc;
    } else {
        h.ld_w = (size_t)l.kp * 2;
        for (int v0 = 0; v0 < V; v0 += l.piece) {
            const int cols = V - v0 < l.piece ? V - v0 : l.piece;
            int rc = pack((const char*)W + (size_t)v0 * ldw * 2, ldw, ws + l.w, cols, K, l.kp, st);
            if (rc != ROV_OK) return rc;
            h.v0 = v0;
            h.part = (float2*)(ws + l.part) + (size_t)(v0 / 128) * M;   // (pieces are whole tiles)
            rc = launch_gemm_head(HEAD_STATS, x, ws + l.w, nullptr, M, cols, kx, scale * kLog2e, 1, h, st);
            if (rc != ROV_OK) return rc;
        }
    }
    hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)((M + 15) / 16)), dim3(256), 0, st, (const float2*)(ws + l.part), 2 * gemm_head_tiles_n(V),
                       h.picked, M, V, targets, ignore, loss, lse);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}

int head_backward(const void* X, const void* W, const int64_t* targets, const float* lse, const float* dloss, const float* dlse, int M, int V, int K,
                  int64_t ldx, int64_t ldw, float scale, int64_t ignore, void* dX, void* dW, int64_t lddx, int64_t lddw, char* ws, const HeadLayout& l,
                  hipStream_t st) {
    HeadArgs h;
    h.targets = targets;
    h.lse = lse;
    h.dloss = dloss;
    h.dlse = dlse;
    h.ignore = ignore;
    h.vocab = V;
    h.scale = scale;
    const void* x = X;
    h.ld_a = (size_t)ldx * 2;
    int kx = K, rc = ROV_OK;
    const bool fit_w = rows_fit(W, ldw, K);
    if (!fit_w || !rows_fit(X, ldx, K)) {
        x = ws + l.x;
        h.ld_a = (size_t)l.kp * 2;
        kx = (int)l.kp;
        rc = pack(X, ldx, ws + l.x, M, K, l.kp, st);
        if (rc != ROV_OK) return rc;
    }
    if (dW != nullptr) {
        rc = transpose(X, ldx, ws + l.xt, l.mp, M, K, targets, ignore, st);
        if (rc != ROV_OK) return rc;
    }
    float* const sum_x = l.shares_x > 1 || l.piece < V ? (float*)(ws + l.sum_x) : nullptr;
    float* const sum_w = l.shares_w > 1 ? (float*)(ws + l.sum_w) : nullptr;
    for (int v0 = 0; v0 < V; v0 += l.piece) {
        const int cols = V - v0 < l.piece ? V - v0 : l.piece;
        const int64_t cp = up_to(cols, 64);
        const char* const w = (const char*)W + (size_t)v0 * ldw * 2;
        const void* wk = w;
        h.ld_w = (size_t)ldw * 2;
        if (!fit_w) {
            rc = pack(w, ldw, ws + l.w, cols, K, l.kp, st);
            if (rc != ROV_OK) return rc;
            wk = ws + l.w;
            h.ld_w = (size_t)l.kp * 2;
        }
        h.v0 = v0;
        h.g = dX != nullptr ? (uint16_t*)(ws + l.g) : nullptr;
        h.gt = dW != nullptr ? (uint16_t*)(ws + l.gt) : nullptr;
        h.ld_g = cp;
        h.ld_gt = l.mp;
        rc = launch_gemm_head(HEAD_GRAD, x, wk, nullptr, M, cols, kx, scale * kLog2e, 1, h, st);
        if (rc != ROV_OK) return rc;
        if (dX != nullptr) {
            rc = transpose(w, ldw, ws + l.w, cp, cols, K, nullptr, 0, st);
            if (rc != ROV_OK) return rc;
            // (the last, shorter piece may have fewer slots of k than shares: the sums of the shares left out stay)
            const int shares = l.shares_x > cp / 64 ? (int)(cp / 64) : l.shares_x;
            rc = product(ws + l.g, cp, ws + l.w, cp, dX, lddx, M, K, cp, shares, sum_x, l.ks, v0 > 0, false, st);
            if (rc != ROV_OK) return rc;
        }
        if (dW != nullptr) {
            rc = product(ws + l.gt, l.mp, ws + l.xt, l.mp, (char*)dW + (size_t)v0 * lddw * 2, lddw, cols, K, l.mp, l.shares_w, sum_w, l.ks, false, true, st);
            if (rc != ROV_OK) return rc;
        }
    }
    if (dX != nullptr && sum_x != nullptr) {
        hipLaunchKernelGGL(xent_fold_kernel, dim3(sweep_grid((int64_t)M * l.ks / 4)), dim3(256), 0, st, sum_x, l.shares_x, l.ks, (uint16_t*)dX, lddx,
                           (int64_t)M, K);
        ROV_LAUNCH_CHECK();
    }
    return ROV_OK;
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

extern "C" int rov_linear_xent(const void* X, const void* W, const int64_t* targets, int M, int V, int K, int64_t ldx, int64_t ldw, int dtype,
                               float scale, int64_t ignore_index, float* loss, float* lse, int vocab_piece, void* workspace,
                               size_t workspace_bytes, void* stream) {
    using namespace rov;
    ROV_STEP(check_xent(X, W, targets, M, V, K, ldx, ldw, dtype, scale, ignore_index, vocab_piece));
    if (loss == nullptr || lse == nullptr || !aligned(loss, 4) || !aligned(lse, 4)) return ROV_ERR_INVALID;
    if (workspace == nullptr || !aligned(workspace, kAlign)) return ROV_ERR_INVALID;
    if (dtype == ROV_BF16) {
        ROV_STEP(check_head(M, V, K, ldx, ldw));
        const HeadLayout hl = head_layout(M, V, K, vocab_piece, false);
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
    if (lse == nullptr || dloss == nullptr || (dX == nullptr && dW == nullptr)) return ROV_ERR_INVALID;
    if (!aligned(lse, 4) || !aligned(dloss, 4) || !aligned(dlse, 4)) return ROV_ERR_INVALID;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    if ((dX != nullptr && (lddx < K || !aligned(dX, esz))) || (dW != nullptr && (lddw < K || !aligned(dW, esz)))) return ROV_ERR_INVALID;
    if (workspace == nullptr || !aligned(workspace, kAlign)) return ROV_ERR_INVALID;
    if (dtype == ROV_BF16) {
        ROV_STEP(check_head(M, V, K, ldx, ldw));
        const HeadLayout hl = head_layout(M, V, K, vocab_piece, true);
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
