// Softmax cross entropy of logits z = scale * X W^T over a large vocabulary, and its gradients, without keeping z:
//     lse_m = log sum_v exp z_mv,   loss_m = lse_m - z_m,target(m)
//     G_mv = scale * (exp(z_mv - lse_m) * (dloss_m + dlse_m) - [v == target(m)] * dloss_m),   dX = G W,   dW = G^T X.
// The vocabulary is walked in pieces: a piece's logits live in the workspace for as long as its statistics, or its
// gradients, are taken (2 and 6 operations per element of M x V x K; the backward pass makes the logits again).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rov_internal.h"
#include "row_device.h"

namespace rov {
namespace {

struct RowState { float top, sum, picked, pad; };   // running maximum, sum of exp(z - top), logit of the target

// A row counts if its target is not the ignored index; a target outside the vocabulary counts and shows as NaN.
__device__ __forceinline__ bool in_vocab(int64_t t, int V) { return t >= 0 && t < V; }

// dst [rows][cols] fp32 = src, rows of ignored targets zero (mask).
template <typename T>
__global__ __launch_bounds__(256) void xent_widen_kernel(const T* __restrict__ src, int64_t ld, float* __restrict__ dst, int64_t rows,
                                                         int cols, const int64_t* __restrict__ targets, int64_t ignore) {
    const int64_t total = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / cols;
        const int c = (int)(i - r * cols);
        Piece<T, 1> v;
        v.load(src + r * ld + c);
        float f[1];
        v.get(f);
        dst[i] = targets != nullptr && targets[r] == ignore ? 0.0f : f[0];
    }
}

// dst [rows][cols] = src fp32.
template <typename T>
__global__ __launch_bounds__(256) void xent_narrow_kernel(const float* __restrict__ src, T* __restrict__ dst, int64_t ld, int64_t rows, int cols) {
    const int64_t total = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / cols;
        const float f[1] = {src[i]};
        Piece<T, 1> v;
        v.set(f);
        v.store(dst + r * ld + (i - r * cols));
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
    __shared__ float red[8];
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

constexpr size_t kAlign = 256;
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

unsigned sweep_grid(int64_t total) {
    const int64_t g = (total + 255) / 256, most = (int64_t)device_cu_count() * 32;
    return (unsigned)(g < most ? g : most);
}

int check_xent(const void* X, const void* W, const int64_t* targets, int M, int V, int K, int64_t ldx, int64_t ldw, int dtype, float scale,
               int64_t ignore, int vocab_piece) {
    if (X == nullptr || W == nullptr || targets == nullptr || M <= 0 || V <= 0 || K <= 0 || ldx < K || ldw < K || vocab_piece < 0)
        return ROV_ERR_INVALID;
    if (!isfinite(scale) || (ignore >= 0 && ignore < V)) return ROV_ERR_INVALID;
    if (dtype != ROV_F32 && dtype != ROV_BF16) return dtype == ROV_FP8_E4M3 ? ROV_ERR_UNSUPPORTED : ROV_ERR_INVALID;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    if (!aligned(X, esz) || !aligned(W, esz) || !aligned(targets, 8)) return ROV_ERR_INVALID;
    return ROV_OK;
}

int widen(const void* src, int64_t ld, float* dst, int64_t rows, int cols, int dtype, const int64_t* targets, int64_t ignore, hipStream_t st) {
    if (dtype == ROV_F32)
        hipLaunchKernelGGL((xent_widen_kernel<float>), dim3(sweep_grid(rows * cols)), dim3(256), 0, st, (const float*)src, ld, dst, rows, cols, targets, ignore);
    else
        hipLaunchKernelGGL((xent_widen_kernel<uint16_t>), dim3(sweep_grid(rows * cols)), dim3(256), 0, st, (const uint16_t*)src, ld, dst, rows, cols, targets, ignore);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
int narrow(const float* src, void* dst, int64_t ld, int64_t rows, int cols, int dtype, hipStream_t st) {
    if (dtype == ROV_F32)
        hipLaunchKernelGGL((xent_narrow_kernel<float>), dim3(sweep_grid(rows * cols)), dim3(256), 0, st, src, (float*)dst, ld, rows, cols);
    else
        hipLaunchKernelGGL((xent_narrow_kernel<uint16_t>), dim3(sweep_grid(rows * cols)), dim3(256), 0, st, src, (uint16_t*)dst, ld, rows, cols);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}

#define ROV_STEP(expr)               \
    do {                             \
        const int rc_ = (expr);      \
        if (rc_ != ROV_OK) return rc_; \
    } while (0)

}  // namespace
}  // namespace rov

extern "C" size_t rov_linear_xent_workspace_bytes(int M, int V, int K, int dtype, int backward, int vocab_piece) {
    if (M <= 0 || V <= 0 || K <= 0 || vocab_piece < 0 || (dtype != ROV_F32 && dtype != ROV_BF16)) return 0;
    return rov::layout(M, V, K, vocab_piece, backward != 0).total;
}

extern "C" int rov_linear_xent(const void* X, const void* W, const int64_t* targets, int M, int V, int K, int64_t ldx, int64_t ldw, int dtype,
                               float scale, int64_t ignore_index, float* loss, float* lse, int vocab_piece, void* workspace,
                               size_t workspace_bytes, void* stream) {
    using namespace rov;
    ROV_STEP(check_xent(X, W, targets, M, V, K, ldx, ldw, dtype, scale, ignore_index, vocab_piece));
    if (loss == nullptr || lse == nullptr || !aligned(loss, 4) || !aligned(lse, 4)) return ROV_ERR_INVALID;
    if (workspace == nullptr || !aligned(workspace, kAlign)) return ROV_ERR_INVALID;
    const XentLayout l = layout(M, V, K, vocab_piece, false);
    if (workspace_bytes < l.total) return ROV_ERR_WORKSPACE;
    char* const ws = (char*)workspace;
    float *x = (float*)(ws + l.x), *w = (float*)(ws + l.w), *z = (float*)(ws + l.z);
    hipStream_t st = (hipStream_t)stream;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    ROV_STEP(check_gemm(x, w, z, nullptr, EPI_ADD, M, l.piece, K, ROV_F32, 1));
    ROV_STEP(widen(X, ldx, x, M, K, dtype, nullptr, 0, st));
    for (int v0 = 0; v0 < V; v0 += l.piece) {
        const int cols = V - v0 < l.piece ? V - v0 : l.piece;
        ROV_STEP(widen((const char*)W + (size_t)v0 * ldw * esz, ldw, w, cols, K, dtype, nullptr, 0, st));
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
    const XentLayout l = layout(M, V, K, vocab_piece, true);
    if (workspace_bytes < l.total) return ROV_ERR_WORKSPACE;
    char* const ws = (char*)workspace;
    float *x = (float*)(ws + l.x), *w = (float*)(ws + l.w), *z = (float*)(ws + l.z), *gt = (float*)(ws + l.gt);
    float *part = (float*)(ws + l.part), *sum = (float*)(ws + l.sum);
    hipStream_t st = (hipStream_t)stream;
    ROV_STEP(check_gemm(x, w, z, nullptr, EPI_ADD, M, l.piece, K, ROV_F32, 1));
    ROV_STEP(check_gemm(z, w, part, nullptr, EPI_ADD, M, K, l.piece, ROV_F32, 0));
    ROV_STEP(check_gemm(gt, x, part, nullptr, EPI_ADD, l.piece, K, M, ROV_F32, 0));
    ROV_STEP(widen(X, ldx, x, M, K, dtype, targets, ignore_index, st));
    for (int v0 = 0; v0 < V; v0 += l.piece) {
        const int cols = V - v0 < l.piece ? V - v0 : l.piece;
        ROV_STEP(widen((const char*)W + (size_t)v0 * ldw * esz, ldw, w, cols, K, dtype, nullptr, 0, st));
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
            ROV_STEP(launch_gemm(gt, x, part, cols, K, M, ROV_F32, 0, 1.0f, 1.0f, st));
            ROV_STEP(narrow(part, (char*)dW + (size_t)v0 * lddw * esz, lddw, cols, K, dtype, st));
        }
    }
    return dX != nullptr ? narrow(sum, dX, lddx, M, K, dtype, st) : ROV_OK;
}
