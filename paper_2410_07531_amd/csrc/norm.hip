// The norms behind one block and before the next (paper Fig. 2's normalisation layers in their RMS form), fused with
// the branch's gate and the residual scale, forward and backward:
//     y  = x_scale * x + h_scale * gate * P(h),   P(h) = h / sqrt(mean h^2 + eps) * w_post   (h itself without w_post)
//     yn = y / sqrt(mean y^2 + eps) * w_pre                                                   (absent without w_pre)
// and, with dy, dn the gradients of y and yn, r = 1/sqrt(mean + eps), t = w_pre dn, hat = y r:
//     g  = dy + r (t - hat mean(hat t));  dx = x_scale g;  q = h_scale gate g
//     dh = r_h (w_post q - h r_h mean(h r_h w_post q));   dw_pre = sum dn hat;  dw_post = sum q h r_h;
//     dgate = sum over the gate's rows of h_scale g P(h).
// What bounds both: memory (4 and 6 passes over rows x n).  A workgroup holds a row in registers, so each tensor
// passes once (backward, rows of more than 1024 pieces are read twice); all sums are fp32 in a fixed order.
// 16384 x 4096 in bf16, both norms: 90 us; 8192 x 8192 backward: 171 us, 4.7 TB/s; 4096 x 16384 backward: 370 us, two vector passes over it.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fp8_device.h"
#include "rov_internal.h"
#include "row_device.h"

namespace rov {
namespace {

constexpr int kMaxRow = 32768;

struct NormParams {
    const void* x;
    const void* h;
    const void* w_post;
    const void* gate;
    const void* w_pre;
    void* y;
    void* yn;
    int64_t ld_x, ld_h, ld_y, ld_yn;
    int rows, n, rows_per_gate;
    float x_scale, h_scale, eps, inv_n, yn_inv;   // yn_inv: 1 / (scale of the e4m3 result)
};

// W consecutive fp32 values, 16 bytes at a time where there are four
template <bool RAGGED, int W>
__device__ __forceinline__ void store_floats(float* row, const float (&v)[W], int e, int n) {
    if constexpr (W == 1) {
        row[e] = v[0];
    } else {
#pragma unroll
        for (int j = 0; j < W; j += 4) {
            Piece<float, 4> out;
            out.raw = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            if (!RAGGED || e + j < n) put_piece<RAGGED>(out, row, e + j, n);
        }
    }
}

template <bool RAGGED, typename T, int W>
__device__ __forceinline__ void load_or(const void* base, int at, int n, float (&f)[W], float otherwise) {
    if (base != nullptr) {
        Piece<T, W> v;
        fetch_piece<RAGGED>(v, (const T*)base, at, n);
        settle<RAGGED>(v, at, n);
        v.get(f);
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j) f[j] = otherwise;
    }
}

// One workgroup of NT threads a row, VPT pieces of W elements a thread.  OUT8: yn is e4m3 bytes.  RAGGED: n % W != 0.
template <typename T, int W, int NT, int VPT, bool OUT8, bool RAGGED>
__global__ __launch_bounds__(NT) void norm_fwd_kernel(const NormParams p) {
    __shared__ float red[2][16];
    __builtin_amdgcn_s_setprio(3);   // beside a co-resident RNG grid: ahead of its long integer multiplies
    const int64_t row = blockIdx.x;
    const T* const x = (const T*)p.x + row * p.ld_x;
    const T* const h = (const T*)p.h + row * p.ld_h;
    const T* const gate = p.gate != nullptr ? (const T*)p.gate + (row / p.rows_per_gate) * p.n : nullptr;
    Piece<T, W> xv[VPT], hv[VPT];
#pragma unroll
    for (int c = 0; c < VPT; ++c) {
        const int e = (c * NT + (int)threadIdx.x) * W;
        xv[c].zero();
        hv[c].zero();
        if (e < p.n) {
            fetch_piece<RAGGED>(hv[c], h, e, p.n);
            fetch_piece<RAGGED>(xv[c], x, e, p.n);
        }
    }
#pragma unroll
    for (int c = 0; c < VPT; ++c) {
        settle<RAGGED>(hv[c], (c * NT + (int)threadIdx.x) * W, p.n);
        settle<RAGGED>(xv[c], (c * NT + (int)threadIdx.x) * W, p.n);
    }
    float inv_h = 1.0f;
    if (p.w_post != nullptr) {
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < VPT; ++c) {
            float f[W];
            hv[c].get(f);
#pragma unroll
            for (int j = 0; j < W; ++j) s = __builtin_fmaf(f[j], f[j], s);
        }
        inv_h = 1.0f / sqrtf(workgroup_sum<NT>(s, red[0]) * p.inv_n + p.eps);
    }
    float y[VPT][W], s = 0.0f;
#pragma unroll
    for (int c = 0; c < VPT; ++c) {
        const int e = (c * NT + (int)threadIdx.x) * W;
        float f[W];
        hv[c].get(f);
        xv[c].get(y[c]);
        if (e < p.n) {
            float wp[W], g[W];
            load_or<RAGGED, T, W>(p.w_post, e, p.n, wp, 1.0f);
            load_or<RAGGED, T, W>(gate, e, p.n, g, 1.0f);
#pragma unroll
            for (int j = 0; j < W; ++j) y[c][j] = p.x_scale * y[c][j] + p.h_scale * g[j] * (f[j] * inv_h * wp[j]);
            Piece<T, W> out;
            out.set(y[c]);
            put_piece<RAGGED>(out, (T*)p.y + row * p.ld_y, e, p.n);
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j) y[c][j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < W; ++j) s = __builtin_fmaf(y[c][j], y[c][j], s);
    }
    if (p.w_pre == nullptr) return;
    const float inv_y = 1.0f / sqrtf(workgroup_sum<NT>(s, red[1]) * p.inv_n + p.eps);
#pragma unroll
    for (int c = 0; c < VPT; ++c) {
        const int e = (c * NT + (int)threadIdx.x) * W;
        if (e >= p.n) continue;
        float w[W];
        load_or<RAGGED, T, W>(p.w_pre, e, p.n, w, 1.0f);
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] *= y[c][j] * inv_y;   // (y not yet rounded: yn is one rounding away from the formula)
        if constexpr (OUT8) {
            uint8_t* const out = (uint8_t*)p.yn + row * p.ld_yn + e;
            if constexpr (W == 1) {
                out[0] = (uint8_t)f32_to_e4m3(w[0] * p.yn_inv);
            } else {
                const uint32_t q[2] = {pack_e4m3x4(w[0] * p.yn_inv, w[1] * p.yn_inv, w[2] * p.yn_inv, w[3] * p.yn_inv),
                                       pack_e4m3x4(w[4] * p.yn_inv, w[5] * p.yn_inv, w[6] * p.yn_inv, w[7] * p.yn_inv)};
                if (!RAGGED || e + W <= p.n) {
                    __builtin_memcpy(out, q, 8);
                } else {
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        if (e + j < p.n) out[j] = (uint8_t)(q[j >> 2] >> (8 * (j & 3)));
                }
            }
        } else {
            Piece<T, W> out;
            out.set(w);
            put_piece<RAGGED>(out, (T*)p.yn + row * p.ld_yn, e, p.n);
        }
    }
}

struct NormBwdParams {
    const void* y;
    const void* h;
    const void* w_post;
    const void* gate;
    const void* w_pre;
    const void* dy;
    const void* dn;
    void* dx;
    void* dh;
    float* dgate;       // written here only where a workgroup holds whole groups
    float* part_h;      // [workgroups][n]: sums of g h r_h (times the gate where a workgroup holds whole groups)
    float* part_y;      // [workgroups][n]: sums of dn y r
    int64_t ld_y, ld_h, ld_dy, ld_dn, ld_dx, ld_dh;
    int rows, n, rows_per_gate;
    int chunks;         // workgroups that share a group (rows of one gate)
    int groups;
    float x_scale, h_scale, eps, inv_n;
};

// A workgroup walks over rows of one group (chunk blockIdx.x % chunks of group blockIdx.x / chunks) or, WHOLE, over
// whole groups (blockIdx.x, blockIdx.x + gridDim.x, ...), and keeps the column sums of its rows in registers.
// Row sums: the sum behind dh's mean is linear in g, so its three parts are summed beside mean(y^2), mean(y t) and
// mean(h^2) and one barrier a row is enough (two sets of scratch by the parity of the row).
// With at most eight elements a thread the next row is on its way while a row is worked on, and the weights stay in registers; with more, the
// column sums fill them, and a row is read a second time, out of the caches, for its results.
template <typename T, int W, int NT, int VPT, bool WHOLE, bool RAGGED>
__global__ __launch_bounds__(NT, VPT * W <= 8 ? 4 : 1) void norm_bwd_kernel(const NormBwdParams p) {
    constexpr bool AHEAD = VPT * W <= 8;
    __shared__ float red[2][6 * 16];
    __builtin_amdgcn_s_setprio(3);
    float col_h[VPT][W], col_y[VPT][W], col_g[WHOLE ? VPT : 1][W];
#pragma unroll
    for (int c = 0; c < VPT; ++c)
#pragma unroll
        for (int j = 0; j < W; ++j) {
            col_h[c][j] = 0.0f;
            col_y[c][j] = 0.0f;
            if constexpr (WHOLE) col_g[c][j] = 0.0f;
        }
    const bool has_pre = p.w_pre != nullptr, has_post = p.w_post != nullptr;
    const bool with_h = p.h != nullptr;
    struct Part { Piece<T, W> y, h, dy, dn; };
    struct Row { Part part[AHEAD ? VPT : 1]; };
    auto fetch_part = [&](Part& r, int64_t row, int c) {
        const int e = (c * NT + (int)threadIdx.x) * W;
        r.y.zero(); r.h.zero(); r.dy.zero(); r.dn.zero();
        if (e < p.n) {
            if (has_pre) {
                fetch_piece<RAGGED>(r.y, (const T*)p.y + row * p.ld_y, e, p.n);
                fetch_piece<RAGGED>(r.dn, (const T*)p.dn + row * p.ld_dn, e, p.n);
            }
            if (with_h) fetch_piece<RAGGED>(r.h, (const T*)p.h + row * p.ld_h, e, p.n);
            if (p.dy != nullptr) fetch_piece<RAGGED>(r.dy, (const T*)p.dy + row * p.ld_dy, e, p.n);
        }
    };
    auto fetch = [&](Row& r, int64_t row) {
#pragma unroll
        for (int c = 0; c < VPT; ++c) fetch_part(r.part[AHEAD ? c : 0], row, c);
    };
    auto settle_part = [&](Part& r, int c) {
        const int e = (c * NT + (int)threadIdx.x) * W;
        settle<RAGGED>(r.y, e, p.n);
        settle<RAGGED>(r.h, e, p.n);
        settle<RAGGED>(r.dy, e, p.n);
        settle<RAGGED>(r.dn, e, p.n);
    };
    Piece<T, W> ones, kept_pre[AHEAD ? VPT : 1], kept_post[AHEAD ? VPT : 1], kept_gate[AHEAD ? VPT : 1];
    {
        float f[W];
#pragma unroll
        for (int j = 0; j < W; ++j) f[j] = 1.0f;
        ones.set(f);
    }
    // a weight or gate of this thread's columns (ones without it)
    auto keep = [&](Piece<T, W>* kept, const T* base) {
#pragma unroll
        for (int c = 0; c < VPT; ++c) {
            const int e = (c * NT + (int)threadIdx.x) * W;
            kept[c] = ones;
            if (base != nullptr && e < p.n) fetch_piece<RAGGED>(kept[c], base, e, p.n);
            settle<RAGGED>(kept[c], e, p.n);
        }
    };
    auto vec = [&](const Piece<T, W>* kept, const void* base, int c) {
        Piece<T, W> v = AHEAD ? kept[c] : ones;
        if (!AHEAD && base != nullptr) {   // (columns that exist)
            fetch_piece<RAGGED>(v, (const T*)base, (c * NT + (int)threadIdx.x) * W, p.n);
            settle<RAGGED>(v, (c * NT + (int)threadIdx.x) * W, p.n);
        }
        return v;
    };
    if constexpr (AHEAD) {
        keep(kept_pre, (const T*)p.w_pre);
        keep(kept_post, (const T*)p.w_post);
    }
    int parity = 0;
    // (64 bits: the step behind the last of 2^31 - 1 groups)
    for (int64_t group = WHOLE ? (int)blockIdx.x : (int)blockIdx.x / p.chunks; group < p.groups; group += WHOLE ? (int)gridDim.x : p.groups) {
        int64_t r0 = group * p.rows_per_gate, r1 = r0 + p.rows_per_gate;
        if constexpr (!WHOLE) {
            const int64_t len = p.rows_per_gate, chunk = (int)blockIdx.x % p.chunks;
            r1 = r0 + len * (chunk + 1) / p.chunks;
            r0 += len * chunk / p.chunks;
        }
        const T* const gate = p.gate != nullptr ? (const T*)p.gate + group * p.n : nullptr;
        if constexpr (AHEAD) keep(kept_gate, gate);
        Row cur, next;
        if (AHEAD && r0 < r1) fetch(next, r0);
        for (int64_t row = r0; row < r1; ++row) {
            if constexpr (AHEAD) {
                cur = next;
                if (row + 1 < r1) fetch(next, row + 1);
                if constexpr (RAGGED) {
#pragma unroll
                    for (int c = 0; c < VPT; ++c) settle_part(cur.part[c], c);
                }
            }
            // the row's elements of piece c, which longer rows read again
            auto take = [&](int c) {
                if constexpr (!AHEAD) {
                    fetch_part(cur.part[0], row, c);
                    if constexpr (RAGGED) settle_part(cur.part[0], c);
                }
                return cur.part[AHEAD ? c : 0];
            };
            float sum[6] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < VPT; ++c) {
                const int e = (c * NT + (int)threadIdx.x) * W;
                if (e >= p.n) continue;
                const Piece<T, W> w = vec(kept_pre, p.w_pre, c), wp = vec(kept_post, p.w_post, c), g = vec(kept_gate, gate, c);
                const Part now = take(c);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float y = now.y.at(j), h = now.h.at(j), t = now.dn.at(j) * w.at(j), u = h * wp.at(j) * g.at(j);
                    sum[0] = __builtin_fmaf(y, y, sum[0]);
                    sum[1] = __builtin_fmaf(y, t, sum[1]);
                    sum[2] = __builtin_fmaf(h, h, sum[2]);
                    sum[3] = __builtin_fmaf(u, now.dy.at(j), sum[3]);
                    sum[4] = __builtin_fmaf(u, t, sum[4]);
                    sum[5] = __builtin_fmaf(u, y, sum[5]);
                    __builtin_amdgcn_sched_barrier(0);   // one element at a time: unpacked ahead they would spill
                }
            }
            workgroup_sums<NT, 6>(sum, red[parity]);
            parity ^= 1;
            const float r = has_pre ? 1.0f / sqrtf(sum[0] * p.inv_n + p.eps) : 0.0f;
            const float rh = has_post ? 1.0f / sqrtf(sum[2] * p.inv_n + p.eps) : 1.0f;
            // means of hat t and of (h r_h) w_post q.  Each factor r goes to an element or a sum of its row, never r * r alone, so that everything
            // between is of the size of results (the cube of r leaves fp32 for rows beyond 1e13, or 1e-13 with a tiny eps)
            const float my = has_pre ? r * sum[1] * p.inv_n : 0.0f;
            const float mh = has_post ? rh * (sum[3] + r * sum[4] - r * sum[5] * (r * my)) * p.inv_n * p.h_scale : 0.0f;
#pragma unroll
            for (int c = 0; c < VPT; ++c) {
                const int e = (c * NT + (int)threadIdx.x) * W;
                if (e >= p.n) continue;
                const Piece<T, W> w = vec(kept_pre, p.w_pre, c), wp = vec(kept_post, p.w_post, c), g = vec(kept_gate, gate, c);
                const Part now = take(c);
                float dx[W], dh[W];
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float y = now.y.at(j), h = now.h.at(j), dn = now.dn.at(j);
                    const float hat = y * r, hat_h = h * rh;
                    const float gy = now.dy.at(j) + r * (w.at(j) * dn - hat * my);
                    col_y[c][j] = __builtin_fmaf(dn, hat, col_y[c][j]);
                    col_h[c][j] = __builtin_fmaf(gy, hat_h, col_h[c][j]);
                    dx[j] = p.x_scale * gy;
                    // (without w_post h may be infinite: times mh = 0 it would be NaN)
                    dh[j] = rh * (wp.at(j) * (p.h_scale * g.at(j) * gy) - (has_post ? hat_h * mh : 0.0f));
                    __builtin_amdgcn_sched_barrier(0);
                }
                Piece<T, W> out;
                if (p.dx != nullptr) {
                    out.set(dx);
                    put_piece<RAGGED>(out, (T*)p.dx + row * p.ld_dx, e, p.n);
                }
                if (p.dh != nullptr) {
                    out.set(dh);
                    put_piece<RAGGED>(out, (T*)p.dh + row * p.ld_dh, e, p.n);
                }
            }
        }
        if constexpr (WHOLE) {
#pragma unroll
            for (int c = 0; c < VPT; ++c) {
                const int e = (c * NT + (int)threadIdx.x) * W;
                if (e >= p.n) continue;
                float wp[W], g[W];
                load_or<RAGGED, T, W>(p.w_post, e, p.n, wp, 1.0f);
                load_or<RAGGED, T, W>(gate, e, p.n, g, 1.0f);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    if (p.dgate != nullptr && (!RAGGED || e + j < p.n)) p.dgate[group * p.n + e + j] = p.h_scale * wp[j] * col_h[c][j];
                    col_g[c][j] = __builtin_fmaf(g[j], col_h[c][j], col_g[c][j]);
                    col_h[c][j] = 0.0f;
                }
            }
        }
    }
#pragma unroll
    for (int c = 0; c < VPT; ++c) {
        const int e = (c * NT + (int)threadIdx.x) * W;
        if (e >= p.n) continue;
        if (p.part_h != nullptr) {
            if constexpr (WHOLE) store_floats<RAGGED, W>(p.part_h + (int64_t)blockIdx.x * p.n, col_g[c], e, p.n);
            else store_floats<RAGGED, W>(p.part_h + (int64_t)blockIdx.x * p.n, col_h[c], e, p.n);
        }
        if (p.part_y != nullptr) store_floats<RAGGED, W>(p.part_y + (int64_t)blockIdx.x * p.n, col_y[c], e, p.n);
    }
}

struct NormSumParams {
    const float* part_h;
    const float* part_y;
    const void* w_post;
    const void* gate;
    float* dw_post;
    float* dgate;
    float* dw_pre;
    int n, parts, groups, chunks;   // parts = groups * chunks rows of partial sums; whole: parts rows, groups = 1
    float h_scale;
    int whole;
};

// Column sums of the workgroups' partial sums: 16 columns a workgroup, 64 threads a column.  BY_GROUP (many gates): a thread adds up whole
// groups; else a column's threads share the rows of each group.
template <typename T, bool BY_GROUP>
__global__ __launch_bounds__(1024) void norm_sum_kernel(const NormSumParams p) {
    __shared__ float red[2][16][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * 16 + (lane & 15), slice = wave * 4 + (lane >> 4);
    const bool in = col < p.n;
    int parity = 0;
    auto strided = [&](const float* part, int64_t first, int count, int from, int step) {
        float s = 0.0f;
        if (in)
#pragma unroll 8
            for (int i = from; i < count; i += step) s += part[(first + i) * p.n + col];
        return s;
    };
    // every thread's s, summed over a column's 64 threads
    auto over_column = [&](float s) {
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (lane < 16) red[parity][wave][lane] = s;
        __syncthreads();
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += red[parity][i][lane & 15];
        parity ^= 1;   // (the next sum's scratch: this one may still be read)
        return s;
    };
    auto gate_of = [&](int64_t g) {
        float f[1];
        load_or<false, T, 1>(p.gate != nullptr ? (const T*)p.gate + g * p.n : nullptr, col, p.n, f, 1.0f);
        return f[0];
    };
    const bool writes = slice == 0 && in;
    if (p.dw_pre != nullptr) {
        const float s = over_column(strided(p.part_y, 0, p.parts, slice, 64));
        if (writes) p.dw_pre[col] = s;
    }
    if (p.part_h == nullptr) return;
    float wp[1] = {1.0f}, total = 0.0f;
    if (in) load_or<false, T, 1>(p.w_post, col, p.n, wp, 1.0f);
    if constexpr (BY_GROUP) {
        if (in)
            for (int g = slice; g < p.groups; g += 64) {
                const float s = strided(p.part_h, (int64_t)g * p.chunks, p.chunks, 0, 1);
                if (p.dgate != nullptr) p.dgate[(int64_t)g * p.n + col] = p.h_scale * wp[0] * s;
                total = __builtin_fmaf(gate_of(g), s, total);
            }
        if (p.dw_post == nullptr) return;
        total = over_column(total);
    } else {
        for (int g = 0; g < p.groups; ++g) {
            const float s = over_column(strided(p.part_h, (int64_t)g * p.chunks, p.chunks, slice, 64));
            if (!writes) continue;
            if (p.dgate != nullptr) p.dgate[(int64_t)g * p.n + col] = p.h_scale * wp[0] * s;
            total = __builtin_fmaf(p.whole ? 1.0f : gate_of(g), s, total);
        }
    }
    if (writes && p.dw_post != nullptr) p.dw_post[col] = p.h_scale * total;
}

// Threads of a workgroup and pieces of w elements a thread for rows of n elements.  A piece is 16 bytes.  Up to 1024 elements that are no whole
// pieces move one by one, up to four a thread: the last piece's extra work would not hide (20000 x 127 in bf16, forward / backward: 9.6 / 31 us
// by elements, 14.2 / 51 by pieces; 8192 x 4099: 273 / 940 and 77 / 133).
struct RowShape { int w, nt, vpt; bool ragged; };
RowShape row_shape(int n, int dtype) {
    const int w = dtype == ROV_F32 ? 4 : 8, pieces = (n + w - 1) / w;
    if (n % w != 0 && n <= 1024) return {1, n <= 256 ? 64 : n <= 512 ? 128 : 256, n <= 64 ? 1 : 4, false};
    if (pieces > 1024) return {w, 1024, pieces <= 4096 ? 4 : 8, n % w != 0};
    int nt = 64;
    while (nt < pieces) nt *= 2;
    return {w, nt, 1, n % w != 0};
}

// F(W, NT, VPT, RAGGED) for the shape s of rows of type T
#define ROV_BY_SHAPE(F)                                             \
    do {                                                            \
        constexpr int PW = 16 / sizeof(T);                          \
        if (s.w == 1) {                                             \
            if (s.vpt == 1) F(1, 64, 1, false);                     \
            else if (s.nt == 64) F(1, 64, 4, false);                \
            else if (s.nt == 128) F(1, 128, 4, false);              \
            else F(1, 256, 4, false);                               \
        } else if (s.ragged) {                                      \
            if (s.nt == 256) F(PW, 256, 1, true);                   \
            else if (s.nt == 512) F(PW, 512, 1, true);              \
            else if (s.vpt == 1) F(PW, 1024, 1, true);              \
            else if (PW == 8 || s.vpt == 4) F(PW, 1024, 4, true);   \
            else if constexpr (PW == 4) F(PW, 1024, 8, true);       \
        } else if (s.nt == 64) F(PW, 64, 1, false);                 \
        else if (s.nt == 128) F(PW, 128, 1, false);                 \
        else if (s.nt == 256) F(PW, 256, 1, false);                 \
        else if (s.nt == 512) F(PW, 512, 1, false);                 \
        else if (s.vpt == 1) F(PW, 1024, 1, false);                 \
        else if (PW == 8 || s.vpt == 4) F(PW, 1024, 4, false);      \
        else if constexpr (PW == 4) F(PW, 1024, 8, false);          \
    } while (0)

template <typename T, bool OUT8>
void launch_fwd(const NormParams& p, const RowShape s, hipStream_t stream) {
    const dim3 grid((unsigned)p.rows);
#define ROV_FWD(W, NT, VPT, RAGGED) hipLaunchKernelGGL((norm_fwd_kernel<T, W, NT, VPT, OUT8, RAGGED>), grid, dim3(NT), 0, stream, p)
    ROV_BY_SHAPE(ROV_FWD);
#undef ROV_FWD
}

template <typename T, bool WHOLE>
void launch_bwd(const NormBwdParams& p, const RowShape s, int blocks, hipStream_t stream) {
    const dim3 grid((unsigned)blocks);
#define ROV_BWD(W, NT, VPT, RAGGED) hipLaunchKernelGGL((norm_bwd_kernel<T, W, NT, VPT, WHOLE, RAGGED>), grid, dim3(NT), 0, stream, p)
    ROV_BY_SHAPE(ROV_BWD);
#undef ROV_BWD
}
#undef ROV_BY_SHAPE

// How the rows are shared: `blocks` workgroups, `chunks` of them a group of rows with one gate, or (whole) every
// workgroup takes whole groups.
struct RowSplit { int blocks, chunks; bool whole; };
RowSplit split_rows(int64_t rows, int64_t rows_per_gate, int n, int dtype) {
    const int64_t groups = rows / rows_per_gate, ncu = device_cu_count();
    // a workgroup a compute unit where each gets two rows (few rows wait for their loads: 1003 x 1001 in fp32 with 250 workgroups 15 us); more only
    // with eight rows each, so that the partial sums stay a fraction of the rows' bytes
    const int64_t most = ncu * (1024 / row_shape(n, dtype).nt);
    int64_t want = rows / 8 < ncu ? (rows / 2 < ncu ? rows / 2 : ncu) : rows / 8;
    if (want > most) want = most;
    if (want < 1) want = 1;
    if (groups > want) return {(int)want, 1, true};
    int64_t chunks = want / groups;
    if (chunks > rows_per_gate) chunks = rows_per_gate;
    return {(int)(groups * chunks), (int)chunks, false};
}

int check_norm_sizes(int64_t rows, int n, int64_t rows_per_gate, int dtype, float x_scale, float h_scale, float eps) {
    if (rows <= 0 || n <= 0 || rows_per_gate <= 0 || rows % rows_per_gate != 0) return ROV_ERR_INVALID;
    if (!(eps > 0.0f) || !isfinite(eps) || !isfinite(x_scale) || !isfinite(h_scale)) return ROV_ERR_INVALID;
    if (dtype != ROV_F32 && dtype != ROV_BF16) return dtype == ROV_FP8_E4M3 ? ROV_ERR_UNSUPPORTED : ROV_ERR_INVALID;
    if (n > kMaxRow || rows > 0x7FFFFFFF) return ROV_ERR_UNSUPPORTED;
    return ROV_OK;
}

}  // namespace

int check_norm_residual(const void* x, const void* h, const void* w_post, const void* gate, const void* w_pre, const void* y,
                        const void* yn, int64_t rows, int n, const int64_t ld[4], int64_t rows_per_gate, int dtype, float x_scale,
                        float h_scale, float eps, float yn_fp8_scale) {
    if (x == nullptr || h == nullptr || y == nullptr || ld == nullptr || (w_pre == nullptr) != (yn == nullptr)) return ROV_ERR_INVALID;
    const int rc = check_norm_sizes(rows, n, rows_per_gate, dtype, x_scale, h_scale, eps);
    if (rc != ROV_OK) return rc;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    const bool out8 = yn_fp8_scale != 0.0f;
    if (out8 && !(yn_fp8_scale > 0.0f && isfinite(yn_fp8_scale))) return ROV_ERR_INVALID;
    if (out8 && dtype != ROV_BF16) return ROV_ERR_UNSUPPORTED;
    const void* const all[] = {x, h, w_post, gate, w_pre, y, out8 ? nullptr : yn};
    for (const void* q : all)
        if (!aligned(q, esz)) return ROV_ERR_INVALID;
    for (int i = 0; i < (w_pre != nullptr ? 4 : 3); ++i)
        if (ld[i] < n && rows > 1) return ROV_ERR_INVALID;
    // in place is element by element: the same stride and type, and one result a buffer
    if (y == yn || (out8 && (yn == x || yn == h))) return ROV_ERR_INVALID;
    const void* const ins[2] = {x, h};
    const void* const outs[2] = {y, yn};
    for (int i = 0; i < 2; ++i)
        for (int o = 0; o < 2; ++o)
            if (outs[o] == ins[i] && ld[2 + o] != ld[i] && rows > 1) return ROV_ERR_INVALID;
    return grid_fits(rows, row_shape(n, dtype).nt) ? ROV_OK : ROV_ERR_UNSUPPORTED;   // (a workgroup a row)
}

int launch_norm_residual(const void* x, const void* h, const void* w_post, const void* gate, const void* w_pre, void* y, void* yn,
                         int64_t rows, int n, const int64_t ld[4], int64_t rows_per_gate, int dtype, float x_scale, float h_scale,
                         float eps, float yn_fp8_scale, hipStream_t stream) {
    {
        const int rc = check_norm_residual(x, h, w_post, gate, w_pre, y, yn, rows, n, ld, rows_per_gate, dtype, x_scale, h_scale, eps,
                                           yn_fp8_scale);
        if (rc != ROV_OK) return rc;
    }
    const bool out8 = yn_fp8_scale != 0.0f;
    NormParams p{x, h, w_post, gate, w_pre, y, yn, ld[0], ld[1], ld[2], ld[3], (int)rows, n, (int)rows_per_gate,
                 x_scale, h_scale, eps, 1.0f / (float)n, out8 ? 1.0f / yn_fp8_scale : 1.0f};
    const RowShape shape = row_shape(n, dtype);
    if (dtype == ROV_F32) launch_fwd<float, false>(p, shape, stream);
    else if (out8) launch_fwd<uint16_t, true>(p, shape, stream);
    else launch_fwd<uint16_t, false>(p, shape, stream);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}

}  // namespace rov

extern "C" int rov_norm_residual(const void* x, const void* h, const void* w_post, const void* gate, const void* w_pre, void* y,
                                 void* yn, int64_t rows, int n, const int64_t ld[4], int64_t rows_per_gate, int dtype, float x_scale,
                                 float h_scale, float eps, float yn_fp8_scale, void* stream) {
    return rov::launch_norm_residual(x, h, w_post, gate, w_pre, y, yn, rows, n, ld, rows_per_gate, dtype, x_scale, h_scale, eps,
                                     yn_fp8_scale, (hipStream_t)stream);
}

extern "C" size_t rov_norm_residual_bwd_workspace_bytes(int64_t rows, int n, int64_t rows_per_gate, int dtype) {
    if (rov::check_norm_sizes(rows, n, rows_per_gate, dtype, 1.0f, 1.0f, 1.0f) != ROV_OK) return 0;
    return 2 * sizeof(float) * (size_t)n * (size_t)rov::split_rows(rows, rows_per_gate, n, dtype).blocks;
}

extern "C" int rov_norm_residual_bwd(const void* y, const void* h, const void* w_post, const void* gate, const void* w_pre,
                                     const void* dy, const void* dn, void* dx, void* dh, float* dw_post, float* dgate, float* dw_pre,
                                     int64_t rows, int n, const int64_t ld[6], int64_t rows_per_gate, int dtype, float x_scale,
                                     float h_scale, float eps, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace rov;
    int rc = check_norm_sizes(rows, n, rows_per_gate, dtype, x_scale, h_scale, eps);
    if (rc != ROV_OK && rc != ROV_ERR_UNSUPPORTED) return rc;
    const bool pre = w_pre != nullptr, sums_h = dw_post != nullptr || dgate != nullptr;
    if (ld == nullptr || (dx == nullptr && dh == nullptr && !sums_h && dw_pre == nullptr)) return ROV_ERR_INVALID;
    if (pre != (dn != nullptr) || (pre && y == nullptr) || (!pre && dy == nullptr)) return ROV_ERR_INVALID;
    if ((dw_pre != nullptr && !pre) || (dw_post != nullptr && w_post == nullptr) || (dgate != nullptr && gate == nullptr))
        return ROV_ERR_INVALID;
    if ((w_post != nullptr || dgate != nullptr) && h == nullptr) return ROV_ERR_INVALID;
    const size_t esz = dtype == ROV_F32 ? 4 : 2;
    const void* const vectors[] = {w_post, gate, w_pre};
    const void* const tensors[6] = {pre ? y : nullptr, h, dy, dn, dx, dh};
    for (const void* q : vectors)
        if (!aligned(q, esz)) return ROV_ERR_INVALID;
    for (int i = 0; i < 6; ++i) {
        if (!aligned(tensors[i], esz)) return ROV_ERR_INVALID;
        if (tensors[i] != nullptr && rows > 1 && ld[i] < n) return ROV_ERR_INVALID;
    }
    if (!aligned(dw_post, 4) || !aligned(dgate, 4) || !aligned(dw_pre, 4)) return ROV_ERR_INVALID;
    if (dx != nullptr && dx == dh) return ROV_ERR_INVALID;
    for (int o = 4; o < 6; ++o)   // in place: the same stride
        for (int i = 0; i < 4; ++i)
            if (tensors[o] != nullptr && tensors[o] == tensors[i] && ld[o] != ld[i] && rows > 1) return ROV_ERR_INVALID;
    if (rc != ROV_OK) return rc;
    const RowSplit sp = split_rows(rows, rows_per_gate, n, dtype);
    const bool sums = sums_h || dw_pre != nullptr;
    if (sums) {
        if (workspace == nullptr || !aligned(workspace, 16)) return ROV_ERR_INVALID;
        if (workspace_bytes < rov_norm_residual_bwd_workspace_bytes(rows, n, rows_per_gate, dtype)) return ROV_ERR_WORKSPACE;
    }
    float* const part = (float*)workspace;
    NormBwdParams p{y, h, w_post, gate, w_pre, dy, dn, dx, dh, sp.whole ? dgate : nullptr,
                    sums_h ? part : nullptr, dw_pre != nullptr ? part + (size_t)sp.blocks * n : nullptr,
                    ld[0], ld[1], ld[2], ld[3], ld[4], ld[5], (int)rows, n, (int)rows_per_gate, sp.chunks,
                    (int)(rows / rows_per_gate), x_scale, h_scale, eps, 1.0f / (float)n};
    hipStream_t st = (hipStream_t)stream;
    const RowShape shape = row_shape(n, dtype);
    if (dtype == ROV_F32) sp.whole ? launch_bwd<float, true>(p, shape, sp.blocks, st) : launch_bwd<float, false>(p, shape, sp.blocks, st);
    else sp.whole ? launch_bwd<uint16_t, true>(p, shape, sp.blocks, st) : launch_bwd<uint16_t, false>(p, shape, sp.blocks, st);
    ROV_LAUNCH_CHECK();
    if (!sums) return ROV_OK;
    NormSumParams s{p.part_h, p.part_y, w_post, gate, dw_post, sp.whole ? nullptr : dgate, dw_pre, n, sp.blocks,
                    sp.whole ? 1 : p.groups, sp.whole ? sp.blocks : sp.chunks, h_scale, sp.whole ? 1 : 0};
    const dim3 grid((unsigned)((n + 15) / 16)), block(1024);
    if (s.groups >= 16) {
        if (dtype == ROV_F32) hipLaunchKernelGGL((norm_sum_kernel<float, true>), grid, block, 0, st, s);
        else hipLaunchKernelGGL((norm_sum_kernel<uint16_t, true>), grid, block, 0, st, s);
    } else {
        if (dtype == ROV_F32) hipLaunchKernelGGL((norm_sum_kernel<float, false>), grid, block, 0, st, s);
        else hipLaunchKernelGGL((norm_sum_kernel<uint16_t, false>), grid, block, 0, st, s);
    }
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}
