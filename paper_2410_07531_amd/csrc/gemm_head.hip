// The products of the loss over the vocabulary (xent.hip): logits that stay in the accumulators of a matrix-core tile, and the
// two products of their gradients.  bf16 operands, fp32 accumulation, rows of any stride.
//
// The main loop is that of the bf16 256-row kernel of gemm.hip (256 x 256 or 256 x 128 tile, four waves in a 2 x 2 grid, MFMA 16x16x32, two
// 64 KiB LDS slots of 128-byte rows filled by loads that write LDS, fragments read a k-step ahead; its comments say why), with three
// differences:
//   - the epilogue: HEAD_STATS keeps the row statistics of the tile's logits, HEAD_GRAD turns them into gradients, HEAD_DX and HEAD_DW
//     store the product, or fp32 sums of it over shares of k;
//   - HEAD_DX: the second operand lies as [K, N] (rows of k), HEAD_DW: both do.  Such an operand's part of a slot is 64 rows of k by the
//     tile's columns; fragments come by the transposing LDS load, two a fragment, with the k order of the other operand's.
//   - a workgroup takes one tile after the other, and the loads of a tile's last two slots' time are the next tile's first: its loop goes on
//     behind the epilogue as if there were one longer k.  A tile a workgroup / this, in turn on one box, us: loss with gradients 1000 x 50257 x 1024
//     500 / 488, 8192 x 50257 x 1024 3017 / 2990, 4096 x 50304 x 256 775 / 727, 8192 x 131072 x 4096 24990 / 24800; loss alone 2048 x 131072 x 4096
//     1549 / 1523.  What the epilogue reads is asked for before the loop, and no wait stands before its stores: loads sent out between loop and epilogue gained nothing.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "rov_internal.h"

namespace rov {
namespace {

constexpr int BM = 256, BN = 256;                   // tile height; width of the widest tile
constexpr int kRowBytes = 128;                      // k per LDS row: 64 values
constexpr int kLdsBytes = 2 * (BM + BN) * kRowBytes;   // two slots of A rows then W rows: 128 KiB

typedef __attribute__((address_space(3))) void* lptr_t;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4* lds_i16x4_ptr;

// Reads one accumulator value where it is needed: the "a" constraint keeps it in its accumulation register until then.
__device__ __forceinline__ float acc_read(float v) {
    float r;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(r) : "a"(v));
    return r;
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    f32x2 v = {lo, hi};
    bf16x2 h = __builtin_convertvector(v, bf16x2);
    return *reinterpret_cast<uint32_t*>(&h);
}

// A lane's value and that of the lane 16 (32) away, in an order that both lanes share: two vector moves, where a shuffle would go
// through the LDS unit and be waited for.
template <int D>
__device__ __forceinline__ f32x2 exchanged(float v) {
    const uint32_t u = __float_as_uint(v);
    if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
    }
}

// NJ: weight blocks of 16 rows a wave, 8 or 4 (tiles of 256 or 128 columns).  RAGGED (both operands with k contiguous): rows of any
// multiple of 16 bytes; the last slot's lanes beyond k are aimed outside the operands and read zeros.  gridDim.y: shares of k (HEAD_DX, HEAD_DW).
template <int NJ, bool RAGGED, int HEAD>
__global__ __launch_bounds__(256, 1) void gemm_head_kernel(const char* __restrict__ A, const char* __restrict__ Wt, uint16_t* __restrict__ C,
                                                          const int M, const int N, const int K, const float alpha, const int tiles_m,
                                                          const int tiles_n, const HeadArgs head) {
    static_assert(NJ == 8 || NJ == 4, "256 or 128 columns");
    constexpr bool KNW = HEAD == HEAD_DX || HEAD == HEAD_DW, KNA = HEAD == HEAD_DW;
    static_assert(!RAGGED || !KNW, "k along the rows");
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    // beside a co-resident RNG grid: its waves get the issue slots these leave
    __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    constexpr int BNT = 32 * NJ, ESZ = 2, kRow = kRowBytes;
    constexpr int kSlot = (BM + BN) * kRow;      // slot stride (the widest tile's); W rows follow the A rows

    // 16-byte chunk swizzles of LDS rows: of rows of k (see gemm.hip), and of rows of columns, where the lanes that the transposing load serves
    // together read rows {0-3, 8-11} (+4, +16) x 32 bytes, so that the 32-byte groups of those rows have to differ
    auto swz = [](int row) { return (row >> 1) & 7; };
    auto swz_kn = [](int row) { return ((row & 3) | (((row >> 3) & 1) << 2)) << 1; };
    // fragment of MFMA 16x16x32: lane holds row lane%16, k-chunk (8 bf16) lane/16 of k-step h
    const int frow = lane & 15, fchunk = lane >> 4;
    int foff[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) foff[h] = frow * kRow + (((4 * h + fchunk) ^ swz(frow)) << 4);   // block bases are multiples of 16
    const int a_base = (wm * 128) * kRow;
    const int w_base = BM * kRow + (wn * 16 * NJ) * kRow;

    // this workgroup's share of k
    const size_t ld_a = head.ld_a, ld_w = head.ld_w, row_bytes = (size_t)K * ESZ;
    int ns = (int)((row_bytes + (RAGGED || KNW ? kRow - 1 : 0)) / kRow);   // slots to walk
    int k_rows = 0;             // rows of k from the share on
    if constexpr (KNW) {
        const int s0 = (int)((int64_t)ns * blockIdx.y / gridDim.y), s1 = (int)((int64_t)ns * (blockIdx.y + 1) / gridDim.y);
        ns = s1 - s0;
        k_rows = K - s0 * 64;
        A += KNA ? (size_t)s0 * 64 * ld_a : (size_t)s0 * kRow;
        Wt += (size_t)s0 * 64 * ld_w;
    }
    // bytes of k that a row holds from the base on (the last row's end bounds the operand)
    const size_t k_bytes = KNW ? (size_t)ns * kRow : row_bytes;
    // RAGGED: does the lane's chunk (the same in every load: row / 2 % 8 does not depend on j) lie beyond k in the last slot?
    const bool beyond_k = RAGGED && ((lane & 7) ^ swz(wave * 8 + (lane >> 3))) * 16 >= (int)(row_bytes - (size_t)(ns - 1) * kRow);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(lptr_t)lds;

    // The tile that the loads are aimed at: lanes' byte offsets of load j of each operand, buffer resources, start of the walk over k
    uint32_t voff_a[8], voff_w[NJ];
    i32x4 rsrc_a, rsrc_w;
    int kstart = 0, aim_m0 = 0, aim_n0 = 0, aim_tn = 0;
    const int T = tiles_m * tiles_n;
    auto aim = [&](int pid) __attribute__((always_inline)) {
        // XCD-aware tile id: workgroup ids are dealt round-robin to the 8 XCDs; give each XCD a contiguous
        // range of logical tiles, ordered in bands of 8 tile-rows with the row fastest
        const int per = T >> 3, rem = T & 7, xcd = pid & 7, loc = pid >> 3;
        const int id = xcd < rem ? xcd * (per + 1) + loc : rem * (per + 1) + (xcd - rem) * per + loc;
        constexpr int GM = 8;
        const int band = id / (GM * tiles_n);
        const int band_rows = (tiles_m - band * GM) < GM ? (tiles_m - band * GM) : GM;
        const int in_band = id - band * GM * tiles_n;
        const int tm = band * GM + in_band % band_rows;
        aim_tn = __builtin_amdgcn_readfirstlane(in_band / band_rows);
        aim_m0 = __builtin_amdgcn_readfirstlane(tm * BM);
        aim_n0 = aim_tn * BNT;
        // the slot at which the cyclic walk over k starts: tile-rows that run together read W apart
        kstart = __builtin_amdgcn_readfirstlane((int)((unsigned)tm % (unsigned)ns));
        const int rows_a = M - aim_m0 < BM ? M - aim_m0 : BM;
        const int rows_w = N - aim_n0 < BNT ? N - aim_n0 : BNT;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = (wave + 4 * j) * 8 + (lane >> 3);
            const int chunk = (lane & 7) ^ swz(row);
            // HEAD_GRAD: LDS row 128*h + 16*i + r holds activation row 128*h + 8*r + i, and weight row 32*j + 16*k + 4*g + e (k = 0, 1) weight
            // row 32*j + 8*g + 4*k + e, so that a lane ends up with eight consecutive rows and groups of eight consecutive columns of the
            // tile, and the four lanes of a row with 32
            const int arow = HEAD == HEAD_GRAD ? (row & 128) | ((row & 15) << 3) | ((row >> 4) & 7) : row;
            const int wrow = HEAD == HEAD_GRAD ? (row & ~31) | (((row >> 2) & 3) << 3) | (((row >> 4) & 1) << 2) | (row & 3) : row;
            if constexpr (KNA) {   // a load is two rows of k of 256 columns, or four of 128
                const int krow = (wave + 4 * j) * 2 + (lane >> 5);
                voff_a[j] = (uint32_t)krow * (uint32_t)ld_a + (uint32_t)(((lane & 31) ^ swz_kn(krow)) * 16);
            } else {
                const int ra = arow < rows_a ? arow : rows_a - 1;   // rows past the edge are never stored
                voff_a[j] = (uint32_t)((size_t)ra * ld_a) + (uint32_t)(chunk * 16);
            }
            if (j >= NJ) continue;
            if constexpr (KNW) {
                constexpr int CH = 4 * NJ;   // chunks of a row
                const int krow = (wave + 4 * j) * (64 / CH) + lane / CH;
                voff_w[j] = (uint32_t)krow * (uint32_t)ld_w + (uint32_t)(((lane % CH) ^ swz_kn(krow)) * 16);
            } else {
                const int rw = wrow < rows_w ? wrow : rows_w - 1;
                voff_w[j] = (uint32_t)((size_t)rw * ld_w) + (uint32_t)(chunk * 16);
            }
        }
        // buffer resources over the two panels: scalar base, per-lane 32-bit offset, scalar k offset; the range ends with the last valid row, so
        // that an offset beyond it reads zeros
        auto make_rsrc = [](const char* base, size_t bytes) {
            const uint64_t b = (uint64_t)(uintptr_t)base;
            i32x4 r;
            r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)b);
            r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)((b >> 32) & 0xFFFFu));
            r[2] = __builtin_amdgcn_readfirstlane((int)(uint32_t)bytes);
            r[3] = 0x00020000;
            return r;
        };
        // ([K, N]: up to the last column of the last row of k, in whole chunks, so that rows beyond k read as zeros)
        auto kn_bytes = [&](size_t ld, int cols) { return (size_t)(k_rows - 1) * ld + (size_t)((cols + 7) / 8 * 16); };
        rsrc_a = make_rsrc(A + (KNA ? (size_t)aim_m0 * ESZ : (size_t)aim_m0 * ld_a),
                           KNA ? kn_bytes(ld_a, M - aim_m0) : (size_t)(rows_a - 1) * ld_a + k_bytes);
        rsrc_w = make_rsrc(Wt + (KNW ? (size_t)aim_n0 * ESZ : (size_t)aim_n0 * ld_w),
                           KNW ? kn_bytes(ld_w, N - aim_n0) : (size_t)(rows_w - 1) * ld_w + k_bytes);
    };

    // Load instruction q (0..7 = A, 8..7+NJ = W) of the slot at place `st` of k into the slot at LDS byte address `slot`.  Inline assembly, so that
    // the compiler's wait-count pass does not see an LDS write it cannot tell apart from the fragment reads; the waits are placed by hand below.
    // M0 (the LDS base of the transfer) is a reserved register that compiled code only sets right before its own uses.
    auto issue = [&](int q, int st, uint32_t slot) __attribute__((always_inline)) {
        const int koff = (q < 8 ? KNA : KNW) ? (int)((uint32_t)st * 64u * (uint32_t)(q < 8 ? ld_a : ld_w)) : st * kRow;
        const uint32_t dst = slot + (uint32_t)(q < 8 ? (wave + 4 * q) * 1024 : BM * kRow + (wave + 4 * (q - 8)) * 1024);
        const i32x4 rsrc = q < 8 ? rsrc_a : rsrc_w;
        const uint32_t vo = RAGGED && st == ns - 1 && beyond_k ? (uint32_t)rsrc[2] : q < 8 ? voff_a[q] : voff_w[q - 8];
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"(dst), "v"(vo), "s"(rsrc), "s"(koff) : "memory");
    };

    i32x4 af[2][8], wf[2][NJ];   // fragments of the two k-steps of a slot
    // [K, N] operands: lane 16g + 4r + s supplies rows 32h + 8g (+4) + r, columns 4s of the block, and receives its own column's values
    const int kn_r = (lane >> 2) & 3, kn_g = lane >> 4, kn_f = kn_r | ((kn_g & 1) << 2);
    auto read_kn = [&](const char* base, int pitch, int h, int b) {
        const char* const at = base + (32 * h + 8 * kn_g + kn_r) * pitch + ((b ^ kn_f) << 5) + (lane & 3) * 8;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)at);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(at + 4 * pitch));
        return __builtin_bit_cast(i32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read_frag = [&](int h, const char* slot, int f /*0..7 = A block, 8..7+NJ = W block*/) {
        if (KNA && f < 8)
            af[h][f] = read_kn(slot + wm * 256, 512, h, f);
        else if (KNW && f >= 8)
            wf[h][f - 8] = NJ == 8 ? read_kn(slot + BM * kRow + wn * 256, 512, h, f - 8) : read_kn(slot + BM * kRow, 256, h, 4 * wn + f - 8);
        else if (f < 8)
            af[h][f] = *reinterpret_cast<const i32x4*>(slot + a_base + f * 16 * kRow + foff[h]);
        else
            wf[h][f - 8] = *reinterpret_cast<const i32x4*>(slot + w_base + (f - 8) * 16 * kRow + foff[h]);
    };

    // The schedule of gemm.hip's bf16 loop: slot-step S lives in slot S % 2 and is two k-steps of NM MFMAs each; loads of slot-step S + 2 go out
    // one per G MFMAs, P1 of them in (S,1), the rest in (S+1,0); at the barrier inside (S,1) a wave has issued VMB younger loads.
    constexpr int NM = 8 * NJ, NF = 8 + NJ, NL = 8 + NJ;
    constexpr int G = NJ >= 5 ? 6 : 5;
    constexpr int HB = NM - 2 * NF;
    constexpr int P1 = (NM - 2) / G + 1;               // load slots idx % G == 1 of a k-step
    constexpr int P0 = NM >= 4 ? (NM - 4) / G + 1 : 0; // load slots idx % G == 3 of a k-step
    constexpr int VMB = HB >= 2 ? (HB - 2) / G + 1 : 0;
    static_assert(HB >= 0 && P1 <= NL && NL - P1 <= P0 && VMB < 16, "load schedule fits the k-steps");
    auto next_of = [&](int st) { return st + 1 >= ns ? 0 : st + 1; };   // (one slot: it again)
    aim(blockIdx.x);
    int st1 = next_of(kstart);   // where in k the next slot-step lies
#pragma unroll
    for (int q = 0; q < NL; ++q) issue(q, kstart, lds_base);
#pragma unroll
    for (int q = 0; q < P1; ++q) issue(q, next_of(kstart), lds_base + kSlot);   // its other loads go out in (0,0) like everywhere below
    __builtin_amdgcn_s_waitcnt(0x0F70 | P1);   // vmcnt(P1): slot-step 0 has landed
    __syncthreads();
#pragma unroll
    for (int f = 0; f < NF; ++f) read_frag(0, lds, f);

    const int mrow = lane & 15;
    const int nsub = (lane >> 4) * 4;
    int at = 0;   // slot of the slot-step
    // (what has to be there before is waited for by hand; a fence would wait for an epilogue's stores too)
    auto barrier = []() __attribute__((always_inline)) { asm volatile("s_barrier" ::: "memory"); };
    for (int pid = blockIdx.x;; pid += gridDim.x) {
        const int m0 = aim_m0, n0 = aim_n0, tn = aim_tn;
        const bool more = pid + (int)gridDim.x < T;   // is there a next tile?
        // what the epilogue reads, on its way meanwhile
        int64_t target[8];
        float4 row[8];   // HeadArgs::rows
        float times[8];
        if constexpr (HEAD == HEAD_STATS)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int m = m0 + wm * 128 + i * 16 + mrow;
                target[i] = m < M ? head.targets[m] : -1;
            }
        if constexpr (HEAD == HEAD_GRAD)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int m = m0 + wm * 128 + 8 * mrow + i;
                row[i] = head.rows[m < M ? m : M - 1];
            }
        if constexpr (KNW)
            if (head.sum == nullptr)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int m = m0 + wm * 128 + i * 16 + mrow;
                    times[i] = head.factor[head.factor_step * (m < M ? m : M - 1)];
                }
        f32x4 acc[NJ][8];   // [weight-row block j (16 rows)][activation-row block i (16 rows)]
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][i][e] = 0.0f;
        // written as inline assembly with explicit register classes (accumulators in AGPRs, fragments in VGPRs): see gemm.hip
        auto mfma_one = [&](int h, int j, int i) {
            asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[j][i]) : "v"(wf[h][j]), "v"(af[h][i]));
        };

        for (int S = 0; S < ns; ++S) {
            const char* cur = lds + at * kSlot;
            const char* nxt = lds + (at ^ 1) * kSlot;
            __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): fragments of (S,0)
            asm volatile("s_nop 3");              // accumulators written just before
#pragma unroll
            for (int idx = 0; idx < NM; ++idx) {
                mfma_one(0, idx >> 3, idx & 7);
                if (idx < 2 * NF && (idx & 1) == 0) read_frag(1, cur, idx >> 1);
                if (idx % G == 3 && P1 + idx / G < NL) issue(P1 + idx / G, st1, lds_base + (at ^ 1) * kSlot);   // the other loads of slot-step S+1
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): fragments of (S,1)
            barrier();
            // the slot-step after the next: the next tile's first where this tile's end, past the last tile's end any (harmless)
            int st2 = next_of(st1);
            if (more && S == ns - 2) {
                aim(pid + gridDim.x);
                st2 = kstart;
            }
#pragma unroll
            for (int idx = 0; idx < NM; ++idx) {
                if (idx == HB) {
                    __builtin_amdgcn_s_waitcnt(0x0F70 | VMB);   // vmcnt(VMB)
                    barrier();
                }
                mfma_one(1, idx >> 3, idx & 7);
                if (idx % G == 1) issue(idx / G, st2, lds_base + at * kSlot);          // loads 0..P1-1 of slot-step S+2
                if (idx >= HB && ((idx - HB) & 1) == 0) read_frag(0, nxt, (idx - HB) >> 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            st1 = st2;
            at ^= 1;
        }
        if (!more) __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0): no LDS load or read may outlive the workgroup
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");   // the last MFMA results are in the accumulators before they are read

        // D'[r][c] = C[m = c][n = r]: lane holds activation row lane%16 and weight rows 4*(lane/16) + e
        if constexpr (HEAD == HEAD_STATS) {
            // per row: maximum and sum of exp2 over this wave's 16*NJ columns (logits in units of log 2: alpha carries log2 e), and the
            // target's logit where it is one of them
            const int nw = n0 + wn * 16 * NJ;
            const bool edge = nw + 16 * NJ > N;
            int limit = N - nw - nsub;   // the lane's columns 16*j + e (counted from nw + nsub) below this exist
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                const int m = m0 + wm * 128 + i * 16 + mrow;
                float v[NJ][4], top = -INFINITY;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j][e] = acc_read(acc[j][i][e]);
                if (edge) {
                    asm volatile("" : "+v"(limit));   // (compared anew for every row: 32 masks kept between rows do not fit the scalar registers)
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (16 * j + e >= limit) v[j][e] = -INFINITY;
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, v[j][e]);
                top = fmaxf(exchanged<16>(top)[0], exchanged<16>(top)[1]);
                top = fmaxf(exchanged<32>(top)[0], exchanged<32>(top)[1]);
                top *= alpha;
                const float base = top > -INFINITY ? top : 0.0f;   // (no column, or all minus infinity: the sum is 0, not NaN)
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(v[j][e], alpha, -base));
                sum = exchanged<16>(sum)[0] + exchanged<16>(sum)[1];
                sum = exchanged<32>(sum)[0] + exchanged<32>(sum)[1];
                if (lane < 16 && m < M) head.part[(size_t)(2 * tn + wn) * M + m] = make_float2(top, sum);
                // the target's column among the lane's
                const int64_t t = target[i] - head.v0 - nw;
                const int tcol = t >= 0 && t < 16 * NJ && t < N - nw && (((int)t >> 2) & 3) == (lane >> 4) ? (int)t - nsub : -1;
                if (__ballot(tcol >= 0) != 0) {   // (few rows of few tiles)
                    float z = 0.0f;
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) z = tcol == 16 * j + e ? v[j][e] : z;
                    if (tcol >= 0) head.picked[m] = z * alpha;
                }
            }
        }
        if constexpr (HEAD == HEAD_GRAD) {
            // gradients of the logits over the row's factor, G[m][n]; rows that are ignored and columns beyond N are zero, so that G can be
            // walked in whole slots as the next product's k
            const int mw = m0 + wm * 128 + 8 * mrow;          // first of this lane's eight rows
            const int nl = n0 + wn * 16 * NJ + 2 * nsub;      // first of its columns nl + 32*j + 0..7
            int tcol[8];
            bool keep[8], whole = n0 + (wn + 1) * 16 * NJ <= N, hit = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = __float_as_int(row[i].w);
                keep[i] = t != INT_MIN;
                whole = whole && keep[i];
                const int64_t c = (int64_t)t - head.v0 - nl;   // 32*j + 0..7: this lane's
                tcol[i] = t >= 0 && c >= 0 && c < 16 * NJ && (c & 31) < 8 ? (int)c : -1;
                hit = hit || tcol[i] >= 0;
            }
            // most waves see neither an ignored row, nor an edge, nor a target
            const bool plain = __ballot(!whole || hit) == 0;
#pragma unroll
            for (int jj = 0; jj < NJ; jj += 2) {
                __builtin_amdgcn_sched_barrier(0);
                const int n = nl + 16 * jj;
                float g[8][8];   // [row][column n + c]
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        g[i][c] = row[i].y * __builtin_amdgcn_exp2f(__builtin_fmaf(acc_read(acc[jj + (c >> 2)][i][c & 3]), alpha, -row[i].x));
                if (!plain) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            if (tcol[i] == 16 * jj + c) g[i][c] -= row[i].z;
                            if (!keep[i] || n + c >= N) g[i][c] = 0.0f;
                        }
                }
                if (n < head.g_cols)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (mw + i < M)
                            *reinterpret_cast<uint4*>(head.g + (size_t)(mw + i) * head.ld_g + n) =
                                make_uint4(pack_bf16x2(g[i][0], g[i][1]), pack_bf16x2(g[i][2], g[i][3]), pack_bf16x2(g[i][4], g[i][5]),
                                           pack_bf16x2(g[i][6], g[i][7]));
            }
        }
        if constexpr (KNW) {
            // fp32 sums of the shares of k, rows of ld_sum values; or the result itself, bf16
            float* const sums = head.sum != nullptr ? head.sum + (size_t)blockIdx.y * M * head.ld_sum : nullptr;
            if (sums == nullptr)
#pragma unroll
                for (int i = 0; i < 8; ++i) times[i] *= head.scale;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                const int m = m0 + wm * 128 + i * 16 + mrow;
                if (m >= M) continue;
                if (sums != nullptr) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const int n = n0 + wn * 16 * NJ + j * 16 + nsub;
                        if (n >= N) continue;
                        f32x4 c;
#pragma unroll
                        for (int e = 0; e < 4; ++e) c[e] = acc_read(acc[j][i][e]);
                        f32x4* const at = reinterpret_cast<f32x4*>(sums + (size_t)m * head.ld_sum + n);   // (rows are padded to four columns)
                        if (head.add) c += *at;
                        *at = c;
                    }
                    continue;
                }
                // rows of 16 lanes swap halves of two blocks: a lane has eight neighbours of one of them, four lanes 64 bytes of a row
#pragma unroll
                for (int j = 0; j < NJ; j += 2) {
                    uint32_t w[2][2];
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            w[b][e] = pack_bf16x2(times[i] * acc_read(acc[j + b][i][2 * e]), times[i] * acc_read(acc[j + b][i][2 * e + 1]));
                    const auto lo = __builtin_amdgcn_permlane16_swap(w[0][0], w[1][0], false, false);
                    const auto hi = __builtin_amdgcn_permlane16_swap(w[0][1], w[1][1], false, false);
                    const uint32_t v[4] = {lo[0], hi[0], lo[1], hi[1]};
                    const int n = n0 + wn * 16 * NJ + (j + ((lane >> 4) & 1)) * 16 + (lane >> 5) * 8;
                    uint16_t* const out = C + (size_t)m * head.ld_out + n;
                    if (n + 7 < N) {
                        __builtin_memcpy(out, v, 16);   // (one store, whatever the rows' alignment)
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (n + e < N) out[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
                    }
                }
            }
        }
        if (!more) return;
    }
}

// A workgroup a compute unit, whose tiles are a multiple of eight apart, so that they belong to one XCD (with two slots of k or more: a next
// tile's first two are loaded during a tile's last two)?  Else a workgroup a tile.
long long walkers() { return device_cu_count() & ~7; }
bool walks(long long tiles, int K, int shares) { return walkers() > 0 && tiles > walkers() && shares == 1 && K >= 128; }

int launch_head_part(int kind, int nj, const void* A, const void* W, void* C, int M, int N, int K, float alpha, int shares, const HeadArgs& head,
                     hipStream_t stream) {
    const bool ragged = kind <= HEAD_GRAD && K % 64 != 0;
    typedef void (*kern_t)(const char*, const char*, uint16_t*, int, int, int, float, int, int, const HeadArgs);
    static const kern_t kerns[12] = {
        gemm_head_kernel<8, false, HEAD_STATS>, gemm_head_kernel<4, false, HEAD_STATS>, gemm_head_kernel<8, true, HEAD_STATS>, gemm_head_kernel<4, true, HEAD_STATS>,
        gemm_head_kernel<8, false, HEAD_GRAD>,  gemm_head_kernel<4, false, HEAD_GRAD>,  gemm_head_kernel<8, true, HEAD_GRAD>,  gemm_head_kernel<4, true, HEAD_GRAD>,
        gemm_head_kernel<8, false, HEAD_DX>,    gemm_head_kernel<4, false, HEAD_DX>,    gemm_head_kernel<8, false, HEAD_DW>,   gemm_head_kernel<4, false, HEAD_DW>};
    const kern_t kern = kerns[(kind == HEAD_STATS ? 0 : kind == HEAD_GRAD ? 4 : kind == HEAD_DX ? 8 : 10) + (ragged ? 2 : 0) + (nj == 4 ? 1 : 0)];
    const int rc = set_max_dynamic_lds((const void*)kern, kLdsBytes);
    if (rc != ROV_OK) return rc;
    const long long tiles_m = (M + BM - 1) / BM, tiles_n = (N + 32 * nj - 1) / (32 * nj);
    if (!grid_fits(tiles_m * tiles_n, 256)) return ROV_ERR_UNSUPPORTED;
    const long long tiles = tiles_m * tiles_n;
    hipLaunchKernelGGL(kern, dim3((unsigned)(walks(tiles, K, shares) ? walkers() : tiles), (unsigned)shares), dim3(256), kLdsBytes, stream, (const char*)A, (const char*)W,
                       (uint16_t*)C, M, N, K, alpha, (int)tiles_m, (int)tiles_n, head);
    ROV_LAUNCH_CHECK();
    return ROV_OK;
}

// How many of `lines` lines of `across` 256 x 256 tiles each run as such: those in full rounds over the compute units, where the rest, cut
// into tiles of 256 x 128, fits one round of 0.63 times a round's time (a slot of k 890 against 1410 ns); else all.  (1000 x
// 50257 x 1024: 788 tiles are four rounds, of which the last has 20 tiles.)
long long wide_lines(long long lines, long long across) {
    const long long ncu = device_cu_count(), full = lines * across / ncu * ncu / across;
    return 2 * across * (lines - full) <= ncu ? full : lines;
}
// Of M x N: the columns (HEAD_STATS, HEAD_GRAD) or rows (HEAD_DX, HEAD_DW) that run as 256 x 256 tiles.
long long wide_part(bool kn, int M, int N, int shares) {
    const long long tiles_m = ((long long)M + BM - 1) / BM, tiles_n = ((long long)N + BN - 1) / BN;
    return !kn ? wide_lines(tiles_n, tiles_m) * BN : shares > 1 ? M : wide_lines(tiles_m, tiles_n) * BM;
}
}  // namespace

bool gemm_head_walks(int kind, int M, int N, int K, int shares) {
    const bool kn = kind == HEAD_DX || kind == HEAD_DW;
    const long long all = kn ? M : N, part = wide_part(kn, M, N, shares), wide = part < all ? part : all, rest = all - wide;
    auto tiles = [&](long long along, int width) {
        return kn ? (along + BM - 1) / BM * (((long long)N + width - 1) / width) : ((long long)M + BM - 1) / BM * ((along + width - 1) / width);
    };
    return walks(tiles(wide, BN), K, shares) || walks(tiles(rest, BN / 2), K, shares);
}

int gemm_head_parts(int M, int N) {
    const long long lines = (N + BN - 1) / BN, wide = wide_lines(lines, (M + BM - 1) / BM);
    return (int)(2 * wide + (wide < lines ? 2 * ((N - wide * BN + 127) / 128) : 0));
}

int launch_gemm_head(int kind, const void* A, const void* W, void* C, int M, int N, int K, float alpha, int shares, const HeadArgs& head,
                     hipStream_t stream) {
    const bool kn = kind == HEAD_DX || kind == HEAD_DW, kna = kind == HEAD_DW;
    if (A == nullptr || W == nullptr || M <= 0 || N <= 0 || K <= 0 || shares <= 0 || shares > 65535) return ROV_ERR_INVALID;
    if (!aligned(A, 16) || !aligned(W, 16) || head.ld_a % 16 != 0 || head.ld_w % 16 != 0 || (!kn && K % 8 != 0)) return ROV_ERR_INVALID;
    const int64_t slots = ((int64_t)K + 63) / 64;
    if (head.ld_a < (size_t)(kna ? (M + 7) / 8 * 16 : kn ? slots * kRowBytes : (int64_t)K * 2)) return ROV_ERR_INVALID;
    if (head.ld_w < (size_t)(kn ? (N + 7) / 8 * 16 : (int64_t)K * 2) || (!kn && shares > 1) || shares > slots) return ROV_ERR_INVALID;
    // an operand's panel (256 rows, or all rows of k) is addressed with 32-bit byte offsets
    if ((unsigned long long)(kna ? slots * 64 : BM) * head.ld_a + 1024 > 0xFFFFFFFFull ||
        (unsigned long long)(kn ? slots * 64 : BN) * head.ld_w + 1024 > 0xFFFFFFFFull)
        return ROV_ERR_UNSUPPORTED;
    HeadArgs h = head;
    const long long part = wide_part(kn, M, N, shares);
    if (!kn) {   // columns beyond the full rounds: narrower tiles
        const int wide = part < N ? (int)part : N;
        if (wide >= N) return launch_head_part(kind, 8, A, W, C, M, N, K, alpha, 1, head, stream);
        if (wide > 0) {
            h.g_cols = wide;
            const int rc = launch_head_part(kind, 8, A, W, C, M, wide, K, alpha, 1, h, stream);
            if (rc != ROV_OK) return rc;
        }
        h.v0 += wide;
        h.g_cols = head.g_cols - wide;
        if (h.g != nullptr) h.g += wide;
        if (h.part != nullptr) h.part += (size_t)(wide / 128) * M;
        return launch_head_part(kind, 4, A, (const char*)W + (size_t)wide * head.ld_w, C, M, N - wide, K, alpha, 1, h, stream);
    }
    const int wide = part < M ? (int)part : M;   // rows
    if (wide >= M) return launch_head_part(kind, 8, A, W, C, M, N, K, alpha, shares, head, stream);
    if (wide > 0) {
        const int rc = launch_head_part(kind, 8, A, W, C, wide, N, K, alpha, 1, head, stream);
        if (rc != ROV_OK) return rc;
    }
    if (h.sum != nullptr) h.sum += (size_t)wide * h.ld_sum;
    h.factor += h.factor_step * wide;
    return launch_head_part(kind, 4, (const char*)A + (kna ? (size_t)wide * 2 : (size_t)wide * head.ld_a), W, (uint16_t*)C + (size_t)wide * head.ld_out,
                            M - wide, N, K, alpha, 1, h, stream);
}

}  // namespace rov
