// bf16 contractions of the transformer layers, each with what follows it done
// on the sums while they are in registers:
//   kEpiGate      z = x W^T + b over W = [gate; up]: y = act(z_gate) z_up, and
//                 optionally z itself (kept for the backward)
//   kEpiGateGrad  z again, then the gradient of z for that of y: dz_gate = dy
//                 z_up act'(z_gate), dz_up = dy act(z_gate)
//   kEpiLse       z = x W^T + b over a vocabulary: the maximum and the sum of
//                 exponentials of each row's part of a column tile, its target
//                 left out, and the target's logit; z is not written
//   kEpiXent      z again, then dz = exp(z - lse) scale, in the target's column its
//                 own entry times scale, and optionally the column sums of dz before
//                 it is rounded
//   kEpiProb      z, then exp(z - r) of the other words than the target, r a
//                 reference of each row's part of a wave's columns, with those parts'
//                 sums of exponentials and the target's logit
//   kEpiAdd       dx += dz W for one piece of the vocabulary, in fp32 (the gated unit's
//                 dx too, in one piece)
//   kEpiStore     the weight gradient dz^T x over the rows that count, times a factor
//   kEpiRows      the same into rows of another width, whole vectors or not
// The main loop is gemm_block_body.inc's.  Everything before the one rounding
// of what is stored is in fp32.  dz and the kept exponentials are stored in bf16 as they
// are the next contraction's operand, and the matrix cores take no wider one at their
// rate: 2^-9 of each term, which averages out over the sums (gradients are 2.0 to 2.4e-3
// from 64 bits, normwise, where the rounding of the result alone is 1.7e-3).
//
// Bound: the matrix cores, of which a tile's beginning and end leave a share idle: a
// 256 x 256 tile takes 1.58 us for 64 of k with all CUs at it, and some 3 us to begin
// and end, with the softmax's statistics 7.7, with dz of the cross entropy 12.  At k =
// 768, 12 such steps, that is the difference between 914 (kEpiLse) or 780 TFLOP/s
// (kEpiXent) and the 1276 that a large product reaches; at k = 4096 kEpiProb has 1178,
// kEpiGate (k = 2048) 1093.  128 x 128 tiles, two a CU, would run one's end under the
// other's steps, but their steps are a fifth slower: est_us() has both.
#pragma once

#include <cstdlib>
#include <cstring>

#include <hip/hip_ext.h>

#include "block_math.h"
#include "gemm_bf16.h"

namespace ms {
namespace g2 {

enum Epi { kEpiStore = 0, kEpiGate = 1, kEpiGateGrad = 2, kEpiLse = 3, kEpiXent = 4, kEpiAdd = 5, kEpiProb = 6, kEpiRows = 7 };

struct FusedArgs : Args {
    const int *count;      // rows that count (weight gradient: of the reduction), on the device; null: all
    const bf16 *fbias;     // bias of the columns (gated: [2F]); null: none
    // gated
    int F;
    uint16_t *proj;        // kEpiGate: z in 24 bits (null: not kept): a plane of the leading 16, [M][2F],
    uint8_t *proj_lo;      // and one of the others
    const bf16 *dh;        // kEpiGateGrad: dy[M][F]; c is dz[M][2F]
    // cross entropy; rows are those that count
    const int *target;     // each row's target in the vocabulary
    int v0;                // the piece's first word
    floatx2 *stat;         // kEpiLse, kEpiProb: softmax statistics as join_lse()'s, [column tile][rows], [64 columns][rows]
    float *tlogit;         // with them: the target's logit; kEpiXent: what rounding took from the target's dz
    int64_t stat_ld;
    const float *lse, *scale;   // kEpiXent: of each row
    const float *ct;       // with them: the target's entry of dz but for the scale
    const float *out_scale;     // kEpiStore, kEpiRows: the sums' factor
    int add;               // kEpiAdd: add to the partials (0: write them)
    const int *nsplit;     // kEpiAdd: their number, on the device,
    int fixed_splits;      // or (null) here
};

// Output column of row `row` of a gated tile's B operand, from the tile's first.
__device__ __forceinline__ int gate_col(int row) { return (row >> 6) * 32 + (row & 31); }

// Between a wave's writes to its staging rows and its reads of them, and back: LDS
// serves a wave's instructions in order, so only the compiler has to keep to it.
__device__ __forceinline__ void stage_order() {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Bias of columns n .. n + 3, zeros past the descriptor's end; `quads`: its length
// and n are whole fours.
__device__ __forceinline__ void bias4(__amdgpu_buffer_rsrc_t r, int n, bool quads, float (&o)[4]) {
    if (quads) {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, n * 2, 0, 0);
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] = __uint_as_float((v & 1) ? (w[v >> 1] & 0xffff0000u) : (w[v >> 1] << 16));
    } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] = __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b16(r, (n + v) * 2, 0, 0) << 16);
    }
}

// Rows of COLS bf16 (a multiple of 8) that a wave has staged in LDS, `pitch`
// apart: 32 of them to dst + row * ld, columns below `ncol`, rows below `nrow`.
template <int COLS>
__device__ __forceinline__ void store_rows(const bf16 *stage, int pitch, bf16 *dst, int64_t ld, int nrow, int ncol, int lane) {
    constexpr int SEG = COLS / 8, RPP = 64 / SEG;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RPP) {
        const int r = r0 + lane / SEG, c = (lane % SEG) * 8;
        Vec16<bf16> v;
        v.u = *reinterpret_cast<const u32x4 *>(stage + r * pitch + c);
        if (r >= nrow || c >= ncol) continue;
        bf16 *d = dst + (int64_t)r * ld + c;
        if (c + 8 <= ncol) {
            *reinterpret_cast<u32x4 *>(d) = v.u;   // (any alignment of the rows)
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < ncol) d[e] = v.e[e];
        }
    }
}

// Rows of COLS bytes, four of a lane packed in each word of b, through the wave's
// staging bytes to dst + row * ld.
template <int COLS, int TG>
__device__ __forceinline__ void put_bytes(uint8_t *stage, const uint32_t (&b)[TG][4], uint8_t *dst, int64_t ld, int nrow, int ncol,
                                          int fr, int fh, int lane) {
    constexpr int PITCH = COLS + 16, SEG = COLS / 16, RPP = 64 / SEG;
    stage_order();
#pragma unroll
    for (int j = 0; j < TG; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<uint32_t *>(stage + fr * PITCH + 32 * j + 8 * q + 4 * fh) = b[j][q];
    stage_order();
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RPP) {
        const int r = r0 + lane / SEG, c = (lane % SEG) * 16;
        if (r >= nrow || c >= ncol || r >= 32) continue;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(stage + r * PITCH + c);
        uint8_t *d = dst + (int64_t)r * ld + c;
        if (c + 16 <= ncol) {
            *reinterpret_cast<u32x4 *>(d) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c + e < ncol) d[e] = (uint8_t)(v[e / 4] >> (8 * (e % 4)));
        }
    }
}

// What the sums start from: the bias of their columns and, in the softmax, minus
// infinity past the last word (nothing is added to it there: W's rows read zeros).
// Loaded before the operands' first loads are issued, put into the sums after.
template <int EPI, class G>
struct FusedInit {
    static constexpr bool GATED = EPI == kEpiGate || EPI == kEpiGateGrad, SOFTMAX = EPI == kEpiLse || EPI == kEpiXent || EPI == kEpiProb;
    float b[G::TN][4][4];

    __device__ __forceinline__ FusedInit(const FusedArgs &P, int n0, int wn0, int lane) {
        const int fh = lane >> 5, nb = GATED ? 2 * P.F : P.N;
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int v = 0; v < 4; ++v) b[j][q][v] = 0.f;
        if (!P.fbias) return;
        const __amdgpu_buffer_rsrc_t r = rsrc(P.fbias, (uint32_t)nb * 2u);
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = 8 * q + 4 * fh;
                // (gated columns past F read the other half's: not stored)
                if constexpr (GATED) bias4(r, (n0 + wn0) / 2 + 32 * (j / 2) + c + (j & 1) * P.F, (P.F & 3) == 0, b[j][q]);
                else bias4(r, n0 + wn0 + 32 * j + c, (nb & 3) == 0, b[j][q]);
            }
    }
    __device__ __forceinline__ void put(const FusedArgs &P, floatx16 (&acc)[G::TM][G::TN], int n0, int wn0, int lane) {
        const int fh = lane >> 5;
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    if (SOFTMAX && n0 + wn0 + 32 * j + 8 * q + 4 * fh + v >= P.N) b[j][q][v] = -INFINITY;
#pragma unroll
                    for (int i = 0; i < G::TM; ++i) acc[i][j][4 * q + v] = b[j][q][v];
                }
    }
};

// The lane's 16 sums of tile (i, j) are row 32 i + lane % 32 and columns
// 32 j + 8 q + 4 (lane / 32) + v, q and v = 0..3.
template <int EPI, int ACT, class G>
__device__ __forceinline__ void fused_epilogue(const FusedArgs &P, char *smem, floatx16 (&acc)[G::TM][G::TN], int M, int m0, int n0,
                                               int wm0, int wn0, int wave, int lane, int tn, int zsplit) {
    constexpr int TM = G::TM, TN = G::TN;
    const int fr = lane & 31, fh = lane >> 5;
    const int N = P.N;
    bf16 *stage = reinterpret_cast<bf16 *>(smem) + wave * G::EPI_ROWS * G::EPI_PITCH;
    if constexpr (EPI == kEpiGate || EPI == kEpiGateGrad) {
        constexpr int TG = TN / 2, COLS = 32 * TG, PITCH = COLS + 8;
        static_assert(TN % 2 == 0, "gated tiles pair the column tiles of a wave");
        const int F = P.F, f0 = (n0 + wn0) / 2;
        const int ncol = min(F - f0, COLS);
        // dy's tile, whole vectors where they are, every pass's loads in flight at once
        constexpr int SEG = COLS / 8, RPP = 64 / SEG;
        Vec16<bf16> dh[EPI == kEpiGateGrad ? TM : 1][32 / RPP];
        if constexpr (EPI == kEpiGateGrad) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int h = 0; h < 32 / RPP; ++h) {
                    const int m = m0 + wm0 + 32 * i + h * RPP + lane / SEG, c = (lane % SEG) * 8;
                    dh[i][h] = zero16<bf16>();
                    if (m >= M || c >= ncol) continue;
                    const bf16 *s = P.dh + (int64_t)m * F + f0 + c;
                    if (c + 8 <= ncol) {
                        dh[i][h].u = *reinterpret_cast<const u32x4 *>(s);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (c + e < ncol) dh[i][h].e[e] = s[e];
                    }
                }
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int mb = m0 + wm0 + 32 * i, nrow = M - mb;   // rows of this pass
            if constexpr (EPI == kEpiGateGrad) {
#pragma unroll
                for (int h = 0; h < 32 / RPP; ++h)
                    *reinterpret_cast<u32x4 *>(stage + (h * RPP + lane / SEG) * PITCH + (lane % SEG) * 8) = dh[i][h].u;
                stage_order();
            }
            // what the second pass stores: gradients, or (gate, up) projections
            bf16x4 og[TG][4], ou[TG][4];
            uint32_t lg[TG][4], lu[TG][4];   // their third bytes
#pragma unroll
            for (int j = 0; j < TG; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = 32 * j + 8 * q + 4 * fh;
                    bf16x4 d4;
                    if constexpr (EPI == kEpiGateGrad) d4 = *reinterpret_cast<const bf16x4 *>(stage + fr * PITCH + c);
                    lg[j][q] = lu[j][q] = 0u;
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float zg = acc[i][2 * j][4 * q + v], zu = acc[i][2 * j + 1][4 * q + v];
                        if constexpr (EPI == kEpiGate) {
                            acc[i][2 * j][4 * q + v] = act::value<true>(ACT, zg) * zu;
                            if (P.proj) {
                                const uint32_t kg = to_f24(zg), ku = to_f24(zu);
                                og[j][q][v] = __builtin_bit_cast(bf16, (uint16_t)(kg >> 8));
                                ou[j][q][v] = __builtin_bit_cast(bf16, (uint16_t)(ku >> 8));
                                lg[j][q] |= (kg & 255u) << (8 * v);
                                lu[j][q] |= (ku & 255u) << (8 * v);
                            }
                        } else {
                            float a, da;
                            act::both<true>(ACT, zg, a, da);
                            const float d = (float)d4[v];
                            og[j][q][v] = (bf16)(d * zu * da);
                            ou[j][q][v] = (bf16)(d * a);
                        }
                    }
                }
            auto put = [&](auto get, bf16 *dst, int64_t ld) __attribute__((always_inline)) {
                stage_order();
#pragma unroll
                for (int j = 0; j < TG; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<bf16x4 *>(stage + fr * PITCH + 32 * j + 8 * q + 4 * fh) = get(j, q);
                stage_order();
                store_rows<COLS>(stage, PITCH, dst + (int64_t)mb * ld + f0, ld, nrow, ncol, lane);
            };
            if constexpr (EPI == kEpiGate) {
                put([&](int j, int q) {
                    bf16x4 o;
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[v] = (bf16)acc[i][2 * j][4 * q + v];
                    return o;
                }, P.c, F);
                if (P.proj) {
                    bf16 *z = reinterpret_cast<bf16 *>(P.proj);
                    put([&](int j, int q) { return og[j][q]; }, z, 2 * (int64_t)F);
                    put([&](int j, int q) { return ou[j][q]; }, z + F, 2 * (int64_t)F);
                    put_bytes<COLS>(reinterpret_cast<uint8_t *>(stage), lg, P.proj_lo + (int64_t)mb * 2 * F + f0, 2 * (int64_t)F, nrow,
                                    ncol, fr, fh, lane);
                    put_bytes<COLS>(reinterpret_cast<uint8_t *>(stage), lu, P.proj_lo + (int64_t)mb * 2 * F + F + f0, 2 * (int64_t)F,
                                    nrow, ncol, fr, fh, lane);
                }
            } else {
                put([&](int j, int q) { return og[j][q]; }, P.c, 2 * (int64_t)F);
                put([&](int j, int q) { return ou[j][q]; }, P.c + F, 2 * (int64_t)F);
            }
            stage_order();
        }
    } else if constexpr (EPI == kEpiLse || EPI == kEpiXent || EPI == kEpiProb) {
        // the rows' values, every pass's loads in flight at once
        int tgt[TM];
        float lse[EPI == kEpiXent ? TM : 1], scale[EPI == kEpiXent ? TM : 1];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = min(m0 + wm0 + 32 * i + fr, M - 1);
            tgt[i] = P.target[m];
            if constexpr (EPI == kEpiXent) {
                lse[i] = P.lse[m];
                scale[i] = P.scale[m];
            }
        }
        if constexpr (EPI == kEpiLse) {
            constexpr int BM = G::A_BYTES / (BK * 2), WC = G::B_BYTES / (BK * 2) / G::WN;   // waves along the columns
            floatx2 *red = reinterpret_cast<floatx2 *>(smem);   // [WC][BM]
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                __builtin_amdgcn_sched_barrier(0);   // one pass at a time: the sums leave few registers
                const int m = m0 + wm0 + 32 * i + fr;
                const int t = m < M ? tgt[i] - P.v0 - (n0 + wn0) : -1;   // within this wave's columns?
                if (__any((unsigned)t < (unsigned)G::WN)) {   // the target leaves the sums
                    float z = 0.f;
                    bool mine = false;
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int v = 0; v < 4; ++v)
                                if (t == 32 * j + 8 * q + 4 * fh + v) {
                                    z = acc[i][j][4 * q + v];
                                    acc[i][j][4 * q + v] = -INFINITY;
                                    mine = true;
                                }
                    if (mine && n0 + wn0 + t < N) P.tlogit[m] = z;
                }
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) top = fmaxf(top, acc[i][j][v]);
                top = fmaxf(top, __shfl_xor(top, 32));
                // (fmaxf passes over NaN: the sum below meets it)
                const float t0 = top == -INFINITY ? 0.f : top;
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) s += exp_below(acc[i][j][v], t0);
                s += __shfl_xor(s, 32);
                if (fh == 0) red[(wn0 / G::WN) * BM + wm0 + 32 * i + fr] = floatx2{top, s};
            }
            __syncthreads();
            for (int r = wave * 64 + lane; r < BM; r += G::NT) {
                if (m0 + r >= M) continue;
                floatx2 a = red[r];
#pragma unroll
                for (int w = 1; w < WC; ++w) a = join_lse(a, red[w * BM + r]);
                P.stat[(int64_t)tn * P.stat_ld + m0 + r] = a;
            }
        } else if constexpr (EPI == kEpiProb) {
            static_assert(G::WN == kProbCols, "statistics of 64 columns");
            constexpr int PITCH = G::EPI_PITCH;
            const int ncol = min(P.ldc - (n0 + wn0), G::WN);   // the padding columns are zeros
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                __builtin_amdgcn_sched_barrier(0);   // one pass at a time: the sums leave few registers
                const int mb = m0 + wm0 + 32 * i, m = mb + fr;
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) top = fmaxf(top, acc[i][j][v]);
                const float r = prob_ref(fmaxf(top, __shfl_xor(top, 32)));
                const float t0 = r == -INFINITY ? 0.f : r;
                const int t = m < M ? tgt[i] - (n0 + wn0) : -1;
                const bool any = __any((unsigned)t < (unsigned)G::WN);
                float s = 0.f, z = 0.f;
                bool mine = false;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        bf16x4 o;
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            float p = exp_below(acc[i][j][4 * q + v], t0);
                            if (any && t == 32 * j + 8 * q + 4 * fh + v) {
                                z = acc[i][j][4 * q + v];
                                mine = true;
                                p = 0.f;
                            }
                            s += p;
                            o[v] = (bf16)p;
                        }
                        *reinterpret_cast<bf16x4 *>(stage + fr * PITCH + 32 * j + 8 * q + 4 * fh) = o;
                    }
                s += __shfl_xor(s, 32);
                if (fh == 0 && m < M) P.stat[(int64_t)((n0 + wn0) / G::WN) * P.stat_ld + m] = floatx2{r, s};
                if (mine && n0 + wn0 + t < N) P.tlogit[m] = z;
                stage_order();
                store_rows<G::WN>(stage, PITCH, P.c + (int64_t)mb * P.ldc + n0 + wn0, P.ldc, M - mb, ncol, lane);
                stage_order();
            }
        } else {
            constexpr int PITCH = G::EPI_PITCH;
            const int ncol = min(P.ldc - (n0 + wn0), G::WN);   // the padding columns are zeros
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                __builtin_amdgcn_sched_barrier(0);   // one pass at a time: the sums leave few registers
                const int mb = m0 + wm0 + 32 * i, m = mb + fr;
                const bool in = m < M;
                const float l = in ? lse[i] : 0.f, sc = in ? scale[i] : 0.f;
                int t = in ? tgt[i] - P.v0 - (n0 + wn0) : -1;
                if (t >= N - (n0 + wn0)) t = -1;   // (a later piece's: this one may end within a tile)
                const bool any = __any((unsigned)t < (unsigned)G::WN);
                const float ct = any && in ? P.ct[m] : 0.f;
                float rest = 0.f;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        bf16x4 o;
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            float p = exp_below(acc[i][j][4 * q + v], l);
                            if (any && t == 32 * j + 8 * q + 4 * fh + v) p = ct;
                            p = in ? p * sc : 0.f;   // (the other rows hold anything)
                            o[v] = (bf16)p;
                            acc[i][j][4 * q + v] = p;
                            if (any && t == 32 * j + 8 * q + 4 * fh + v) rest = p - (float)o[v];
                        }
                        *reinterpret_cast<bf16x4 *>(stage + fr * PITCH + 32 * j + 8 * q + 4 * fh) = o;
                    }
                stage_order();
                // (of the two lanes of a row the one that has the column: (t / 4) odd in the upper half)
                if ((unsigned)t < (unsigned)G::WN && ((t >> 2) & 1) == fh) P.tlogit[m] = rest;
                store_rows<G::WN>(stage, PITCH, P.c + (int64_t)mb * P.ldc + n0 + wn0, P.ldc, M - mb, ncol, lane);
                stage_order();
            }
            if (P.dbpart) {
                // Column sums of the wave's rows: each of the 32 lanes that share a column's
                // rows sends half of its columns and keeps the other, five times.
                float *row = P.dbpart + (int64_t)((m0 + wm0) / G::WM) * N;
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    float s[16];
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        s[v] = acc[0][j][v];
#pragma unroll
                        for (int i = 1; i < TM; ++i) s[v] += acc[i][j][v];
                    }
#pragma unroll
                    for (int h = 8; h > 0; h >>= 1)
#pragma unroll
                        for (int v = 0; v < h; ++v) {
                            const bool up = (fr & h) != 0;
                            const float mine = up ? s[v + h] : s[v], give = up ? s[v] : s[v + h];
                            s[v] = mine + __shfl_xor(give, h);
                        }
                    s[0] += __shfl_xor(s[0], 16);
                    const int v = fr & 15, n = n0 + wn0 + 32 * j + 8 * (v / 4) + 4 * fh + v % 4;
                    if (fr < 16 && n < N) row[n] = s[0];
                }
            }
        }
    } else if constexpr (EPI == kEpiRows) {
        constexpr int PITCH = G::EPI_PITCH;
        const int ncol = min(P.ldc - (n0 + wn0), G::WN);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int mb = m0 + wm0 + 32 * i;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    bf16x4 o;
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[v] = (bf16)acc[i][j][4 * q + v];
                    *reinterpret_cast<bf16x4 *>(stage + fr * PITCH + 32 * j + 8 * q + 4 * fh) = o;
                }
            stage_order();
            store_rows<G::WN>(stage, PITCH, P.c + (int64_t)mb * P.ldc + n0 + wn0, P.ldc, M - mb, ncol, lane);
            stage_order();
        }
    } else {
        static_assert(EPI == kEpiAdd, "epilogue");
        float *W = P.part + (int64_t)zsplit * P.part_stride;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = m0 + wm0 + 32 * i + fr;
            if (m >= M) continue;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = n0 + wn0 + 32 * j + 8 * q + 4 * fh;
                    if (n >= N) continue;   // (N is a multiple of 8)
                    floatx4 *d = reinterpret_cast<floatx4 *>(W + (int64_t)m * N + n);
                    floatx4 o = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    if (P.add) o += *d;
                    *d = o;
                }
        }
    }
}

#define GEMM_FUSED
template <int EPI, int MODE, int BM, int BN, int WR, int WC, int STAGES, int OCC, int ACT = 0, bool A3 = false>
__global__ __launch_bounds__(WR * WC * 64, OCC) void gemm_fused_kernel(const FusedArgs P) {
    constexpr bool UNIT = true, TS = false, D3 = false;
    constexpr int KG = 1;
    using C = Cfg<MODE, BM, BN, WR, WC, STAGES, KG>;
    __shared__ __attribute__((aligned(1024))) char smem[A3 ? 3 * C::A_BYTES + 2 * C::B_BYTES : C::SMEM_BYTES];
    const int bx = (int)blockIdx.x, bz = (int)blockIdx.z;
#include "gemm_block_body.inc"
}
#undef GEMM_FUSED

// ------------------------------------------------------------------ host
namespace {

uint32_t bytes_of(int64_t elems) { return (uint32_t)(elems * 2); }

// Tiles of the contractions over k-contiguous operands (gated, cross entropy).
// Efficiencies as in gemm_bf16.hip's table.
constexpr Tile kRowTiles[] = {
    {"256x256", 256, 256, 2, 4, 2, 1, 1.20f, 1.20f},
    {"128x128", 128, 128, 2, 2, 2, 2, 0.78f, 1.00f},
    {"128x128s4", 128, 128, 2, 2, 4, 1, 0.90f, 0.90f},
};
struct FusedPlan {
    int tile, splits;
};

// MEMSAVE_FUSED_TILE=<name> forces one tile where the table has it (a testing
// knob); returns its index or -1.
template <int NT>
int forced_tile(const Tile (&tiles)[NT], int ntiles) {
    const char *e = getenv("MEMSAVE_FUSED_TILE");
    if (!e || !*e) return -1;
    for (int t = 0; t < ntiles; ++t)
        if (strcmp(tiles[t].name, e) == 0) return t;
    return -1;
}

template <int NT>
FusedPlan plan(const Tile (&tiles)[NT], int ntiles, long M, long N, long K, int max_splits) {
    FusedPlan p{0, 1};
    double best = 1e300;
    const int forced = forced_tile(tiles, ntiles);
    for (int t = std::max(forced, 0); t < (forced < 0 ? ntiles : forced + 1); ++t)
        for (int s = 1; s <= max_splits; ++s) {
            const double us = est_us(tiles[t], M, N, K, 1, s);
            if (us < best * 0.999) {
                best = us;
                p = FusedPlan{t, s};
            }
        }
    return p;
}

template <int EPI, int MODE, int BM, int BN, int WR, int WC, int STAGES, int OCC, int ACT = 0, bool A3 = false>
int go(unsigned prof, const FusedArgs &a, hipStream_t st, int times = 1) {
    void *eb = nullptr, *ee = nullptr;
    const bool timed = prof_pair(prof, &eb, &ee);
    hipExtLaunchKernelGGL((gemm_fused_kernel<EPI, MODE, BM, BN, WR, WC, STAGES, OCC, ACT, A3>), dim3(a.ntm * a.ntn * times, 1, a.splits),
                          dim3(WR * WC * 64), 0, st, (hipEvent_t)eb, (hipEvent_t)ee, 0, a);
    const int err = (int)hipGetLastError();
    if (timed) prof_pair_done(prof, eb, ee, err == 0);
    return err;
}

template <int EPI, int ACT = 0>
int go_rows(int tile, unsigned prof, const FusedArgs &a, hipStream_t st) {
    switch (tile) {
    case 0: return go<EPI, kFwd, 256, 256, 2, 4, 2, 1, ACT>(prof, a, st);
    case 1: return go<EPI, kFwd, 128, 128, 2, 2, 2, 2, ACT>(prof, a, st);
    default:
        // (the softmax's tables leave the third tile out)
        if constexpr (EPI == kEpiGate || EPI == kEpiGateGrad) return go<EPI, kFwd, 128, 128, 2, 2, 4, 1, ACT>(prof, a, st);
        else return (int)hipErrorInvalidValue;
    }
}

// x[M][D] w[N][D]^T
FusedArgs rows_args(const Tile &t, int64_t M, int64_t N, int64_t D, const void *x, const void *w, int64_t w_rows) {
    FusedArgs a{};
    a.a = (const bf16 *)x;
    a.b = (const bf16 *)w;
    a.g.N = (int)M; a.g.C = (int)D; a.g.K = (int)N;
    a.g.H = a.g.W = a.g.R = a.g.S = a.g.P = a.g.Q = a.g.sh = a.g.sw = 1;
    a.M = (int)M; a.N = (int)N; a.K = (int)D;
    a.ntm = (int)((M + t.bm - 1) / t.bm);
    a.ntn = (int)((N + t.bn - 1) / t.bn);
    a.splits = 1;
    a.k_split = (int)D;
    a.a_bytes = bytes_of(M * D);
    a.b_bytes = bytes_of(w_rows * D);
    return a;
}

}  // namespace
}  // namespace g2
}  // namespace ms
