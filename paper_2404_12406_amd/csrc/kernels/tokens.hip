// The row contractions z = x W^T of the gated unit and the cross entropy for at
// most 16 rows: single tokens while a model answers, or a few to be scored.
//
// Bound: the read of W, once.  A tile of the large contractions would stage W
// through LDS for rows that are not there; here W goes from memory into the
// registers that feed the matrix instruction.  16 rows of W are its first operand,
// the (up to) 16 rows of x its second: 16x16x32 for bf16, 16x16x4 for fp32.
//  * a wave reads 128 bytes of each of its 32 rows of W a step (two 16-byte loads a
//    lane and tile, k permuted alike in both operands), four steps in flight;
//  * the KS waves of a block take every KS-th step and meet in LDS;
//  * x is read from the caches, by every block; rows past M repeat the last one and
//    their columns of the result are dropped.
// The gated unit pairs a tile of gate rows with one of up rows, so that a lane has
// both projections; the softmax keeps running statistics of its words per lane.
// Measured, us a call, here and with the large contraction, W not in the caches: one
// token, bf16, 4096 x 2 x 10944 73 and 79 (from the last-level cache 33 and 30), 2048
// x 2 x 1024 14 and 21, 1024 x 2 x 4096 12 and 15.  16 rows are what the matrix
// instruction takes: one more would read W twice.  (Which sizes of the cross entropy
// and of fp32 come here: few_rows() in xent.hip, launch_gated_fwd().)
#include <algorithm>

#include "block_math.h"
#include "lds_dma.h"
#include "limits.h"

namespace ms {
namespace tok {

constexpr int kRows = 16;   // rows of x at most
constexpr int KS = 4;       // waves of a block, each a share of k
constexpr int DEEP = 4;     // steps in flight

struct Args {
    const void *x, *w, *bias;
    int M, K;
    uint32_t x_bytes, w_bytes;
    // gated
    int F, act;
    void *y;
    void *proj;                  // z as the large contraction keeps it (null: not kept)
    // cross entropy
    int V;
    const int64_t *target;
    floatx2 *stat;               // [block][kRows]
    float *tlogit;               // [kRows]
};

template <typename T> struct Step;
template <> struct Step<bf16> {
    static constexpr int K = 64;
    // element of load s of lane group g within a step
    static __device__ __forceinline__ int at(int g, int s) { return 16 * g + 8 * s; }
    static constexpr int N = 8;
    static __device__ __forceinline__ floatx4 mac(u32x4 a, u32x4 b, floatx4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Step<float> {
    static constexpr int K = 32;
    static __device__ __forceinline__ int at(int g, int s) { return 16 * s + 4 * g; }
    static constexpr int N = 4;
    static __device__ __forceinline__ floatx4 mac(u32x4 a, u32x4 b, floatx4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
        return c;
    }
};

// Walks `groups` groups of two 16-row tiles of W, group i's tiles starting at rows
// first + i stride (+ apart for the second) and ending at end[t]; after the last of
// a group's steps done(i, acc) has the sums with the rows of x over this wave's
// steps: lane l holds row 4 (l / 16) + v of tile t and row l % 16 of x.  The loads
// run DEEP steps ahead, into the next group where this one ends.
template <typename T, class Done>
__device__ __forceinline__ void products(const Args &P, int first, int stride, int apart, const int (&end)[2], int groups, int wave,
                                         int lane, Done done) {
    using S = Step<T>;
    const __amdgpu_buffer_rsrc_t rw = g2::rsrc(P.w, P.w_bytes), rx = g2::rsrc(P.x, P.x_bytes);
    const int g = lane >> 4, r16 = lane & 15;
    const uint32_t ox = (uint32_t)min(r16, P.M - 1) * (uint32_t)P.K;
    const int steps = ((P.K + S::K - 1) / S::K + KS - 1) / KS;   // of each wave (some past the end)
    int li = 0, ls = 0;   // group and step to be loaded
    u32x4 fw[DEEP][2][2], fx[DEEP][2];
    auto load = [&](u32x4 (&w)[2][2], u32x4 (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = (wave + ls * KS) * S::K + S::at(g, s);
            const bool in = k < P.K && li < groups;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int row = first + li * stride + t * apart + r16;
                const uint32_t off = in && row < end[t] ? ((uint32_t)row * (uint32_t)P.K + (uint32_t)k) * (uint32_t)sizeof(T) : g2::kOOB;
                w[t][s] = __builtin_amdgcn_raw_buffer_load_b128(rw, (int)off, 0, 0);
            }
            const uint32_t off = in ? (ox + (uint32_t)k) * (uint32_t)sizeof(T) : g2::kOOB;
            x[s] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)off, 0, 0);
            if constexpr (sizeof(T) == 4) {   // a row's last elements, where its width is no multiple of 4
                if (k + 4 > P.K) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool past = k + e >= P.K;
                        x[s][e] = past ? 0u : x[s][e];
#pragma unroll
                        for (int t = 0; t < 2; ++t) w[t][s][e] = past ? 0u : w[t][s][e];
                    }
                }
            }
        }
        if (++ls == steps) {
            ls = 0;
            ++li;
        }
    };
#pragma unroll
    for (int d = 0; d < DEEP; ++d) load(fw[d], fx[d]);
    floatx4 acc[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
    int i = 0, s0 = 0;   // group and step worked on
    while (i < groups) {
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            if (i >= groups) break;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) acc[t] = S::mac(fw[d][t][s], fx[d][s], acc[t]);
            load(fw[d], fx[d]);   // (past the end: zeros, no memory read)
            if (++s0 == steps) {
                done(i, acc);
                acc[0] = acc[1] = floatx4{0.f, 0.f, 0.f, 0.f};
                s0 = 0;
                ++i;
            }
        }
    }
}

// Wave 0's sums become the block's.
__device__ __forceinline__ void meet(floatx4 (&acc)[2], float *red, int wave, int lane) {
    floatx4 *r = reinterpret_cast<floatx4 *>(red);
    if (wave > 0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) r[((wave - 1) * 2 + t) * 64 + lane] = acc[t];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 0; w < KS - 1; ++w)
#pragma unroll
            for (int t = 0; t < 2; ++t) acc[t] += r[(w * 2 + t) * 64 + lane];
    }
}

template <typename T>
__global__ __launch_bounds__(KS * 64) void gate_kernel(const Args P) {
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ float red[(KS - 1) * 2 * 64 * 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int f0 = (int)blockIdx.x * 16, F = P.F;
    const int end[2] = {F, 2 * F};
    floatx4 acc[2];
    products<T>(P, f0, 0, F, end, 1, wave, lane, [&](int, floatx4 (&sums)[2]) {
        acc[0] = sums[0];
        acc[1] = sums[1];
    });
    meet(acc, red, wave, lane);
    const int m = lane & 15, f = f0 + 4 * (lane >> 4);
    if (wave != 0 || m >= P.M) return;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (f + v >= F) continue;
        const float zg = acc[0][v] + (P.bias ? to_f32(((const T *)P.bias)[f + v]) : 0.f);
        const float zu = acc[1][v] + (P.bias ? to_f32(((const T *)P.bias)[F + f + v]) : 0.f);
        ((T *)P.y)[(int64_t)m * F + f + v] = from_f32<T>(act::value<FAST>(P.act, zg) * zu);
        if (!P.proj) continue;
        const int64_t at = (int64_t)m * 2 * F + f + v;
        if constexpr (FAST) {
            uint16_t *hi = (uint16_t *)P.proj;
            uint8_t *lo = (uint8_t *)P.proj + (int64_t)P.M * 4 * F;
            const uint32_t kg = to_f24(zg), ku = to_f24(zu);
            hi[at] = (uint16_t)(kg >> 8);
            hi[at + F] = (uint16_t)(ku >> 8);
            lo[at] = (uint8_t)kg;
            lo[at + F] = (uint8_t)ku;
        } else {
            ((float *)P.proj)[at] = zg;
            ((float *)P.proj)[at + F] = zu;
        }
    }
}

// Statistics of the words that this block's groups of 32 hold.
template <typename T>
__global__ __launch_bounds__(KS * 64) void lse_kernel(const Args P) {
    __shared__ float red[(KS - 1) * 2 * 64 * 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15;
    const int64_t t = wave == 0 && m < P.M ? P.target[m] : -1;
    floatx2 a = {-INFINITY, 0.f};
    const int end[2] = {P.V, P.V}, all = (P.V + 31) / 32;
    const int mine = (all - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    products<T>(P, (int)blockIdx.x * 32, (int)gridDim.x * 32, 16, end, mine, wave, lane, [&](int g, floatx4 (&acc)[2]) {
        const int v0 = ((int)blockIdx.x + g * (int)gridDim.x) * 32;
        if (g > 0) __syncthreads();   // wave 0 has read the others' last sums
        meet(acc, red, wave, lane);
        if (wave == 0) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int n = v0 + 16 * i + 4 * (lane >> 4) + v;
                    const bool in = n < P.V;
                    if (P.bias && in) acc[i][v] += to_f32(((const T *)P.bias)[n]);
                    acc[i][v] = in ? acc[i][v] : -INFINITY;
                    if (in && t == n) {   // the target leaves the sums
                        P.tlogit[m] = acc[i][v];
                        acc[i][v] = -INFINITY;
                    }
                    top = fmaxf(top, acc[i][v]);
                }
            const float t0 = top == -INFINITY ? 0.f : top;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) s += exp_below(acc[i][v], t0);
            a = join_lse(a, floatx2{top, s});
        }
    });
    if (wave != 0) return;
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) a = join_lse(a, floatx2{__shfl_xor(a.x, o), __shfl_xor(a.y, o)});
    if (lane < kRows) P.stat[(int64_t)blockIdx.x * kRows + lane] = a;
}

// The rows' losses from the blocks' statistics, a wave a row, and their reduction.
__global__ __launch_bounds__(1024) void loss_kernel(const floatx2 *__restrict__ stat, int parts, const float *__restrict__ tlogit,
                                                    const int64_t *__restrict__ target, int64_t ignore, int M, int V, int reduction,
                                                    float *__restrict__ loss, float *__restrict__ others) {
    __shared__ float each[kRows];
    const int lane = threadIdx.x & 63, m = threadIdx.x >> 6;
    if (m < M) {
        floatx2 a = {-INFINITY, 0.f};
        for (int p = lane; p < parts; p += 64) a = join_lse(a, stat[(int64_t)p * kRows + m]);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) a = join_lse(a, floatx2{__shfl_xor(a.x, o), __shfl_xor(a.y, o)});
        if (lane == 0) {
            const int64_t t = target[m];
            float l = 0.f, c = 0.f;
            if (t != ignore) {
                const RowLoss q = row_loss(a, t >= 0 && t < V ? tlogit[m] : NAN);
                l = q.others;
                c = q.loss;
            }
            if (others) others[m] = l;
            if (reduction == 2) loss[m] = c;
            each[m] = c;
        }
    }
    __syncthreads();
    if (threadIdx.x != 0 || reduction == 2) return;
    double s = 0.0;
    int n = 0;
    for (int i = 0; i < M; ++i) {
        s += (double)each[i];
        n += target[i] != ignore;
    }
    *loss = (float)(reduction == 0 ? s / (double)n : s);
}

namespace {

constexpr int kMostBlocks = 768;

template <typename T>
Args args(int64_t M, int64_t N, int64_t K, const void *x, const void *w, const void *bias) {
    Args a{};
    a.x = x;
    a.w = w;
    a.bias = bias;
    a.M = (int)M;
    a.K = (int)K;
    a.x_bytes = (uint32_t)(M * K * (int64_t)sizeof(T));
    a.w_bytes = (uint32_t)(N * K * (int64_t)sizeof(T));
    return a;
}

template <typename T>
int gate_t(int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *b, void *y, void *proj, hipStream_t st) {
    Args a = args<T>(M, 2 * F, D, x, w, b);
    a.F = (int)F;
    a.act = act;
    a.y = y;
    a.proj = proj;
    hipLaunchKernelGGL(gate_kernel<T>, dim3((unsigned)((F + 15) / 16)), dim3(KS * 64), 0, st, a);
    return (int)hipGetLastError();
}

// As many blocks as the card holds at once, each with as many groups as the others.
int blocks(int64_t V) {
    const int64_t groups = (V + 31) / 32, each = (groups + kMostBlocks - 1) / kMostBlocks;
    return (int)((groups + each - 1) / each);
}

template <typename T>
int lse_t(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *b, const int64_t *target, floatx2 *stat, float *tlogit,
          hipStream_t st) {
    Args a = args<T>(M, V, D, x, w, b);
    a.V = (int)V;
    a.target = target;
    a.stat = stat;
    a.tlogit = tlogit;
    hipLaunchKernelGGL(lse_kernel<T>, dim3(blocks(V)), dim3(KS * 64), 0, st, a);
    return (int)hipGetLastError();
}

}  // namespace

// Operands below 2^32 bytes; bf16 rows of whole 16-byte vectors so aligned, fp32
// rows as they are.
bool applies(int dtype, int64_t M, int64_t N, int64_t K, const void *x, const void *w) {
    const int64_t e = dtype == kBF16 ? 2 : 4;
    if (M < 1 || M > kRows || N * K * e > (int64_t)g2::kOOB - 64) return false;
    return dtype != kBF16 || (K % 8 == 0 && ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(w)) & 15u) == 0);
}

int gate(int dtype, int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *b, void *y, void *proj,
         hipStream_t st) {
    return dtype == kBF16 ? gate_t<bf16>(M, D, F, act, x, w, b, y, proj, st) : gate_t<float>(M, D, F, act, x, w, b, y, proj, st);
}

size_t xent_workspace() { return (size_t)kMostBlocks * kRows * sizeof(floatx2) + 256; }

int xent(int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *b, const int64_t *target, int64_t ignore,
         int reduction, float *loss, float *lse, void *ws, hipStream_t st) {
    floatx2 *stat = static_cast<floatx2 *>(ws);
    float *tlogit = reinterpret_cast<float *>(stat + kMostBlocks * kRows);
    const int err = dtype == kBF16 ? lse_t<bf16>(M, D, V, x, w, b, target, stat, tlogit, st)
                                   : lse_t<float>(M, D, V, x, w, b, target, stat, tlogit, st);
    if (err) return err;
    hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, st, stat, blocks(V), tlogit, target, ignore, (int)M, (int)V, reduction, loss,
                       lse);
    return (int)hipGetLastError();
}

}  // namespace tok
}  // namespace ms
