// Attention over whole prompts, forward: for each query row of each packed sequence and head
//   o = sum over visible keys of exp(c s_j - m) v_j / sum of exp(c s_j - m),  s_j = q k_j
// with one pass over the keys.  A block takes 128 queries of a head, 32 a wave, and walks
// the keys BN at a time: S^T = K Q^T, so that a lane holds one query's scores (its maximum
// and sum are registers of that lane and one exchange with the lane 32 away), and O^T =
// V^T P^T straight from those registers (attn_tile.h).
//
// Bound: matrix cores, 4 D operations a visible pair, and the vector units next to them
// (an exponential takes four times an addition's time).  bf16, 32 on 8 heads of 128, causal: two prompts of
// 8192 rows 1.07 ms, 1.03 PFLOP/s of visible pairs where a library product of 8192^3 reaches 1.24; 8192 rows in 7
// sequences 178 us, 600 TFLOP/s.  16 x 512 rows, 12 heads of 64, all keys: 25 us, 520 TFLOP/s.  fp32, 1777 rows, 6 on 2 heads
// of 72: 36 us and 8 for the join.
// Queries of a block: 128, four waves of a tile's 32 columns each, so that two blocks share a CU and one's
// matrix instructions run beside the other's exponentials.  The tiles come straight from memory into LDS a
// step ahead: loads that hit L2 alone took 12 of 212 us off.  Exponentials of one part between matrix instructions
// of another, by hand, and longer blocks at a higher wave priority gave nothing.
#include <algorithm>

#include "attn_tile.h"

namespace ms {
namespace att {

constexpr int kRows = 128;   // queries of a block

template <typename T, int DC>
struct FwdShape {
    static constexpr int BN = kPitch<DC> * (int)sizeof(T) <= 256 ? 64 : 32;   // keys of a step
    static constexpr int OCC = DC <= 128 ? 2 : 1;   // blocks a CU
};

// Partial results of a block that takes some of the keys alone: sums[split][Hq][Tq][DC] and
// floatx2 {reference, sum}[split][Hq][Tq] behind them.
struct Parts {
    int splits;
    float *sums;
    floatx2 *stat;
};

// WG: groups of four waves.  Two take every other step each, from stages of their own, and meet at the end.
template <typename T, int DC, int WG>
__global__ __launch_bounds__(256 * WG, (FwdShape<T, DC>::OCC / WG)) void fwd_kernel(AttnArgs a, Parts part) {
    constexpr int DP = kPitch<DC>;
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    typedef typename M::Frag Frag;
    constexpr int BN = FwdShape<T, DC>::BN, NS = BN / 32, NP = 32 / M::KC, BYTES = BN * Ti::RB;
    __shared__ __align__(256) char lds[4 * BYTES * WG];
    const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6) & 3, side = WG > 1 ? uniform(threadIdx.x >> 8) : 0;
    int head, rank;
    find_head((int)blockIdx.x, a.Hq, head, rank);
    const int hk = head / (a.Hq / a.Hk);
    const Span s = find_ranked(a.qoff, a.koff, a.n, (int)a.Tq, (int)a.Tk, rank, kRows, a.causal, true);
    const int row0 = s.tile * kRows;
    if (s.tile < 0 || row0 >= s.na) return;
    const int shift = s.nb - s.na;                 // query i sees keys to i + shift
    const int seen = a.causal ? max(0, min(s.nb, min(row0 + kRows, s.na) + shift)) : s.nb, steps = (seen + BN - 1) / BN;
    const int begin = (int)((int64_t)steps * blockIdx.y / part.splits) * BN;   // of the block's keys
    const int end = min(seen, (int)((int64_t)steps * (blockIdx.y + 1) / part.splits) * BN);
    const int wrow = row0 + 32 * w, rows = min(32, s.na - wrow);                 // the wave's
    const int wend = rows <= 0 ? 0 : a.causal ? min(s.nb, wrow + rows + shift) : s.nb;
    const int wfull = a.causal ? min(s.nb, wrow + 1 + shift) : s.nb;             // keys that all its rows see
    const int last = a.causal ? min(s.nb - 1, wrow + (lane & 31) + shift) : s.nb - 1;   // the lane's row sees

    const T *qp = static_cast<const T *>(a.q.p) + (int64_t)(s.a0 + wrow) * a.q.ts + head * a.q.hs;
    const char *kp = reinterpret_cast<const char *>(static_cast<const T *>(a.k.p) + (int64_t)s.b0 * a.k.ts + hk * a.k.hs);
    const char *vp = reinterpret_cast<const char *>(static_cast<const T *>(a.v.p) + (int64_t)s.b0 * a.v.ts + hk * a.v.hs);
    Loader<T, DP, BN, 4> lk, lv;
    lk.init(a.k.ts, a.D, w, lane);
    lv.init(a.v.ts, a.D, w, lane);
    char *stages = lds + side * 4 * BYTES;
    auto issue = [&](int k) {
        char *to = stages + (k / (BN * WG) & 1) * 2 * BYTES;
        lk.issue(kp + k * lk.ts, s.nb - k, a.D, to, w);
        lv.issue(vp + k * lv.ts, s.nb - k, a.D, to + BYTES, w);
    };
    if (begin + side * BN < end) issue(begin + side * BN);
    Rows<T, DC> q;
    q.init(qp, a.q.ts, rows, a.D, lane);

    const float c = a.scale * kLog2e;
    float m = -INFINITY, l[4] = {0.f, 0.f, 0.f, 0.f};
    floatx16 acc[DC / 32];
#pragma unroll
    for (int t = 0; t < DC / 32; ++t) acc[t] = zero16x();
    // N 32-key tiles from row r0 of the stage on, of which some rows may not see all.
    auto attend = [&](const char *kt, const char *vt, int k, int r0, bool masked, auto tiles) __attribute__((always_inline)) {
        constexpr int N = decltype(tiles)::value;
        floatx16 x[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            x[n] = zero16x();
#pragma unroll
            for (int i = 0; i < DC / M::KC; ++i) x[n] = M::mma(Ti::row_frag(kt, r0 + 32 * n, i, lane), q.get(i, lane), x[n]);
        }
        if (masked) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[n][i] = k + r0 + 32 * n + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) > last ? -INFINITY : x[n][i];
        }
        float top = x[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[n][i]);
        top = both_max(top);
        // The reference follows the maximum only where that is 2^8 above it: what is summed
        // is then below 2^8 a key, and the sums are seldom multiplied again.
        if (__any((top - m) * c > 8.f)) {
            const float to = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
#pragma unroll
            for (int j = 0; j < 4; ++j) l[j] *= f;
#pragma unroll
            for (int t = 0; t < DC / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][i] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m, minus = -ref * c;   // (no key yet)
        Frag p[N * NP];
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[n][i] = power<T>(x[n][i], ref, minus, c);
                l[i & 3] += x[n][i];
            }
            // (in bf16 rounded to 8 bits, an operand; the sum has all of them)
#pragma unroll
            for (int i = 0; i < NP; ++i) p[n * NP + i] = as_frag<T>(x[n], i);
        }
        if (masked && any_wild<T, DP, 32 * N>(vt, r0, lane)) wild_product<T, DP, DC, N * NP>(acc, vt, r0, p, 0, last - k - r0, lane);
        else add_product<T, DP, DC, N * NP>(acc, vt, r0, p, lane);
    };
    // The keys that all of the block's rows see, in whole steps; then the others, 32 at a time.
    // (Two loops: around the rare path of masked keys the compiler copies all sums, 64 moves a step.)
    const int clear = max(begin, min(end, max(0, a.causal ? min(s.nb, row0 + 1 + shift) : s.nb) / BN * BN));
    int k = begin;
    auto stage = [&](int own) __attribute__((always_inline)) {
        tile_sync();
        if (own + BN * WG < end) issue(own + BN * WG);
        return stages + (own / (BN * WG) & 1) * 2 * BYTES;
    };
    for (; k + (WG - 1) * BN < clear; k += BN * WG) {
        const int own = k + side * BN;
        const char *kt = stage(own);
        attend(kt, kt + BYTES, own, 0, false, Number<NS>{});
    }
    for (; k < end; k += BN * WG) {
        const int own = k + side * BN;
        const char *kt = stage(own);
#pragma unroll
        for (int r = 0; r < BN; r += 32)
            if (own + r < min(wend, end)) attend(kt, kt + BYTES, own, r, own + r + 32 > wfull, Number<1>{});
    }
    tile_sync();   // no wave reads the tiles any more
    float sum = both_sum((l[0] + l[1]) + (l[2] + l[3]));
    if constexpr (WG > 1) {   // the second group's sums, maximum and sum of weights to the first
        char *to = lds + w * (DC * 128 + 512);
        floatx4 *sums = reinterpret_cast<floatx4 *>(to) + lane;
        floatx2 *stat = reinterpret_cast<floatx2 *>(to + DC * 128) + lane;
        if (side) {
            *stat = floatx2{m, sum};
#pragma unroll
            for (int t = 0; t < DC / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) sums[64 * (4 * t + g)] = floatx4{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]};
        }
        tile_sync();
        if (!side) {
            const floatx2 st = *stat;
            const float top = fmaxf(m, st.x), f = m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * c),
                        h = st.x == top ? 1.f : __builtin_amdgcn_exp2f((st.x - top) * c);
            m = top;
            sum = f * sum + h * st.y;
#pragma unroll
            for (int t = 0; t < DC / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const floatx4 v = sums[64 * (4 * t + g)];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[t][4 * g + j] = f * acc[t][4 * g + j] + h * v[j];
                }
        }
        tile_sync();
        if (side) return;
    }
    if (rows <= 0) return;
    const bool none = last < 0;   // a row that sees no key: zeros
    if (part.splits > 1) {
        const int64_t at = ((int64_t)blockIdx.y * a.Hq + head) * a.Tq + s.a0 + wrow;
        store_sums<DC>(acc, part.sums + at * DC, DC, rows, lane);
        if (lane < rows) part.stat[at + lane] = floatx2{m, none ? -1.f : sum};
        return;
    }
    if (a.lse && lane < rows)
        a.lse[(int64_t)head * a.Tq + s.a0 + wrow + lane] = none ? INFINITY : m * c + __builtin_amdgcn_logf(sum);
    store_rows<T, DP, DC>(acc, 1.f / sum, none, lds + w * 32 * Ti::RB,
                      static_cast<T *>(a.o.p) + (int64_t)(s.a0 + wrow) * a.o.ts + head * a.o.hs, a.o.ts, rows, a.D, lane);
}

// o and lse from the partial results: a vector a thread.
template <typename T, int DC>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a, Parts part) {
    constexpr int V = Vec16<T>::N;
    const int per = a.D / V;
    const int64_t rows = a.Tq * a.Hq, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * per) return;
    const int64_t row = i / per, t = row / a.Hq;
    const int u = (int)(i - row * per), h = (int)(row - t * a.Hq);
    const int64_t at = h * a.Tq + t;
    const float c = a.scale * kLog2e;
    float top = -INFINITY, sum = 0.f, o[V];
    bool none = false;
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = 0.f;
    for (int s = 0; s < part.splits; ++s) top = fmaxf(top, part.stat[s * rows + at].x);
    for (int s = 0; s < part.splits; ++s) {
        const floatx2 st = part.stat[s * rows + at];
        const float f = st.x == top ? 1.f : __builtin_amdgcn_exp2f((st.x - top) * c);
        none |= st.y < 0.f;
        sum += f * st.y;
        const float *p = part.sums + (s * rows + at) * DC + u * V;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] += f * p[e];
    }
    Vec16<T> v;
#pragma unroll
    for (int e = 0; e < V; ++e) v.e[e] = from_f32<T>(none ? 0.f : o[e] / sum);
    store16(static_cast<T *>(a.o.p) + t * a.o.ts + h * a.o.hs + u * V, v);
    if (a.lse && u == 0) a.lse[at] = none ? INFINITY : top * c + __builtin_amdgcn_logf(sum);
}

// dst[T][H][Dp]: a vector a thread.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T *__restrict__ src, int64_t ts, int64_t hs, int64_t ds, int64_t n, int H, int D,
                                                   T *__restrict__ dst, int Dp) {
    constexpr int V = Vec16<T>::N;
    const int per = Dp / V;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per, t = row / H;
        const int u = (int)(i - row * per), h = (int)(row - t * H);
        const T *p = src + t * ts + h * hs;
        Vec16<T> v;
#pragma unroll
        for (int e = 0; e < V; ++e) v.e[e] = u * V + e < D ? p[(u * V + e) * ds] : (T)0.f;
        store16(dst + i * V, v);
    }
}

namespace {

int64_t rows_slots(const AttnArgs &a) { return span_slots(a.qoff != nullptr, a.n, a.Tq, kRows); }

template <typename T, int DC>
int64_t fwd_steps(const AttnArgs &a) {   // of a sequence
    return (a.qoff ? a.Tk / std::max(a.n, 1) : a.Tk) / FwdShape<T, DC>::BN;
}

template <typename T, int DC>
int fwd_splits(const AttnArgs &a) {
    return span_splits<T>(rows_slots(a) * a.Hq, fwd_steps<T, DC>(a), a.Tq * a.Hq * DC * 4);
}

template <typename T, int DC>
size_t fwd_space(const AttnArgs &a) {
    const size_t n = fwd_splits<T, DC>(a);
    return n > 1 ? (n * a.Tq * a.Hq * (DC * sizeof(float) + sizeof(floatx2)) + 255) / 256 * 256 : 0;
}

template <typename T, int DC>
int fwd_run(const AttnArgs &a, void *ws, hipStream_t st) {
    const int64_t slots = rows_slots(a), rows = a.Tq * a.Hq;
    Parts part{fwd_splits<T, DC>(a), static_cast<float *>(ws), nullptr};
    part.stat = reinterpret_cast<floatx2 *>(part.sums + part.splits * rows * DC);
    const dim3 grid((unsigned)(slots * a.Hq), (unsigned)part.splits);
    constexpr bool pairs = sizeof(T) == 2 && FwdShape<T, DC>::OCC == 2;
    if (pairs && wide_blocks((int64_t)grid.x * grid.y, fwd_steps<T, DC>(a) / part.splits, 24)) {
        if constexpr (pairs) hipLaunchKernelGGL((fwd_kernel<T, DC, 2>), grid, dim3(512), 0, st, a, part);
    } else {
        hipLaunchKernelGGL((fwd_kernel<T, DC, 1>), grid, dim3(256), 0, st, a, part);
    }
    if (part.splits > 1) {
        const int64_t n = rows * (a.D / Vec16<T>::N);
        hipLaunchKernelGGL((join_kernel<T, DC>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, part);
    }
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace att

size_t attention_fwd_workspace(int dtype, const AttnArgs &a) {
    if (a.Tq == 0) return 0;
    return dtype == kBF16 ? ATT_COLUMNS(att::fwd_space, bf16, a) : ATT_COLUMNS(att::fwd_space, float, a);
}

int launch_attention_fwd(int dtype, const AttnArgs &a, void *ws, void *stream) {
    if (a.Tq == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    return dtype == kBF16 ? ATT_COLUMNS(att::fwd_run, bf16, a, ws, st) : ATT_COLUMNS(att::fwd_run, float, a, ws, st);
}

int launch_pack_heads(int dtype, const void *src, int64_t ts, int64_t hs, int64_t ds, int64_t T, int H, int D, void *dst, int Dp,
                      void *stream) {
    const int64_t n = T * H * (Dp / (dtype == kBF16 ? 8 : 4));
    if (n == 0) return 0;
    const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, 8192));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == kBF16)
        hipLaunchKernelGGL(att::pack_kernel<bf16>, grid, dim3(256), 0, st, (const bf16 *)src, ts, hs, ds, n, H, D, (bf16 *)dst, Dp);
    else
        hipLaunchKernelGGL(att::pack_kernel<float>, grid, dim3(256), 0, st, (const float *)src, ts, hs, ds, n, H, D, (float *)dst, Dp);
    return (int)hipGetLastError();
}

}  // namespace ms
