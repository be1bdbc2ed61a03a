// Attention over whole prompts, backward: from q, k, v, o, the gradient g of o and the kept
// log-sum-exp of each row (base 2, attention.hip),
//   P = 2^(c q k^T - lse),  dP = g v^T,  delta = sum over the head of g o,  dS = P (dP - delta),
//   dq = scale dS k,  dk = scale dS^T q,  dv = P^T g;  dk and dv summed over a group's heads.
// P and dS are taken again a tile at a time and never written.
//
// One kernel for dq (a block owns queries and walks the keys) and one for dk and dv (a block
// owns keys and walks the queries of all heads that share them), so every sum has one
// owner and a fixed order, without atomics; each is launched only where its gradients are asked for.
// Both at once would take S and dP once instead of twice, five products instead of seven,
// but one of the sums would then go through memory.  dv alone needs neither v nor o.
//
// Bound: matrix cores, 3 products in dq, 2 in dv alone, 3 in dk alone, 4 in both (in bf16 that with dS twice),
// and the vector units: 8 operations and an exponential an element of P beside them.  bf16, 8192 rows in 7 sequences,
// 32 on 8 heads of 128: dq 300 us, 530 TFLOP/s by three products, dv alone 170 to 200, 530 to 620; 16 x 512 rows, 12 heads of
// 64: dq 38 us, dk and dv 46.  fp32, 1777 rows, 6 on 2 heads of 72: dq 55 us, dk and dv 72, sums of the parts 6 each.
//
// P is taken from one float a row, whose rounding moves a row of it by up to 2^-25 ln 2 times the log-sum-exp.  The scores'
// own rounding in 32 bits is some eight times that: 500 rows of 64 with a score of 700 in common are off by 1.2e-4 here as with
// softmax taken again, and by 1.6e-5 where every product of q and k is exact.
#include <algorithm>

#include "attn_tile.h"

namespace ms {
namespace att {

// delta of a wave's 32 rows from row `first` on: the sum of o g over row l % 32 (a lane
// takes every other unit), in one order wherever it is taken.
template <typename T, int DC, bool HOLD>
__device__ __forceinline__ float row_delta(const AttnArgs &a, int head, int64_t first, int rows, const Rows<T, DC, HOLD> &g, int lane) {
    typedef Mat<T> M;
    const T *o = static_cast<const T *>(a.o.p) + first * a.o.ts + head * a.o.hs;
    float delta = 0.f;
    auto add = [&](int i) __attribute__((always_inline)) {
        const typename M::Frag x = load_row<T>(o, a.o.ts, rows, a.D, i, lane), y = g.get(i, lane);
#pragma unroll
        for (int j = 0; j < M::V; ++j) delta = __builtin_fmaf(to_f32(x[j]), to_f32(y[j]), delta);
    };
    if constexpr (HOLD) {
#pragma unroll
        for (int i = 0; i < DC / M::KC; ++i) add(i);
    } else {
#pragma unroll 2
        for (int i = 0; i < DC / M::KC; ++i) add(i);
    }
    return both_sum(delta);
}

// delta[h][t], for dk without dq: 128 rows a block, blockIdx.y the head.
template <typename T, int DC>
__global__ __launch_bounds__(256) void delta_kernel(AttnArgs a, float *__restrict__ delta) {
    const int lane = threadIdx.x & 63, head = (int)blockIdx.y;
    const int64_t first = (int64_t)blockIdx.x * 128 + (threadIdx.x >> 6) * 32;
    const int rows = (int)min((int64_t)32, a.Tq - first);
    if (rows <= 0) return;
    Rows<T, DC, false> g;
    g.init(static_cast<const T *>(a.go.p) + first * a.go.ts + head * a.go.hs, a.go.ts, rows, a.D, lane);
    const float v = row_delta<T, DC, false>(a, head, first, rows, g, lane);
    if (lane < rows) delta[head * a.Tq + first + lane] = v;
}

// acc += columns of `tile` times b = dS, in bf16 as the rounded values and what that leaves off: rounded once, dq and
// dk would have two roundings next to delta's error, which is o's (7 packed sequences: off by 2.6e-3 and 2.5e-3; now 1.9e-3
// and 2.0e-3, one rounding alone being 1.7e-3).  (7 sequences, 8192 rows, 32 on 8 heads of 128: dq 250 -> 300 us, dk alone 263 ->
// 310, all gradients 655 -> 702.)
template <typename T, int DP, int DC>
__device__ __forceinline__ void add_exactly(floatx16 (&acc)[DC / 32], const char *tile, int r0, const floatx16 &b, int lane) {
    typedef Mat<T> M;
#pragma unroll
    for (int i = 0; i < 32 / M::KC; ++i) {
        const typename M::Frag d = as_frag<T>(b, i);
        typename M::Frag r;
#pragma unroll
        for (int j = 0; j < M::V; ++j) r[j] = from_f32<T>(b[i * M::V + j] - to_f32(d[j]));
#pragma unroll
        for (int t = 0; t < DC / 32; ++t) {
            const typename M::Frag f = Tile<T, DP>::col_frag(tile, r0, t, i, lane);
            acc[t] = M::mma(f, d, acc[t]);
            acc[t] = M::mma(f, r, acc[t]);
        }
    }
}

// The sums of a block's second group of four waves (side 1) to the wave of the first that has the
// same rows, through the latter's part of LDS; nobody reads LDS before or after.
template <int N, typename F>
__device__ __forceinline__ void add_side(char *lds, int side, int lane, F acc) {
    floatx4 *sums = reinterpret_cast<floatx4 *>(lds) + lane;
    if (side) {
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const floatx16 &s = acc(t);
                sums[64 * (4 * t + g)] = floatx4{s[4 * g], s[4 * g + 1], s[4 * g + 2], s[4 * g + 3]};
            }
    }
    tile_sync();
    if (!side) {
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const floatx4 v = sums[64 * (4 * t + g)];
#pragma unroll
                for (int j = 0; j < 4; ++j) acc(t)[4 * g + j] += v[j];
            }
    }
    tile_sync();
}

// ------------------------------------------------------------------ dq
constexpr int kRows = 128;   // queries of a block of dq, keys of a block of dk and dv

// Whether a wave has registers for the first, and for the second of the two operands that
// it keeps: not for 256, for 192 fp32 elements.
template <typename T, int DC> constexpr bool kHold1 = DC * sizeof(T) < 1024;
template <typename T, int DC> constexpr bool kHold = DC * sizeof(T) < 768;

// What the kernels take besides: delta, which dq_kernel writes, and where they leave sums in fp32 if the
// other side is divided, or a gradient has to wait until everything is read: [split][rows][heads][DC].  (8192 rows in 7
// sequences, 32 on 8 heads of 128, bf16, forward and all gradients: 860 us, 960 with dq where o was.)
struct Parts {
    float *delta;
    int splits;
    bool sums;
    float *a, *b;
};

template <typename T, int DC>
struct DqShape {
    static constexpr int BN = kPitch<DC> * (int)sizeof(T) <= 256 ? 64 : 32;
    static constexpr int OCC = DC * (int)sizeof(T) <= 256 ? 2 : 1;
};

// WG: groups of four waves.  Two take every other step each, from stages of their own, and add
// their sums at the end: a block that fills a CU alone.
template <typename T, int DC, int WG>
__global__ __launch_bounds__(256 * WG, (DqShape<T, DC>::OCC / WG)) void dq_kernel(AttnArgs a, Parts part) {
    constexpr int DP = kPitch<DC>;
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    typedef typename M::Frag Frag;
    constexpr int BN = DqShape<T, DC>::BN, NP = 32 / M::KC, BYTES = BN * Ti::RB;
    __shared__ __align__(256) char lds[4 * BYTES * WG];
    const int lane = threadIdx.x & 63, w = WG > 1 ? uniform(threadIdx.x >> 6) & 3 : uniform(threadIdx.x >> 6), side = WG > 1 ? uniform(threadIdx.x >> 8) : 0;
    int head, rank;
    find_head((int)blockIdx.x, a.Hq, head, rank);
    const int hk = head / (a.Hq / a.Hk);
    const Span s = find_ranked(a.qoff, a.koff, a.n, (int)a.Tq, (int)a.Tk, rank, kRows, a.causal, true);
    const int row0 = s.tile * kRows;
    if (s.tile < 0 || row0 >= s.na) return;
    const int shift = s.nb - s.na;
    const int seen = a.causal ? max(0, min(s.nb, min(row0 + kRows, s.na) + shift)) : s.nb, steps = (seen + BN - 1) / BN;
    const int begin = (int)((int64_t)steps * blockIdx.y / part.splits) * BN;
    const int end = min(seen, (int)((int64_t)steps * (blockIdx.y + 1) / part.splits) * BN);
    const int wrow = row0 + 32 * w, rows = min(32, s.na - wrow);
    const int wend = rows <= 0 ? 0 : a.causal ? min(s.nb, wrow + rows + shift) : s.nb;
    const int wfull = a.causal ? min(s.nb, wrow + 1 + shift) : s.nb;
    const int last = a.causal ? min(s.nb - 1, wrow + (lane & 31) + shift) : s.nb - 1;

    const int64_t first = s.a0 + wrow;
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
    Rows<T, DC, kHold1<T, DC>> q;
    Rows<T, DC, kHold<T, DC>> g;
    q.init(static_cast<const T *>(a.q.p) + first * a.q.ts + head * a.q.hs, a.q.ts, rows, a.D, lane);
    g.init(static_cast<const T *>(a.go.p) + first * a.go.ts + head * a.go.hs, a.go.ts, rows, a.D, lane);
    float lse = INFINITY;
    const float delta = row_delta<T, DC, kHold<T, DC>>(a, head, first, rows, g, lane);
    if ((lane & 31) < rows) {
        const int64_t at = (int64_t)head * a.Tq + first + (lane & 31);
        lse = a.lse[at];
        if (part.delta && blockIdx.y == 0 && side == 0 && lane < 32) part.delta[at] = delta;
    }
    const float c = a.scale * kLog2e;
    floatx16 acc[DC / 32];
#pragma unroll
    for (int t = 0; t < DC / 32; ++t) acc[t] = zero16x();
    // 32 keys, from row n of the stage on.
    auto tile = [&](const char *kt, const char *vt, int k, int n, auto mode) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(mode)::value;
        const bool masked = MASKED && k + n + 32 > wfull;
        floatx16 x = zero16x(), y = zero16x();
#pragma unroll
        for (int i = 0; i < DC / M::KC; ++i) {
            x = M::mma(Ti::row_frag(kt, n, i, lane), q.get(i, lane), x);
            y = M::mma(Ti::row_frag(vt, n, i, lane), g.get(i, lane), y);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -lse)) * (y[i] - delta);
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = k + n + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) > last ? 0.f : x[i];
        }
        // (there dS is rounded once: rows that see the infinity or NaN are none, the others have a rounding more)
        const bool wild = masked && any_wild<T, DP, 32>(kt, n, lane);
        if (sizeof(T) == 4 || wild) {
            Frag d[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) d[i] = as_frag<T>(x, i);
            if (wild) wild_product<T, DP, DC, NP>(acc, kt, n, d, 0, last - k - n, lane);
            else add_product<T, DP, DC, NP>(acc, kt, n, d, lane);
            return;
        }
        add_exactly<T, DP, DC>(acc, kt, n, x, lane);
    };
    auto step = [&](int k, auto mode) __attribute__((always_inline)) {
        tile_sync();
        if (k + BN * WG < end) issue(k + BN * WG);
        if (WG > 1 && k >= end) return;
        const char *kt = stages + (k / (BN * WG) & 1) * 2 * BYTES, *vt = kt + BYTES;
        if constexpr (sizeof(T) == 2 && decltype(mode)::value) {   // (in turn: unrolled, what the rare path holds would not fit the registers)
#pragma unroll 1
            for (int n = 0; n < BN && k + n < wend; n += 32) {
                int row = n;
                asm volatile("" : "+s"(row));   // (nothing of it is worked out before the loop and held)
                tile(kt, vt, k, row, mode);
            }
        } else {
#pragma unroll
            for (int n = 0; n < BN; n += 32)
                if (!decltype(mode)::value || k + n < wend) tile(kt, vt, k, n, mode);
        }
    };
    // Keys that all of the block's rows see, in whole steps; then the others.
    const int clear = max(begin, min(end, max(0, a.causal ? min(s.nb, row0 + 1 + shift) : s.nb) / BN * BN));
    int k = begin;
    for (; k + (WG - 1) * BN < clear; k += BN * WG) step(k + side * BN, Full{});
    for (; k < end; k += BN * WG) step(k + side * BN, Masked{});
    tile_sync();
    if constexpr (WG > 1) {   // the second group's sums to the first
        add_side<DC / 32>(lds + w * DC * 128, side, lane, [&](int t) -> floatx16 & { return acc[t]; });
        if (side) return;
    }
    if (rows <= 0) return;
    if (part.sums) {
        store_sums<DC>(acc, part.a + ((blockIdx.y * a.Tq + first) * a.Hq + head) * DC, (int64_t)a.Hq * DC, rows, lane);
        return;
    }
    store_rows<T, DP, DC>(acc, a.scale, last < 0, lds + w * 32 * Ti::RB, static_cast<T *>(a.dq.p) + first * a.dq.ts + head * a.dq.hs, a.dq.ts,
                      rows, a.D, lane);
}

// ------------------------------------------------------------------ dk, dv
template <typename T, int DC, bool DK, bool DV>
struct DkvShape {
    static constexpr int BM = kPitch<DC> * (int)sizeof(T) <= 256 ? 64 : 32;   // queries of a step
    // two blocks a CU where the sums and operands that a wave keeps leave registers for the rest
    static constexpr int KEPT = DC / 2 * (DK + DV) + DC / 8 * (int)sizeof(T) * (DK ? 2 : 1);
    static constexpr int OCC = kPitch<DC> * (int)sizeof(T) <= 256 && KEPT <= (sizeof(T) == 2 ? 128 : 96) ? 2 : 1;
};

// WG as dq_kernel's.
template <typename T, int DC, bool DK, bool DV, int WG>
__global__ __launch_bounds__(256 * WG, (DkvShape<T, DC, DK, DV>::OCC / WG)) void dkv_kernel(AttnArgs a, Parts part) {
    constexpr int DP = kPitch<DC>;
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    typedef typename M::Frag Frag;
    constexpr int BM = DkvShape<T, DC, DK, DV>::BM, NP = 32 / M::KC, BYTES = BM * Ti::RB, C = DC / M::KC;
    constexpr int STAGE = 2 * BYTES + 512;   // q, g, and 64 each of lse and delta
    __shared__ __align__(256) char lds[2 * STAGE * WG];
    const int lane = threadIdx.x & 63, w = WG > 1 ? uniform(threadIdx.x >> 6) & 3 : uniform(threadIdx.x >> 6), side = WG > 1 ? uniform(threadIdx.x >> 8) : 0;
    int hk, rank;
    find_head((int)blockIdx.x, a.Hk, hk, rank);
    const int group = a.Hq / a.Hk;
    const Span s = find_ranked(a.koff, a.qoff, a.n, (int)a.Tk, (int)a.Tq, rank, kRows, a.causal, false);
    const int key0 = s.tile * kRows;
    if (s.tile < 0 || key0 >= s.na) return;
    const int shift = s.na - s.nb;   // query i sees keys to i + shift
    const int begin = a.causal ? max(0, key0 - shift) / BM * BM : 0;
    const int steps = begin < s.nb ? (s.nb - begin + BM - 1) / BM : 0;   // of one head
    // Of these, the first ones, where some of the block's keys are hidden from some queries, are a loop
    // of their own before the others; both go through the heads of the group.
    const int edge = a.causal ? min(steps, (max(0, key0 + kRows - 1 - shift - begin) + BM - 1) / BM) : 0;
    const int wkey = key0 + 32 * w, keys = min(32, s.na - wkey);
    const int key = wkey + (lane & 31);

    const int64_t first = s.a0 + wkey;
    Loader<T, DP, BM, 4> lq, lg;
    lq.init(a.q.ts, a.D, w, lane);
    lg.init(a.go.ts, a.D, w, lane);
    const uint32_t word = lane < BM ? lane * 4 : 0x80000000u;
    // Step n of group * steps: a head of the group and its first query; the next one's.
    struct Place {
        int h, at;
    };
    const int split = begin + edge * BM, stop = begin + steps * BM;
    auto place_of = [&](int n) {
        const bool first = n < edge * group;
        const int m = first ? n : n - edge * group, per = first ? edge : steps - edge, h = m / per;
        return Place{h, (first ? begin : split) + (m - h * per) * BM};
    };
    auto after = [&](Place p) {
        const bool first = p.at < split;
        p.at += BM;
        if (p.at >= (first ? split : stop)) {
            ++p.h;
            p.at = first && p.h < group ? begin : split;
            if (p.h == group) p.h = 0;
        }
        return p;
    };
    char *stages = lds + side * 2 * STAGE;
    auto issue = [&](int n, const Place &p) {
        char *to = stages + (n / WG & 1) * STAGE;
        const int head = hk * group + p.h, at = p.at;
        const int64_t row = s.b0 + at;
        lq.issue(reinterpret_cast<const char *>(static_cast<const T *>(a.q.p) + row * a.q.ts + head * a.q.hs), s.nb - at, a.D, to, w);
        lg.issue(reinterpret_cast<const char *>(static_cast<const T *>(a.go.p) + row * a.go.ts + head * a.go.hs), s.nb - at, a.D, to + BYTES, w);
        if (w < (DK ? 2 : 1))
            g2::dma4s(g2::rsrc((w ? part.delta : a.lse) + head * a.Tq + row, (uint32_t)min(BM, s.nb - at) * 4), to + 2 * BYTES + 256 * w, word, 0);
    };
    const int first_step = (int)((int64_t)steps * group * blockIdx.y / part.splits);
    const int total = (int)((int64_t)steps * group * (blockIdx.y + 1) / part.splits);
    Place now{0, 0}, next{0, 0};
    if (first_step + side < total) {
        next = place_of(first_step + side);
        issue(first_step + side, next);
    }
    Rows<T, DC, kHold1<T, DC>> kf;
    Rows<T, DC, DK && kHold<T, DC>> vf;
    kf.init(static_cast<const T *>(a.k.p) + first * a.k.ts + hk * a.k.hs, a.k.ts, keys, a.D, lane);
    if constexpr (DK) vf.init(static_cast<const T *>(a.v.p) + first * a.v.ts + hk * a.v.hs, a.v.ts, keys, a.D, lane);
    const float c = a.scale * kLog2e;
    floatx16 dk[DC / 32], dv[DC / 32];
#pragma unroll
    for (int t = 0; t < DC / 32; ++t) dk[t] = dv[t] = zero16x();
    // 32 queries, from row m of the stage on.
    auto tile = [&](int at, const char *qt, const char *gt, int m, auto mode) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(mode)::value;
        const float *lt = reinterpret_cast<const float *>(gt + BYTES), *dt = lt + 64;
        if (DK && DV && WG > 1) __builtin_amdgcn_sched_barrier(0);   // (both tiles at once do not fit the registers)
        // (rows past the last query are zeros; a wave without keys has nothing to do)
        if (MASKED && (keys <= 0 || min(at + m + 32, s.nb) - 1 + shift < wkey)) return;
        const bool masked = MASKED && at + m + shift < wkey + 31;
        floatx16 x = zero16x(), y = zero16x();
#pragma unroll
        for (int i = 0; i < C; ++i) {
            x = M::mma(Ti::row_frag(qt, m, i, lane), kf.get(i, lane), x);
            if constexpr (DK) y = M::mma(Ti::row_frag(gt, m, i, lane), vf.get(i, lane), y);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int r = m + 8 * g + 4 * (lane >> 5);
            const floatx4 l4 = *reinterpret_cast<const floatx4 *>(lt + r);
            floatx4 d4{};
            if constexpr (DK) d4 = *reinterpret_cast<const floatx4 *>(dt + r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool hidden = masked && key > at + r + j + shift;
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * g + j], c, -l4[j]));
                x[4 * g + j] = hidden ? 0.f : p;
                if constexpr (DK) y[4 * g + j] = hidden ? 0.f : p * (y[4 * g + j] - d4[j]);
            }
        }
        // Past the last query: zeros, also where a score is none, such as 0 times a key's infinity.
        if (at + m + 32 > s.nb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool past = at + m + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) >= s.nb;
                x[i] = past ? 0.f : x[i];
                y[i] = past ? 0.f : y[i];
            }
        }
        // (an operand: in bf16 rounded, P to 8 bits)
        Frag f[NP];
        const int lo = a.causal ? key - shift - at - m : 0, hi = s.nb - 1 - at - m;   // rows that see the lane's key
        if constexpr (DV) {
#pragma unroll
            for (int i = 0; i < NP; ++i) f[i] = as_frag<T>(x, i);
            if (masked && any_wild<T, DP, 32>(gt, m, lane)) wild_product<T, DP, DC, NP>(dv, gt, m, f, lo, hi, lane);
            else add_product<T, DP, DC, NP>(dv, gt, m, f, lane);
        }
        if constexpr (DK) {
            const bool wild = masked && any_wild<T, DP, 32>(qt, m, lane);
            if (sizeof(T) == 4 || wild) {
#pragma unroll
                for (int i = 0; i < NP; ++i) f[i] = as_frag<T>(y, i);
                if (wild) wild_product<T, DP, DC, NP>(dk, qt, m, f, lo, hi, lane);
                else add_product<T, DP, DC, NP>(dk, qt, m, f, lane);
            } else {
                add_exactly<T, DP, DC>(dk, qt, m, y, lane);
            }
        }
    };
    auto step = [&](int n, auto mode) __attribute__((always_inline)) {
        tile_sync();
        now = next;
#pragma unroll
        for (int k = 0; k < WG; ++k) next = after(next);
        if (n + WG < total) issue(n + WG, next);
        if (WG > 1 && n >= total) return;
        const int at = now.at;
        const char *qt = stages + (n / WG & 1) * STAGE, *gt = qt + BYTES;
        if constexpr (sizeof(T) == 2 && decltype(mode)::value && DK) {   // (in turn, as dq_kernel's)
#pragma unroll 1
            for (int m = 0; m < BM; m += 32) {
                int row = m;
                asm volatile("" : "+s"(row));
                tile(at, qt, gt, row, mode);
            }
        } else {
#pragma unroll
            for (int m = 0; m < BM; m += 32) tile(at, qt, gt, m, mode);
        }
    };
    const int hidden_to = max(first_step, min(total, edge * group));
    int n = first_step;
    for (; n < hidden_to; n += WG) step(n + side, Masked{});
    for (; n < total; n += WG) step(n + side, Full{});
    tile_sync();
    if constexpr (WG > 1) {   // the second group's sums to the first
        if constexpr (DK) add_side<DC / 32>(lds + w * DC * 128, side, lane, [&](int t) -> floatx16 & { return dk[t]; });
        if constexpr (DV) add_side<DC / 32>(lds + w * DC * 128, side, lane, [&](int t) -> floatx16 & { return dv[t]; });
        if (side) return;
    }
    if (keys <= 0) return;
    if (part.sums) {
        const int64_t at = ((blockIdx.y * a.Tk + first) * a.Hk + hk) * DC;
        if constexpr (DK) store_sums<DC>(dk, part.a + at, (int64_t)a.Hk * DC, keys, lane);
        if constexpr (DV) store_sums<DC>(dv, part.b + at, (int64_t)a.Hk * DC, keys, lane);
        return;
    }
    char *mine = lds + w * 32 * Ti::RB;
    if constexpr (DK)
        store_rows<T, DP, DC>(dk, a.scale, false, mine, static_cast<T *>(a.dk.p) + first * a.dk.ts + hk * a.dk.hs, a.dk.ts, keys, a.D, lane);
    if constexpr (DV)
        store_rows<T, DP, DC>(dv, 1.f, false, mine, static_cast<T *>(a.dv.p) + first * a.dv.ts + hk * a.dv.hs, a.dv.ts, keys, a.D, lane);
}

// A gradient from its sums: a vector a thread.
struct Sum {
    HeadsView out;
    const float *part;
    float scale;
};

template <typename T>
__global__ __launch_bounds__(256) void sum_kernel(Sum a, Sum b, int64_t rows, int H, int D, int cols, int splits) {
    constexpr int V = Vec16<T>::N;
    const Sum &s = blockIdx.y ? b : a;
    const int per = D / V;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * H * per) return;
    const int64_t row = i / per, t = row / H;
    const int u = (int)(i - row * per), h = (int)(row - t * H);
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    for (int n = 0; n < splits; ++n) {
        const float *p = s.part + (n * rows * H + row) * cols + u * V;
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += p[e];
    }
    Vec16<T> o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(v[e] * s.scale);
    store16(static_cast<T *>(s.out.p) + t * s.out.ts + h * s.out.hs + u * V, o);
}

// ------------------------------------------------------------------ host
namespace {

size_t al256(size_t n) { return (n + 255) / 256 * 256; }

// What a backward lays out: delta, then sums of dq, dk and dv; the steps of their blocks.
struct Plan {
    int dq_splits, dkv_splits;
    bool dq_sums, dkv_sums;
    int64_t dq_steps, dkv_steps;
    size_t dq_at, dk_at, dv_at, bytes;
};

template <typename T, int DC>
Plan plan(const AttnArgs &a, bool dq, bool dk, bool dv) {
    const bool packed = a.qoff != nullptr;
    const int64_t n = packed ? std::max(a.n, 1) : 1, group = a.Hq / a.Hk;
    Plan p{1, 1, false, false, a.Tk / n / DqShape<T, DC>::BN, a.Tq / n * group / DkvShape<T, DC, true, true>::BM, 0, 0, 0, 0};
    if (dq) p.dq_splits = span_splits<T>(span_slots(packed, a.n, a.Tq, kRows) * a.Hq, p.dq_steps, a.Tq * a.Hq * DC * 4);
    if (dk || dv) p.dkv_splits = span_splits<T>(span_slots(packed, a.n, a.Tk, kRows) * a.Hk, p.dkv_steps, a.Tk * a.Hk * DC * 8);
    p.dq_steps /= p.dq_splits;
    p.dkv_steps /= p.dkv_splits;
    p.dq_sums = dq && (p.dq_splits > 1 || a.shared);
    p.dkv_sums = p.dkv_splits > 1 || a.shared;
    const size_t keys = p.dkv_sums ? al256((size_t)p.dkv_splits * a.Tk * a.Hk * DC * sizeof(float)) : 0;
    p.dq_at = dk ? al256((size_t)a.Tq * a.Hq * sizeof(float)) : 0;
    p.dk_at = p.dq_at + (p.dq_sums ? al256((size_t)p.dq_splits * a.Tq * a.Hq * DC * sizeof(float)) : 0);
    p.dv_at = p.dk_at + (dk ? keys : 0);
    p.bytes = p.dv_at + (dv ? keys : 0);
    return p;
}

template <typename T, int DC>
size_t space(const AttnArgs &a, bool dq, bool dk, bool dv) {
    return plan<T, DC>(a, dq, dk, dv).bytes;
}

template <typename T, int DC, bool DK, bool DV>
void dkv_run(dim3 grid, bool few, const AttnArgs &a, const Parts &part, hipStream_t st) {
    if constexpr (sizeof(T) == 2 && DkvShape<T, DC, DK, DV>::OCC == 2) {
        if (few) {
            hipLaunchKernelGGL((dkv_kernel<T, DC, DK, DV, 2>), grid, dim3(512), 0, st, a, part);
            return;
        }
    }
    hipLaunchKernelGGL((dkv_kernel<T, DC, DK, DV, 1>), grid, dim3(256), 0, st, a, part);
}

template <typename T, int DC>
int run(const AttnArgs &a, char *ws, hipStream_t st) {
    const bool packed = a.qoff != nullptr, dq = a.dq.p, dk = a.dk.p, dv = a.dv.p;
    const Plan p = plan<T, DC>(a, dq, dk, dv);
    constexpr int V = Vec16<T>::N;
    float *delta = reinterpret_cast<float *>(ws), *dq_sums = reinterpret_cast<float *>(ws + p.dq_at),
          *dk_sums = reinterpret_cast<float *>(ws + p.dk_at), *dv_sums = reinterpret_cast<float *>(ws + p.dv_at);
    if (dk && !dq && a.Tq > 0) {
        hipLaunchKernelGGL((delta_kernel<T, DC>), dim3((unsigned)((a.Tq + 127) / 128), (unsigned)a.Hq), dim3(256), 0, st, a, delta);
    }
    if (dq && a.Tq > 0) {
        const int64_t slots = span_slots(packed, a.n, a.Tq, kRows);
        const Parts part{dk ? delta : nullptr, p.dq_splits, p.dq_sums, dq_sums, nullptr};
        const dim3 grid((unsigned)(slots * a.Hq), (unsigned)part.splits);
        constexpr bool pairs = sizeof(T) == 2 && DqShape<T, DC>::OCC == 2;
        if (pairs && wide_blocks((int64_t)grid.x * grid.y, p.dq_steps, 24)) {
            if constexpr (pairs) hipLaunchKernelGGL((dq_kernel<T, DC, 2>), grid, dim3(512), 0, st, a, part);
        } else {
            hipLaunchKernelGGL((dq_kernel<T, DC, 1>), grid, dim3(256), 0, st, a, part);
        }
    }
    if ((dk || dv) && a.Tk > 0) {
        const int64_t slots = span_slots(packed, a.n, a.Tk, kRows);
        const Parts part{delta, p.dkv_splits, p.dkv_sums, dk_sums, dv_sums};
        const dim3 grid((unsigned)(slots * a.Hk), (unsigned)part.splits);
        // Both at once up to where both sums and their operands are in a wave's registers: four products
        // instead of five (1777 x 2 heads of 72 in fp32: 74 us against 57 and 49).
        constexpr bool both = DC <= (sizeof(T) == 2 ? 128 : 96);
        // Blocks of two groups (attn_tile.h): dk and dv each for itself where a CU does not hold both sums of eight waves,
        // the same for all masks, so that a gradient's bits do not depend on which others are asked for.  (7 sequences of
        // 8192 rows, 32 on 8 heads, bf16: dv alone of 128 columns 208 -> 169 us, dk alone 390 -> 311, both 450 -> 475; of 64
        // columns 136 -> 110, 243 -> 195, 266 -> 230.  4 x 2048 rows, 8 heads of 128, 32 steps: both 127 -> 151.  In fp32 two
        // kernels instead of one cost more, 8 on 2 heads of 64 483 -> 591.)
        const bool few = sizeof(T) == 2 && DkvShape<T, DC, true, false>::OCC == 2 && wide_blocks((int64_t)grid.x * grid.y, p.dkv_steps, 40);
        if (both && dk && dv && !(few && DkvShape<T, DC, true, true>::OCC == 1)) {
            if constexpr (both) dkv_run<T, DC, true, true>(grid, few, a, part, st);
        } else {
            if (dk) dkv_run<T, DC, true, false>(grid, few, a, part, st);
            if (dv) dkv_run<T, DC, false, true>(grid, few, a, part, st);
        }
    }
    // (gradients may lie where the kernels above read)
    if (p.dq_sums && a.Tq > 0) {
        const Sum s{a.dq, dq_sums, a.scale};
        hipLaunchKernelGGL(sum_kernel<T>, dim3((unsigned)((a.Tq * a.Hq * (a.D / V) + 255) / 256)), dim3(256), 0, st, s, s, a.Tq, a.Hq, a.D, DC,
                           p.dq_splits);
    }
    if ((dk || dv) && p.dkv_sums && a.Tk > 0) {
        const Sum k{a.dk, dk_sums, a.scale}, v{a.dv, dv_sums, 1.f};
        hipLaunchKernelGGL(sum_kernel<T>, dim3((unsigned)((a.Tk * a.Hk * (a.D / V) + 255) / 256), dk && dv ? 2 : 1), dim3(256), 0, st,
                           dk ? k : v, v, a.Tk, a.Hk, a.D, DC, p.dkv_splits);
    }
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace att

size_t attention_bwd_workspace(int dtype, const AttnArgs &a, bool dq, bool dk, bool dv) {
    return dtype == kBF16 ? ATT_COLUMNS(att::space, bf16, a, dq, dk, dv) : ATT_COLUMNS(att::space, float, a, dq, dk, dv);
}

int launch_attention_bwd(int dtype, const AttnArgs &a, void *ws, void *stream) {
    char *w = static_cast<char *>(ws);
    hipStream_t st = (hipStream_t)stream;
    return dtype == kBF16 ? ATT_COLUMNS(att::run, bf16, a, w, st) : ATT_COLUMNS(att::run, float, a, w, st);
}

}  // namespace ms
