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
// Bound: matrix cores, 3 products in dq, 2 in dv alone, 3 in dk alone, 4 in both.
#include <algorithm>

#include "attn_tile.h"

namespace ms {
namespace att {

// delta[h][t] = sum over d of g o, a row by L lanes.
template <typename T, int L>
__global__ __launch_bounds__(256) void delta_kernel(AttnArgs a) {
    constexpr int V = Vec16<T>::N;
    const int l = threadIdx.x % L;
    const int64_t n = a.Tq * a.Hq;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L; i < n; i += (int64_t)gridDim.x * (256 / L)) {
        const int64_t t = i / a.Hq;
        const int h = (int)(i - t * a.Hq);
        float s = 0.f;
        if (l * V < a.D) {
            const Vec16<T> x = load16(static_cast<const T *>(a.o.p) + t * a.o.ts + h * a.o.hs + l * V);
            const Vec16<T> y = load16(static_cast<const T *>(a.go.p) + t * a.go.ts + h * a.go.hs + l * V);
#pragma unroll
            for (int e = 0; e < V; ++e) s += to_f32(x.e[e]) * to_f32(y.e[e]);
        }
#pragma unroll
        for (int d = 1; d < L; d *= 2) s += __shfl_xor(s, d);
        if (l == 0) a.delta[h * a.Tq + t] = s;
    }
}

// ------------------------------------------------------------------ dq
constexpr int kRows = 128;   // queries of a block of dq, keys of a block of dk and dv

// Whether a wave has registers for both operands that it keeps: not for 256 fp32 elements.
template <typename T, int DP> constexpr bool kHold = DP * sizeof(T) < 1024;

template <typename T, int DP>
struct DqShape {
    static constexpr int BN = DP * (int)sizeof(T) <= 256 ? 64 : 32;
    static constexpr int OCC = DP * (int)sizeof(T) <= 256 ? 2 : 1;
};

template <typename T, int DP>
__global__ __launch_bounds__(256, (DqShape<T, DP>::OCC)) void dq_kernel(AttnArgs a, int slots) {
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    typedef typename M::Frag Frag;
    constexpr int BN = DqShape<T, DP>::BN, NP = 32 / M::KC, BYTES = BN * Ti::RB;
    __shared__ __align__(16) char lds[4 * BYTES];
    const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
    const int logical = xcd_remap((int)blockIdx.x, (int)gridDim.x);
    const int head = logical / slots, hk = head / (a.Hq / a.Hk);
    const Span s = find_span(a.qoff, a.koff, a.n, (int)a.Tq, (int)a.Tk, slots - 1 - logical % slots, kRows);
    const int row0 = s.tile * kRows;
    if (s.tile < 0 || row0 >= s.na) return;
    const int shift = s.nb - s.na;
    const int end = a.causal ? min(s.nb, min(row0 + kRows, s.na) + shift) : s.nb;
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
    auto issue = [&](int k) {
        char *to = lds + (k / BN & 1) * 2 * BYTES;
        lk.issue(kp + k * lk.ts, s.nb - k, a.D, to, w);
        lv.issue(vp + k * lv.ts, s.nb - k, a.D, to + BYTES, w);
    };
    if (end > 0) issue(0);
    Rows<T, DP> q;
    Rows<T, DP, kHold<T, DP>> g;
    q.init(static_cast<const T *>(a.q.p) + first * a.q.ts + head * a.q.hs, a.q.ts, rows, a.D, lane);
    g.init(static_cast<const T *>(a.go.p) + first * a.go.ts + head * a.go.hs, a.go.ts, rows, a.D, lane);
    float lse = INFINITY, delta = 0.f;
    if ((lane & 31) < rows) {
        lse = a.lse[(int64_t)head * a.Tq + first + (lane & 31)];
        delta = a.delta[(int64_t)head * a.Tq + first + (lane & 31)];
    }
    const float c = a.scale * kLog2e;
    floatx16 acc[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = zero16x();
    for (int k = 0; k < end; k += BN) {
        tile_sync();
        if (k + BN < end) issue(k + BN);
        const char *kt = lds + (k / BN & 1) * 2 * BYTES, *vt = kt + BYTES;
#pragma unroll
        for (int n = 0; n < BN; n += 32) {
            if (k + n >= wend) continue;
            floatx16 x = zero16x(), y = zero16x();
#pragma unroll
            for (int i = 0; i < DP / M::KC; ++i) {
                x = M::mma(Ti::row_frag(kt, n, i, lane), q.get(i, lane), x);
                y = M::mma(Ti::row_frag(vt, n, i, lane), g.get(i, lane), y);
            }
            const bool masked = k + n + 32 > wfull;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -lse)) * (y[i] - delta);
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (k + n + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) > last) x[i] = 0.f;
            }
            Frag d[NP];   // (an operand: in bf16 rounded)
#pragma unroll
            for (int i = 0; i < NP; ++i) d[i] = as_frag<T>(x, i);
            if (masked && any_wild<T, DP, 32>(kt, n, lane)) wild_product<T, DP, NP>(acc, kt, n, d, lane);
            else add_product<T, DP, NP>(acc, kt, n, d, lane);
        }
    }
    tile_sync();
    if (rows <= 0) return;
    store_rows<T, DP>(acc, a.scale, last < 0, lds + w * 32 * Ti::RB, static_cast<T *>(a.dq.p) + first * a.dq.ts + head * a.dq.hs, a.dq.ts,
                      rows, a.D, lane);
}

// ------------------------------------------------------------------ dk, dv
template <typename T, int DP>
struct DkvShape {
    static constexpr int BM = DP * (int)sizeof(T) <= 256 ? 64 : 32;   // queries of a step
};

template <typename T, int DP, bool DK, bool DV>
__global__ __launch_bounds__(256, DP == 64 && sizeof(T) == 2 ? 2 : 1) void dkv_kernel(AttnArgs a, int slots) {
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    typedef typename M::Frag Frag;
    constexpr int BM = DkvShape<T, DP>::BM, NP = 32 / M::KC, BYTES = BM * Ti::RB, C = DP / M::KC;
    constexpr int STAGE = 2 * BYTES + 512;   // q, g, and 64 each of lse and delta
    __shared__ __align__(16) char lds[2 * STAGE];
    const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
    const int logical = xcd_remap((int)blockIdx.x, (int)gridDim.x);
    const int hk = logical / slots, group = a.Hq / a.Hk;
    // (the first keys of a causal sequence take longest: first)
    const Span s = find_span(a.koff, a.qoff, a.n, (int)a.Tk, (int)a.Tq, logical % slots, kRows);
    const int key0 = s.tile * kRows;
    if (s.tile < 0 || key0 >= s.na) return;
    const int shift = s.na - s.nb;   // query i sees keys to i + shift
    const int begin = a.causal ? max(0, key0 - shift) / BM * BM : 0;
    const int steps = begin < s.nb ? (s.nb - begin + BM - 1) / BM : 0;   // of one head
    const int wkey = key0 + 32 * w, keys = min(32, s.na - wkey);
    const int key = wkey + (lane & 31);

    const int64_t first = s.a0 + wkey;
    Loader<T, DP, BM, 4> lq, lg;
    lq.init(a.q.ts, a.D, w, lane);
    lg.init(a.go.ts, a.D, w, lane);
    const uint32_t word = lane < BM ? lane * 4 : 0x80000000u;
    auto issue = [&](int n) {   // step n of group * steps
        char *to = lds + (n & 1) * STAGE;
        const int head = hk * group + n / steps, at = begin + n % steps * BM;
        const int64_t row = s.b0 + at;
        lq.issue(reinterpret_cast<const char *>(static_cast<const T *>(a.q.p) + row * a.q.ts + head * a.q.hs), s.nb - at, a.D, to, w);
        lg.issue(reinterpret_cast<const char *>(static_cast<const T *>(a.go.p) + row * a.go.ts + head * a.go.hs), s.nb - at, a.D, to + BYTES, w);
        if (w < (DK ? 2 : 1))
            g2::dma4s(g2::rsrc((w ? a.delta : a.lse) + head * a.Tq + row, (uint32_t)min(BM, s.nb - at) * 4), to + 2 * BYTES + 256 * w, word, 0);
    };
    const int total = steps * group;
    if (total > 0) issue(0);
    Rows<T, DP> kf;
    Rows<T, DP, DK && kHold<T, DP>> vf;
    kf.init(static_cast<const T *>(a.k.p) + first * a.k.ts + hk * a.k.hs, a.k.ts, keys, a.D, lane);
    if constexpr (DK) vf.init(static_cast<const T *>(a.v.p) + first * a.v.ts + hk * a.v.hs, a.v.ts, keys, a.D, lane);
    const float c = a.scale * kLog2e;
    floatx16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) dk[t] = dv[t] = zero16x();
    for (int n = 0; n < total; ++n) {
        tile_sync();
        if (n + 1 < total) issue(n + 1);
        const int at = begin + n % steps * BM;
        const char *qt = lds + (n & 1) * STAGE, *gt = qt + BYTES;
        const float *lt = reinterpret_cast<const float *>(gt + BYTES), *dt = lt + 64;
#pragma unroll
        for (int m = 0; m < BM; m += 32) {
            const int top = min(at + m + 32, s.nb);   // queries below it
            if (keys <= 0 || at + m >= s.nb || (a.causal && top - 1 + shift < wkey)) continue;
            floatx16 x = zero16x(), y = zero16x();
#pragma unroll
            for (int i = 0; i < C; ++i) {
                x = M::mma(Ti::row_frag(qt, m, i, lane), kf.get(i, lane), x);
                if constexpr (DK) y = M::mma(Ti::row_frag(gt, m, i, lane), vf.get(i, lane), y);
            }
            const bool masked = a.causal && at + m + shift < wkey + 31;
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
            // (both are operands: in bf16 rounded)
            Frag f[NP];
            if constexpr (DV) {
#pragma unroll
                for (int i = 0; i < NP; ++i) f[i] = as_frag<T>(x, i);
                if (masked && any_wild<T, DP, 32>(gt, m, lane)) wild_product<T, DP, NP>(dv, gt, m, f, lane);
                else add_product<T, DP, NP>(dv, gt, m, f, lane);
            }
            if constexpr (DK) {
#pragma unroll
                for (int i = 0; i < NP; ++i) f[i] = as_frag<T>(y, i);
                if (masked && any_wild<T, DP, 32>(qt, m, lane)) wild_product<T, DP, NP>(dk, qt, m, f, lane);
                else add_product<T, DP, NP>(dk, qt, m, f, lane);
            }
        }
    }
    tile_sync();
    if (keys <= 0) return;
    char *mine = lds + w * 32 * Ti::RB;
    if constexpr (DK)
        store_rows<T, DP>(dk, a.scale, false, mine, static_cast<T *>(a.dk.p) + first * a.dk.ts + hk * a.dk.hs, a.dk.ts, keys, a.D, lane);
    if constexpr (DV)
        store_rows<T, DP>(dv, 1.f, false, mine, static_cast<T *>(a.dv.p) + first * a.dv.ts + hk * a.dv.hs, a.dv.ts, keys, a.D, lane);
}

// ------------------------------------------------------------------ host
namespace {

template <typename T, int DP>
void run(const AttnArgs &a, hipStream_t st) {
    const bool packed = a.qoff != nullptr;
    if ((a.dq.p || a.dk.p) && a.Tq > 0) {
        constexpr int L = DP / Vec16<T>::N;
        const int64_t blocks = (a.Tq * a.Hq + 256 / L - 1) / (256 / L);
        hipLaunchKernelGGL((delta_kernel<T, L>), dim3((unsigned)std::min<int64_t>(blocks, 8192)), dim3(256), 0, st, a);
    }
    if (a.dq.p && a.Tq > 0) {
        const int64_t slots = span_slots(packed, a.n, a.Tq, kRows);
        hipLaunchKernelGGL((dq_kernel<T, DP>), dim3((unsigned)(slots * a.Hq)), dim3(256), 0, st, a, (int)slots);
    }
    if ((a.dk.p || a.dv.p) && a.Tk > 0) {
        const int64_t slots = span_slots(packed, a.n, a.Tk, kRows);
        const dim3 grid((unsigned)(slots * a.Hk));
        // (both sums of 512 bytes a row, and their operands, are more than a wave's registers)
        constexpr bool both = DP * sizeof(T) < 512;
        if constexpr (both) {
            if (a.dk.p && a.dv.p) {
                hipLaunchKernelGGL((dkv_kernel<T, DP, true, true>), grid, dim3(256), 0, st, a, (int)slots);
                return;
            }
        }
        if (a.dk.p) hipLaunchKernelGGL((dkv_kernel<T, DP, true, false>), grid, dim3(256), 0, st, a, (int)slots);
        if (a.dv.p) hipLaunchKernelGGL((dkv_kernel<T, DP, false, true>), grid, dim3(256), 0, st, a, (int)slots);
    }
}

template <typename T>
int bwd_t(const AttnArgs &a, hipStream_t st) {
    if (a.D <= 64) run<T, 64>(a, st);
    else if (a.D <= 128) run<T, 128>(a, st);
    else run<T, 256>(a, st);
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace att

int launch_attention_bwd(int dtype, const AttnArgs &a, void *stream) {
    return dtype == kBF16 ? att::bwd_t<bf16>(a, (hipStream_t)stream) : att::bwd_t<float>(a, (hipStream_t)stream);
}

}  // namespace ms
