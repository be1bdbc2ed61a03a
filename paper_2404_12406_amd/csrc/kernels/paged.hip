// Attention of one query a sequence over a paged cache: o = softmax(scale q k^T) v over the
// first lengths[b] places of the pages that tables[b] lists.
//
// Bound: memory, one read of the keys and values that are used, however many query heads
// share them: these are the columns of a 32x32 tile (attn_tile.h), up to 32 at once.
//  * A block takes `per` keys of one sequence and head of the cache, and each of its waves
//    32 keys at a time on its own: a wave's loads go straight into its own part of LDS, and
//    nothing waits for another wave before the end.  The next keys are loaded as soon as
//    this step's scores are taken, the next values after its sums; eight such waves a CU
//    keep some 100 KiB in flight.  (Two steps ahead, with half as many waves, was slower:
//    one wave a SIMD has to wait for each of its own instructions.)
//  * The pages of a step's keys are loaded a step before these, into LDS too, so that
//    the loads follow each other in one order and the waits count them.
//  * A key's row is looked up by itself, so pages may have any size and end anywhere.  Rows
//    past the length read as zeros, whatever lies there; rows of a page that is none make
//    their scores NaN.
//  * Softmax statistics and sums of a block's waves meet in LDS, those of a
//    sequence's blocks in join_kernel, in a fixed order.
// bf16, 32 on 8 heads of 128: 64 sequences of 400000 keys in all 290 us, 5.6 TB/s (a device copy reaches 5.1); one of
// 4111 keys in pages of 16 some 10 us, two launches.
#include <algorithm>

#include "../paged_plan.h"
#include "attn_tile.h"

namespace ms {
namespace att {

static __device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};

// 16 (4) bytes a lane from its own address to lds + 16 l (4 l); as g2::dma16<true>.
__device__ __forceinline__ void far16(const void *p, char *lds) {
    const uint32_t base = (uint32_t)(uintptr_t)(g2::lds_void_t *)lds;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(base));
}
__device__ __forceinline__ void far4(const void *p, char *lds) {
    const uint32_t base = (uint32_t)(uintptr_t)(g2::lds_void_t *)lds;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(p), "s"(base));
}

// What a wave's loads have left in LDS may be read: the compiler knows of neither.
template <int N>
__device__ __forceinline__ void landed() {
    g2::wait_vmcnt<(N < 63 ? N : 63)>();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

template <typename T, int DP>
struct PagedShape {
    static constexpr int RB = DP * (int)sizeof(T);
    static constexpr int NW = RB <= 256 ? 4 : 1024 / RB;               // waves of a block
    static constexpr int HALF = 32 * RB, WAVE = 2 * HALF + 768;        // keys, values, pages of two steps
    static constexpr int LOADS = HALF / 1024;                          // of a step's keys, of its values
    static constexpr int PER_SIMD = RB <= 256 ? 2 : 1;                 // waves: two blocks a CU
    static constexpr int LD = DP + 4;                                  // a row of sums at the end
    static_assert(32 * LD * 4 <= WAVE, "the sums fit where the keys were");
};

// FAST: rows of the cache are whole 16-byte vectors, so aligned; else they go through
// registers, any number of elements side by side.
template <typename T, int DP, bool FAST>
__global__ __launch_bounds__((64 * PagedShape<T, DP>::NW), (PagedShape<T, DP>::PER_SIMD)) void paged_kernel(PagedArgs a, int splits, int per, float *__restrict__ part) {
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    typedef PagedShape<T, DP> Sh;
    typedef typename M::Frag Frag;
    constexpr int NW = Sh::NW, NP = 32 / M::KC, LD = Sh::LD;
    __shared__ __align__(256) char lds[NW * Sh::WAVE + NW * 256];
    const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), hh = lane >> 5;
    const int group = a.Hq / a.Hk;
    const int split = (int)(blockIdx.x % splits), hk = (int)(blockIdx.x / splits % a.Hk), b = (int)(blockIdx.x / splits / a.Hk);
    const int g0 = (int)blockIdx.y * 32, heads = min(32, group - g0);   // the block's queries
    const int head = hk * group + g0;
    const int64_t room = (int64_t)a.width * a.page;
    int len = uniform(a.lengths[b]);
    const bool wrong = len > room;
    if (wrong || len < 0) len = 0;
    const int begin = (int)min((int64_t)split * per, (int64_t)len), end = (int)min((int64_t)begin + per, (int64_t)len);
    if (split > 0 && begin >= end) return;   // (the join knows how many there are)

    char *mine = lds + w * Sh::WAVE, *kt = mine, *vt = mine + Sh::HALF, *pages = mine + 2 * Sh::HALF;
    const int32_t *table = a.tables + (int64_t)b * a.width;
    const uint32_t magic = a.page > 1 ? (uint32_t)((uint64_t(1) << 32) / (uint32_t)a.page) : ~0u;
    auto divide = [&](int key, int &in) {   // by the page size
        int q = (int)__umulhi((uint32_t)key, magic);
        in = key - q * a.page;
        if (in >= a.page) {
            in -= a.page;
            ++q;
        }
        return q;
    };
    // Step i: the places of its keys in their pages; their pages are asked for.
    auto look = [&](int i) {
        const int key = min(begin + (i * NW + w) * 32 + (lane & 31), len - 1);
        int in;
        far4(table + divide(key, in), pages + (i & 1) * 256);
        return in;
    };
    uint32_t row = ~0u;       // of the cache, of key l % 32; ~0 for none
    auto at = [&](int n) { return (uint32_t)__shfl((int)row, (n * 64 + lane) / Ti::U); };   // of load n's
    bool whole;               // of 32 keys and all of the columns
    // The rows of step i; which keys have a page that is none.
    auto find = [&](int i, int in) {
        const int k = begin + (i * NW + w) * 32;
        const int pg = *reinterpret_cast<const int *>(pages + (i & 1) * 256 + 4 * (lane & 31));
        const bool used = k + (lane & 31) < end, none = used && (uint32_t)pg >= (uint32_t)a.pages;
        row = used && !none ? ((uint32_t)pg * (uint32_t)a.Hk + (uint32_t)hk) * (uint32_t)a.page + (uint32_t)in : ~0u;
        const uint32_t bad = (uint32_t)__ballot(none);
        whole = k + 32 <= end && !bad && a.D == DP;
        return bad;
    };
    auto issue = [&](const void *from, char *to) {
        const char *base = static_cast<const char *>(from);
        const uint32_t bytes = (uint32_t)a.D * (uint32_t)sizeof(T);
        if (FAST && whole) {
#pragma unroll
            for (int n = 0; n < Sh::LOADS; ++n) {
                const int idx = n * 64 + lane, unit = (idx % Ti::U) ^ Ti::swz(idx / Ti::U);
                far16(base + ((uint64_t)at(n) * bytes + (uint32_t)(unit * 16)), to + n * 1024);
            }
            return;
        }
#pragma unroll
        for (int n = 0; n < Sh::LOADS; ++n) {
            const int idx = n * 64 + lane, unit = (idx % Ti::U) ^ Ti::swz(idx / Ti::U);
            const uint32_t r = at(n);
            const bool there = r != ~0u && unit * M::V < a.D;
            const char *p = base + (uint64_t)r * bytes;
            if constexpr (FAST) {
                far16(there ? (const void *)(p + unit * 16) : &kZeros, to + n * 1024);
            } else {
                Vec16<T> v = zero16<T>();
                if (there) v = load_vec<T>(reinterpret_cast<const T *>(p), unit * M::V, a.D);
                store16(reinterpret_cast<T *>(to + n * 1024 + lane * 16), v);
            }
        }
    };
    const int keys = end - begin - w * 32, steps = keys > 0 ? (keys + 32 * NW - 1) / (32 * NW) : 0;   // the wave's
    Rows<T, DP, (DP * sizeof(T) < 1024)> q;   // (256 fp32 elements are too many to hold)
    q.init(static_cast<const T *>(a.q) + b * a.qts + head * a.qhs, a.qhs, heads, a.D, lane);
    q.settle();
    uint32_t bad = 0u, bad1 = 0u;   // of this step and the next
    int in = 0;
    if (steps > 0) {
        in = look(0);
        landed<0>();
        bad = find(0, in);
        in = look(1);
        issue(a.kp, kt);
        issue(a.vp, vt);
    }
    const float c = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    floatx16 acc[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = zero16x();
    // On their way at the start of a step, in order: the next one's pages, its keys, its values.
    for (int i = 0; i < steps; ++i) {
        const bool more = i + 1 < steps;
        landed<FAST ? Sh::LOADS : 0>();   // all but the values
        floatx16 x = zero16x();
#pragma unroll
        for (int n = 0; n < DP / M::KC; ++n) x = M::mma(Ti::row_frag(kt, 0, n, lane), q.get(n, lane), x);
        if (more) {
            bad1 = find(i + 1, in);
            in = look(i + 2);
            __atomic_signal_fence(__ATOMIC_SEQ_CST);
            g2::wait_lgkm0();   // (the keys have been read)
            issue(a.kp, kt);
        }
        const int k = begin + (i * NW + w) * 32;
        if (k + 32 > end || bad) {
#pragma unroll
            for (int n = 0; n < 16; ++n) {
                const int r = 8 * (n >> 2) + 4 * hh + (n & 3);
                x[n] = bad >> r & 1 ? NAN : x[n];
                x[n] = k + r >= end ? -INFINITY : x[n];
            }
        }
        float top = x[0];
#pragma unroll
        for (int n = 1; n < 16; ++n) top = fmaxf(top, x[n]);
        top = both_max(top);
        if (__any(top > m)) {
            const float to = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
            l *= f;
#pragma unroll
            for (int t = 0; t < DP / 32; ++t)
#pragma unroll
                for (int n = 0; n < 16; ++n) acc[t][n] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            x[n] = __builtin_amdgcn_exp2f((x[n] - ref) * c);
            l += x[n];
        }
        Frag p[NP];
#pragma unroll
        for (int n = 0; n < NP; ++n) p[n] = as_frag<T>(x, n);
        if (more) landed<FAST ? Sh::LOADS + 1 : 0>();   // the values
        else landed<0>();
        add_product<T, DP, DP, NP>(acc, vt, 0, p, lane);
        if (more) {
            __atomic_signal_fence(__ATOMIC_SEQ_CST);
            g2::wait_lgkm0();   // (and the values)
            issue(a.vp, vt);
        }
        bad = bad1;
    }
    l = both_sum(l);
    // the waves' sums side by side: [queries][LD] each, and their statistics
    g2::wait_lgkm0();
    float *own = reinterpret_cast<float *>(mine);
    floatx2 *stat = reinterpret_cast<floatx2 *>(lds + NW * Sh::WAVE);
    if ((lane & 31) < heads) {
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                floatx4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = acc[t][4 * g + j];
                *reinterpret_cast<floatx4 *>(own + (lane & 31) * LD + 32 * t + 8 * g + 4 * hh) = v;
            }
    }
    if (lane < 32) stat[w * 32 + lane] = floatx2{m, l};
    __syncthreads();
    for (int i = threadIdx.x; i < heads * DP; i += 64 * NW) {
        const int n = i / DP, d = i % DP;
        if (d >= a.D) continue;
        float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
        for (int v = 0; v < NW; ++v) top = fmaxf(top, stat[v * 32 + n].x);
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const floatx2 s = stat[v * 32 + n];
            const float f = s.x == top ? 1.f : __builtin_amdgcn_exp2f((s.x - top) * c);
            sum += f * s.y;
            o += f * reinterpret_cast<const float *>(lds + v * Sh::WAVE)[n * LD + d];
        }
        if (splits == 1) {
            static_cast<T *>(a.o)[b * a.ots + (head + n) * a.ohs + d] = from_f32<T>(wrong ? NAN : len == 0 ? 0.f : o / sum);
        } else {
            const int64_t at = ((int64_t)b * a.Hq + head + n) * splits + split;
            part[2 * (int64_t)a.n * a.Hq * splits + at * a.D + d] = o;
            if (d == 0) reinterpret_cast<floatx2 *>(part)[at] = floatx2{top, sum};
        }
    }
}

// o of the splits that a sequence has: a block a query head.  Its threads are DL columns
// and 256 / DL groups, of every so many splits each.
template <typename T, int DL>
__global__ __launch_bounds__(256) void join_kernel(PagedArgs a, int splits, int per, const float *__restrict__ part) {
    constexpr int G = 256 / DL;
    __shared__ float weight[256], red[8], meet[G][DL + 1];
    const int b = (int)(blockIdx.x / a.Hq), head = (int)(blockIdx.x % a.Hq), d = threadIdx.x % DL, g = threadIdx.x / DL;
    const int len = a.lengths[b];
    const bool wrong = len > (int64_t)a.width * a.page;
    const int n = wrong ? 0 : (int)(((int64_t)max(len, 0) + per - 1) / per);
    const float c = a.scale * kLog2e;
    const floatx2 *stat = reinterpret_cast<const floatx2 *>(part) + (int64_t)blockIdx.x * splits;
    const float *p = part + 2 * (int64_t)a.n * a.Hq * splits + (int64_t)blockIdx.x * splits * a.D;
    float top = -INFINITY;
    for (int s = threadIdx.x; s < n; s += 256) top = fmaxf(top, stat[s].x);
#pragma unroll
    for (int k = 1; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float o = 0.f, sum = 0.f;
    for (int s0 = 0; s0 < n; s0 += 256) {
        const int m = min(256, n - s0);
        if (threadIdx.x < m) {
            const floatx2 st = stat[s0 + threadIdx.x];
            const float f = st.x == top ? 1.f : __builtin_amdgcn_exp2f((st.x - top) * c);
            weight[threadIdx.x] = f;
            sum += f * st.y;
        }
        __syncthreads();
        if (d < a.D) {
#pragma unroll 4
            for (int s = g; s < m; s += G) o += weight[s] * p[(int64_t)(s0 + s) * a.D + d];
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) red[4 + (threadIdx.x >> 6)] = sum;
    meet[g][d] = o;
    __syncthreads();
    if (g > 0 || d >= a.D) return;
    sum = red[4] + red[5] + red[6] + red[7];
#pragma unroll
    for (int k = 1; k < G; ++k) o += meet[k][d];
    static_cast<T *>(a.o)[b * a.ots + head * a.ohs + d] = from_f32<T>(wrong ? NAN : n == 0 ? 0.f : o / sum);
}

namespace {

template <typename T, int DP, bool FAST>
void paged_run(const PagedArgs &a, float *ws, hipStream_t st) {
    const PagedPlan p = paged_plan(a);
    const dim3 grid((unsigned)(p.splits * (int64_t)a.n * a.Hk), (unsigned)((a.Hq / a.Hk + 31) / 32));
    hipLaunchKernelGGL((paged_kernel<T, DP, FAST>), grid, dim3(64 * PagedShape<T, DP>::NW), 0, st, a, p.splits, p.per, ws);
    if (p.splits > 1)
        hipLaunchKernelGGL((join_kernel<T, DP>), dim3((unsigned)((int64_t)a.n * a.Hq)), dim3(256), 0, st, a, p.splits, p.per, ws);
}

template <typename T, int DP>
void paged_any(const PagedArgs &a, float *ws, hipStream_t st) {
    const bool fast = a.D * sizeof(T) % 16 == 0 && (((uintptr_t)a.kp | (uintptr_t)a.vp) & 15) == 0;
    if (fast) paged_run<T, DP, true>(a, ws, st);
    else paged_run<T, DP, false>(a, ws, st);
}

template <typename T>
int paged_t(const PagedArgs &a, float *ws, hipStream_t st) {
    if (a.D <= 64) paged_any<T, 64>(a, ws, st);
    else if (a.D <= 128) paged_any<T, 128>(a, ws, st);
    else paged_any<T, 256>(a, ws, st);
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace att

int64_t paged_blocks(const PagedArgs &a) {
    if (a.n == 0 || a.Hq == 0) return 0;
    return std::max<int64_t>((int64_t)att::paged_plan(a).splits * a.n * a.Hk, (int64_t)a.n * a.Hq);
}

size_t paged_workspace(int, const PagedArgs &a) {
    if (a.n == 0 || a.Hq == 0) return 0;
    const att::PagedPlan p = att::paged_plan(a);
    return p.splits > 1 ? ((size_t)a.n * a.Hq * p.splits * (a.D + 2) * sizeof(float) + 255) / 256 * 256 : 0;
}

int launch_paged(int dtype, const PagedArgs &a, void *ws, void *stream) {
    if (a.n == 0 || a.Hq == 0) return 0;
    return dtype == kBF16 ? att::paged_t<bf16>(a, static_cast<float *>(ws), (hipStream_t)stream)
                          : att::paged_t<float>(a, static_cast<float *>(ws), (hipStream_t)stream);
}

}  // namespace ms
