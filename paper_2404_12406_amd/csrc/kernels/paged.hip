// Attention of one query a sequence over a paged cache: o = softmax(scale q k^T) v over the
// first lengths[b] places of the pages that tables[b] lists.
//
// Bound: memory, one read of the keys and values that are used, however many query heads
// share them: these are the columns of a 32x32 tile (attn_tile.h), up to 32 at once.
//  * A block takes `per` keys of one sequence and head of the cache, and each of its waves
//    32 keys at a time on its own: a wave's loads go straight into its own part of LDS, two
//    steps of them in flight, and nothing waits for another wave before the end.
//  * The pages of a step's keys are loaded a step before its keys, into LDS too, so that
//    the loads follow each other in one order and the waits count them.
//  * A key's row is looked up by itself, so pages may have any size and end anywhere.  Rows
//    past the length read as zeros, whatever lies there; rows of a page that is none make
//    their scores NaN.
//  * Softmax statistics and sums of a block's waves meet in LDS, those of a
//    sequence's blocks in join_kernel, in a fixed order.
#include <algorithm>

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
    static constexpr int NW = RB <= 256 ? 4 : 1024 / RB;       // waves: two steps of 64 rows each in 128 KiB
    static constexpr int STAGE = 64 * RB, WAVE = 2 * STAGE + 3 * 256;   // + pages of two steps, rows of one
    static constexpr int LOADS = STAGE / 1024;
};

// FAST: rows of the cache are whole 16-byte vectors, so aligned; else they go through
// registers, any number of elements side by side.
template <typename T, int DP, bool FAST>
__global__ __launch_bounds__((64 * PagedShape<T, DP>::NW), 1) void paged_kernel(PagedArgs a, int splits, int per, float *__restrict__ part) {
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    typedef PagedShape<T, DP> Sh;
    typedef typename M::Frag Frag;
    constexpr int NW = Sh::NW, NP = 32 / M::KC, LD = DP + 4;
    __shared__ __align__(16) char lds[NW * Sh::WAVE + NW * 256];
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

    char *mine = lds + w * Sh::WAVE, *pages = mine + 2 * Sh::STAGE, *rows = pages + 512;
    const int32_t *table = a.tables + (int64_t)b * a.width;
    // the pages of step i's keys
    auto look = [&](int i) {
        const int key = min(begin + (i * NW + w) * 32 + (lane & 31), len - 1);
        far4(table + key / a.page, pages + (i & 1) * 256);
    };
    uint32_t bad_of[2] = {0u, 0u};   // keys whose page is none
    auto issue = [&](int i, uint32_t &bad) {
        const int key = begin + (i * NW + w) * 32 + (lane & 31);
        const int pg = *reinterpret_cast<const int *>(pages + (i & 1) * 256 + 4 * (lane & 31));
        const bool used = key < end, none = used && (pg < 0 || pg >= a.pages);
        bad = (uint32_t)__ballot(none);
        const uint32_t row = used && !none ? ((uint32_t)pg * (uint32_t)a.Hk + (uint32_t)hk) * (uint32_t)a.page + (uint32_t)(key % a.page) : ~0u;
        *reinterpret_cast<uint32_t *>(rows + 4 * lane) = row;   // (twice: both halves hold the same keys)
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        char *to = mine + (i & 1) * Sh::STAGE;
#pragma unroll
        for (int n = 0; n < Sh::LOADS / 2; ++n) {
            const int idx = n * 64 + lane, r = idx / Ti::U, unit = (idx % Ti::U) ^ Ti::swz(r);
            const uint32_t at = *reinterpret_cast<const uint32_t *>(rows + 4 * r);
            const bool there = at != ~0u && unit * M::V < a.D;
            const T *k = static_cast<const T *>(a.kp) + (int64_t)at * a.D, *v = static_cast<const T *>(a.vp) + (int64_t)at * a.D;
            if constexpr (FAST) {
                far16(there ? (const void *)(k + unit * M::V) : &kZeros, to + n * 1024);
                far16(there ? (const void *)(v + unit * M::V) : &kZeros, to + Sh::STAGE / 2 + n * 1024);
            } else {
                Vec16<T> kv = zero16<T>(), vv = zero16<T>();
                if (there) {
                    kv = load_vec<T>(k, unit * M::V, a.D);
                    vv = load_vec<T>(v, unit * M::V, a.D);
                }
                store16(reinterpret_cast<T *>(to + n * 1024 + lane * 16), kv);
                store16(reinterpret_cast<T *>(to + Sh::STAGE / 2 + n * 1024 + lane * 16), vv);
            }
        }
    };
    const int keys = end - begin - w * 32, steps = keys > 0 ? (keys + 32 * NW - 1) / (32 * NW) : 0;   // the wave's
    Rows<T, DP, (DP * sizeof(T) < 1024)> q;   // (256 fp32 elements are too many to hold)
    q.init(static_cast<const T *>(a.q) + b * a.qts + head * a.qhs, a.qhs, heads, a.D, lane);
    if (steps > 0) {
        look(0);
        landed<0>();
        if (steps > 1) look(1);
        issue(0, bad_of[0]);
    }
    const float c = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    floatx16 acc[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = zero16x();
    for (int i = 0; i < steps; ++i) {
        if (i + 1 < steps) {
            landed<Sh::LOADS>();   // the pages of the next step; this step's keys may be under way
            g2::wait_lgkm0();      // the stage that is loaded now has been read
            if (i + 2 < steps) {
                look(i + 2);
                issue(i + 1, bad_of[1]);
                landed<Sh::LOADS + 1>();
            } else {
                issue(i + 1, bad_of[1]);
                landed<Sh::LOADS>();
            }
        } else {
            landed<0>();
        }
        const char *kt = mine + (i & 1) * Sh::STAGE, *vt = kt + Sh::STAGE / 2;
        floatx16 x = zero16x();
#pragma unroll
        for (int n = 0; n < DP / M::KC; ++n) x = M::mma(Ti::row_frag(kt, 0, n, lane), q.get(n, lane), x);
        const int k = begin + (i * NW + w) * 32;
        if (k + 32 > end || bad_of[0]) {
#pragma unroll
            for (int n = 0; n < 16; ++n) {
                const int r = 8 * (n >> 2) + 4 * hh + (n & 3);
                if (k + r >= end) x[n] = -INFINITY;
                else if (bad_of[0] >> r & 1) x[n] = NAN;
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
        add_product<T, DP, NP>(acc, vt, 0, p, lane);
        bad_of[0] = bad_of[1];
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
            float *to = part + (((int64_t)b * a.Hq + head + n) * splits + split) * (a.D + 2);
            to[d] = o;
            if (d == 0) {
                to[a.D] = top;
                to[a.D + 1] = sum;
            }
        }
    }
}

// o of the splits that a sequence has: a block a query head.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(PagedArgs a, int splits, int per, const float *__restrict__ part) {
    const int b = (int)(blockIdx.x / a.Hq), head = (int)(blockIdx.x % a.Hq), d = threadIdx.x;
    if (d >= a.D) return;
    const int len = a.lengths[b];
    const int n = (int)(((int64_t)max(len, 0) + per - 1) / per);
    float out = 0.f;
    if (len > (int64_t)a.width * a.page) {
        out = NAN;
    } else if (n > 0) {
        const float *p = part + (int64_t)blockIdx.x * splits * (a.D + 2);
        const float c = a.scale * kLog2e;
        float top = -INFINITY, sum = 0.f, o = 0.f;
        for (int s = 0; s < n; ++s) top = fmaxf(top, p[s * (a.D + 2) + a.D]);
        for (int s = 0; s < n; ++s) {
            const float m = p[s * (a.D + 2) + a.D], f = m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * c);
            sum += f * p[s * (a.D + 2) + a.D + 1];
            o += f * p[s * (a.D + 2) + d];
        }
        out = o / sum;
    }
    static_cast<T *>(a.o)[b * a.ots + head * a.ohs + d] = from_f32<T>(out);
}

namespace {

struct PagedPlan {
    int splits, per;   // blocks of a sequence at most, keys of each
};

// Keys a block: some 4096 blocks if every sequence filled its table, whole steps of a
// block's waves (128 keys).
PagedPlan paged_plan(const PagedArgs &a) {
    const int64_t room = (int64_t)a.width * a.page, work = (int64_t)a.n * a.Hk * ((a.Hq / a.Hk + 31) / 32);
    const int64_t per = std::max<int64_t>(128, (room * work / 4096 + 127) / 128 * 128);
    return {(int)std::max<int64_t>(1, (room + per - 1) / per), (int)std::min<int64_t>(per, INT32_MAX / 2)};
}

template <typename T, int DP, bool FAST>
void paged_run(const PagedArgs &a, float *ws, hipStream_t st) {
    const PagedPlan p = paged_plan(a);
    const dim3 grid((unsigned)(p.splits * (int64_t)a.n * a.Hk), (unsigned)((a.Hq / a.Hk + 31) / 32));
    hipLaunchKernelGGL((paged_kernel<T, DP, FAST>), grid, dim3(64 * PagedShape<T, DP>::NW), 0, st, a, p.splits, p.per, ws);
    if (p.splits > 1)
        hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)((int64_t)a.n * a.Hq)), dim3(256), 0, st, a, p.splits, p.per, ws);
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
