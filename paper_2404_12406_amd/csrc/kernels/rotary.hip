// Norms of the heads of x[T][H][D] (a scale for the query heads, one for the key heads)
// and the rotation of each by its token's position, in one pass; and the same on the way
// into a paged cache:
//   r = 1 / sqrt(mean x^2 + eps),  z = x r g
//   y_i = z_i cos a - z_j sin a,  y_j = z_j cos a + z_i sin a,  a = position freq
// over the pairs (i, j) of the first R elements: (k, k + R/2) or (2k, 2k + 1).  Backward:
//   dz = dy turned by -a,  q = dz g,  dx = r (q - x r^2 mean(q x)),  dg = sum of dz x r
//
// Bound: memory.  A head lies in the registers of L lanes (a power of two that holds it
// in 16-byte vectors), so it is read once and the norm is a sum within those lanes.  A
// wave takes one token and goes over its heads, 64 / L side by side, so that its loads
// are of one piece and the angles' sines are taken once a token, from position * freq in
// 64 bits: in 32 an angle of 10^6 would be off by 0.06.
// bf16, 8192 x 40 heads of 128: forward 41 us, 4.1 TB/s, backward 56, 4.5 TB/s, and 5 for the scales' sums (a device copy
// reaches 5.1); 16384 tokens of 48 heads into a cache 89 us, 4.5 TB/s.
#include <algorithm>

#include "block_math.h"

namespace ms {
namespace rot {

// The sum over L lanes (a power of two), in every one of them.
template <int L>
__device__ __forceinline__ float group_sum(float v) {
#define ROT_MOVED(ctrl) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false))
    if constexpr (L > 1) v += ROT_MOVED(0xb1);    // the neighbour
    if constexpr (L > 2) v += ROT_MOVED(0x4e);    // the other pair of four
    if constexpr (L > 4) v += ROT_MOVED(0x141);   // mirrored in eight
    if constexpr (L > 8) v += ROT_MOVED(0x140);   // mirrored in sixteen
#undef ROT_MOVED
    if constexpr (L > 16) v += __shfl_xor(v, 16);
    if constexpr (L > 32) v += __shfl_xor(v, 32);
    return v;
}

// How an element finds its partner: within its vector, in another lane's, from memory
// (halves that are no whole vectors).
enum Pairing { kNext, kLane, kLoose };

// A lane's part of the rotation: its elements' frequencies, a token's
// cosines and (signed) sines, and where the partners are.
template <typename T, int L>
struct Turn {
    static constexpr int V = Vec16<T>::N;
    float freq[V], cs[V], sn[V];
    int lane;        // kLane: of the partner
    uint32_t flip;   // elements whose sine counts the other way
    __device__ __forceinline__ void init(const RotaryArgs &a, int c, int l, bool back) {
        const int half = a.R / 2;
        flip = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int d = c + e;
            const bool second = a.next ? d & 1 : d >= half;
            freq[e] = d < 2 * half ? a.freq[a.next ? d >> 1 : second ? d - half : d] : 0.f;
            flip |= second == back ? 1u << e : 0u;
        }
        const int away = half / V, g = c / V;
        lane = g < away ? l + away : g < 2 * away ? l - away : l;
    }
    // (the angle in turns is reduced in 64 bits; what does not turn has frequency 0)
    __device__ __forceinline__ void take(double pos) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const double turns = pos * 0.15915494309189533577 * (double)freq[e];
            float s;
            sincospif(2.f * (float)(turns - rint(turns)), &s, &cs[e]);
            sn[e] = flip >> e & 1 ? -s : s;
        }
    }
    // turned z; partner(e) is the partner's value, for kLoose.  (Without a sine nothing
    // comes from the partner: elements past R stay as they are beside an infinite one.)
    static __device__ __forceinline__ float sum(float z, float p, float k, float s) { return s == 0.f ? z * k : z * k + p * s; }
    template <int PAIR, typename F>
    __device__ __forceinline__ void apply(float (&z)[V], F partner) const {
        if constexpr (PAIR == kNext) {
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                const float p = z[e], q = z[e + 1];
                z[e] = sum(p, q, cs[e], sn[e]);
                z[e + 1] = sum(q, p, cs[e + 1], sn[e + 1]);
            }
        } else if constexpr (PAIR == kLane) {
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = sum(z[e], __shfl(z[e], lane), cs[e], sn[e]);
        } else if constexpr (PAIR == kLoose) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (sn[e] != 0.f || cs[e] != 1.f) z[e] = sum(z[e], partner(e), cs[e], sn[e]);
        }
    }
};

template <typename T>
__device__ __forceinline__ float at(const T *p, int d) { return p ? to_f32(p[d]) : 1.f; }

__device__ __forceinline__ int partner_of(const RotaryArgs &a, int d) {
    const int half = a.R / 2;
    return d < half ? d + half : d < 2 * half ? d - half : d;
}

// Heads of a lane loaded at once, at most; backward, which loads two of each, three leave
// registers for three waves a SIMD.
constexpr int kAhead = 4, kAheadBwd = 3;

// A wave's way through its tokens and their heads, `ahead` heads of each of its G groups of
// lanes at a time; the next ones are loaded before these are worked on.
struct Way {
    int64_t t;
    int h;   // the first group's first head
    __device__ __forceinline__ void next(int ahead_heads, int H) {
        h += (int)gridDim.y * ahead_heads;
        if (h >= H) {
            h = (int)blockIdx.y * ahead_heads;
            t += (int64_t)gridDim.x * 4;
        }
    }
};

// A scale's elements of this lane; ones without it.
template <typename T>
__device__ __forceinline__ Vec16<T> scale_of(const T *p, int c, int D) {
    Vec16<T> v;
    if (p) v = load_vec<T>(p, c, D);
    else
#pragma unroll
        for (int e = 0; e < Vec16<T>::N; ++e) v.e[e] = (T)1.f;
    return v;
}

// Forward.  APPEND: heads past the Hq queries go to the cache, the last Hk of them (the
// values) as they are.
template <typename T, int L, int PAIR, bool APPEND>
__global__ __launch_bounds__(256) void fwd_kernel(RotaryArgs a, int ahead) {
    constexpr int V = Vec16<T>::N, G = 64 / L;
    const int lane = threadIdx.x & 63, c = lane % L * V, g = lane / L;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.y);
    const T *gq = static_cast<const T *>(a.gq), *gk = static_cast<const T *>(a.gk);
    const int H = a.Hq + (APPEND ? 2 : 1) * a.Hk;
    auto load = [&](const Way &w, Vec16<T> (&v)[kAhead]) {
        const T *p = x + w.t * a.xts + (w.h + g) * a.xhs;
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (u < ahead && w.h + g + u * G < H) v[u] = load_vec<T>(p + u * G * a.xhs, c, a.D);
    };
    Way way{(int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), (int)blockIdx.y * ahead * G};
    Vec16<T> in[kAhead], after[kAhead];
    if (way.t < a.T) load(way, in);
    const Vec16<T> wq = scale_of<T>(gq, c, a.D), wk = scale_of<T>(gk, c, a.D);
    Turn<T, L> turn;
    turn.init(a, c, lane, false);
    T *kto = nullptr, *vto = nullptr;   // the token's first head in the cache
    for (int64_t seen = -1; way.t < a.T;) {
        const Way now = way;
        way.next(ahead * G, H);
        if (way.t < a.T) load(way, after);
        if (now.t != seen) {
            seen = now.t;
            const int pos = APPEND || a.R ? a.pos[now.t] : 0;
            if constexpr (APPEND) {
                const int64_t row = a.rows ? (int64_t)a.rows[now.t] : now.t;
                kto = nullptr;
                if (pos >= 0 && row >= 0 && row < a.nseq && pos / a.page < a.width) {
                    const int pg = a.tables[row * a.width + pos / a.page];
                    if (pg >= 0 && pg < a.pages) {
                        const int64_t to = ((int64_t)pg * a.Hk * a.page + pos % a.page) * a.D;
                        kto = static_cast<T *>(a.kp) + to;
                        vto = static_cast<T *>(a.vp) + to;
                    }
                }
            }
            turn.take((double)pos);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int h = now.h + g + u * G;
            if (u >= ahead || h >= H) continue;
            Vec16<T> out = in[u];
            const bool value = APPEND && h >= a.Hq + a.Hk, query = h < a.Hq;
            if (!value) {
                float z[V], r = 1.f;
#pragma unroll
                for (int e = 0; e < V; ++e) z[e] = to_f32(in[u].e[e]);
                if (a.norm) {
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < V; ++e) s += z[e] * z[e];
                    r = 1.f / sqrtf(group_sum<L>(s) / (float)a.D + a.eps);
#pragma unroll
                    for (int e = 0; e < V; ++e) z[e] = z[e] * r * to_f32(query ? wq.e[e] : wk.e[e]);
                }
                turn.template apply<PAIR>(z, [&](int e) {
                    const int p = partner_of(a, c + e);
                    return to_f32(x[now.t * a.xts + h * a.xhs + p]) * r * (a.norm ? at(query ? gq : gk, p) : 1.f);
                });
#pragma unroll
                for (int e = 0; e < V; ++e) out.e[e] = from_f32<T>(z[e]);
            }
            if (c >= a.D) continue;
            if (!APPEND || query) store_vec<T>(y + now.t * a.yts + h * a.yhs, c, a.D, out);
            else if (kto) store_vec<T>((value ? vto : kto) + (int64_t)(h - a.Hq - (value ? a.Hk : 0)) * a.page * a.D, c, a.D, out);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) in[u] = after[u];
    }
}

// dx (may be null) and partial rows of dgq and dgk: part[blocks][2][D] (may be null).
template <typename T, int L, int PAIR>
__global__ __launch_bounds__(256, PAIR == kLoose || L * Vec16<T>::N == 256 ? 2 : 3) void bwd_kernel(RotaryArgs a, int ahead, const T *dy, int64_t dts, int64_t dhs, T *dx, int64_t gts,
                                                  int64_t ghs, float *part) {
    constexpr int V = Vec16<T>::N, G = 64 / L, GROUPS = 256 / L;
    __shared__ float meet[GROUPS][L * V];
    const int lane = threadIdx.x & 63, c = lane % L * V, g = lane / L;
    const T *x = static_cast<const T *>(a.x);
    const T *gq = static_cast<const T *>(a.gq), *gk = static_cast<const T *>(a.gk);
    const int H = a.Hq + a.Hk;
    auto load = [&](const Way &w, Vec16<T> (&v)[kAheadBwd], Vec16<T> (&d)[kAheadBwd]) {
        const T *p = x + w.t * a.xts + (w.h + g) * a.xhs, *q = dy + w.t * dts + (w.h + g) * dhs;
#pragma unroll
        for (int u = 0; u < kAheadBwd; ++u) {
            if (u >= ahead || w.h + g + u * G >= H) continue;
            d[u] = load_vec<T>(q + u * G * dhs, c, a.D);
            if (a.norm) v[u] = load_vec<T>(p + u * G * a.xhs, c, a.D);
        }
    };
    Way way{(int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), (int)blockIdx.y * ahead * G};
    Vec16<T> xi[kAheadBwd], gi[kAheadBwd], xn[kAheadBwd], gn[kAheadBwd];
    if (way.t < a.T) load(way, xi, gi);
    float sq[V], sk[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sq[e] = sk[e] = 0.f;
    const Vec16<T> wq = scale_of<T>(gq, c, a.D), wk = scale_of<T>(gk, c, a.D);
    Turn<T, L> turn;
    turn.init(a, c, lane, true);
    for (int64_t seen = -1; way.t < a.T;) {
        const Way now = way;
        way.next(ahead * G, H);
        if (way.t < a.T) load(way, xn, gn);
        if (now.t != seen) {
            seen = now.t;
            turn.take(a.R ? (double)a.pos[now.t] : 0.0);
        }
#pragma unroll
        for (int u = 0; u < kAheadBwd; ++u) {
            const int h = now.h + g + u * G;
            if (u >= ahead || h >= H) continue;
            const bool query = h < a.Hq;
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = to_f32(gi[u].e[e]);
            turn.template apply<PAIR>(z, [&](int e) { return to_f32(dy[now.t * dts + h * dhs + partner_of(a, c + e)]); });
            if (a.norm) {
                float s = 0.f, m = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float v = to_f32(xi[u].e[e]);
                    s += v * v;
                    m += z[e] * to_f32(query ? wq.e[e] : wk.e[e]) * v;
                }
                const float r = 1.f / sqrtf(group_sum<L>(s) / (float)a.D + a.eps);
                m = group_sum<L>(m) / (float)a.D * r * r;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float v = to_f32(xi[u].e[e]), p = z[e] * v * r;
                    if (query) sq[e] += p;
                    else sk[e] += p;
                    z[e] = r * (z[e] * to_f32(query ? wq.e[e] : wk.e[e]) - v * m);
                }
            }
            if (dx && c < a.D) {
                Vec16<T> out;
#pragma unroll
                for (int e = 0; e < V; ++e) out.e[e] = from_f32<T>(z[e]);
                store_vec<T>(dx + now.t * gts + h * ghs, c, a.D, out);
            }
        }
#pragma unroll
        for (int u = 0; u < kAheadBwd; ++u) {
            xi[u] = xn[u];
            gi[u] = gn[u];
        }
    }
    if (!part) return;
    float *to = part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int e = 0; e < V; ++e) meet[threadIdx.x / L][c + e] = which ? sk[e] : sq[e];
        __syncthreads();
        for (int d = threadIdx.x; d < a.D; d += 256) {
            float s = 0.f;
            for (int k = 0; k < GROUPS; ++k) s += meet[k][d];
            to[which * a.D + d] = s;
        }
        __syncthreads();
    }
}

// out[which][d] = the sum of the partial rows, in a fixed order: 16 columns a block, 64 groups
// of every 64th row.
template <typename T>
__global__ __launch_bounds__(1024) void sum_kernel(const float *__restrict__ part, int rows, int D, T *__restrict__ oq, T *__restrict__ ok) {
    __shared__ float red[64][17];
    const int col = threadIdx.x & 15, grp = threadIdx.x >> 4, c = (int)blockIdx.x * 16 + col;   // a column of [2 D]
    float s = 0.f;
    if (c < 2 * D) {
#pragma unroll 8
        for (int r = grp; r < rows; r += 64) s += part[(int64_t)r * 2 * D + c];
    }
    red[grp][col] = s;
    __syncthreads();
    if (grp == 0 && c < 2 * D) {
#pragma unroll
        for (int q = 1; q < 64; ++q) s += red[q][col];
        T *o = c < D ? oq : ok;
        if (o) o[c < D ? c : c - D] = from_f32<T>(s);
    }
}

// ------------------------------------------------------------------ host
namespace {

// Blocks at most: all at once, so that each wave's way is long (a wave begins with loads that depend on
// each other).  8192 x 40 heads of 128, bf16: forward 512, 1024, 2048 blocks 46, 40, 43 us;
// backward, whose blocks leave a partial row each, 512, 768, 1024 blocks 64, 59, 71.
constexpr int kMostBlocks = 1024, kMostParts = 768;

int lanes(int dtype, int D) {
    const int v = dtype == kBF16 ? 8 : 4, n = (D + v - 1) / v;
    int l = 4;
    while (l < n) l *= 2;
    return l;
}

int pairing(int dtype, const RotaryArgs &a) {
    if (a.R < 2 || a.next) return kNext;
    return (a.R / 2) % (dtype == kBF16 ? 8 : 4) == 0 ? kLane : kLoose;
}

// Blocks of four waves, a token a wave; where these are few, their heads over several
// blocks.  ahead: a token's heads in equal parts.
struct Plan {
    dim3 grid;
    int ahead;
};

Plan plan(int dtype, const RotaryArgs &a, int heads, int at_once, int most) {
    const int G = 64 / lanes(dtype, a.D), per = (heads + G - 1) / G, parts = (per + at_once - 1) / at_once;
    const int64_t bx = std::min<int64_t>((a.T + 3) / 4, most);
    const int64_t by = std::max<int64_t>(1, std::min<int64_t>(parts, most / std::max<int64_t>(bx, 1)));
    return {dim3((unsigned)bx, (unsigned)by), std::max(1, (per + parts - 1) / std::max(parts, 1))};
}

template <typename T, int L, int PAIR>
void fwd_run(const RotaryArgs &a, const Plan &p, bool append, hipStream_t st) {
    if (append) hipLaunchKernelGGL((fwd_kernel<T, L, PAIR, true>), p.grid, dim3(256), 0, st, a, p.ahead);
    else hipLaunchKernelGGL((fwd_kernel<T, L, PAIR, false>), p.grid, dim3(256), 0, st, a, p.ahead);
}

template <typename T, int L, int PAIR>
void bwd_run(const RotaryArgs &a, const Plan &p, const void *dy, const int64_t ds[2], void *dx, const int64_t gs[2], float *part,
             hipStream_t st) {
    hipLaunchKernelGGL((bwd_kernel<T, L, PAIR>), p.grid, dim3(256), 0, st, a, p.ahead, (const T *)dy, ds[0], ds[1], (T *)dx, gs[0], gs[1], part);
}

#define ROT_PAIR(F, L, ...)                                  \
    switch (pairing(dtype, a)) {                             \
    case kNext: F<T, L, kNext>(__VA_ARGS__); break;          \
    case kLane: F<T, L, kLane>(__VA_ARGS__); break;          \
    default: F<T, L, kLoose>(__VA_ARGS__); break;            \
    }
#define ROT_DISPATCH(F, ...)                                 \
    switch (lanes(dtype, a.D)) {                             \
    case 4: ROT_PAIR(F, 4, __VA_ARGS__) break;               \
    case 8: ROT_PAIR(F, 8, __VA_ARGS__) break;               \
    case 16: ROT_PAIR(F, 16, __VA_ARGS__) break;             \
    case 32: ROT_PAIR(F, 32, __VA_ARGS__) break;             \
    default:   /* (256 bf16 elements take 32) */             \
        if constexpr (sizeof(T) == 4) {                      \
            ROT_PAIR(F, 64, __VA_ARGS__)                     \
        }                                                    \
    }

template <typename T>
int fwd_t(int dtype, const RotaryArgs &a, bool append, hipStream_t st) {
    const Plan p = plan(dtype, a, a.Hq + (append ? 2 : 1) * a.Hk, kAhead, kMostBlocks);
    ROT_DISPATCH(fwd_run, a, p, append, st)
    return (int)hipGetLastError();
}

template <typename T>
int bwd_t(int dtype, const RotaryArgs &a, const void *dy, const int64_t ds[2], void *dx, const int64_t gs[2], void *dgq, void *dgk,
          void *ws, hipStream_t st) {
    const bool params = dgq || dgk;
    float *part = params ? static_cast<float *>(ws) : nullptr;
    int rows = 0;
    if (a.T > 0 && a.Hq + a.Hk > 0) {
        const Plan p = plan(dtype, a, a.Hq + a.Hk, kAheadBwd, params ? kMostParts : kMostBlocks);
        ROT_DISPATCH(bwd_run, a, p, dy, ds, dx, gs, part, st)
        rows = (int)(p.grid.x * p.grid.y);
    }
    if (params)
        hipLaunchKernelGGL(sum_kernel<T>, dim3((unsigned)((2 * a.D + 15) / 16)), dim3(1024), 0, st, part, rows, a.D, (T *)dgq, (T *)dgk);
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace rot

int launch_rotary_fwd(int dtype, const RotaryArgs &a, bool append, void *stream) {
    if (a.T == 0 || a.Hq + a.Hk == 0) return 0;
    return dtype == kBF16 ? rot::fwd_t<bf16>(dtype, a, append, (hipStream_t)stream)
                          : rot::fwd_t<float>(dtype, a, append, (hipStream_t)stream);
}

size_t rotary_bwd_workspace(int dtype, const RotaryArgs &a, bool params) {
    if (!params || a.T == 0 || a.Hq + a.Hk == 0) return 0;
    const dim3 g = rot::plan(dtype, a, a.Hq + a.Hk, rot::kAheadBwd, rot::kMostParts).grid;
    return ((size_t)g.x * g.y * 2 * a.D * sizeof(float) + 255) / 256 * 256;
}

int launch_rotary_bwd(int dtype, const RotaryArgs &a, const void *dy, const int64_t dstride[2], void *dx, const int64_t gstride[2],
                      void *dgq, void *dgk, void *ws, void *stream) {
    return dtype == kBF16 ? rot::bwd_t<bf16>(dtype, a, dy, dstride, dx, gstride, dgq, dgk, ws, (hipStream_t)stream)
                          : rot::bwd_t<float>(dtype, a, dy, dstride, dx, gstride, dgq, dgk, ws, (hipStream_t)stream);
}

}  // namespace ms
