// Layer norm over the rows of x[M][D], forward and backward:
//   h = (x - mean) r,  r = 1 / sqrt(var + eps),  y = h gamma + beta
//   q = dy gamma,  dx = r (q - mean(q) - h mean(q h))
//   dgamma = sum over rows of dy h,  dbeta = sum over rows of dy
// with mean and (biased) variance over the row.
//
// Bound: memory.  The forward reads x and writes y; the backward reads x and
// dy and writes dx, and takes the statistics again from the x that it has to
// read anyway, so nothing but x is kept between the two.  A row lies in the
// registers of TPR threads, NV 16-byte vectors each: every element is read
// once, the variance is the sum of squared differences from the mean that was
// found first (no cancellation), and all sums are in 32 bits.
//  * TPR = 64, four rows a block, to 256 vectors a row (2048 bf16): no barrier
//    anywhere in the row loop.  256 and 512 threads a row beyond that, their
//    waves meeting in LDS; rows of more than 1536 vectors take the kernels at
//    the end, which read a row from memory (its L2) for each pass over it.
//  * blocks are persistent: a thread owns the same columns in each of its rows,
//    so gamma and beta are loaded once and dgamma and dbeta are running sums in
//    registers, left as one partial row a block and added up in a fixed order
//    by finalize_kernel.
//  * rows of any width and alignment take 16-byte accesses; only a row's last,
//    incomplete vector goes element by element.
// Measured: 16384 x 4096 bf16, forward 48 us (5.6 TB/s), input gradient 81 us (5.0
// TB/s), where a large copy reaches 5.1; 8192 x 768, all gradients: 9.2, 13.5 and
// 4.0 us, of which some 3 each are a launch's own time and the rest latency.
#include <algorithm>

#include "block_math.h"

namespace ms {
namespace ln {

// The sum over a wave, by moves within the vector registers (an exchange through
// LDS takes some 60 clocks a step, and a row's sums are a chain of 24 steps).
__device__ __forceinline__ float wave_sum(float v) {
    auto add = [&](float m) __attribute__((always_inline)) { v += m; };
#define LN_MOVED(ctrl, rows) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, false))
    add(LN_MOVED(0x111, 0xf));   // from 1, 2, 4 and 8 lanes below, within rows of 16
    add(LN_MOVED(0x112, 0xf));
    add(LN_MOVED(0x114, 0xf));
    add(LN_MOVED(0x118, 0xf));
    add(LN_MOVED(0x142, 0xa));   // the rows before
    add(LN_MOVED(0x143, 0xc));
#undef LN_MOVED
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sums of N values over the TPR threads of a row.  More than one wave: through
// LDS, in one of four slots in turn, so that one barrier a sum is enough (a slot
// is written again only after three more barriers, which a wave reaches after it
// has read it).
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float *red, int &slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (TPR > 64) {
        constexpr int NW = TPR / 64;
        float *s = red + slot * (2 * NW);
        slot = (slot + 1) & 3;
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) s[i * NW + w] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int k = 0; k < NW; ++k) v[i] += s[i * NW + k];
        }
    }
}

template <typename T, int TPR, int NV>
struct Row {
    static constexpr int V = Vec16<T>::N;
    static constexpr int NT = TPR > 256 ? TPR : 256;
    static constexpr int RPB = NT / TPR;   // rows of a block at once
    // mean and 1 / sqrt(var + eps) of the row held in x (zeros past its end)
    static __device__ __forceinline__ void stats(const Vec16<T> (&x)[NV], int t, int D, float eps, float *red, int &slot,
                                                 float &mean, float &r) {
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += to_f32(x[k].e[e]);
        row_sum<TPR>(s, red, slot);
        mean = s[0] / (float)D;
        s[0] = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = to_f32(x[k].e[e]) - mean;
                if ((t + k * TPR) * V + e < D) s[0] += d * d;
            }
        row_sum<TPR>(s, red, slot);
        r = 1.f / sqrtf(s[0] / (float)D + eps);
    }
};

template <typename T, int TPR, int NV>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void fwd_kernel(const T *__restrict__ x, const T *__restrict__ gamma,
                                                                    const T *__restrict__ beta, float eps, int64_t M, int D,
                                                                    T *__restrict__ y) {
    using R = Row<T, TPR, NV>;
    constexpr int V = R::V;
    __shared__ float red[TPR > 64 ? 8 * (TPR / 64) : 1];
    int slot = 0;
    const int t = threadIdx.x % TPR;
    Vec16<T> g[NV], b[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (t + k * TPR) * V;
        if (gamma) g[k] = load_vec(gamma, c, D);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) g[k].e[e] = (T)1.f;
        b[k] = beta ? load_vec(beta, c, D) : zero16<T>();
    }
    for (int64_t row = (int64_t)blockIdx.x * R::RPB + threadIdx.x / TPR; row < M; row += (int64_t)gridDim.x * R::RPB) {
        Vec16<T> v[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = load_vec(x + row * D, (t + k * TPR) * V, D);
        float mean, r;
        R::stats(v, t, D, eps, red, slot, mean, r);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (t + k * TPR) * V;
            if (c >= D) continue;
#pragma unroll
            for (int e = 0; e < V; ++e)
                v[k].e[e] = from_f32<T>((to_f32(v[k].e[e]) - mean) * r * to_f32(g[k].e[e]) + to_f32(b[k].e[e]));
            store_vec(y + row * D, c, D, v[k]);
        }
    }
}

// dx (DX) and partial rows of dgamma and dbeta (DP): pg, pb are [blocks][D],
// either may be null.
template <typename T, int TPR, int NV, bool DX, bool DP>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void bwd_kernel(const T *__restrict__ x, const T *__restrict__ dy,
                                                                    const T *__restrict__ gamma, float eps, int64_t M, int D,
                                                                    T *__restrict__ dx, float *__restrict__ pg,
                                                                    float *__restrict__ pb) {
    using R = Row<T, TPR, NV>;
    constexpr int V = R::V;
    constexpr bool MEET = DP && R::RPB > 1;   // the block's rows meet in LDS at the end
    __shared__ float red[TPR > 64 ? 8 * (TPR / 64) : 1];
    __shared__ float meet[MEET ? 2 * R::RPB * TPR * V : 1];
    int slot = 0;
    const int t = threadIdx.x % TPR;
    Vec16<T> g[DX ? NV : 1];
    if constexpr (DX) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (gamma) g[k] = load_vec(gamma, (t + k * TPR) * V, D);
            else
#pragma unroll
                for (int e = 0; e < V; ++e) g[k].e[e] = (T)1.f;
        }
    }
    float ag[DP ? NV : 1][V], ab[DP ? NV : 1][V];
    if constexpr (DP) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) ag[k][e] = ab[k][e] = 0.f;
    }
    for (int64_t row = (int64_t)blockIdx.x * R::RPB + threadIdx.x / TPR; row < M; row += (int64_t)gridDim.x * R::RPB) {
        Vec16<T> v[NV], d[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            v[k] = load_vec(x + row * D, (t + k * TPR) * V, D);
            d[k] = load_vec(dy + row * D, (t + k * TPR) * V, D);
        }
        float mean, r;
        R::stats(v, t, D, eps, red, slot, mean, r);
        if constexpr (DP) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {   // (dy is zero past the row)
                    const float q = to_f32(d[k].e[e]);
                    ag[k][e] += q * ((to_f32(v[k].e[e]) - mean) * r);
                    ab[k][e] += q;
                }
        }
        if constexpr (DX) {
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float q = to_f32(d[k].e[e]) * to_f32(g[k].e[e]);
                    s[0] += q;
                    s[1] += q * ((to_f32(v[k].e[e]) - mean) * r);
                }
            row_sum<TPR>(s, red, slot);
            const float mq = s[0] / (float)D, mqh = s[1] / (float)D;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = (t + k * TPR) * V;
                if (c >= D) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float h = (to_f32(v[k].e[e]) - mean) * r, q = to_f32(d[k].e[e]) * to_f32(g[k].e[e]);
                    v[k].e[e] = from_f32<T>(r * (q - mq - h * mqh));
                }
                store_vec(dx + row * D, c, D, v[k]);
            }
        }
    }
    if constexpr (DP) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if constexpr (MEET) {
                constexpr int COLS = TPR * V, NW = R::RPB;
                const int w = threadIdx.x / TPR;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    meet[w * COLS + t * V + e] = ag[k][e];
                    meet[(NW + w) * COLS + t * V + e] = ab[k][e];
                }
                __syncthreads();
                for (int i = threadIdx.x; i < COLS; i += R::NT) {
                    const int c = k * COLS + i;
                    float sg = 0.f, sb = 0.f;
#pragma unroll
                    for (int q = 0; q < NW; ++q) {
                        sg += meet[q * COLS + i];
                        sb += meet[(NW + q) * COLS + i];
                    }
                    if (c < D) {
                        if (pg) pg[(int64_t)blockIdx.x * D + c] = sg;
                        if (pb) pb[(int64_t)blockIdx.x * D + c] = sb;
                    }
                }
                __syncthreads();
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int c = (t + k * TPR) * V + e;
                    if (c >= D) continue;
                    if (pg) pg[(int64_t)blockIdx.x * D + c] = ag[k][e];
                    if (pb) pb[(int64_t)blockIdx.x * D + c] = ab[k][e];
                }
            }
        }
    }
}

// out[c] = sum of rows partial rows, in a fixed order: a block owns 16 columns
// (64 bytes of a row), its 16 thread groups every 16th row.  blockIdx.y picks
// the pair (p0, o0) or (p1, o1).
template <typename T>
__global__ __launch_bounds__(256) void finalize_kernel(const float *__restrict__ p0, T *__restrict__ o0,
                                                       const float *__restrict__ p1, T *__restrict__ o1, int rows, int D) {
    __shared__ float red[16][17];
    const float *p = blockIdx.y ? p1 : p0;
    T *o = blockIdx.y ? o1 : o0;
    const int col = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int c = (int)blockIdx.x * 16 + col;
    float s = 0.f;
    if (c < D) {
        int r = grp;
        for (; r + 48 < rows; r += 64) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = p[(int64_t)(r + 16 * u) * D + c];
#pragma unroll
            for (int u = 0; u < 4; ++u) s += v[u];
        }
        for (; r < rows; r += 16) s += p[(int64_t)r * D + c];
    }
    red[grp][col] = s;
    __syncthreads();
    if (grp == 0 && c < D) {
#pragma unroll
        for (int q = 1; q < 16; ++q) s += red[q][col];
        o[c] = from_f32<T>(s);
    }
}

// ------------------------------------------------------------------ rows past the registers
// One block a row, which it reads once for each sum and once for the result.
template <typename T, bool BWD>
__global__ __launch_bounds__(1024) void wide_kernel(const T *__restrict__ x, const T *__restrict__ dy,
                                                    const T *__restrict__ gamma, const T *__restrict__ beta, float eps,
                                                    int64_t M, int64_t D, T *__restrict__ out, float *__restrict__ stat) {
    __shared__ float red[8 * 16];
    int slot = 0;
    for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
        const T *xr = x + row * D;
        float s[1] = {0.f};
        for (int64_t c = threadIdx.x; c < D; c += 1024) s[0] += to_f32(xr[c]);
        row_sum<1024>(s, red, slot);
        const float mean = s[0] / (float)D;
        s[0] = 0.f;
        for (int64_t c = threadIdx.x; c < D; c += 1024) {
            const float d = to_f32(xr[c]) - mean;
            s[0] += d * d;
        }
        row_sum<1024>(s, red, slot);
        const float r = 1.f / sqrtf(s[0] / (float)D + eps);
        if (stat && threadIdx.x == 0) {
            stat[2 * row] = mean;
            stat[2 * row + 1] = r;
        }
        if (!out) continue;
        float q2[2] = {0.f, 0.f};
        if constexpr (BWD) {
            for (int64_t c = threadIdx.x; c < D; c += 1024) {
                const float q = to_f32(dy[row * D + c]) * (gamma ? to_f32(gamma[c]) : 1.f);
                q2[0] += q;
                q2[1] += q * ((to_f32(xr[c]) - mean) * r);
            }
            row_sum<1024>(q2, red, slot);
        }
        for (int64_t c = threadIdx.x; c < D; c += 1024) {
            const float h = (to_f32(xr[c]) - mean) * r, gm = gamma ? to_f32(gamma[c]) : 1.f;
            if constexpr (BWD)
                out[row * D + c] = from_f32<T>(r * (to_f32(dy[row * D + c]) * gm - q2[0] / (float)D - h * (q2[1] / (float)D)));
            else
                out[row * D + c] = from_f32<T>(h * gm + (beta ? to_f32(beta[c]) : 0.f));
        }
    }
}

// Partial rows of dgamma and dbeta, one thread a column, `per` rows a block.
template <typename T>
__global__ __launch_bounds__(256) void wide_params_kernel(const T *__restrict__ x, const T *__restrict__ dy,
                                                          const float *__restrict__ stat, int64_t M, int64_t D, int64_t per,
                                                          float *__restrict__ pg, float *__restrict__ pb) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= D) return;
    const int64_t end = min(M, (int64_t)(blockIdx.y + 1) * per);
    float sg = 0.f, sb = 0.f;
    for (int64_t row = (int64_t)blockIdx.y * per; row < end; ++row) {
        const float q = to_f32(dy[row * D + c]);
        sg += q * ((to_f32(x[row * D + c]) - stat[2 * row]) * stat[2 * row + 1]);
        sb += q;
    }
    if (pg) pg[(int64_t)blockIdx.y * D + c] = sg;
    if (pb) pb[(int64_t)blockIdx.y * D + c] = sb;
}

// ------------------------------------------------------------------ host
namespace {

constexpr int kVecs = 4;         // vectors of a row that one thread holds (three of 512 threads: a fourth spills)
constexpr int kWideChunks = 64;  // partial rows of the wide parameter sums

// Threads a row, vectors a thread (0: past the registers) and blocks.
struct Plan {
    int tpr, nv, blocks;
};

Plan plan(int dtype, int64_t M, int64_t D, bool params) {
    const int64_t nvec = (D + (dtype == kBF16 ? 7 : 3)) / (dtype == kBF16 ? 8 : 4);
    const int tpr = nvec <= 64 * kVecs ? 64 : nvec <= 256 * kVecs ? 256 : nvec <= 512 * 3 ? 512 : 0;
    if (!tpr) return {0, 0, (int)std::min<int64_t>(M, 2048)};
    const int64_t rows = tpr == 64 ? (M + 3) / 4 : M;
    // Parameter sums leave a partial row a block: two blocks of 256 threads a CU.
    // 8192 x 768 bf16: 13.5 us and 4.0 for the sum of the partials; with four 13.6 and
    // 6.6 (loading the next row ahead of the one worked on gave nothing, 14.0).
    const int64_t most = params ? (tpr == 512 ? 256 : 512) : 2048;
    return {tpr, (int)((nvec + tpr - 1) / tpr), (int)std::min(rows, most)};
}

size_t al256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T, int TPR, int NV>
void run_fwd(const Plan &p, const void *x, const void *g, const void *b, float eps, int64_t M, int64_t D, void *y, hipStream_t st) {
    hipLaunchKernelGGL((fwd_kernel<T, TPR, NV>), dim3(p.blocks), dim3(TPR > 256 ? TPR : 256), 0, st, (const T *)x, (const T *)g,
                       (const T *)b, eps, M, (int)D, (T *)y);
}

template <typename T, int TPR, int NV>
void run_bwd(const Plan &p, const void *x, const void *dy, const void *g, float eps, int64_t M, int64_t D, void *dx, float *pg,
             float *pb, hipStream_t st) {
    const dim3 grid(p.blocks), block(TPR > 256 ? TPR : 256);
    const bool dp = pg || pb;
    if (dx && dp)
        hipLaunchKernelGGL((bwd_kernel<T, TPR, NV, true, true>), grid, block, 0, st, (const T *)x, (const T *)dy, (const T *)g,
                           eps, M, (int)D, (T *)dx, pg, pb);
    else if (dx)
        hipLaunchKernelGGL((bwd_kernel<T, TPR, NV, true, false>), grid, block, 0, st, (const T *)x, (const T *)dy, (const T *)g,
                           eps, M, (int)D, (T *)dx, pg, pb);
    else
        hipLaunchKernelGGL((bwd_kernel<T, TPR, NV, false, true>), grid, block, 0, st, (const T *)x, (const T *)dy, (const T *)g,
                           eps, M, (int)D, (T *)dx, pg, pb);
}

// Calls f<TPR, NV>() for the plan's pair.
#define LN_DISPATCH(F, ...)                                        \
    switch (p.tpr * 8 + p.nv) {                                    \
    case 64 * 8 + 1: F<T, 64, 1>(__VA_ARGS__); break;              \
    case 64 * 8 + 2: F<T, 64, 2>(__VA_ARGS__); break;              \
    case 64 * 8 + 3: F<T, 64, 3>(__VA_ARGS__); break;              \
    case 64 * 8 + 4: F<T, 64, 4>(__VA_ARGS__); break;              \
    case 256 * 8 + 2: F<T, 256, 2>(__VA_ARGS__); break;            \
    case 256 * 8 + 3: F<T, 256, 3>(__VA_ARGS__); break;            \
    case 256 * 8 + 4: F<T, 256, 4>(__VA_ARGS__); break;            \
    default: F<T, 512, 3>(__VA_ARGS__); break;                     \
    }

template <typename T>
int fwd_t(int dtype, const void *x, const void *gamma, const void *beta, float eps, int64_t M, int64_t D, void *y, hipStream_t st) {
    const Plan p = plan(dtype, M, D, false);
    if (!p.tpr) {
        hipLaunchKernelGGL((wide_kernel<T, false>), dim3(p.blocks), dim3(1024), 0, st, (const T *)x, (const T *)nullptr,
                           (const T *)gamma, (const T *)beta, eps, M, D, (T *)y, (float *)nullptr);
    } else {
        LN_DISPATCH(run_fwd, p, x, gamma, beta, eps, M, D, y, st)
    }
    return (int)hipGetLastError();
}

template <typename T>
int bwd_t(int dtype, const void *x, const void *dy, const void *gamma, float eps, int64_t M, int64_t D, void *dx, void *dgamma,
          void *dbeta, void *ws, hipStream_t st) {
    const bool dp = dgamma || dbeta;
    const Plan p = plan(dtype, M, D, dp);
    const int64_t per = (M + kWideChunks - 1) / kWideChunks;
    const int rows = M == 0 ? 0 : p.tpr ? p.blocks : (int)((M + per - 1) / per);
    float *pg = dgamma ? static_cast<float *>(ws) : nullptr;
    float *pb = dbeta ? static_cast<float *>(ws) + (dgamma ? (size_t)rows * D : 0) : nullptr;
    if (M > 0 && !p.tpr) {
        float *stat = dp ? static_cast<float *>(ws) + (size_t)rows * D * ((dgamma ? 1 : 0) + (dbeta ? 1 : 0)) : nullptr;
        hipLaunchKernelGGL((wide_kernel<T, true>), dim3(p.blocks), dim3(1024), 0, st, (const T *)x, (const T *)dy,
                           (const T *)gamma, (const T *)nullptr, eps, M, D, (T *)dx, stat);
        if (dp)
            hipLaunchKernelGGL(wide_params_kernel<T>, dim3((unsigned)((D + 255) / 256), rows), dim3(256), 0, st, (const T *)x,
                               (const T *)dy, stat, M, D, per, pg, pb);
    } else if (M > 0) {
        LN_DISPATCH(run_bwd, p, x, dy, gamma, eps, M, D, dx, pg, pb, st)
    }
    if (dp) {
        const bool both = dgamma && dbeta;
        hipLaunchKernelGGL(finalize_kernel<T>, dim3((unsigned)((D + 15) / 16), both ? 2 : 1), dim3(256), 0, st, dgamma ? pg : pb,
                           (T *)(dgamma ? dgamma : dbeta), pb, (T *)dbeta, rows, (int)D);
    }
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace ln

size_t layer_norm_bwd_workspace(int dtype, int64_t M, int64_t D, bool params) {
    if (!params || M == 0) return 0;
    const ln::Plan p = ln::plan(dtype, M, D, true);
    const int64_t rows = p.tpr ? p.blocks : ln::kWideChunks;
    return ln::al256((size_t)(2 * rows * D + (p.tpr ? 0 : 2 * M)) * sizeof(float));
}

int launch_layer_norm_fwd(int dtype, const void *x, const void *gamma, const void *beta, float eps, int64_t M, int64_t D, void *y,
                          void *stream) {
    if (M == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    return dtype == kBF16 ? ln::fwd_t<bf16>(dtype, x, gamma, beta, eps, M, D, y, st)
                          : ln::fwd_t<float>(dtype, x, gamma, beta, eps, M, D, y, st);
}

int launch_layer_norm_bwd(int dtype, const void *x, const void *dy, const void *gamma, float eps, int64_t M, int64_t D, void *dx,
                          void *dgamma, void *dbeta, void *ws, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    if (M == 0 && !dgamma && !dbeta) return 0;
    return dtype == kBF16 ? ln::bwd_t<bf16>(dtype, x, dy, gamma, eps, M, D, dx, dgamma, dbeta, ws, st)
                          : ln::bwd_t<float>(dtype, x, dy, gamma, eps, M, D, dx, dgamma, dbeta, ws, st);
}

}  // namespace ms
