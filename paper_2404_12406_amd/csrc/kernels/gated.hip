// Gated linear unit y = act(z_g) z_u over z = x W^T + b, W = [gate; up][2F][D]:
//   dz_g = dy z_u act'(z_g),  dz_u = dy act(z_g),
// after which the gradients are those of a Linear with the output gradient dz.
//
// bf16 runs on the fused contractions of gemm_fused.hip: the forward never
// writes z unless it is to be kept, and a backward without it takes z again and
// leaves dz in one pass.  fp32 runs the Linear contraction and the elementwise
// kernels below; so does a bf16 backward that kept z.  Those are bound by
// memory: 16 bytes a thread and access, a row's last vector element by element.
#include <algorithm>

#include "block_math.h"

namespace ms {

namespace g2 {
bool rows_ok(int64_t M, int64_t N, int64_t D, const void *x, const void *w);
int gate_fwd(int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *bias, void *y, void *proj,
             hipStream_t st);
int gate_grad(int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *bias, const void *dy, void *dz,
              hipStream_t st);
}  // namespace g2

namespace gated {

// Rows of a block's y index, then every gridDim.y-th; a thread one vector of each.
__global__ __launch_bounds__(256) void act_kernel(const float *__restrict__ z, int64_t M, int F, int kind, float *__restrict__ y) {
    using T = float;
    constexpr int V = Vec16<T>::N;
    constexpr bool FAST = false;
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * V;
    if (c >= F) return;
    for (int64_t r = blockIdx.y; r < M; r += gridDim.y) {
        const T *zr = z + r * 2 * F;
        const Vec16<T> g = load_vec(zr, c, F), u = load_vec(zr + F, c, F);
        Vec16<T> o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(act::value<FAST>(kind, to_f32(g.e[e])) * to_f32(u.e[e]));
        store_vec(y + r * F, c, F, o);
    }
}

// dz may be z itself: a thread reads both halves of its columns before it writes them.
__global__ __launch_bounds__(256) void grad_kernel(const float *z, const float *__restrict__ dy, int64_t M, int F, int kind,
                                                   float *dz) {
    using T = float;
    constexpr int V = Vec16<T>::N;
    constexpr bool FAST = false;
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * V;
    if (c >= F) return;
    for (int64_t r = blockIdx.y; r < M; r += gridDim.y) {
        const T *zr = z + r * 2 * F;
        Vec16<T> g = load_vec(zr, c, F), u = load_vec(zr + F, c, F);
        const Vec16<T> d = load_vec(dy + r * F, c, F);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float a, da;
            act::both<FAST>(kind, to_f32(g.e[e]), a, da);
            const float q = to_f32(d.e[e]);
            g.e[e] = from_f32<T>(q * to_f32(u.e[e]) * da);
            u.e[e] = from_f32<T>(q * a);
        }
        T *dr = dz + r * 2 * F;
        store_vec(dr, c, F, g);
        store_vec(dr + F, c, F, u);
    }
}

// The same from the kept 24-bit z of bf16 tensors: planes of its leading 16 bits
// and of the other 8.
__global__ __launch_bounds__(256) void grad24_kernel(const uint16_t *__restrict__ hi, const uint8_t *__restrict__ lo,
                                                     const bf16 *__restrict__ dy, int64_t M, int F, int kind,
                                                     bf16 *__restrict__ dz) {
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 8;
    if (c >= F) return;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef u32x2 bytes8 __attribute__((aligned(1)));
    auto read = [&](const uint16_t *h, const uint8_t *l, float (&z)[8]) {
        const Vec16<bf16> v = load_vec(reinterpret_cast<const bf16 *>(h), c, F);
        u32x2 b = {0u, 0u};
        if (c + 8 <= F) {
            b = *reinterpret_cast<const bytes8 *>(l + c);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < F) b[e / 4] |= (uint32_t)l[c + e] << (8 * (e % 4));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t w = v.u[e / 2], top = (e & 1) ? (w & 0xffff0000u) : (w << 16);
            z[e] = __uint_as_float(top | ((b[e / 4] >> (8 * (e % 4))) & 255u) << 8);
        }
    };
    for (int64_t r = blockIdx.y; r < M; r += gridDim.y) {
        float zg[8], zu[8];
        read(hi + r * 2 * F, lo + r * 2 * F, zg);
        read(hi + r * 2 * F + F, lo + r * 2 * F + F, zu);
        const Vec16<bf16> d = load_vec(dy + r * F, c, F);
        Vec16<bf16> g, u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a, da;
            act::both<true>(kind, zg[e], a, da);
            const float q = to_f32(d.e[e]);
            g.e[e] = from_f32<bf16>(q * zu[e] * da);
            u.e[e] = from_f32<bf16>(q * a);
        }
        bf16 *dr = dz + r * 2 * F;
        store_vec(dr, c, F, g);
        store_vec(dr + F, c, F, u);
    }
}

// dst[r][0 .. ld) = src[r][0 .. cols), then zeros
template <typename T>
__global__ __launch_bounds__(256) void pad_rows_kernel(const T *__restrict__ src, int64_t rows, int cols, T *__restrict__ dst, int ld) {
    constexpr int V = Vec16<T>::N;
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * V;
    if (c >= ld) return;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const Vec16<T> v = c < cols ? load_vec(src + r * cols, c, cols) : zero16<T>();
        store16(dst + r * ld + c, v);
    }
}

namespace {

dim3 grid(int64_t rows, int64_t cols, int V) {
    const int64_t gx = (cols + 256 * V - 1) / (256 * V);
    return dim3((unsigned)gx, (unsigned)std::max<int64_t>(1, std::min<int64_t>(rows, std::max<int64_t>(1, 8192 / gx))));
}

ConvGeom linear(int64_t M, int64_t K, int64_t N) {
    ConvGeom g{};
    g.N = (int)M;
    g.C = (int)K;
    g.K = (int)N;
    g.H = g.W = g.R = g.S = g.P = g.Q = g.sh = g.sw = 1;
    return g;
}

size_t al256(size_t n) { return (n + 255) / 256 * 256; }

int run_act(const void *z, int64_t M, int64_t F, int kind, void *y, hipStream_t st) {
    hipLaunchKernelGGL(act_kernel, grid(M, F, 4), dim3(256), 0, st, (const float *)z, M, (int)F, kind, (float *)y);
    return (int)hipGetLastError();
}

int run_grad(const void *z, const void *dy, int64_t M, int64_t F, int kind, void *dz, hipStream_t st) {
    hipLaunchKernelGGL(grad_kernel, grid(M, F, 4), dim3(256), 0, st, (const float *)z, (const float *)dy, M, (int)F, kind, (float *)dz);
    return (int)hipGetLastError();
}

int run_grad24(const void *z, const void *dy, int64_t M, int64_t F, int kind, void *dz, hipStream_t st) {
    hipLaunchKernelGGL(grad24_kernel, grid(M, F, 8), dim3(256), 0, st, (const uint16_t *)z, (const uint8_t *)z + M * 4 * F,
                       (const bf16 *)dy, M, (int)F, kind, (bf16 *)dz);
    return (int)hipGetLastError();
}

}  // namespace
}  // namespace gated

int launch_pad_rows(int dtype, const void *src, int64_t rows, int64_t cols, void *dst, int64_t ld, void *stream) {
    if (rows == 0 || ld == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == kBF16)
        hipLaunchKernelGGL(gated::pad_rows_kernel<bf16>, gated::grid(rows, ld, 8), dim3(256), 0, st, (const bf16 *)src, rows,
                           (int)cols, (bf16 *)dst, (int)ld);
    else
        hipLaunchKernelGGL(gated::pad_rows_kernel<float>, gated::grid(rows, ld, 4), dim3(256), 0, st, (const float *)src, rows,
                           (int)cols, (float *)dst, (int)ld);
    return (int)hipGetLastError();
}

bool gated_rows_ok(int64_t M, int64_t D, int64_t F, const void *x, const void *w, const void *b) {
    return g2::rows_ok(M, 2 * F, D, x, w) && (reinterpret_cast<uintptr_t>(b) & 3u) == 0;
}

// fp32: z where it is not kept, then the contraction's
size_t gated_fwd_workspace(int dtype, int64_t M, int64_t D, int64_t F, bool keep) {
    if (dtype == kBF16 || M == 0) return 0;
    return (keep ? 0 : gated::al256((size_t)M * 2 * F * 4)) + conv_fwd_workspace(dtype, gated::linear(M, D, 2 * F));
}

int launch_gated_fwd(int dtype, int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *b, void *y,
                     void *proj, void *ws, void *stream) {
    if (M == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == kBF16) {
        if (!gated_rows_ok(M, D, F, x, w, b)) return (int)hipErrorInvalidValue;
        return g2::gate_fwd(M, D, F, act, x, w, b, y, proj, st);
    }
    char *p = static_cast<char *>(ws);
    void *z = proj ? proj : p;
    if (!proj) p += gated::al256((size_t)M * 2 * F * 4);
    const int err = launch_conv_fwd(dtype, gated::linear(M, D, 2 * F), x, w, b, z, p, stream);
    return err ? err : gated::run_act(z, M, F, act, y, st);
}

// what launch_gated_dz itself needs: the fp32 contraction's
size_t gated_dz_workspace(int dtype, int64_t M, int64_t D, int64_t F, bool kept) {
    return dtype == kBF16 || kept || M == 0 ? 0 : conv_fwd_workspace(dtype, gated::linear(M, D, 2 * F));
}

int launch_gated_dz(int dtype, int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *b,
                    const void *proj, const void *dy, void *dz, void *ws, void *stream) {
    if (M == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    if (proj)
        return dtype == kBF16 ? gated::run_grad24(proj, dy, M, F, act, dz, st) : gated::run_grad(proj, dy, M, F, act, dz, st);
    if (dtype == kBF16) {
        if (!gated_rows_ok(M, D, F, x, w, b)) return (int)hipErrorInvalidValue;
        return g2::gate_grad(M, D, F, act, x, w, b, dy, dz, st);
    }
    const int err = launch_conv_fwd(dtype, gated::linear(M, D, 2 * F), x, w, b, dz, ws, stream);
    return err ? err : gated::run_grad(dz, dy, M, F, act, dz, st);
}

size_t linear_bwd_workspace(int dtype, int64_t M, int64_t K, int64_t N, bool dx, bool dw, bool db) {
    const ConvGeom g = gated::linear(M, K, N);
    size_t ws = 0;
    if (dx) ws = std::max(ws, conv_dgrad_workspace(dtype, g, db && !dw));
    if (dw) ws = std::max(ws, conv_wgrad_workspace(dtype, g, db));
    if (db) ws = std::max(ws, colsum_workspace(dtype, M, (int)N));
    return ws;
}

int launch_linear_bwd(int dtype, int64_t M, int64_t K, int64_t N, const void *dy, const void *x, const void *w, void *dx, void *dw,
                      void *db, void *ws, void *stream) {
    const ConvGeom g = gated::linear(M, K, N);
    bool done = false;
    int err = 0;
    if (dx) err = launch_conv_dgrad(dtype, g, dy, w, nullptr, dx, ws, stream, dw ? nullptr : db, &done);
    if (!err && dw) err = launch_conv_wgrad(dtype, g, dy, x, dw, db, ws, stream, &done);
    if (!err && db && !done) err = launch_colsum(dtype, dy, M, (int)N, db, ws, stream);
    return err;
}

}  // namespace ms
