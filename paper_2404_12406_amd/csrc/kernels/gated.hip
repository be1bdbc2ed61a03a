// Gated linear unit y = act(z_g) z_u over z = x W^T + b, W = [gate; up][2F][D]:
//   dz_g = dy z_u act'(z_g),  dz_u = dy act(z_g),
// after which the gradients are those of a Linear with the output gradient dz.
//
// bf16 runs on the fused contractions of gemm_gate.hip: the forward never
// writes z unless it is to be kept, and a backward without it takes z again and
// leaves dz in one pass.  fp32 runs the Linear contraction and the elementwise
// kernels below; so does a bf16 backward that kept z.  Those are bound by
// memory: 16 bytes a thread and access, a row's last vector element by element.
//
// Measured, us: 8192 x 768 x 2 x 2048 bf16, trained: forward 81, dz from the kept
// projections 33 (184 MB, 5.5 TB/s), dx 60 with W's transpose, dW 84 with the sum of
// its partials.  4096 x 2048 x 2 x 5504, from the input alone: forward 163, dz 175,
// dx 158 from W in place and 13 for the sum of its two partials.  1001 x 515 x 2 x
// 1366 fp32, trained: z 35, dx 40, dW 42, everything else 45 in eight launches.
#include <algorithm>

#include "block_math.h"
#include "limits_f32.h"
#include "../../../include/memsave.h"
#include "../../../include/memsave_testing.h"

namespace ms {

namespace g2 {
bool rows_ok(int64_t M, int64_t N, int64_t D, const void *x, const void *w);
int gate_fwd(int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *bias, void *y, void *proj,
             hipStream_t st);
int gate_grad(int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *bias, const void *dy, void *dz,
              hipStream_t st);
int place_splits(int64_t M, int64_t D, int64_t K);
size_t place_dx_workspace(int64_t M, int64_t D, int64_t K);
int place_dx(int64_t M, int64_t D, int64_t K, const void *dz, const void *w, void *dx, void *ws, hipStream_t st);
}  // namespace g2

namespace tok {
bool applies(int dtype, int64_t M, int64_t N, int64_t K, const void *x, const void *w);
int gate(int dtype, int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *b, void *y, void *proj,
         hipStream_t st);
}  // namespace tok

namespace gated {

// Rows of a block's y index, then every gridDim.y-th; a thread one vector of each.
// z has rows of 2 Fp, its halves at 0 and Fp.
__global__ __launch_bounds__(256) void act_kernel(const float *__restrict__ z, int64_t M, int F, int Fp, int kind,
                                                  float *__restrict__ y) {
    using T = float;
    constexpr int V = Vec16<T>::N;
    constexpr bool FAST = false;
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * V;
    if (c >= F) return;
    for (int64_t r = blockIdx.y; r < M; r += gridDim.y) {
        const T *zr = z + r * 2 * Fp;
        const Vec16<T> g = load_vec(zr, c, F), u = load_vec(zr + Fp, c, F);
        Vec16<T> o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(act::value<FAST>(kind, to_f32(g.e[e])) * to_f32(u.e[e]));
        store_vec(y + r * F, c, F, o);
    }
}

// dz may be z itself: a thread reads both halves of its columns before it writes
// them.  Columns F .. Fp - 1 of both halves become zeros.
__global__ __launch_bounds__(256) void grad_kernel(const float *z, const float *__restrict__ dy, int64_t M, int F, int Fp, int kind,
                                                   float *dz) {
    using T = float;
    constexpr int V = Vec16<T>::N;
    constexpr bool FAST = false;
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * V;
    if (c >= Fp) return;
    for (int64_t r = blockIdx.y; r < M; r += gridDim.y) {
        const T *zr = z + r * 2 * Fp;
        Vec16<T> g = load_vec(zr, c, Fp), u = load_vec(zr + Fp, c, Fp);
        const Vec16<T> d = c < F ? load_vec(dy + r * F, c, F) : zero16<T>();
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float a, da;
            act::both<FAST>(kind, to_f32(g.e[e]), a, da);
            const float q = to_f32(d.e[e]);
            const bool in = c + e < F;
            g.e[e] = in ? q * to_f32(u.e[e]) * da : 0.f;
            u.e[e] = in ? q * a : 0.f;
        }
        T *dr = dz + r * 2 * Fp;
        store_vec(dr, c, Fp, g);
        store_vec(dr + Fp, c, Fp, u);
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

// Up to kCopies copies at once (grid y): dst[r][0 .. dld) = src[r][0 .. cols) and
// zeros for r < rows, zeros for r to drows (cols at most dld, or the other columns
// are left out).
struct Copies {
    CopyJob job[kCopies];
};
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(const Copies k) {
    constexpr int V = Vec16<T>::N;
    const CopyJob &j = k.job[blockIdx.y];
    const T *src = (const T *)j.src;
    T *dst = (T *)j.dst;
    const int cols = (int)min(j.cols, j.dld), dld = (int)j.dld, per = (dld + V - 1) / V;
    // (row, vector of the row) of this thread, moved on by whole steps of the grid
    const int step = (int)gridDim.x * 256, dr = step / per, dc = step % per;
    const int i = (int)blockIdx.x * 256 + (int)threadIdx.x;
    int64_t r = i / per;
    for (int c = i % per; r < j.drows; r += dr) {
        store_vec(dst + r * dld, c * V, dld, r < j.rows && c * V < cols ? load_vec(src + r * j.sld, c * V, cols) : zero16<T>());
        c += dc;
        if (c >= per) {
            c -= per;
            ++r;
        }
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

int run_act(const void *z, int64_t M, int64_t F, int64_t Fp, int kind, void *y, hipStream_t st) {
    hipLaunchKernelGGL(act_kernel, grid(M, F, 4), dim3(256), 0, st, (const float *)z, M, (int)F, (int)Fp, kind, (float *)y);
    return (int)hipGetLastError();
}

int run_grad(const void *z, const void *dy, int64_t M, int64_t F, int64_t Fp, int kind, void *dz, hipStream_t st) {
    hipLaunchKernelGGL(grad_kernel, grid(M, Fp, 4), dim3(256), 0, st, (const float *)z, (const float *)dy, M, (int)F, (int)Fp, kind,
                       (float *)dz);
    return (int)hipGetLastError();
}

int run_grad24(const void *z, const void *dy, int64_t M, int64_t F, int kind, void *dz, hipStream_t st) {
    hipLaunchKernelGGL(grad24_kernel, grid(M, F, 8), dim3(256), 0, st, (const uint16_t *)z, (const uint8_t *)z + M * 4 * F,
                       (const bf16 *)dy, M, (int)F, kind, (bf16 *)dz);
    return (int)hipGetLastError();
}

bool al(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Zero-padded copies of operands that the contractions do not take, or take slowly:
// bf16 rows of D values that are no whole 16-byte vectors, or not so aligned (the
// copies have D rounded up to 8); for fp32, where D is no multiple of 4 or F is
// odd, copies with D and F rounded up to 32 and 16 instead of the contractions'
// 4-byte loads (1001 x 515 -> 2 x 1366, trained: 211 us with those, 165 with copies).
// Few rows are not worth a copy of W.
constexpr int64_t kPadRows = 96;

struct Pads {
    int64_t D, F;            // as the contractions see them
    bool x, w, b, any;
    size_t ox, ow, ob, bytes;
};

Pads pads(int dtype, int64_t M, int64_t D, int64_t F, const void *x, const void *w, const void *b) {
    Pads p{D, F, false, false, false, false, 0, 0, 0, 0};
    const size_t e = dtype == kBF16 ? 2 : 4;
    if (dtype == kBF16) {
        p.D = (D + 7) / 8 * 8;
        p.x = p.D != D || !al(x, 16);
        p.w = p.D != D || !al(w, 16);
        p.b = b && !al(b, 4);
    } else if (M >= kPadRows) {
        const int64_t Dp = (D + 31) / 32 * 32, Fp = (F + 15) / 16 * 16;
        // (not past what the contractions take: the narrowest rows grow many times)
        if ((D % 4 || F % 2) && std::max({M * Dp, M * 2 * Fp, 2 * Fp * Dp}) <= g2::kMostFloats) {
            p.D = Dp;
            p.F = Fp;
        }
        p.x = p.D != D || !al(x, 16);
        p.w = p.D != D || p.F != F || !al(w, 16);
        p.b = b && p.F != F;
    }
    p.any = p.D != D || p.F != F;
    p.ow = p.x ? al256((size_t)M * p.D * e) : 0;
    p.ob = p.ow + (p.w ? al256((size_t)2 * p.F * p.D * e) : 0);
    p.bytes = p.ob + (p.b ? al256((size_t)2 * p.F * e) : 0);
    return p;
}

// the copies, in `base`; x, w and b move to them
int make_pads(const Pads &p, int dtype, int64_t M, int64_t D, int64_t F, char *base, const void **x, const void **w, const void **b,
              void *stream) {
    const size_t e = dtype == kBF16 ? 2 : 4;
    CopyJob j[kCopies];
    int n = 0;
    if (p.x) {
        j[n++] = {*x, D, M, D, base + p.ox, M, p.D};
        *x = base + p.ox;
    }
    if (p.w) {
        const char *s = static_cast<const char *>(*w);
        for (int h = 0; h < 2; ++h) j[n++] = {s + (size_t)h * F * D * e, D, F, D, base + p.ow + (size_t)h * p.F * p.D * e, p.F, p.D};
        *w = base + p.ow;
    }
    if (p.b) {
        const char *s = static_cast<const char *>(*b);
        for (int h = 0; h < 2; ++h) j[n++] = {s + (size_t)h * F * e, F, 1, F, base + p.ob + (size_t)h * p.F * e, 1, p.F};
        *b = base + p.ob;
    }
    return launch_copy_rows(dtype, j, n, stream);
}

}  // namespace
}  // namespace gated

int launch_copy_rows(int dtype, const CopyJob *jobs, int n, void *stream) {
    gated::Copies k{};
    const int V = dtype == kBF16 ? 8 : 4;
    int64_t most = 0;   // vectors of the largest
    int used = 0;
    for (int i = 0; i < n; ++i) {
        if (jobs[i].drows == 0 || jobs[i].dld == 0) continue;
        k.job[used++] = jobs[i];
        most = std::max(most, jobs[i].drows * ((jobs[i].dld + V - 1) / V));
    }
    if (!used) return 0;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)std::min<int64_t>((most + 255) / 256, 4096), (unsigned)used);
    if (dtype == kBF16) hipLaunchKernelGGL(gated::copy_rows_kernel<bf16>, grid, dim3(256), 0, st, k);
    else hipLaunchKernelGGL(gated::copy_rows_kernel<float>, grid, dim3(256), 0, st, k);
    return (int)hipGetLastError();
}

size_t linear_bwd_workspace(int dtype, int64_t M, int64_t K, int64_t N, bool dx, bool dw, bool db) {
    ConvGeom g = gated::linear(M, K, N);
    g.fine = true;
    size_t ws = 0;
    if (dx) ws = std::max(ws, conv_dgrad_workspace(dtype, g, db && !dw));
    if (dw) ws = std::max(ws, conv_wgrad_workspace(dtype, g, db));
    if (db) ws = std::max(ws, colsum_workspace(dtype, M, (int)N));
    return ws;
}

int launch_linear_bwd(int dtype, int64_t M, int64_t K, int64_t N, int64_t wrows, const int *count, const void *dy, const void *x, const void *w,
                      void *dx, void *dw, void *db, void *ws, void *stream) {
    ConvGeom g = gated::linear(M, K, N);
    g.count = count;
    g.wrows = wrows < N ? (int)wrows : 0;
    g.fine = true;
    bool done = false;
    int err = 0;
    if (dx) err = launch_conv_dgrad(dtype, g, dy, w, nullptr, dx, ws, stream, dw ? nullptr : db, &done);
    if (!err && dw) err = launch_conv_wgrad(dtype, g, dy, x, dw, db, ws, stream, &done);
    if (!err && db && !done) err = launch_colsum(dtype, dy, M, (int)N, db, ws, stream);
    return err;
}

// the copies, then (fp32) z where it is not kept and the contraction's workspace
size_t gated_fwd_workspace(int dtype, int64_t M, int64_t D, int64_t F, const void *x, const void *w, const void *b, bool keep) {
    if (M == 0) return 0;
    const gated::Pads p = gated::pads(dtype, M, D, F, x, w, b);
    if (dtype == kBF16) return p.bytes;
    return p.bytes + (keep ? 0 : gated::al256((size_t)M * 2 * p.F * 4)) + conv_fwd_workspace(dtype, gated::linear(M, p.D, 2 * p.F));
}

int launch_gated_fwd(int dtype, int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *b, void *y,
                     void *proj, void *ws, void *stream) {
    if (M == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
    const gated::Pads p = gated::pads(dtype, M, D, F, x, w, b);
    char *c = static_cast<char *>(ws);
    int err = gated::make_pads(p, dtype, M, D, F, c, &x, &w, &b, stream);
    if (err) return err;
    // (p.F is F wherever the few rows' kernel applies)
    // (not where fp32 has few outputs for its inputs: the large contraction splits k.  16 x
    // 4096 x 2 x 256 25 and 33 us from the caches and not, there 16 and 17; 16 x 2048 x 2 x
    // 1024 15 and 22, there 16 and 19; 16 x 1024 x 2 x 4096 10 and 21, there 18 and 25)
    const bool split = dtype != kBF16 && D % 4 == 0 && D > 4 * F;
    if (!split && tok::applies(dtype, M, 2 * F, p.D, x, w)) return tok::gate(dtype, M, p.D, F, act, x, w, b, y, proj, st);
    if (dtype == kBF16) {
        if (!g2::rows_ok(M, 2 * F, p.D, x, w)) return (int)hipErrorInvalidValue;
        return g2::gate_fwd(M, p.D, F, act, x, w, b, y, proj, st);
    }
    c += p.bytes;
    void *z = proj ? proj : c;
    if (!proj) c += gated::al256((size_t)M * 2 * p.F * 4);
    err = launch_conv_fwd(dtype, gated::linear(M, p.D, 2 * p.F), x, w, b, z, c, stream);
    return err ? err : gated::run_act(z, M, F, p.F, act, y, st);
}

namespace gated {
namespace {

// Workspace of a backward: dz, the copies, padded gradients, the contractions'.
struct Bwd {
    Pads p;
    bool place;   // dx from W in place
    size_t dz, pad, gx, gw, gb, work, bytes;
};

Bwd bwd_plan(int dtype, int64_t M, int64_t D, int64_t F, const void *x, const void *w, const void *b, bool kept, bool dx, bool dw, bool db) {
    Bwd k{};
    // bf16 contractions of the backward take any D themselves: copies only to take z again
    k.p = dtype == kBF16 && kept ? Pads{D, F} : pads(dtype, M, D, F, x, w, b);
    const bool f32 = dtype != kBF16;
    const size_t e = f32 ? 4 : 2;
    const int64_t Dp = f32 ? k.p.D : D, Fp = k.p.F;
    k.dz = 0;
    k.pad = al256((size_t)M * 2 * Fp * e);
    k.gx = k.pad + k.p.bytes;
    k.gw = k.gx + (f32 && dx && Dp != D ? al256((size_t)M * Dp * e) : 0);
    k.gb = k.gw + (f32 && dw && k.p.any ? al256((size_t)2 * Fp * Dp * e) : 0);
    k.work = k.gb + (f32 && db && Fp != F ? al256((size_t)2 * Fp * e) : 0);
    k.place = !f32 && dx && (reinterpret_cast<uintptr_t>(w) & 15u) == 0 && g2::place_splits(M, D, 2 * F) > 0;
    size_t ws = linear_bwd_workspace(dtype, M, Dp, 2 * Fp, dx && !k.place, dw, db);
    if (k.place) ws = std::max(ws, g2::place_dx_workspace(M, D, 2 * F));
    if (f32 && !kept && M) ws = std::max(ws, conv_fwd_workspace(dtype, linear(M, Dp, 2 * Fp)));
    k.bytes = k.work + ws;
    return k;
}

// As launch_gated_bwd() lays it out: no rows need no z, as if it were kept.
Bwd launch_plan(int dtype, int64_t M, int64_t D, int64_t F, const void *x, const void *w, const void *b, const void *proj, bool dx, bool dw,
                bool db) {
    return bwd_plan(dtype, M, D, F, x, w, b, proj || M == 0, dx, dw, db);
}

}  // namespace
}  // namespace gated

size_t gated_bwd_workspace(int dtype, int64_t M, int64_t D, int64_t F, const void *x, const void *w, const void *b, bool kept, bool dx,
                           bool dw, bool db) {
    return gated::bwd_plan(dtype, M, D, F, x, w, b, kept, dx, dw, db).bytes;
}

int launch_gated_bwd(int dtype, int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *b, const void *proj,
                     const void *dy, void *dx, void *dw, void *db, void *ws, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    const gated::Bwd k = gated::launch_plan(dtype, M, D, F, x, w, b, proj, dx, dw, db);
    char *c = static_cast<char *>(ws);
    void *dz = c + k.dz;
    const void *xp = x, *wp = w, *bp = b;
    // (a kept z leaves only the operands of the gradients asked for)
    gated::Pads p = k.p;
    if (proj) {
        p.x = p.x && dw;
        p.w = p.w && dx;
        p.b = false;
    }
    int err = M ? gated::make_pads(p, dtype, M, D, F, c + k.pad, &xp, &wp, &bp, stream) : 0;
    if (err) return err;
    if (dtype == kBF16) {
        if (M && proj) {
            err = gated::run_grad24(proj, dy, M, F, act, dz, st);
        } else if (M) {
            if (!g2::rows_ok(M, 2 * F, k.p.D, xp, wp)) return (int)hipErrorInvalidValue;
            err = g2::gate_grad(M, k.p.D, F, act, xp, wp, bp, dy, dz, st);
        }
        if (!err && k.place) err = g2::place_dx(M, D, 2 * F, dz, w, dx, c + k.work, st);
        if (err || (k.place && !dw && !db)) return err;
        return launch_linear_bwd(dtype, M, D, 2 * F, 2 * F, nullptr, dz, x, w, k.place ? nullptr : dx, dw, db, c + k.work, stream);
    }
    const int64_t Dp = k.p.D, Fp = k.p.F;
    if (M && !proj) err = launch_conv_fwd(dtype, gated::linear(M, Dp, 2 * Fp), xp, wp, bp, dz, c + k.work, stream);
    if (!err && M) err = gated::run_grad(proj ? proj : dz, dy, M, F, Fp, act, dz, st);
    const bool tx = dx && Dp != D, tw = dw && k.p.any, tb = db && Fp != F;   // gradients by way of padded ones
    char *gx = c + k.gx, *gw = c + k.gw, *gb = c + k.gb;
    if (!err)
        err = launch_linear_bwd(dtype, M, Dp, 2 * Fp, 2 * Fp, nullptr, dz, xp, wp, tx ? gx : dx, tw ? gw : dw, tb ? gb : db, c + k.work, stream);
    CopyJob j[kCopies];
    int n = 0;
    if (tx) j[n++] = {gx, Dp, M, D, dx, M, D};
    for (int h = 0; h < 2; ++h) {
        if (tw) j[n++] = {gw + (size_t)h * Fp * Dp * 4, Dp, F, D, (float *)dw + (size_t)h * F * D, F, D};
        if (tb) j[n++] = {gb + (size_t)h * Fp * 4, Fp, 1, F, (float *)db + (size_t)h * F, 1, F};
    }
    return err ? err : launch_copy_rows(dtype, j, n, stream);
}

}  // namespace ms

extern "C" void ms_testing_gated_plan(int32_t dtype, int64_t rows, int64_t D, int64_t F, int32_t proj, int32_t aligned, uint32_t mask,
                                      int64_t out[4]) {
    const void *p = aligned ? nullptr : reinterpret_cast<const void *>(uintptr_t(2));   // (nothing is read)
    const void *z = proj && rows ? out : nullptr;
    const bool dx = mask & MS_RG_INPUT, dw = mask & MS_RG_WEIGHT, db = mask & MS_RG_BIAS;
    const ms::gated::Bwd k = ms::gated::launch_plan(dtype, rows, D, F, p, p, nullptr, z, dx, dw, db);
    out[0] = (int64_t)ms::gated_bwd_workspace(dtype, rows, D, F, p, p, nullptr, proj || !rows, dx, dw, db);
    out[1] = (int64_t)k.bytes;
    out[2] = k.p.D;
    out[3] = k.p.F;
}
