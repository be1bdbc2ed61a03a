// Softmax cross entropy of a linear head over a large vocabulary,
//   z = x W^T + b,  loss_i = log sum_v exp(z_iv) - z_it,  t the row's target,
//   dz = (exp(z - lse) - [v = t]) scale_i,  dx = dz W,  dW = dz^T x,  db = sum of dz,
// without keeping z.
//
//  * Rows whose target is the ignored one take no part: the others are gathered
//    first (their number stays on the device and bounds every contraction), so
//    that whatever an ignored row holds, NaN included, reaches no result, and a
//    prompt costs nothing.
//  * bf16: the contraction's epilogue (gemm_fused.hip) leaves, per row and column
//    tile, the maximum and the sum of exponentials; combine_kernel joins them.
//    Backward goes over the vocabulary in pieces of at most kPieceBytes of dz:
//    z again, dz from its epilogue, dx added up in fp32, dW whole.
//  * fp32: the same steps on the fp32 contraction, z a piece at a time in
//    workspace and the softmax's passes by the row kernels below.
// Exponentials are of differences from a maximum or an lse, which no logit of
// any size overflows; a row's lse is kept in fp32.
#include <algorithm>

#include "block_math.h"

namespace ms {

namespace g2 {
bool rows_ok(int64_t M, int64_t N, int64_t D, const void *x, const void *w);
int xent_lse_tiles(int64_t M, int64_t D, int64_t V);
int xent_lse(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
             void *stat, float *tlogit, hipStream_t st);
int xent_grad(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
              int v0, const float *lse, const float *scale, void *dz, int64_t ldz, hipStream_t st);
SplitRule xent_dx_rule(int64_t M, int64_t D, int64_t V);
int xent_dx(int64_t M, int64_t D, int64_t V, int64_t ldz, int64_t piece, const void *dz, const void *w, const int *count,
            const int *nsplit, float *part, bool add, hipStream_t st);
size_t xent_dw_workspace(int64_t M, int64_t D, int64_t Dr, int64_t V, bool db);
int xent_dw(int64_t M, int64_t D, int64_t Dr, int64_t V, int64_t ldz, const void *dz, const void *x, const int *count,
            const float *scale, void *dw, void *db, void *ws, hipStream_t st);
}  // namespace g2

namespace tok {
bool applies(int dtype, int64_t M, int64_t N, int64_t K, const void *x, const void *w);
size_t xent_workspace();
int xent(int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *b, const int64_t *target, int64_t ignore,
         int reduction, float *loss, float *lse, void *ws, hipStream_t st);
}  // namespace tok

namespace xent {

// The rows that count, in order: idx[i] the i-th, pos[r] its place or -1, tgt[i]
// its target (-1 where that is no word), *count their number.  One block: 4096
// rows a turn, their places from the ballots of its 16 waves.
__global__ __launch_bounds__(1024) void rows_kernel(const int64_t *__restrict__ target, int64_t ignore, int64_t M, int64_t V,
                                                    int *__restrict__ pos, int *__restrict__ idx, int *__restrict__ tgt,
                                                    int *__restrict__ count) {
    __shared__ int sums[4 * 16];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int base = 0;
    for (int64_t r0 = 0; r0 < M; r0 += 4096) {
        int64_t t[4];
        unsigned long long in[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t r = r0 + k * 1024 + threadIdx.x;
            t[k] = r < M ? target[r] : ignore;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            in[k] = __ballot(t[k] != ignore);
            if (lane == 0) sums[k * 16 + w] = __popcll(in[k]);
        }
        __syncthreads();
        int before = base;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            int mine = before, all = 0;
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int s = sums[k * 16 + q];
                mine += q < w ? s : 0;
                all += s;
            }
            const int64_t r = r0 + k * 1024 + threadIdx.x;
            if (r < M) {
                const bool c = (in[k] >> lane) & 1;
                const int i = mine + __popcll(in[k] & ((1ull << lane) - 1));
                pos[r] = c ? i : -1;
                if (c) {
                    idx[i] = (int)r;
                    tgt[i] = t[k] >= 0 && t[k] < V ? (int)t[k] : -1;
                }
            }
            before += all;
        }
        base = before;
        __syncthreads();   // the sums are read
    }
    if (threadIdx.x == 0) *count = base;
}

// xc[i][0 .. ld) = x[idx[i]] and zeros past D, for the rows that count; the others'
// rows are zeros where `fill`.  With lse: lsec[i], and the loss's gradient as a
// factor of the row's dz, scale[i], and one of all results, scale[M].  Where it is
// the same for every row (mean, sum) it stays out of dz: that is rounded, and a
// common factor would give every row's largest entry, near -1 times it, the same
// rounding error.
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(const T *__restrict__ x, const int *__restrict__ idx,
                                                     const int *__restrict__ count, int64_t M, int D, int ld, bool fill,
                                                     T *__restrict__ xc, const float *__restrict__ lse,
                                                     const float *__restrict__ gloss, int reduction, float *__restrict__ lsec,
                                                     float *__restrict__ scale, SplitRule rule, int *__restrict__ nsplit) {
    constexpr int V = Vec16<T>::N;
    const int n = *count;
    if (nsplit && blockIdx.x == 0 && threadIdx.x == 64) *nsplit = rule.splits(n);
    // (no row that counts: every result is an empty sum, whatever the factor)
    if (lse && blockIdx.x == 0 && threadIdx.x == 0)
        scale[M] = reduction == 2 || n == 0 ? 1.f : reduction == 1 ? gloss[0] : gloss[0] / (float)n;
    for (int64_t i = blockIdx.x; i < M; i += gridDim.x) {
        if (i >= n && !fill) break;
        const int64_t r = i < n ? idx[i] : 0;
        for (int c = (int)threadIdx.x * V; c < ld; c += 256 * V)
            store_vec(xc + i * ld, c, ld, i < n && c < D ? load_vec(x + r * D, c, D) : zero16<T>());
        if (lse && threadIdx.x == 0) {
            lsec[i] = i < n ? lse[r] : 0.f;
            scale[i] = i >= n ? 0.f : reduction == 2 ? gloss[r] : 1.f;
        }
    }
}

// The loss and lse of every row from `parts` statistics [part][M] of the rows
// that count (32 rows a block, eight threads each).
__global__ __launch_bounds__(256) void combine_kernel(const floatx2 *__restrict__ stat, int parts, const float *__restrict__ tlogit,
                                                      const int *__restrict__ pos, const int *__restrict__ tgt, int64_t M,
                                                      float *__restrict__ each, float *__restrict__ lse) {
    __shared__ floatx2 red[8][32];
    const int row = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int64_t r = (int64_t)blockIdx.x * 32 + row;
    const int i = r < M ? pos[r] : -1;
    floatx2 a = {-INFINITY, 0.f};
    if (i >= 0) {
        int p = grp;
        for (; p + 24 < parts; p += 32) {
            floatx2 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = stat[(int64_t)(p + 8 * u) * M + i];
#pragma unroll
            for (int u = 0; u < 4; ++u) a = join_lse(a, v[u]);
        }
        for (; p < parts; p += 8) a = join_lse(a, stat[(int64_t)p * M + i]);
    }
    red[grp][row] = a;
    __syncthreads();
    if (grp != 0 || r >= M) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) a = join_lse(a, red[q][row]);
    float l = 0.f, loss = 0.f;
    if (i >= 0) {
        // no word at all, or every one of them minus infinity: no distribution
        l = tgt[i] < 0 || a.x == -INFINITY ? NAN : a.x + logf(a.y);
        loss = l - (tgt[i] < 0 ? 0.f : tlogit[i]);
    }
    if (lse) lse[r] = l;
    each[r] = loss;
}

// *out = the sum of each[0 .. M), over *count where it is to be the mean.
__global__ __launch_bounds__(1024) void total_kernel(const float *__restrict__ each, int64_t M, const int *__restrict__ count,
                                                     bool mean, float *__restrict__ out) {
    __shared__ double red[16];
    double s = 0.0;
    for (int64_t r = threadIdx.x; r < M; r += 1024) s += (double)each[r];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 16; ++w) s += red[w];
    *out = (float)(mean ? s / (double)*count : s);
}

// dx[r] = *scale (null: 1) times the sum of the partials of the row's place, or zeros.
template <typename T>
__global__ __launch_bounds__(256) void finish_kernel(const float *__restrict__ part, const int *__restrict__ nsplit, int64_t stride,
                                                     const int *__restrict__ pos, int64_t M, int D, int ld, const float *__restrict__ scale,
                                                     T *__restrict__ dx) {
    constexpr int V = Vec16<T>::N;
    const float f = scale ? *scale : 1.f;
    const int splits = nsplit ? *nsplit : 1;
    for (int64_t r = blockIdx.x; r < M; r += gridDim.x) {
        const int i = pos[r];
        for (int c = (int)threadIdx.x * V; c < D; c += 256 * V) {
            Vec16<T> o = zero16<T>();
            if (i >= 0) {
                float s[V];
#pragma unroll
                for (int e = 0; e < V; ++e) s[e] = 0.f;
                for (int z = 0; z < splits; ++z) {
#pragma unroll
                    for (int h = 0; h < V / 4; ++h) {
                        const Vec16<float> p = load_vec(part + z * stride + (int64_t)i * ld, c + 4 * h, ld);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[4 * h + e] += p.e[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(s[e] * f);
            }
            store_vec(dx + r * D, c, D, o);
        }
    }
}

// db[v] = *scale times the sum over the rows that count of dz[i][v]: 16 columns of eight a
// block, 16 threads each (a bias trained without its weight).
__global__ __launch_bounds__(256) void bias_kernel(const bf16 *__restrict__ dz, int64_t ldz, const int *__restrict__ count, int V,
                                                   const float *__restrict__ scale, bf16 *__restrict__ db) {
    __shared__ float red[16][16 * 8 + 4];
    const int col = threadIdx.x & 15, grp = threadIdx.x >> 4, n = *count;
    const int c = ((int)blockIdx.x * 16 + col) * 8;
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.f;
    if (c < V)
        for (int64_t i = grp; i < n; i += 16) {
            const Vec16<bf16> v = load16(dz + i * ldz + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += to_f32(v.e[e]);
        }
#pragma unroll
    for (int e = 0; e < 8; ++e) red[grp][col * 8 + e] = s[e];
    __syncthreads();
    if (threadIdx.x >= 128) return;
    const int v = (int)blockIdx.x * 128 + (int)threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 16; ++q) t += red[q][threadIdx.x];
    if (v < V) db[v] = (bf16)(t * *scale);
}

// ------------------------------------------------------------------ fp32 pieces
// A piece's logits z[i][0 .. V) in rows of ldz, words v0 on: joins the row's statistics (those
// of the first piece start them) and takes the target's logit.  A block a row.
__global__ __launch_bounds__(256) void lse_rows_kernel(const float *__restrict__ z, int ldz, int V, int v0, const int *__restrict__ count,
                                                       const int *__restrict__ tgt, bool first, floatx2 *__restrict__ stat,
                                                       float *__restrict__ tlogit) {
    __shared__ floatx2 red[4];
    const int n = *count;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const float *zr = z + i * ldz;
        float top = -INFINITY;
        for (int c = (int)threadIdx.x * 4; c < V; c += 1024) {
            const Vec16<float> v = load_vec(zr, c, V);
#pragma unroll
            for (int e = 0; e < 4; ++e) top = c + e < V ? fmaxf(top, v.e[e]) : top;
        }
        const float t0 = top == -INFINITY ? 0.f : top;
        float s = 0.f;
        for (int c = (int)threadIdx.x * 4; c < V; c += 1024) {
            const Vec16<float> v = load_vec(zr, c, V);
#pragma unroll
            for (int e = 0; e < 4; ++e) s += c + e < V ? exp_below(v.e[e], t0) : 0.f;
        }
        floatx2 a = {top, s};
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) a = join_lse(a, floatx2{__shfl_xor(a.x, o), __shfl_xor(a.y, o)});
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 4; ++w) a = join_lse(a, red[w]);
            stat[i] = first ? a : join_lse(stat[i], a);
            const int t = tgt[i] - v0;
            if (tgt[i] >= 0 && t >= 0 && t < V) tlogit[i] = zr[t];
        }
        __syncthreads();
    }
}

// z -> dz in place; the rows that do not count and the columns past V become zeros.
__global__ __launch_bounds__(256) void grad_rows_kernel(float *__restrict__ z, int ldz, int V, int v0, int64_t M, const int *__restrict__ count,
                                                        const int *__restrict__ tgt, const float *__restrict__ lse,
                                                        const float *__restrict__ scale) {
    const int n = *count;
    const float factor = scale[M];   // (what a common rounding error of 2^-24 would do does not matter)
    for (int64_t i = blockIdx.x; i < M; i += gridDim.x) {
        const bool in = i < n;
        const float l = in ? lse[i] : 0.f, sc = in ? scale[i] * factor : 0.f;
        const int t = in ? tgt[i] - v0 : -1;
        for (int c = (int)threadIdx.x * 4; c < ldz; c += 1024) {
            Vec16<float> v = load_vec(z + i * ldz, c, ldz);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = exp_below(v.e[e], l) - (c + e == t ? 1.f : 0.f);
                v.e[e] = in && c + e < V ? p * sc : 0.f;
            }
            store_vec(z + i * ldz, c, ldz, v);
        }
    }
}

__global__ __launch_bounds__(256) void add_kernel(float *__restrict__ acc, const float *__restrict__ v, int64_t n) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
        if (i + 4 <= n) {
            *reinterpret_cast<floatx4 *>(acc + i) += *reinterpret_cast<const floatx4 *>(v + i);
        } else {
            for (int64_t k = i; k < n; ++k) acc[k] += v[k];
        }
    }
}

// ------------------------------------------------------------------ host
namespace {

// dz of a piece: enough words that a contraction fills the card many times over,
// and a small part of its memory.  8192 x 768 x 50000 trained, a third of the rows
// ignored: pieces of 128, 256, 512 and 1024 MiB 2.31, 2.30, 2.24 and 2.15 ms; 4096 x
// 4096 x 128000, the head frozen, 10.5, 10.4, 10.3 and 10.3.
constexpr int64_t kPieceBytes = int64_t(1) << 30;

size_t al256(size_t n) { return (n + 255) / 256 * 256; }

int64_t piece(int dtype, int64_t M, int64_t V) {
    const int64_t bytes = std::max<int64_t>(M, 1) * V * (dtype == kBF16 ? 2 : 4);
    const int64_t n = (bytes + kPieceBytes - 1) / kPieceBytes;
    return std::min(V, ((V + n - 1) / n + 255) / 256 * 256);
}

ConvGeom linear(int64_t M, int64_t K, int64_t N) {
    ConvGeom g{};
    g.N = (int)M;
    g.C = (int)K;
    g.K = (int)N;
    g.H = g.W = g.R = g.S = g.P = g.Q = g.sh = g.sw = 1;
    return g;
}

// fp32 contractions take 16-byte loads where widths are multiples of 4 and take
// twice as long or more where they are not: from kPadRows rows on (fewer are not
// worth a copy of W) such a piece runs on zero-padded copies of its rows of W and
// its biases, as wide and as many as these say.
constexpr int64_t kPadRows = 96;
int64_t f32_width(int64_t M, int64_t D) { return M >= kPadRows && D % 4 ? (D + 31) / 32 * 32 : D; }
int64_t f32_words(int64_t M, int64_t V) { return M >= kPadRows && V % 4 ? (V + 31) / 32 * 32 : V; }

// A piece's operands as the contractions take them.
struct Piece {
    int64_t n, np;          // words, and columns of z
    const float *w, *b;
    float *dw, *db;         // the gradients' places, padded or the caller's
    bool own;               // padded
};

// Workspace of a call, carved in order.
struct Carve {
    char *base;
    size_t off = 0;
    template <typename T>
    T *get(int64_t n) {
        T *p = base ? reinterpret_cast<T *>(base + off) : nullptr;
        off += al256((size_t)std::max<int64_t>(n, 0) * sizeof(T));
        return p;
    }
    void *raw(size_t bytes) {
        void *p = base ? base + off : nullptr;
        off += al256(bytes);
        return p;
    }
};

struct Rows {
    int *pos, *idx, *tgt, *count;
    void *xc, *wp, *bp;   // gathered rows; padded weight and bias where they are needed
    int64_t D8;
};

Rows carve_rows(Carve &c, int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb) {
    Rows r{};
    r.D8 = dtype == kBF16 ? (D + 7) / 8 * 8 : f32_width(M, D);
    r.pos = c.get<int>(M);
    r.idx = c.get<int>(M);
    r.tgt = c.get<int>(M);
    r.count = c.get<int>(1);
    r.xc = c.raw((size_t)M * r.D8 * (dtype == kBF16 ? 2 : 4));
    r.wp = padw ? c.raw((size_t)V * r.D8 * 2) : nullptr;
    r.bp = padb ? c.raw((size_t)((V + 7) / 8 * 8) * 2) : nullptr;
    return r;
}

struct Fwd {
    Rows r;
    void *stat;
    float *tlogit, *each;
    float *z;      // fp32: a piece's logits,
    float *wp, *bp;   // its padded operands
    void *conv;    // and the contraction's workspace
};

Fwd carve_fwd(Carve &c, int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb, bool each) {
    Fwd f{};
    f.r = carve_rows(c, dtype, M, D, V, padw, padb);
    f.stat = c.get<floatx2>((dtype == kBF16 && M ? g2::xent_lse_tiles(M, f.r.D8, V) : 1) * M);
    f.tlogit = c.get<float>(M);
    f.each = each ? c.get<float>(M) : nullptr;
    if (dtype != kBF16) {
        const int64_t p = piece(dtype, M, V), last = V - (V - 1) / p * p, most = std::max(f32_words(M, p), f32_words(M, last));
        f.z = c.get<float>(M * most);
        f.wp = M >= kPadRows ? c.get<float>(most * f.r.D8) : nullptr;
        f.bp = M >= kPadRows ? c.get<float>(most) : nullptr;
        size_t ws = 0;
        for (int64_t v : {p, last}) ws = std::max(ws, conv_fwd_workspace(dtype, linear(M, f.r.D8, f32_words(M, v))));
        f.conv = c.raw(ws);
    }
    return f;
}

struct Bwd {
    Rows r;
    float *lse, *scale;
    void *dz;
    float *part;     // partials of dx (fp32: the sum and a piece's)
    float *wp, *bp, *gwp, *gbp;   // fp32: a piece's padded operands and gradients
    void *work;      // the contractions' workspace
    SplitRule rule;  // bf16: of the contraction for dx
    int *nsplit;
};

Bwd carve_bwd(Carve &c, int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb, bool dx, bool dw, bool db) {
    Bwd b{};
    b.r = carve_rows(c, dtype, M, D, V, padw, padb);
    b.lse = c.get<float>(M);
    b.scale = c.get<float>(M + 1);
    const int64_t p = piece(dtype, M, V), last = V - (V - 1) / p * p;
    const int64_t most = dtype == kBF16 ? (p + 7) / 8 * 8 : std::max(f32_words(M, p), f32_words(M, last));
    b.dz = c.raw((size_t)M * most * (dtype == kBF16 ? 2 : 4));
    if (dtype != kBF16 && M >= kPadRows) {
        b.wp = c.get<float>(most * b.r.D8);
        b.bp = c.get<float>(most);
        b.gwp = dw ? c.get<float>(most * b.r.D8) : nullptr;
        b.gbp = db ? c.get<float>(most) : nullptr;
    }
    size_t ws = 0;
    for (int64_t v : {p, last}) {
        if (dtype == kBF16) {
            if (dw) ws = std::max(ws, g2::xent_dw_workspace(M, b.r.D8, D, v, db));
        } else {
            ws = std::max(ws, conv_fwd_workspace(dtype, linear(M, b.r.D8, f32_words(M, v))));
            ws = std::max(ws, linear_bwd_workspace(dtype, M, b.r.D8, f32_words(M, v), dx, dw, db));
        }
    }
    if (dx) {
        if (dtype == kBF16) {
            b.rule = g2::xent_dx_rule(M, b.r.D8, p);
            b.nsplit = c.get<int>(1);
        }
        b.part = c.get<float>((dtype == kBF16 ? b.rule.most : p < V ? 2 : 1) * M * b.r.D8);
    }
    b.work = c.raw(ws);
    return b;
}

int row_grid(int64_t M) { return (int)std::max<int64_t>(1, std::min<int64_t>(M, 8192)); }

// The rows that count and what the contractions read.
int start(const Rows &r, int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void **w, const void **b,
          const int64_t *target, int64_t ignore, const float *lse, const float *gloss, int reduction, float *lsec, float *scale,
          const SplitRule &rule, int *nsplit, hipStream_t st) {
    hipLaunchKernelGGL(rows_kernel, dim3(1), dim3(1024), 0, st, target, ignore, M, V, r.pos, r.idx, r.tgt, r.count);
    if (dtype == kBF16)
        hipLaunchKernelGGL(gather_kernel<bf16>, dim3(row_grid(M)), dim3(256), 0, st, (const bf16 *)x, r.idx, r.count, M, (int)D,
                           (int)r.D8, false, (bf16 *)r.xc, lse, gloss, reduction, lsec, scale, rule, nsplit);
    else
        hipLaunchKernelGGL(gather_kernel<float>, dim3(row_grid(M)), dim3(256), 0, st, (const float *)x, r.idx, r.count, M, (int)D,
                           (int)r.D8, true, (float *)r.xc, lse, gloss, reduction, lsec, scale, rule, nsplit);
    int err = (int)hipGetLastError();
    CopyJob j[kCopies];
    int n = 0;
    if (r.wp) {
        j[n++] = {*w, D, V, D, r.wp, V, r.D8};
        *w = r.wp;
    }
    if (r.bp && *b) {
        j[n++] = {*b, V, 1, V, r.bp, 1, V};
        *b = r.bp;
    }
    if (!err) err = launch_copy_rows(kBF16, j, n, st);
    return err;
}

// fp32: the words v0 .. v0 + n - 1, their operands copied where they are to be padded.
int take_piece(Piece *q, int64_t M, int64_t D, int64_t D8, int64_t v0, int64_t n, const void *w, const void *b, float *wp, float *bp,
               hipStream_t st) {
    q->n = n;
    q->np = f32_words(M, n);
    q->w = (const float *)w + v0 * D;
    q->b = b ? (const float *)b + v0 : nullptr;
    q->own = wp && (q->np != n || D8 != D || (reinterpret_cast<uintptr_t>(q->w) & 15u));
    if (!q->own) return 0;
    CopyJob j[kCopies] = {{q->w, D, n, D, wp, q->np, D8}};
    q->w = wp;
    if (b) {
        j[1] = {q->b, n, 1, n, bp, 1, q->np};
        q->b = bp;
    }
    return launch_copy_rows(kF32, j, b ? 2 : 1, st);
}

int logits(const Piece &q, const Rows &r, int64_t M, float *z, void *ws, hipStream_t st) {
    ConvGeom g = linear(M, r.D8, q.np);
    g.count = r.count;
    return launch_conv_fwd(kF32, g, r.xc, q.w, q.b, z, ws, st);
}

}  // namespace
}  // namespace xent

size_t xent_fwd_workspace(int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb, int reduction) {
    xent::Carve c{nullptr};
    xent::carve_fwd(c, dtype, M, D, V, padw, padb, reduction != 2);
    return std::max(c.off, tok::xent_workspace());
}

int launch_xent_fwd(int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *b, bool padw, bool padb,
                    const int64_t *target, int64_t ignore, int reduction, float *loss, float *lse, void *ws, void *stream) {
    using namespace xent;
    hipStream_t st = (hipStream_t)stream;
    if (tok::applies(dtype, M, V, D, x, w)) return tok::xent(dtype, M, D, V, x, w, b, target, ignore, reduction, loss, lse, ws, st);
    Carve c{static_cast<char *>(ws)};
    const Fwd f = carve_fwd(c, dtype, M, D, V, padw, padb, reduction != 2);
    int err = start(f.r, dtype, M, D, V, x, &w, &b, target, ignore, nullptr, nullptr, reduction, nullptr, nullptr, SplitRule{}, nullptr, st);
    if (err) return err;
    int parts = 1;
    if (M == 0) {
    } else if (dtype == kBF16) {
        if (!g2::rows_ok(M, V, f.r.D8, f.r.xc, w)) return (int)hipErrorInvalidValue;
        parts = g2::xent_lse_tiles(M, f.r.D8, V);
        err = g2::xent_lse(M, f.r.D8, V, f.r.xc, w, b, f.r.count, f.r.tgt, f.stat, f.tlogit, st);
    } else {
        const int64_t p = piece(dtype, M, V);
        for (int64_t v0 = 0; v0 < V && !err; v0 += p) {
            const int64_t n = std::min(p, V - v0);
            Piece q;
            err = take_piece(&q, M, D, f.r.D8, v0, n, w, b, f.wp, f.bp, st);
            if (!err) err = logits(q, f.r, M, f.z, f.conv, st);
            if (err) break;
            hipLaunchKernelGGL(lse_rows_kernel, dim3(row_grid(M)), dim3(256), 0, st, f.z, (int)q.np, (int)n, (int)v0, f.r.count, f.r.tgt,
                               v0 == 0, (floatx2 *)f.stat, f.tlogit);
            err = (int)hipGetLastError();
        }
    }
    if (err) return err;
    float *each = reduction == 2 ? loss : f.each;
    if (M > 0)
        hipLaunchKernelGGL(combine_kernel, dim3((unsigned)((M + 31) / 32)), dim3(256), 0, st, (const floatx2 *)f.stat, parts, f.tlogit,
                           f.r.pos, f.r.tgt, M, each, lse);
    if (reduction != 2)
        hipLaunchKernelGGL(total_kernel, dim3(1), dim3(1024), 0, st, each, M, f.r.count, reduction == 0, loss);
    return (int)hipGetLastError();
}

size_t xent_bwd_workspace(int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb, bool dx, bool dw, bool db) {
    xent::Carve c{nullptr};
    xent::carve_bwd(c, dtype, M, D, V, padw, padb, dx, dw, db);
    return c.off;
}

int launch_xent_bwd(int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *b, bool padw, bool padb,
                    const int64_t *target, int64_t ignore, int reduction, const float *gloss, const float *lse, void *dx, void *dw,
                    void *db, void *ws, void *stream) {
    using namespace xent;
    hipStream_t st = (hipStream_t)stream;
    Carve c{static_cast<char *>(ws)};
    const Bwd k = carve_bwd(c, dtype, M, D, V, padw, padb, dx, dw, db);
    int err = start(k.r, dtype, M, D, V, x, &w, &b, target, ignore, lse, gloss, reduction, k.lse, k.scale, k.rule, k.nsplit, st);
    if (err) return err;
    const int64_t p = piece(dtype, M, V), D8 = k.r.D8;
    if (dtype == kBF16 && M > 0 && !g2::rows_ok(M, V, D8, k.r.xc, w)) return (int)hipErrorInvalidValue;
    for (int64_t v0 = 0; v0 < V && !err; v0 += p) {
        const int64_t n = std::min(p, V - v0);
        if (dtype == kBF16) {
            const int64_t ldz = (n + 7) / 8 * 8;
            const bf16 *wv = (const bf16 *)w + v0 * D8;
            if (M > 0)
                err = g2::xent_grad(M, D8, n, k.r.xc, wv, b ? (const bf16 *)b + v0 : nullptr, k.r.count, k.r.tgt, (int)v0, k.lse, k.scale,
                                    k.dz, ldz, st);
            if (!err && dx && M > 0) err = g2::xent_dx(M, D8, n, ldz, p, k.dz, wv, k.r.count, k.nsplit, k.part, v0 > 0, st);
            bf16 *dbv = db ? (bf16 *)db + v0 : nullptr;
            if (!err && dw)
                err = g2::xent_dw(M, D8, D, n, ldz, k.dz, k.r.xc, k.r.count, k.scale + M, (bf16 *)dw + v0 * D, dbv, k.work, st);
            else if (!err && db) {
                hipLaunchKernelGGL(bias_kernel, dim3((unsigned)((n + 127) / 128)), dim3(256), 0, st, (const bf16 *)k.dz, ldz, k.r.count,
                                   (int)n, k.scale + M, dbv);
                err = (int)hipGetLastError();
            }
        } else {
            float *z = (float *)k.dz, *tmp = k.part + (v0 > 0 ? M * D8 : 0);
            float *dwv = dw ? (float *)dw + v0 * D : nullptr, *dbv = db ? (float *)db + v0 : nullptr;
            Piece q;
            err = take_piece(&q, M, D, D8, v0, n, w, b, k.wp, k.bp, st);
            if (!err && M > 0) {
                err = logits(q, k.r, M, z, k.work, st);
                if (err) break;
                hipLaunchKernelGGL(grad_rows_kernel, dim3(row_grid(M)), dim3(256), 0, st, z, (int)q.np, (int)n, (int)v0, M, k.r.count,
                                   k.r.tgt, k.lse, k.scale);
                err = (int)hipGetLastError();
            }
            const bool tw = dw && (q.np != n || D8 != D), tb = db && q.np != n;
            if (!err)
                err = launch_linear_bwd(dtype, M, D8, q.np, k.r.count, z, k.r.xc, q.w, dx && M > 0 ? tmp : nullptr, tw ? k.gwp : dwv,
                                        tb ? k.gbp : dbv, k.work, stream);
            CopyJob j[kCopies];
            int jobs = 0;
            if (tw) j[jobs++] = {k.gwp, D8, n, D, dwv, n, D};
            if (tb) j[jobs++] = {k.gbp, n, 1, n, dbv, 1, n};
            if (!err) err = launch_copy_rows(kF32, j, jobs, stream);
            if (!err && dx && v0 > 0 && M > 0) {
                hipLaunchKernelGGL(add_kernel, dim3((unsigned)std::min<int64_t>((M * D8 + 1023) / 1024, 4096)), dim3(256), 0, st, k.part,
                                   tmp, M * D8);
                err = (int)hipGetLastError();
            }
        }
    }
    if (err || !dx || M == 0) return err;
    if (dtype == kBF16)
        hipLaunchKernelGGL(finish_kernel<bf16>, dim3(row_grid(M)), dim3(256), 0, st, k.part, k.nsplit, M * D8, k.r.pos, M, (int)D, (int)D8,
                           k.scale + M, (bf16 *)dx);
    else
        hipLaunchKernelGGL(finish_kernel<float>, dim3(row_grid(M)), dim3(256), 0, st, k.part, (const int *)nullptr, M * D8, k.r.pos, M, (int)D, (int)D8,
                           (const float *)nullptr, (float *)dx);   // (its dz has the factor)
    return (int)hipGetLastError();
}

}  // namespace ms
