// Softmax cross entropy of a linear head over a large vocabulary,
//   z = x W^T + b,  loss_i = log sum_v exp(z_iv) - z_it,  t the row's target,
//   dz = (exp(z - lse) - [v = t]) scale_i,  dx = dz W,  dW = dz^T x,  db = sum of dz,
// without keeping z.
//
//  * A target with nearly all of the probability leaves a loss and a dz that are small
//    differences of numbers near 1.  So it stays out of the sums: with l the log of the
//    sum of the others' exponentials, loss = log(1 + exp(l - z_t)) and dz_t = -scale /
//    (1 + exp(z_t - l)) (row_loss()).  A record keeps l; backward takes z_t of each row
//    again where it gathers the rows, and has both lse and dz_t from the two.
//  * Rows whose target is the ignored one take no part: the others are gathered
//    first (their number stays on the device and bounds every contraction), so
//    that whatever an ignored row holds, NaN included, reaches no result, and a
//    prompt costs nothing.
//  * bf16: the contraction's epilogue (gemm_xent.hip) leaves, per row and column
//    tile, the maximum and the sum of exponentials; combine_kernel joins them.
//    Backward goes over the vocabulary in pieces of at most kPieceBytes of dz:
//    z again, dz from its epilogue, dx added up in fp32, dW whole.
//  * fp32: the same steps on the fp32 contraction, z a piece at a time in
//    workspace and the softmax's passes by the row kernels below.
//  * dx alone (a frozen head) is taken in the forward, while the exponentials are
//    at hand, and kept in place of x: two contractions in all instead of three.  It
//    is dx without the loss's gradient, which backward multiplies it by.  bf16: by
//    chunks of rows, whose exponentials p = exp(z - r) are written as bf16 beside
//    their sums, r a reference that combine_kernel() then makes one of each row:
//      dx = (1 / sum) p W - (1 - p_t) W_t
//    with the target's p left out of p W, so that what is left of it at a large
//    p_t is no difference of rounded numbers.
// Exponentials are of differences from a maximum or an lse, which no logit of
// any size overflows; what is kept of a row, and its lse, are in fp32.
//
// Measured, us.  8192 x 768 x 50000 bf16, a third of the rows ignored, head trained:
// statistics 414, dz 498, dx 397, dW 414, everything else 84.  4096 x 4096 x 128000,
// head frozen: exponentials 3632, dx 3313, the rest 120.  777 x 514 x 10007 fp32,
// trained: z 72 (twice), dx 81 and 7 for the sum of its partials, dW 75, the softmax's
// passes 23, padded copies 25, eight small launches 42.
#include <algorithm>
#include <type_traits>

#include "block_math.h"
#include "limits_f32.h"
#include "../../../include/memsave_testing.h"

namespace ms {

namespace g2 {
bool rows_ok(int64_t M, int64_t N, int64_t D, const void *x, const void *w);
int xent_lse_tiles(int64_t M, int64_t D, int64_t V);
int xent_lse(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
             void *stat, float *tlogit, hipStream_t st);
int xent_grad(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
              int v0, const float *lse, const float *scale, const float *ct, void *dz, int64_t ldz, float *rest, float *dbpart,
              hipStream_t st);
void xent_bias_rows(int64_t M, int64_t D, int64_t V, int *tile, int *rows);
int xent_prob_parts(int64_t M, int64_t D, int64_t V);
int xent_prob(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
              void *stat, int64_t stat_ld, float *tlogit, void *prob, int64_t ldz, hipStream_t st);
SplitRule xent_dx_rule(int64_t M, int64_t D, int64_t V);
int xent_dx(int64_t M, int64_t D, int64_t V, int64_t ldz, int64_t piece, const void *dz, const void *w, const int *count,
            const int *nsplit, float *part, bool add, hipStream_t st);
size_t xent_dw_workspace(int64_t M, int64_t D, int64_t V);
int xent_dw(int64_t M, int64_t D, int64_t Dr, int64_t V, int64_t ldz, const void *dz, const void *x, const int *count,
            const float *scale, void *dw, void *ws, hipStream_t st);
}  // namespace g2

namespace tok {
bool applies(int dtype, int64_t M, int64_t N, int64_t K, const void *x, const void *w);
size_t xent_workspace();
int xent(int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *b, const int64_t *target, int64_t ignore,
         int reduction, float *loss, float *others, void *ws, hipStream_t st);
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
// rows are zeros where `fill`.  With others (the kept log-sums of the words but the
// targets, w and bias then being theirs): the row's lse[i] and the target's entry of its
// dz, ct[i], from the target's logit, and the loss's gradient as a
// factor of the row's dz, scale[i], and one of all results, scale[M].  Where it is
// the same for every row (mean, sum) it stays out of dz: that is rounded, and a
// common factor would give every row's largest entry, near -1 times it, the same
// rounding error.  With nsplit: the splits of dx's contraction for each chunk of
// `chunk` rows, and (ccount) the chunks' numbers of rows.
// SCAN: rows_kernel() is part of it: each block counts the rows before its own, for up
// to kScanRows (one launch less; 16 bits hold a count).
constexpr int kScanRows = 2048;
template <typename T, bool SCAN>
__global__ __launch_bounds__(256) void gather_kernel(const int64_t *__restrict__ target, int64_t ignore, int64_t words, int *__restrict__ pos,
                                                     int *__restrict__ tgt, const T *__restrict__ x, const int *__restrict__ idx,
                                                     int *__restrict__ count, int64_t M, int D, int ld, bool fill,
                                                     T *__restrict__ xc, const float *__restrict__ others,
                                                     const T *__restrict__ w, const T *__restrict__ bias,
                                                     const float *__restrict__ gloss, int reduction, float *__restrict__ lse,
                                                     float *__restrict__ ct, float *__restrict__ scale, SplitRule rule,
                                                     int *__restrict__ nsplit, int64_t chunk, int *__restrict__ ccount) {
    constexpr int V = Vec16<T>::N;
    __shared__ float red[4];
    int n, at = 0;        // the rows that count; SCAN: the place of this block's row
    bool counts = true;
    if constexpr (SCAN) {
        __shared__ int sums[4];
        const int r = (int)blockIdx.x;
        int c = 0;   // all of them in the low half, those before r in the high one
        for (int k = (int)threadIdx.x; k < M; k += 256) c += target[k] != ignore ? (k < r ? 0x10001 : 1) : 0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o);
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = c;
        __syncthreads();
        c = sums[0] + sums[1] + sums[2] + sums[3];
        n = c & 0xffff;
        at = c >> 16;
        if (threadIdx.x == 0) {
            if (r == 0) *count = n;
            if (r < M) {
                const int64_t t = target[r];
                counts = t != ignore;
                pos[r] = counts ? at : -1;
                if (counts) tgt[at] = t >= 0 && t < words ? (int)t : -1;
            }
        }
        if (r < M) counts = target[r] != ignore;
        if (!counts) at = n + r - at;   // the others' places come after
    } else {
        n = *count;
    }
    if (nsplit && blockIdx.x == 0)
        for (int64_t k = (int)threadIdx.x; k * chunk < M; k += 256) {
            const int rows = (int)min(max(n - k * chunk, (int64_t)0), chunk);
            nsplit[k] = rule.splits(rows);
            if (ccount) ccount[k] = rows;
        }
    // (no row that counts: every result is an empty sum, whatever the factor)
    if (scale && blockIdx.x == 0 && threadIdx.x == 0)   // (nothing is kept of no rows, which still have a factor)
        scale[M] = reduction == 2 || n == 0 ? 1.f : reduction == 1 ? gloss[0] : gloss[0] / (float)n;
    for (int64_t k = blockIdx.x; k < M; k += gridDim.x) {
        const int64_t i = SCAN ? at : k;
        if (i >= n && !fill) break;
        const int64_t r = i >= n ? 0 : SCAN ? k : idx[i];
        const int64_t t = others && i < n ? target[r] : -1;
        const bool word = t >= 0 && t < words;
        float z = 0.f;   // this thread's part of the target's logit
        for (int c = (int)threadIdx.x * V; c < ld; c += 256 * V) {
            const Vec16<T> v = i < n && c < D ? load_vec(x + r * D, c, D) : zero16<T>();
            store_vec(xc + i * ld, c, ld, v);
            if (word && c < D) {
                const Vec16<T> wt = load_vec(w + t * D, c, D);
#pragma unroll
                for (int e = 0; e < V; ++e) z += to_f32(v.e[e]) * to_f32(wt.e[e]);
            }
        }
        if (!others) continue;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = z;
        __syncthreads();
        if (threadIdx.x == 0) {
            float l = 0.f, c = 0.f;
            if (i < n) {
                z = word ? red[0] + red[1] + red[2] + red[3] + (bias ? to_f32(bias[t]) : 0.f) : NAN;
                const float rest = others[r], d = rest - z;   // (one of them may be minus infinity)
                l = fmaxf(rest, z) + log1pf(expf(-fabsf(d)));
                c = target_entry(d);
            }
            lse[i] = l;
            ct[i] = c;
            scale[i] = i >= n ? 0.f : reduction == 2 ? gloss[r] : 1.f;
        }
        __syncthreads();   // red is read
    }
}

// What dx needs of a row that counts, by its place: the reference of its
// exponentials, 1 / their sum, and the coefficient -(1 - p_t) of W_t.
struct Kept {
    float *ref, *f, *ct;
};

// The loss of every row and what is kept of it, others[], from `parts` statistics [part][ld] of the rows that
// count, of which this launch has those from place i0 to i0 + ld - 1 (8 rows a
// block, 32 threads each).  With prob (exponentials [ld][ldz] of kProbCols columns a
// part): the parts of a row with another reference than the row's are brought to it.
__global__ __launch_bounds__(256) void combine_kernel(const floatx2 *__restrict__ stat, int parts, int64_t ld, int64_t i0,
                                                      const float *__restrict__ tlogit, const int *__restrict__ pos,
                                                      const int *__restrict__ tgt, int64_t M, float *__restrict__ each,
                                                      float *__restrict__ others, Kept kept, bf16 *__restrict__ prob, int64_t ldz) {
    constexpr int ROWS = 8, GROUPS = 256 / ROWS;
    __shared__ floatx2 red[GROUPS][ROWS];
    const int row = threadIdx.x % ROWS, grp = threadIdx.x / ROWS;
    const int64_t r = (int64_t)blockIdx.x * ROWS + row;
    const int i = r < M ? pos[r] : -1;
    const bool here = i >= i0 && i < i0 + ld;
    const floatx2 *s = stat + (here ? i - i0 : 0);
    floatx2 a = {-INFINITY, 0.f};
    if (here) {
        int p = grp;
        for (; p + 3 * GROUPS < parts; p += 4 * GROUPS) {
            floatx2 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = s[(int64_t)(p + GROUPS * u) * ld];
#pragma unroll
            for (int u = 0; u < 4; ++u) a = join_lse(a, v[u]);
        }
        for (; p < parts; p += GROUPS) a = join_lse(a, s[(int64_t)p * ld]);
    }
    red[grp][row] = a;
    __syncthreads();
    if (grp == 0) {
        for (int q = 1; q < GROUPS; ++q) a = join_lse(a, red[q][row]);
        red[0][row] = a;
        if (r < M && (i < 0 || here)) {
            float l = 0.f, loss = 0.f;
            if (here) {
                const float z = tgt[i] < 0 ? NAN : tlogit[i];
                const RowLoss q = row_loss(a, z);
                l = q.others;
                loss = q.loss;
                if (kept.ref) {   // (bf16: the exponentials have their reference already)
                    const floatx2 all = prob ? floatx2{a.x, a.y + exp_below(z, a.x)} : join_lse(a, floatx2{z, 1.f});
                    kept.ref[i] = all.x;
                    kept.f[i] = q.loss != q.loss ? NAN : 1.f / all.y;
                    kept.ct[i] = q.ct;
                }
            }
            if (others) others[r] = l;
            each[r] = loss;
        }
    }
    if (!prob) return;
    __syncthreads();
    if (!here) return;
    const float to = red[0][row].x;
    for (int p = grp; p < parts; p += GROUPS) {
        const float from = s[(int64_t)p * ld].x;
        if (from == to || from == -INFINITY) continue;   // (nothing but zeros there)
        const float f = exp_below(from, to);
        bf16 *at = prob + (i - i0) * ldz + (int64_t)p * kProbCols;
        for (int c = 0; c < kProbCols && (int64_t)p * kProbCols + c < ldz; c += 8) {
            Vec16<bf16> v = load16(at + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) v.e[e] = from_f32<bf16>(to_f32(v.e[e]) * f);
            *reinterpret_cast<u32x4 *>(at + c) = v.u;
        }
    }
}

// *out = the sum of each[0 .. M), over *count where it is to be the mean: a block of N.
template <int N>
__device__ __forceinline__ void total(const float *__restrict__ each, int64_t M, const int *__restrict__ count, bool mean,
                                      float *__restrict__ out) {
    __shared__ double red[N / 64];
    double s = 0.0;
    for (int64_t r = threadIdx.x; r < M; r += N) s += (double)each[r];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < N / 64; ++w) s += red[w];
    *out = (float)(mean ? s / (double)*count : s);
}

__global__ __launch_bounds__(1024) void total_kernel(const float *__restrict__ each, int64_t M, const int *__restrict__ count,
                                                     bool mean, float *__restrict__ out) {
    total<1024>(each, M, count, mean, out);
}

// The kept gradient of the rows at places i0 .. i0 + chunk - 1, and zeros (by the first
// chunk's launch) for the rows that do not count: the sum of the partials, with f
// times it and ct times the target's row of w; over their number where the loss is
// the mean.  bf16: in 24 bits, a plane [M][D] of the leading 16 and one of the others
// (rounded once more when backward has multiplied it: 2^-17 does not show).  With
// loss, one more block takes its sum from each row's.
template <typename T>
__global__ __launch_bounds__(256) void keep_kernel(const float *__restrict__ part, const int *__restrict__ nsplit, int64_t stride,
                                                   const int *__restrict__ pos, int64_t M, int D, int ld, int64_t i0, int64_t chunk,
                                                   const int *__restrict__ count, bool mean, const float *__restrict__ f,
                                                   const float *__restrict__ ct, const int *__restrict__ tgt, const T *__restrict__ w,
                                                   void *__restrict__ kept, const float *__restrict__ each, float *__restrict__ loss) {
    constexpr int V = Vec16<T>::N;
    const int blocks = (int)gridDim.x - (loss ? 1 : 0);
    if ((int)blockIdx.x == blocks) {
        total<256>(each, M, count, mean, loss);
        return;
    }
    const int splits = nsplit ? *nsplit : 1;
    const float all = mean ? 1.f / (float)*count : 1.f;
    for (int64_t r = blockIdx.x; r < M; r += blocks) {
        const int i = pos[r];
        if (i < 0 ? i0 > 0 : i < i0 || i >= i0 + chunk) continue;
        const int t = i < 0 || !f ? -1 : tgt[i];
        for (int c = (int)threadIdx.x * V; c < D; c += 256 * V) {
            float s[V];
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] = 0.f;
            if (i >= 0) {
                for (int z = 0; z < splits; ++z) {
#pragma unroll
                    for (int h = 0; h < V / 4; ++h) {
                        const Vec16<float> p = load_vec(part + z * stride + (i - i0) * ld, c + 4 * h, ld);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[4 * h + e] += p.e[e];
                    }
                }
                if (f) {
                    const Vec16<T> wt = t >= 0 ? load_vec(w + (int64_t)t * ld, c, ld) : zero16<T>();
#pragma unroll
                    for (int e = 0; e < V; ++e) s[e] = s[e] * f[i] + ct[i] * to_f32(wt.e[e]);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) s[e] *= all;   // (not for a row that does not count: it may be that none does)
            }
            if constexpr (V == 8) {
                Vec16<bf16> hi;
                uint8_t *lo = (uint8_t *)kept + 2 * M * D + r * D + c;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t u = to_f24(s[e]);
                    hi.e[e] = __builtin_bit_cast(bf16, (uint16_t)(u >> 8));
                    if (c + e < D) lo[e] = (uint8_t)u;
                }
                store_vec((bf16 *)kept + r * D, c, D, hi);
            } else {
                Vec16<float> o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o.e[e] = s[e];
                store_vec((float *)kept + r * D, c, D, o);
            }
        }
    }
}

// dx = the kept gradient times the loss's.
template <typename T>
__global__ __launch_bounds__(256) void scale_kernel(const void *__restrict__ kept, int64_t M, int D, const float *__restrict__ gloss,
                                                    bool each, T *__restrict__ dx) {
    constexpr int V = Vec16<T>::N;
    for (int64_t r = blockIdx.x; r < M; r += gridDim.x) {
        const float g = gloss[each ? r : 0];
        for (int c = (int)threadIdx.x * V; c < D; c += 256 * V) {
            Vec16<T> o = load_vec((const T *)kept + r * D, c, D);
            const uint8_t *lo = (const uint8_t *)kept + 2 * M * D + r * D + c;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float v = to_f32(o.e[e]);
                if constexpr (V == 8)
                    v = __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, o.e[e]) << 16 | (c + e < D ? (uint32_t)lo[e] << 8 : 0u));
                // (a row that does not count stays zero whatever the gradient)
                o.e[e] = from_f32<T>(v == 0.f ? 0.f : v * g);
            }
            store_vec(dx + r * D, c, D, o);
        }
    }
}

// dx[r] = *scale (null: 1) times the sum of the partials of the row's place, or zeros.
// With rest: the partials are those of rounded dz, of which a target's entry is most
// of a row: what rounding took from it, times the target's row of w, is put back.
template <typename T>
__global__ __launch_bounds__(256) void finish_kernel(const float *__restrict__ part, const int *__restrict__ nsplit, int64_t stride,
                                                     const int *__restrict__ pos, int64_t M, int D, int ld, const float *__restrict__ scale,
                                                     const float *__restrict__ rest, const int *__restrict__ tgt, const T *__restrict__ w,
                                                     T *__restrict__ dx) {
    constexpr int V = Vec16<T>::N;
    const float f = scale ? *scale : 1.f;
    const int splits = nsplit ? *nsplit : 1;
    for (int64_t r = blockIdx.x; r < M; r += gridDim.x) {
        const int i = pos[r], t = rest && i >= 0 ? tgt[i] : -1;
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
                if (t >= 0) {
                    const Vec16<T> wt = load_vec(w + (int64_t)t * ld, c, ld);
#pragma unroll
                    for (int e = 0; e < V; ++e) s[e] += rest[i] * to_f32(wt.e[e]);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(s[e] * f);
            }
            store_vec(dx + r * D, c, D, o);
        }
    }
}

// db[v] = *scale times the sum of the contraction's column sums, one row of them for
// `rows` rows of dz: those of dz before it was rounded.  (A target's entry of dz is
// near -1 in every row, so a rounded one would be off by much the same in all.)
__global__ __launch_bounds__(256) void bias_kernel(const float *__restrict__ part, int tile, int rows, const int *__restrict__ count, int V,
                                                   const float *__restrict__ scale, bf16 *__restrict__ db) {
    const int v = (int)blockIdx.x * 256 + (int)threadIdx.x, n = (*count + tile - 1) / tile * (tile / rows);
    if (v >= V) return;
    float s = 0.f;
    int r = 0;
    for (; r + 4 <= n; r += 4) {
        float p[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) p[u] = part[(int64_t)(r + u) * V + v];
#pragma unroll
        for (int u = 0; u < 4; ++u) s += p[u];
    }
    for (; r < n; ++r) s += part[(int64_t)r * V + v];
    db[v] = (bf16)(s * *scale);
}

// ------------------------------------------------------------------ fp32 pieces
// A piece's logits z[i][0 .. V) in rows of ldz, words v0 on: joins the row's statistics (those
// of the first piece start them), without its target, whose logit it takes.  A block a row.
__global__ __launch_bounds__(256) void lse_rows_kernel(const float *__restrict__ z, int ldz, int V, int v0, const int *__restrict__ count,
                                                       const int *__restrict__ tgt, bool first, floatx2 *__restrict__ stat,
                                                       float *__restrict__ tlogit) {
    __shared__ floatx2 red[4];
    const int n = *count;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const float *zr = z + i * ldz;
        const int t = tgt[i] < 0 ? -1 : tgt[i] - v0;
        float top = -INFINITY;
        for (int c = (int)threadIdx.x * 4; c < V; c += 1024) {
            const Vec16<float> v = load_vec(zr, c, V);
#pragma unroll
            for (int e = 0; e < 4; ++e) top = c + e < V && c + e != t ? fmaxf(top, v.e[e]) : top;
        }
        const float t0 = top == -INFINITY ? 0.f : top;
        float s = 0.f;
        for (int c = (int)threadIdx.x * 4; c < V; c += 1024) {
            const Vec16<float> v = load_vec(zr, c, V);
#pragma unroll
            for (int e = 0; e < 4; ++e) s += c + e < V && c + e != t ? exp_below(v.e[e], t0) : 0.f;
        }
        floatx2 a = {top, s};
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) a = join_lse(a, floatx2{__shfl_xor(a.x, o), __shfl_xor(a.y, o)});
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 4; ++w) a = join_lse(a, red[w]);
            stat[i] = first ? a : join_lse(stat[i], a);
            if (t >= 0 && t < V) tlogit[i] = zr[t];
        }
        __syncthreads();
    }
}

// z -> dz in place; the rows that do not count and the columns past V become zeros.
// The softmax is exp(z - lse), or (inv) inv exp(z - lse), lse then being a reference
// and inv the sum's inverse; ct: the target's entry.
__global__ __launch_bounds__(256) void grad_rows_kernel(float *__restrict__ z, int ldz, int V, int v0, int64_t M, const int *__restrict__ count,
                                                        const int *__restrict__ tgt, const float *__restrict__ lse,
                                                        const float *__restrict__ inv, const float *__restrict__ ct,
                                                        const float *__restrict__ scale) {
    const int n = *count;
    const float factor = scale ? scale[M] : 1.f;   // (what a common rounding error of 2^-24 would do does not matter)
    for (int64_t i = blockIdx.x; i < M; i += gridDim.x) {
        const bool in = i < n;
        const float l = in ? lse[i] : 0.f, f = in && inv ? inv[i] : 1.f, sc = in ? (scale ? scale[i] : 1.f) * factor : 0.f;
        const int t = in ? tgt[i] - v0 : -1;
        const float pt = in ? ct[i] : 0.f;
        for (int c = (int)threadIdx.x * 4; c < ldz; c += 1024) {
            Vec16<float> v = load_vec(z + i * ldz, c, ldz);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = c + e == t ? pt : exp_below(v.e[e], l) * f;
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

// The contractions' byte offsets have 32 bits: with rows by the million a piece is
// fewer than the 256 words of a tile, in eights (there are some: kMaxHeadRows).
int64_t piece(int dtype, int64_t M, int64_t V) {
    M = std::max<int64_t>(M, 1);
    const int64_t bytes = M * V * (dtype == kBF16 ? 2 : 4);
    const int64_t n = (bytes + kPieceBytes - 1) / kPieceBytes;
    const int64_t p = std::min(V, ((V + n - 1) / n + 255) / 256 * 256);
    const int64_t most = dtype == kBF16 ? (g2::kOOB / 2 - 8) / M / 8 * 8 : g2::kMostFloats / M / 8 * 8;
    return std::min(p, most);
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
// twice as long or more where they are not.  So z has as many columns as f32_words()
// says, of which the contractions know those that are words (ConvGeom::wrows), and
// from kPadRows rows on (fewer are not worth a copy of W) rows of W of another width
// run on zero-padded copies as wide as f32_width() says.
// us, forward alone / with all gradients, with 4-byte loads and on copies:
//   40 x 511 x 39536    81 / 284 and  93 / 307    70 x 511 x 39536   102 / 381 and 109 / 372
//   36 x 3485 x 30640  216 / 934 and 303 / 1098   71 x 3485 x 30640  344 / 1488 and 395 / 1473
constexpr int64_t kPadRows = 96;
// (not past what the contractions take: with the narrowest rows the copies are many times
// the tensors, and of more elements than any contraction's indexes reach)
int64_t f32_width(int64_t M, int64_t D, int64_t V) {
    const int64_t wide = (D + 31) / 32 * 32;
    return M >= kPadRows && D % 4 && std::max(M, V) * wide <= g2::kMostFloats ? wide : D;
}
int64_t f32_words(int64_t M, int64_t D8, int64_t V) {
    const int64_t n = (V + 31) / 32 * 32;
    // (larger operands take a contraction that does not know them)
    return V % 4 && std::max({M * D8, n * D8, M * n}) <= g2::kMostFloats ? n : V;
}

// A piece's operands as the contractions take them.
struct Piece {
    int64_t n, np;          // words, and columns of z
    const float *w, *b;
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
    r.D8 = dtype == kBF16 ? (D + 7) / 8 * 8 : f32_width(M, D, V);
    r.pos = c.get<int>(M);
    r.idx = c.get<int>(M);
    r.tgt = c.get<int>(M);
    r.count = c.get<int>(1);
    r.xc = c.raw((size_t)M * r.D8 * (dtype == kBF16 ? 2 : 4));
    r.wp = padw ? c.raw((size_t)V * r.D8 * 2) : nullptr;
    r.bp = padb ? c.raw((size_t)((V + 7) / 8 * 8) * 2) : nullptr;
    return r;
}

// Rows at once where dx is kept: kPieceBytes of exponentials, whole tiles.
int64_t chunk_rows(int64_t M, int64_t V) { return std::min(M, kPieceBytes / ((V + 7) / 8 * 16) / 256 * 256); }

struct Fwd {
    Rows r;
    void *stat;
    float *tlogit, *each;
    float *z;      // fp32: a piece's logits,
    float *wp, *bp;   // its padded operands
    void *conv;    // and the contractions' workspace
    // where dx is kept
    Kept kept;
    int64_t chunk;
    bf16 *prob;      // bf16: a chunk's exponentials
    float *part;     // partials of dx
    SplitRule rule;
    int *nsplit, *ccount;   // of each chunk
};

Fwd carve_fwd(Carve &c, int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb, bool each, bool keep) {
    Fwd f{};
    f.r = carve_rows(c, dtype, M, D, V, padw, padb);
    f.chunk = keep && dtype == kBF16 ? chunk_rows(M, V) : M;
    f.stat = c.get<floatx2>((dtype != kBF16 || !M ? 1 : keep ? (V + 255) / 256 * (256 / kProbCols) : g2::xent_lse_tiles(M, f.r.D8, V)) *
                            f.chunk);
    f.tlogit = c.get<float>(M);
    f.each = each ? c.get<float>(M) : nullptr;
    if (keep) {
        f.kept.ref = c.get<float>(M);
        f.kept.f = c.get<float>(M);
        f.kept.ct = c.get<float>(M);
        if (dtype == kBF16) {
            f.prob = c.get<bf16>(f.chunk * ((V + 7) / 8 * 8));
            f.rule = g2::xent_dx_rule(f.chunk, f.r.D8, V);
            f.nsplit = c.get<int>((M + f.chunk - 1) / f.chunk);
            f.ccount = c.get<int>((M + f.chunk - 1) / f.chunk);
        }
        f.part = c.get<float>((dtype == kBF16 ? f.rule.most * f.chunk : M) * f.r.D8);
    }
    if (dtype != kBF16) {
        const int64_t p = piece(dtype, M, V), last = V - (V - 1) / p * p, most = std::max(f32_words(M, f.r.D8, p), f32_words(M, f.r.D8, last));
        f.z = c.get<float>(M * most);
        f.wp = f.r.D8 != D ? c.get<float>(p * f.r.D8) : nullptr;
        f.bp = c.get<float>(most);
        size_t ws = 0;
        for (int64_t v : {p, last}) ws = std::max(ws, conv_fwd_workspace(dtype, linear(M, f.r.D8, f32_words(M, f.r.D8, v))));
        if (keep) ws = std::max(ws, linear_bwd_workspace(dtype, M, f.r.D8, f32_words(M, f.r.D8, V), true, false, false));
        f.conv = c.raw(ws);
    }
    return f;
}

struct Bwd {
    Rows r;
    float *lse, *ct, *scale, *rest;
    void *dz;
    float *part;     // partials of dx (fp32: the sum and a piece's)
    float *wp, *bp, *gwp, *gbp;   // fp32: a piece's padded operands and gradients
    float *dbpart;                // bf16: column sums of dz
    void *work;      // the contractions' workspace
    SplitRule rule;  // bf16: of the contraction for dx
    int *nsplit;
};

Bwd carve_bwd(Carve &c, int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb, bool dx, bool dw, bool db) {
    Bwd b{};
    b.r = carve_rows(c, dtype, M, D, V, padw, padb);
    b.lse = c.get<float>(M);
    b.ct = c.get<float>(M);
    b.scale = c.get<float>(M + 1);
    b.rest = dtype == kBF16 ? c.get<float>(M) : nullptr;
    const int64_t p = piece(dtype, M, V), last = V - (V - 1) / p * p;
    const int64_t most = dtype == kBF16 ? (p + 7) / 8 * 8 : std::max(f32_words(M, b.r.D8, p), f32_words(M, b.r.D8, last));
    b.dz = c.raw((size_t)M * most * (dtype == kBF16 ? 2 : 4));
    if (dtype != kBF16) {
        b.wp = b.r.D8 != D ? c.get<float>(p * b.r.D8) : nullptr;
        b.bp = c.get<float>(most);
        b.gwp = dw && b.r.D8 != D ? c.get<float>(p * b.r.D8) : nullptr;
        b.gbp = db ? c.get<float>(most) : nullptr;
    }
    size_t ws = 0;
    for (int64_t v : {p, last}) {
        if (dtype == kBF16) {
            if (dw) ws = std::max(ws, g2::xent_dw_workspace(M, b.r.D8, v));
        } else {
            ws = std::max(ws, conv_fwd_workspace(dtype, linear(M, b.r.D8, f32_words(M, b.r.D8, v))));
            ws = std::max(ws, linear_bwd_workspace(dtype, M, b.r.D8, f32_words(M, b.r.D8, v), dx, dw, db));
        }
    }
    if (dtype == kBF16 && db) b.dbpart = c.get<float>((M + 63) / 64 * 4 * most);   // (rows of 64 or more, in whole tiles)
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
          const int64_t *target, int64_t ignore, const float *others, const float *gloss, int reduction, float *lse, float *ct, float *scale,
          const SplitRule &rule, int *nsplit, int64_t chunk, int *ccount, hipStream_t st) {
    const bool scan = M <= kScanRows;   // (a block a row)
    if (!scan) hipLaunchKernelGGL(rows_kernel, dim3(1), dim3(1024), 0, st, target, ignore, M, V, r.pos, r.idx, r.tgt, r.count);
    auto gather = [&](auto kernel, auto *xs, auto *xc, bool fill) {   // (before w and b move to their copies)
        using T = std::remove_reference_t<decltype(*xc)>;
        hipLaunchKernelGGL(kernel, dim3(row_grid(M)), dim3(256), 0, st, target, ignore, V, r.pos, r.tgt, xs, r.idx, r.count, M, (int)D, (int)r.D8,
                           fill, xc, others, (const T *)*w, (const T *)*b, gloss, reduction, lse, ct, scale, rule, nsplit, chunk, ccount);
    };
    if (dtype == kBF16) gather(scan ? gather_kernel<bf16, true> : gather_kernel<bf16, false>, (const bf16 *)x, (bf16 *)r.xc, false);
    else gather(scan ? gather_kernel<float, true> : gather_kernel<float, false>, (const float *)x, (float *)r.xc, true);
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
    q->np = f32_words(M, D8, n);
    q->w = (const float *)w + v0 * D;
    q->b = b ? (const float *)b + v0 : nullptr;
    CopyJob j[kCopies];
    int jobs = 0;
    if (D8 != D) {
        j[jobs++] = {q->w, D, n, D, wp, n, D8};
        q->w = wp;
    }
    if (b && q->np != n) {
        j[jobs++] = {q->b, n, 1, n, bp, 1, q->np};
        q->b = bp;
    }
    return launch_copy_rows(kF32, j, jobs, st);
}

// Whether the kernels for few rows take the forward.  bf16: not W of more than 64 MiB,
// which the large contraction's tiles read faster than its two more launches cost.  us,
// few rows' / large (W in the last-level cache where it fits, and not):
//   16 x 2048 x 2000   13 / 31, 19 / 44     4 x 768 x 50000   28 / 26, 47 / 47
//   16 x 1024 x 10000  15 / 22, 22 / 33    16 x 768 x 50000   32 / 26, 51 / 47
//                                           1 x 4096 x 100000 221 / 171, 250 / 232
// (Between W of 20 and of 77 MB nothing was measured.)
// fp32: 16 x 768 x 50000 50 / 90, 85 / 112; 16 x 2048 x 2000 19 / 27, 26 / 32.
bool few_rows(int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void *w) {
    return (dtype != kBF16 || V * D * 2 <= int64_t(64) << 20) && tok::applies(dtype, M, V, D, x, w);
}

int logits(const Piece &q, const Rows &r, int64_t M, float *z, void *ws, hipStream_t st) {
    ConvGeom g = linear(M, r.D8, q.np);
    g.count = r.count;
    g.wrows = q.np != q.n ? (int)q.n : 0;
    return launch_conv_fwd(kF32, g, r.xc, q.w, q.b, z, ws, st);
}

}  // namespace
}  // namespace xent

// Where dx is the only gradient, the forward takes it: from sizes on at which a
// contraction and two launches less are worth a kept gradient larger than x (fp32: where
// its logits are one piece).  us of forward and backward, so and with the backward's own
// contractions, M x 768 x V:
//                bf16 64 x 5461  512 x 10922  4096 x 5461    fp32 64 x 5461  512 x 10922  4096 x 5461
//   in the forward         50           68          136               68          213          612
//   in the backward        59           79          177               88          305          895
// and 4096 x 4096 x 128000 bf16 7.2 and 10.5 ms.
bool xent_keeps_gradient(int dtype, int64_t M, int64_t D, int64_t V, bool dx, bool dw, bool db) {
    if (!dx || dw || db || M <= 16 || (double)M * D * V < double(int64_t(1) << 28)) return false;
    return dtype == kBF16 ? xent::chunk_rows(M, V) > 0 : xent::piece(dtype, M, V) == V;
}

size_t xent_kept_bytes(int dtype, int64_t M, int64_t D) { return (size_t)M * D * (dtype == kBF16 ? 3 : 4); }

size_t xent_fwd_workspace(int dtype, int64_t M, int64_t D, int64_t V, bool padw, bool padb, int reduction, bool keep) {
    xent::Carve c{nullptr};
    xent::carve_fwd(c, dtype, M, D, V, padw, padb, reduction != 2, keep);
    return std::max(c.off, tok::xent_workspace());
}

int launch_xent_fwd(int dtype, int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *b, bool padw, bool padb,
                    const int64_t *target, int64_t ignore, int reduction, float *loss, float *lse, void *kept, void *ws, void *stream) {
    using namespace xent;
    hipStream_t st = (hipStream_t)stream;
    if (!kept && few_rows(dtype, M, D, V, x, w)) return tok::xent(dtype, M, D, V, x, w, b, target, ignore, reduction, loss, lse, ws, st);
    Carve c{static_cast<char *>(ws)};
    const Fwd f = carve_fwd(c, dtype, M, D, V, padw, padb, reduction != 2, kept != nullptr);
    const int64_t D8 = f.r.D8;
    int err = start(f.r, dtype, M, D, V, x, &w, &b, target, ignore, nullptr, nullptr, reduction, nullptr, nullptr, nullptr, f.rule, f.nsplit,
                    f.chunk, f.ccount, st);
    if (err) return err;
    if (dtype == kBF16 && M > 0 && !g2::rows_ok(M, V, D8, f.r.xc, w)) return (int)hipErrorInvalidValue;
    float *each = reduction == 2 ? loss : f.each;
    auto combine = [&](int parts, int64_t ld, int64_t i0, bf16 *prob, int64_t ldz) {
        hipLaunchKernelGGL(combine_kernel, dim3((unsigned)((M + 7) / 8)), dim3(256), 0, st, (const floatx2 *)f.stat, parts, ld, i0, f.tlogit,
                           f.r.pos, f.r.tgt, M, each, lse, f.kept, prob, ldz);
        return (int)hipGetLastError();
    };
    auto keep = [&](auto kernel, auto *w0, const int *splits, int64_t i0, int64_t R, const float *kf, const float *ct) {
        float *out = reduction == 2 || i0 + R < M ? nullptr : loss;
        hipLaunchKernelGGL(kernel, dim3(row_grid(M) + (out ? 1 : 0)), dim3(256), 0, st, f.part, splits, R * D8, f.r.pos, M, (int)D, (int)D8, i0, R,
                           f.r.count, reduction == 0, kf, ct, f.r.tgt, w0, kept, each, out);
        return (int)hipGetLastError();
    };
    if (M == 0) {
    } else if (kept && dtype == kBF16) {
        const int64_t ldz = (V + 7) / 8 * 8, R = f.chunk;
        for (int64_t i0 = 0, k = 0; i0 < M && !err; i0 += R, ++k) {
            const bf16 *xc = (const bf16 *)f.r.xc + i0 * D8;
            const int64_t m = std::min(R, M - i0);
            const int parts = g2::xent_prob_parts(m, D8, V);
            err = g2::xent_prob(m, D8, V, xc, w, b, f.ccount + k, f.r.tgt + i0, f.stat, R, f.tlogit + i0, f.prob, ldz, st);
            if (!err) err = combine(parts, R, i0, f.prob, ldz);
            if (!err) err = g2::xent_dx(R, D8, V, ldz, V, f.prob, w, f.ccount + k, f.nsplit + k, f.part, false, st);
            if (!err) err = keep(keep_kernel<bf16>, (const bf16 *)w, f.nsplit + k, i0, R, f.kept.f, f.kept.ct);
        }
    } else if (dtype == kBF16) {
        err = g2::xent_lse(M, D8, V, f.r.xc, w, b, f.r.count, f.r.tgt, f.stat, f.tlogit, st);
        if (!err) err = combine(g2::xent_lse_tiles(M, D8, V), M, 0, nullptr, 0);
    } else {
        const int64_t p = piece(dtype, M, V);
        Piece q;
        for (int64_t v0 = 0; v0 < V && !err; v0 += p) {
            const int64_t n = std::min(p, V - v0);
            err = take_piece(&q, M, D, D8, v0, n, w, b, f.wp, f.bp, st);
            if (!err) err = logits(q, f.r, M, f.z, f.conv, st);
            if (err) break;
            hipLaunchKernelGGL(lse_rows_kernel, dim3(row_grid(M)), dim3(256), 0, st, f.z, (int)q.np, (int)n, (int)v0, f.r.count, f.r.tgt,
                               v0 == 0, (floatx2 *)f.stat, f.tlogit);
            err = (int)hipGetLastError();
        }
        if (!err) err = combine(1, M, 0, nullptr, 0);
        if (!err && kept) {   // (one piece)
            hipLaunchKernelGGL(grad_rows_kernel, dim3(row_grid(M)), dim3(256), 0, st, f.z, (int)q.np, (int)V, 0, M, f.r.count, f.r.tgt,
                               f.kept.ref, f.kept.f, f.kept.ct, (const float *)nullptr);
            err = (int)hipGetLastError();
            if (!err)
                err = launch_linear_bwd(dtype, M, D8, q.np, q.n, f.r.count, f.z, f.r.xc, q.w, f.part, nullptr, nullptr, f.conv, stream);
            if (!err) err = keep(keep_kernel<float>, (const float *)w, nullptr, 0, M, nullptr, nullptr);
        }
    }
    if (err) return err;
    if (reduction != 2 && !kept)
        hipLaunchKernelGGL(total_kernel, dim3(1), dim3(1024), 0, st, each, M, f.r.count, reduction == 0, loss);
    return (int)hipGetLastError();
}

int launch_xent_scale(int dtype, int64_t M, int64_t D, const void *kept, const float *gloss, int reduction, void *dx, void *stream) {
    using namespace xent;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == kBF16)
        hipLaunchKernelGGL(scale_kernel<bf16>, dim3(row_grid(M)), dim3(256), 0, st, kept, M, (int)D, gloss, reduction == 2, (bf16 *)dx);
    else
        hipLaunchKernelGGL(scale_kernel<float>, dim3(row_grid(M)), dim3(256), 0, st, kept, M, (int)D, gloss, reduction == 2, (float *)dx);
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
    int err = start(k.r, dtype, M, D, V, x, &w, &b, target, ignore, lse, gloss, reduction, k.lse, k.ct, k.scale, k.rule, k.nsplit, M, nullptr,
                    st);
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
                                    k.ct, k.dz, ldz, k.rest, k.dbpart, st);
            if (!err && dx && M > 0) err = g2::xent_dx(M, D8, n, ldz, p, k.dz, wv, k.r.count, k.nsplit, k.part, v0 > 0, st);
            bf16 *dbv = db ? (bf16 *)db + v0 : nullptr;
            if (!err && dw)
                err = g2::xent_dw(M, D8, D, n, ldz, k.dz, k.r.xc, k.r.count, k.scale + M, (bf16 *)dw + v0 * D, k.work, st);
            if (!err && db) {
                int tile = 256, rows = 64;
                if (M > 0) g2::xent_bias_rows(M, D8, n, &tile, &rows);
                hipLaunchKernelGGL(bias_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, k.dbpart, tile, rows, k.r.count, (int)n,
                                   k.scale + M, dbv);
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
                                   k.r.tgt, k.lse, (const float *)nullptr, k.ct, k.scale);
                err = (int)hipGetLastError();
            }
            const bool tw = dw && D8 != D, tb = db && q.np != n;
            if (!err)
                err = launch_linear_bwd(dtype, M, D8, q.np, q.n, k.r.count, z, k.r.xc, q.w, dx && M > 0 ? tmp : nullptr, tw ? k.gwp : dwv,
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
                           k.scale + M, k.rest, k.r.tgt, (const bf16 *)w, (bf16 *)dx);
    else
        hipLaunchKernelGGL(finish_kernel<float>, dim3(row_grid(M)), dim3(256), 0, st, k.part, (const int *)nullptr, M * D8, k.r.pos, M, (int)D, (int)D8,
                           (const float *)nullptr, (const float *)nullptr, k.r.tgt, (const float *)w, (float *)dx);   // (its dz has the factor)
    return (int)hipGetLastError();
}

}  // namespace ms

extern "C" void ms_testing_cross_entropy_plan(int32_t dtype, int64_t rows, int64_t D, int64_t V, int64_t out[4]) {
    using namespace ms::xent;
    const int64_t p = piece(dtype, rows, V), last = V - (V - 1) / p * p;
    out[0] = p;
    out[2] = dtype == ms::kBF16 ? (D + 7) / 8 * 8 : f32_width(rows, D, V);
    out[3] = f32_words(rows, out[2], last);
    out[1] = rows * (dtype == ms::kBF16 ? (p + 7) / 8 * 8 : std::max(f32_words(rows, out[2], p), out[3]));
}
