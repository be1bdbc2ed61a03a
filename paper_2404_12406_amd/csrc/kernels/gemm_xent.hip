// The cross entropy's bf16 contractions (gemm_fused.h).
#include "gemm_fused.h"

namespace ms {
namespace g2 {

int sum_wgrad_partials(const float *part, int splits, int M, int C8, int C, void *out, const float *dbpart, void *db, hipStream_t st);

namespace {
// Tiles of the gradients of the cross entropy (an operand along m or n).
constexpr Tile kGradTiles[] = {
    {"256x256", 256, 256, 2, 4, 2, 1, 1.20f, 1.20f},
    {"256x128", 256, 128, 2, 4, 3, 1, 1.00f, 1.00f},
    {"128x128w8", 128, 128, 2, 4, 2, 2, 0.85f, 1.02f},
};

template <int EPI, int MODE>
int go_grad(int tile, unsigned prof, const FusedArgs &a, hipStream_t st, int times = 1) {
    switch (tile) {
    case 0: return go<EPI, MODE, 256, 256, 2, 4, 2, 1, 0, EPI == kEpiAdd>(prof, a, st, times);
    case 1: return go<EPI, MODE, 256, 128, 2, 4, 3, 1>(prof, a, st, times);
    default: return go<EPI, MODE, 128, 128, 2, 4, 2, 2>(prof, a, st, times);
    }
}
}  // namespace

// Column tiles of the statistics (rows of `stat`).
int xent_lse_tiles(int64_t M, int64_t D, int64_t V) {
    const Tile &t = kRowTiles[plan(kRowTiles, 2, M, V, D, 1).tile];
    return (int)((V + t.bn - 1) / t.bn);
}

int xent_lse(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
             void *stat, float *tlogit, hipStream_t st) {
    const FusedPlan p = plan(kRowTiles, 2, M, V, D, 1);
    FusedArgs a = rows_args(kRowTiles[p.tile], M, V, D, x, w, V);
    a.fbias = (const bf16 *)bias;
    a.count = count;
    a.target = target;
    a.stat = (floatx2 *)stat;
    a.stat_ld = M;
    a.tlogit = tlogit;
    return go_rows<kEpiLse>(p.tile, kProfFwd, a, st);
}

// Rows of xent_grad()'s column sums: one for each `rows` rows of dz, of whole tiles
// of `tile` rows.
void xent_bias_rows(int64_t M, int64_t D, int64_t V, int *tile, int *rows) {
    const Tile &t = kRowTiles[plan(kRowTiles, 2, M, V, D, 1).tile];
    *tile = t.bm;
    *rows = t.bm / t.wr;
}

// dz[M][ldz] of the words v0 .. v0 + V - 1, whose rows of W and biases w and
// bias are; columns V .. ldz - 1 are zeros.  ct: the targets' entries.  rest: what rounding took from the entry of
// each row whose target is among them.  dbpart (null: not wanted): the column sums,
// rows of V.
int xent_grad(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
              int v0, const float *lse, const float *scale, const float *ct, void *dz, int64_t ldz, float *rest, float *dbpart,
              hipStream_t st) {
    const FusedPlan p = plan(kRowTiles, 2, M, V, D, 1);
    FusedArgs a = rows_args(kRowTiles[p.tile], M, V, D, x, w, V);
    a.fbias = (const bf16 *)bias;
    a.count = count;
    a.target = target;
    a.v0 = v0;
    a.lse = lse;
    a.scale = scale;
    a.ct = ct;
    a.tlogit = rest;
    a.dbpart = dbpart;
    a.c = (bf16 *)dz;
    a.ldc = (int)ldz;
    return go_rows<kEpiXent>(p.tile, kProfFwd, a, st);
}

// Statistics of 64 columns each (rows of xent_prob()'s `stat`).
int xent_prob_parts(int64_t M, int64_t D, int64_t V) {
    const Tile &t = kRowTiles[plan(kRowTiles, 2, M, V, D, 1).tile];
    return (int)((V + t.bn - 1) / t.bn) * (t.bn / kProbCols);
}

// prob[M][ldz] = exp(z - r) for the words that are not the row's target, zeros there
// and in columns V .. ldz - 1; r and their sums go to stat.
int xent_prob(int64_t M, int64_t D, int64_t V, const void *x, const void *w, const void *bias, const int *count, const int *target,
              void *stat, int64_t stat_ld, float *tlogit, void *prob, int64_t ldz, hipStream_t st) {
    const FusedPlan p = plan(kRowTiles, 2, M, V, D, 1);
    FusedArgs a = rows_args(kRowTiles[p.tile], M, V, D, x, w, V);
    a.fbias = (const bf16 *)bias;
    a.count = count;
    a.target = target;
    a.stat = (floatx2 *)stat;
    a.stat_ld = stat_ld;
    a.tlogit = tlogit;
    a.c = (bf16 *)prob;
    a.ldc = (int)ldz;
    return go_rows<kEpiProb>(p.tile, kProfFwd, a, st);
}

namespace {
int dx_tile(int64_t M, int64_t D, int64_t V) { return plan(kGradTiles, 3, M, D, V, (int)std::clamp<int64_t>(V / (4 * BK), 1, 16)).tile; }
}  // namespace

// dx += dz w over the words of a piece, in up to rule.most arrays [M][D] of partials.
// Few rows of a wide vocabulary are few tiles of many steps: how many ways to split
// them follows from the rows that count, which only the device knows
// (SplitRule::splits()).
SplitRule xent_dx_rule(int64_t M, int64_t D, int64_t V) {
    const Tile &t = kGradTiles[dx_tile(M, D, V)];
    SplitRule r;
    r.bm = t.bm;
    r.ntn = (int)((D + t.bn - 1) / t.bn);
    r.steps = (int)((V + BK - 1) / BK);
    r.slots = kCUs * t.per_cu;
    r.row_us = (float)(8.0 * D / 5.0e6);   // a partial row, written and read
    r.step_us = (float)(1.5 * t.bm * t.bn * t.per_cu / (256.0 * 256.0));
    // at most a quarter gigabyte of partials
    r.most = (int)std::clamp<int64_t>((int64_t(256) << 20) / std::max<int64_t>(1, M * D * 4), 1, 16);
    return r;
}

namespace {
// part[M][D] (+)= dz[M][ldz] w[V][D], its split arrays one after another
FusedArgs dx_args(const Tile &t, int64_t M, int64_t D, int64_t V, int64_t ldz, const void *dz, const void *w, float *part) {
    FusedArgs a{};
    a.a = (const bf16 *)dz;
    a.b = (const bf16 *)w;
    a.g.N = (int)M; a.g.C = (int)D; a.g.K = (int)ldz;
    a.g.H = a.g.W = a.g.R = a.g.S = a.g.P = a.g.Q = a.g.sh = a.g.sw = 1;
    a.M = (int)M; a.N = (int)D; a.K = (int)ldz;
    a.ntm = (int)((M + t.bm - 1) / t.bm);
    a.ntn = (int)((D + t.bn - 1) / t.bn);
    a.splits = 1;
    a.k_split = (int)ldz;
    a.a_bytes = bytes_of(M * ldz);
    a.b_bytes = bytes_of(V * D);
    a.part = part;
    a.part_stride = M * D;
    return a;
}
}  // namespace

int xent_dx(int64_t M, int64_t D, int64_t V, int64_t ldz, int64_t piece, const void *dz, const void *w, const int *count,
            const int *nsplit, float *part, bool add, hipStream_t st) {
    const int tile = dx_tile(M, D, piece);   // (a last, smaller piece runs as the others)
    FusedArgs a = dx_args(kGradTiles[tile], M, D, V, ldz, dz, w, part);
    a.count = count;
    a.nsplit = nsplit;
    a.add = add;
    return go_grad<kEpiAdd, kDgradN>(tile, kProfDgrad, a, st, xent_dx_rule(M, D, piece).most);
}

// A Linear's dx[M][D] = dz[M][K] w[K][D] so, bf16: in how many splits, 0 where it is not
// to be.  It costs partials of M x D, where the general contraction transposes w, K x D:
// for K of at least 2 M.  us of a gated unit, forward and input gradient, general / so:
//   4096 x 2048 x 11008  540 / 513    512 x 2048 x 11008  119 / 104    100 x 4096 x 21888  201 / 107
//   4096 x 512 x 16384   282 / 268    1024 x 1024 x 2048   50 / 45     300 x 256 x 1024     28 / 26
// and past that
//   8192 x 768 x 4096    173 / 188    8192 x 4096 x 2048  336 / 403
int place_splits(int64_t M, int64_t D, int64_t K) {
    if (M < 1 || K < 2 * M || D % 8 || K % 8 || !operand_fits(M * K) || !operand_fits(K * D)) return 0;
    return xent_dx_rule(M, D, K).splits((int)M);
}
size_t place_dx_workspace(int64_t M, int64_t D, int64_t K) { return (size_t)place_splits(M, D, K) * M * D * sizeof(float); }
int place_dx(int64_t M, int64_t D, int64_t K, const void *dz, const void *w, void *dx, void *ws, hipStream_t st) {
    const int tile = dx_tile(M, D, K), s = place_splits(M, D, K);
    FusedArgs a = dx_args(kGradTiles[tile], M, D, K, K, dz, w, static_cast<float *>(ws));
    a.fixed_splits = s;
    const int err = go_grad<kEpiAdd, kDgradN>(tile, kProfDgrad, a, st, s);
    return err ? err : sum_wgrad_partials(a.part, s, (int)M, (int)D, (int)D, dx, nullptr, nullptr, st);
}

// dw[V][Dr] = *scale dz^T x over the rows that count (x has D >= Dr columns).

namespace {
FusedPlan dw_plan(int64_t M, int64_t D, int64_t V) {
    return plan(kGradTiles, 3, V, D, M, (int)std::clamp<int64_t>(M / (4 * BK), 1, 16));
}
}  // namespace

size_t xent_dw_workspace(int64_t M, int64_t D, int64_t V) {
    const FusedPlan p = dw_plan(M, D, V);
    return p.splits > 1 ? (size_t)p.splits * V * D * sizeof(float) : 0;
}

int xent_dw(int64_t M, int64_t D, int64_t Dr, int64_t V, int64_t ldz, const void *dz, const void *x, const int *count,
            const float *scale, void *dw, void *ws, hipStream_t st) {
    const FusedPlan p = dw_plan(M, D, V);
    const Tile &t = kGradTiles[p.tile];
    FusedArgs a{};
    a.a = (const bf16 *)dz;
    a.b = (const bf16 *)x;
    a.g.N = (int)M; a.g.C = (int)D; a.g.K = (int)ldz;
    a.g.H = a.g.W = a.g.R = a.g.S = a.g.P = a.g.Q = a.g.sh = a.g.sw = 1;
    a.M = (int)V; a.N = (int)D; a.K = (int)M;
    a.ntm = (int)((V + t.bm - 1) / t.bm);
    a.ntn = (int)((D + t.bn - 1) / t.bn);
    a.splits = p.splits;
    a.k_split = (int)M;
    a.a_bytes = bytes_of(M * ldz);
    a.b_bytes = bytes_of(M * D);
    a.count = count;
    a.out_scale = scale;
    if (p.splits > 1) {
        a.part = static_cast<float *>(ws);
        a.part_stride = V * D;
    } else {
        a.c = (bf16 *)dw;
        a.ldc = (int)Dr;
    }
    // (the sum of the partials leaves the padding out by itself)
    const int err = p.splits == 1 && D != Dr ? go_grad<kEpiRows, kWgrad>(p.tile, kProfWgrad, a, st)
                                             : go_grad<kEpiStore, kWgrad>(p.tile, kProfWgrad, a, st);
    if (err || p.splits == 1) return err;
    return sum_wgrad_partials(a.part, p.splits, (int)V, (int)D, (int)Dr, dw, nullptr, nullptr, st);
}

}  // namespace g2
}  // namespace ms
