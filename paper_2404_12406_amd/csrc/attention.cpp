// Host runtime of a transformer's attention: norms and rotation of its heads, attention
// over whole prompts, the paged cache and the attention of single tokens over it.
// Validation, the save rule and the records follow blocks.cpp.
#include "blocks.h"
#include "overlap.h"

using namespace ms::rt;

namespace {

// ------------------------------------------------------------------ tensors [rows][heads][D]
// Elements of a row of D padded to whole 16-byte vectors.
int64_t padded(int64_t D, int32_t dtype) {
    const int64_t v = dtype == MS_BF16 ? 8 : 4;
    return (D + v - 1) / v * v;
}

ms_status check_heads(const ms_tensor *t, const char *name, int32_t dtype, bool output) {
    ms_status st = check_tensor(t, name, 3, true);
    if (st) return st;
    if (t->dtype != dtype) return fail(MS_E_DTYPE, "%s dtype differs from the first tensor's", name);
    if (output ? !non_overlapping(t) : !strides_ok(t))
        return fail(MS_E_LAYOUT, output ? "%s must not overlap itself" : "%s needs non-negative strides", name);
    return MS_OK;
}

// What the kernels are handed for a tensor: itself, or a dense stand-in of padded rows at
// `off` of the workspace.  WHOLE: rows have to be whole aligned vectors, a row's bytes
// within 2^24 of the next one's; otherwise elements have to lie side by side.
struct Stand {
    const ms_tensor *t = nullptr;
    size_t off = kNoStage;
    bool whole = true;
};

bool in_place(const ms_tensor *t, bool whole) {
    const int64_t D = t->shape[2], e = (int64_t)elt_size(t->dtype);
    if (D > 1 && t->stride[2] != 1) return false;
    if (!whole) return true;
    if (D * e % 16 || !aligned(t->data, 16)) return false;
    if (t->shape[1] > 1 && t->stride[1] * e % 16) return false;
    return t->shape[0] <= 1 || (t->stride[0] * e % 16 == 0 && t->stride[0] >= D && t->stride[0] * e <= (int64_t(1) << 24));
}

struct Stands {
    size_t bytes = 0;
    // apart: not in its own memory
    Stand add(const ms_tensor *t, bool whole, bool apart = false) {
        Stand s{t, kNoStage, whole};
        if (!t || numel(t) == 0 || (in_place(t, whole) && !apart)) return s;
        s.off = bytes;
        bytes += al256((size_t)(t->shape[0] * t->shape[1] * padded(t->shape[2], t->dtype)) * elt_size(t->dtype));
        return s;
    }
};

// Whether y lies where x does, but not its heads where x's are: kernels write a head where they have read it.
Shared crosses(const ms_tensor *x, const ms_tensor *y) {
    return !x || !y || same_places(x, y) ? Shared::kNo : shared(x, y);
}

// The workspace that a tensor like t takes in a backward, where its gradient is expected
// in the same layout.
size_t stand_bytes(const ms_tensor *t, bool whole) {
    Stands s;
    s.add(t, whole);
    return s.bytes;
}

ms::HeadsView view(const Stand &s, char *base) {
    const ms_tensor *t = s.t;
    if (!t) return {nullptr, 0, 0};
    const int64_t Dp = padded(t->shape[2], t->dtype);
    if (s.off != kNoStage) return {base + s.off, t->shape[1] * Dp, Dp};
    // (a single row's stride may be anything)
    return {t->data, t->shape[0] > 1 ? t->stride[0] : Dp, t->shape[1] > 1 ? t->stride[1] : 0};
}

int put_in(const Stand &s, char *base, void *stream) {
    if (s.off == kNoStage) return 0;
    const ms_tensor *t = s.t;
    return ms::launch_pack_heads(t->dtype, t->data, t->stride[0], t->stride[1], t->stride[2], t->shape[0], (int)t->shape[1],
                                 (int)t->shape[2], base + s.off, (int)padded(t->shape[2], t->dtype), stream);
}

int put_out(const Stand &s, char *base, void *stream) {
    if (s.off == kNoStage) return 0;
    const ms_tensor *t = s.t;
    const int64_t Dp = padded(t->shape[2], t->dtype);
    const int64_t ext[4] = {t->shape[0], 1, t->shape[1], t->shape[2]}, from[4] = {t->shape[1] * Dp, 0, Dp, 1},
                  to[4] = {t->stride[0], 0, t->stride[1], t->stride[2]};
    return ms::launch_copy4(t->dtype, base + s.off, ext, from, t->data, to, stream);
}

constexpr int64_t kMaxBlocks = (int64_t(1) << 24) - 1;   // of 256 threads in a launch

// ------------------------------------------------------------------ head norms with rotation
// What a call needs of ms_rotary; heads: of x.
ms_status check_rotary(const ms_rotary *r, const ms_tensor *gq, const ms_tensor *gk, int64_t T, int64_t heads, int64_t D, int32_t dtype,
                       bool place) {
    if (!r) return fail(MS_E_NULL, "rotary is NULL");
    if (D < 1 || D > ms::kMaxHeadDim) return fail(MS_E_UNSUPPORTED, "heads of 1 to %d elements; got %lld", ms::kMaxHeadDim, (long long)D);
    if (r->q_heads < 0 || r->q_heads > heads) return fail(MS_E_SHAPE, "q_heads must lie in 0 to %lld", (long long)heads);
    if (r->rotary_dim < 0 || r->rotary_dim > D || r->rotary_dim % 2) return fail(MS_E_ARG, "rotary_dim must be even and at most a head's size");
    if (r->rotary_dim > 0 && !r->inv_freq) return fail(MS_E_NULL, "inv_freq is NULL");
    if (T > 0 && (r->rotary_dim > 0 || place) && !r->positions) return fail(MS_E_NULL, "positions is NULL");
    if (!aligned(r->positions, 4) || !aligned(r->inv_freq, 4)) return fail(MS_E_ARG, "positions and inv_freq must be 4-byte aligned");
    if (!r->norm && (gq || gk)) return fail(MS_E_ARG, "scales without a norm");
    if (r->norm && (!(r->eps >= 0.f) || !std::isfinite(r->eps))) return fail(MS_E_ARG, "eps must be finite and >= 0");
    ms_status st = check_vector(gq, "gamma_q", D, dtype);
    return st ? st : check_vector(gk, "gamma_k", D, dtype);
}

ms::RotaryArgs rotary_args(const ms_rotary *r, const ms_tensor *x, const ms_tensor *gq, const ms_tensor *gk) {
    ms::RotaryArgs a{};
    a.gq = gq ? gq->data : nullptr;
    a.gk = gk ? gk->data : nullptr;
    a.pos = r->positions;
    a.freq = r->inv_freq;
    a.T = x->shape[0];
    a.Hq = (int)r->q_heads;
    a.Hk = (int)(x->shape[1] - r->q_heads);
    a.D = (int)x->shape[2];
    a.R = r->rotary_dim;
    a.next = r->interleaved != 0;
    a.norm = r->norm != 0;
    a.eps = r->eps;
    return a;
}

ms_status rotary_backward(ms_record *r, const ms_tensor *gy, const ms_tensor *gx, const ms_tensor *gq, const ms_tensor *gk, void *stream,
                          bool fixed) {
    const int32_t dt = r->plan.dtype;
    const ms_rotary rot{r->blk.heads, r->blk.turned, r->blk.next, r->blk.norm, r->eps, r->blk.positions, r->blk.freq};
    ms::RotaryArgs a = rotary_args(&rot, &r->x, &r->W, &r->b);
    const bool read_x = a.norm && r->x.data;
    Stands sg;
    const Stand sx = sg.add(read_x ? &r->x : nullptr, false), sy = sg.add(gy, false);
    const bool apart = (sx.off == kNoStage && crosses(sx.t, gx) != Shared::kNo) || (sy.off == kNoStage && crosses(gy, gx) != Shared::kNo);
    const Stand so = sg.add(gx, false, apart);
    const size_t kb = ms::rotary_bwd_workspace(dt, a, gq || gk);
    Work w;
    ms_status st = take(&w, sg.bytes + kb, stream, fixed);
    if (st) return st;
    int err = put_in(sy, w.base, stream);
    if (!err) err = put_in(sx, w.base, stream);
    const ms::HeadsView vx = view(sx, w.base), vy = view(sy, w.base), vo = view(so, w.base);
    a.x = vx.p;
    a.xts = vx.ts;
    a.xhs = vx.hs;
    const int64_t ds[2] = {vy.ts, vy.hs}, os[2] = {vo.ts, vo.hs};
    if (!err)
        err = ms::launch_rotary_bwd(dt, a, vy.p, ds, vo.p, os, gq ? gq->data : nullptr, gk ? gk->data : nullptr,
                                    kb ? w.base + sg.bytes : nullptr, stream);
    if (!err) err = put_out(so, w.base, stream);
    return err ? hip_fail(err, "backward launch") : MS_OK;
}

// ------------------------------------------------------------------ attention
ms::AttnArgs attention_args(const ms_tensor *q, const ms_tensor *k, const BlockState &b) {
    ms::AttnArgs a{};
    a.Tq = q->shape[0];
    a.Tk = k->shape[0];
    a.Hq = (int)q->shape[1];
    a.Hk = (int)k->shape[1];
    a.D = (int)padded(q->shape[2], q->dtype);
    a.n = (int)b.n;
    a.qoff = b.qoff;
    a.koff = b.koff;
    a.causal = b.causal;
    a.scale = b.scale;
    return a;
}

ms_status attention_backward(ms_record *r, const ms_tensor *go, const ms_tensor *gq, const ms_tensor *gk, const ms_tensor *gv, void *stream,
                             bool fixed) {
    const int32_t dt = r->plan.dtype;
    const bool both = gq || gk;   // dP is needed
    Stands sg;
    const Stand q = sg.add(&r->x, true), k = sg.add(&r->W, true), v = sg.add(both ? &r->b : nullptr, true),
                o = sg.add(both ? &r->y : nullptr, true), g = sg.add(go, true), dq = sg.add(gq, true), dk = sg.add(gk, true),
                dv = sg.add(gv, true);
    ms::AttnArgs a = attention_args(&r->x, &r->W, r->blk);
    // (stand-ins are read, and written, before and after all kernels)
    for (const Stand *out : {&dq, &dk, &dv})
        for (const Stand *in : {&q, &k, &v, &o, &g})
            a.shared |= out->off == kNoStage && in->off == kNoStage && shared(out->t, in->t) != Shared::kNo;
    const size_t kb = ms::attention_bwd_workspace(dt, a, gq, gk, gv);
    Work w;
    ms_status st = take(&w, sg.bytes + kb, stream, fixed);
    if (st) return st;
    int err = 0;
    for (const Stand *s : {&q, &k, &v, &o, &g})
        if (!err) err = put_in(*s, w.base, stream);
    a.q = view(q, w.base);
    a.k = view(k, w.base);
    a.v = view(v, w.base);
    a.o = view(o, w.base);
    a.go = view(g, w.base);
    a.dq = view(dq, w.base);
    a.dk = view(dk, w.base);
    a.dv = view(dv, w.base);
    a.lse = r->blk.lse;
    if (!err) err = ms::launch_attention_bwd(dt, a, kb ? w.base + sg.bytes : nullptr, stream);
    for (const Stand *s : {&dq, &dk, &dv})
        if (!err) err = put_out(*s, w.base, stream);
    return err ? hip_fail(err, "backward launch") : MS_OK;
}

// A cache's pages [pages][heads][page][D], row-major; as many elements as memory holds.
ms_status check_pages(const ms_tensor *t, const char *name, int32_t dtype) {
    if (!t) return fail(MS_E_NULL, "%s is NULL", name);
    if (t->ndim != 4) return fail(MS_E_SHAPE, "%s: expected 4 dims, got %d", name, t->ndim);
    if (t->dtype != dtype) return fail(MS_E_DTYPE, "%s dtype differs from the first tensor's", name);
    int64_t rows = 1;
    for (int i = 0; i < 4; ++i) {
        if (t->shape[i] < 0) return fail(MS_E_SHAPE, "%s: negative extent", name);
        if (t->shape[i] > kMaxElems) return fail(MS_E_UNSUPPORTED, "%s: extent too large", name);
        if (i < 3) {
            rows = t->shape[i] == 0 ? 0 : rows > (int64_t(1) << 32) / t->shape[i] ? int64_t(1) << 32 : rows * t->shape[i];
            if (rows >= int64_t(1) << 32) return fail(MS_E_UNSUPPORTED, "%s: 2^32 or more rows", name);
        }
    }
    const int64_t H = t->shape[1], P = t->shape[2], D = t->shape[3];
    if (H < 1 || P < 1) return fail(MS_E_SHAPE, "%s: pages need heads and rows", name);
    if (D < 1 || D > ms::kMaxHeadDim) return fail(MS_E_UNSUPPORTED, "heads of 1 to %d elements; got %lld", ms::kMaxHeadDim, (long long)D);
    const int64_t want[4] = {H * P * D, P * D, D, 1};
    for (int i = 0; i < 4; ++i)
        if (t->shape[0] > 0 && t->shape[i] > 1 && t->stride[i] != want[i]) return fail(MS_E_LAYOUT, "%s must be contiguous", name);
    if (t->shape[0] > 0 && !t->data) return fail(MS_E_NULL, "%s.data is NULL", name);
    return MS_OK;
}

ms_status check_tables(const int32_t *tables, int64_t sequences, int64_t width) {
    if (sequences < 0 || sequences > kMaxElems || width < 0 || width > kMaxElems) return fail(MS_E_SHAPE, "tables must be [sequences, width]");
    if (sequences > 0 && width > 0 && !tables) return fail(MS_E_NULL, "tables is NULL");
    if (!aligned(tables, 4)) return fail(MS_E_ARG, "tables must be 4-byte aligned");
    return MS_OK;
}

}  // namespace

extern "C" {

ms_status ms_head_norm_rotary_forward(const ms_tensor *x, const ms_tensor *gamma_q, const ms_tensor *gamma_k, const ms_rotary *rotary,
                                      uint32_t mask, const ms_tensor *y, ms_record **rec, void *stream) {
    clear_err();
    if (!rec) return fail(MS_E_NULL, "rec is NULL");
    *rec = nullptr;
    ms_status st = check_mask(mask, gamma_q, gamma_k);
    if (!st) st = check_tensor(x, "x", 3, true);
    if (!st) st = check_heads(x, "x", x->dtype, false);
    if (!st) st = check_rotary(rotary, gamma_q, gamma_k, x->shape[0], x->shape[1], x->shape[2], x->dtype, false);
    if (!st) st = check_heads(y, "y", x->dtype, true);
    if (st) return st;
    if (!same_shape(x, y)) return fail(MS_E_SHAPE, "y must have the shape of x");
    if (mask && rotary->norm && shared(x, y) == Shared::kYes) return fail(MS_E_ARG, "y must not be x, which the backward reads");
    if (crosses(x, y) == Shared::kYes) return fail(MS_E_ARG, "y may be x, but not other heads of x");
    ms::RotaryArgs a = rotary_args(rotary, x, gamma_q, gamma_k);
    Stands sg;
    const Stand sx = sg.add(x, false), sy = sg.add(y, false);
    Work w;
    if ((st = take(&w, sg.bytes, stream, false))) return st;
    ms_record *r = nullptr;
    if (mask) {
        const bool keep_x = a.norm, scales = a.norm && (mask & MS_RG_INPUT);
        const uint32_t borrowed = (keep_x ? (uint32_t)MS_SAVED_X : 0u) | (scales && gamma_q ? (uint32_t)MS_SAVED_W : 0u) |
                                  (scales && gamma_k ? (uint32_t)MS_SAVED_B : 0u) | (a.R ? (uint32_t)MS_SAVED_INDEX : 0u);
        r = new_record(MS_HEAD_NORM_ROTARY, x, gamma_q, gamma_k, y, mask, borrowed, rotary_backward);
        if (!r) return fail(MS_E_NOMEM, "record allocation failed");
        if (borrowed & MS_SAVED_B) {
            r->b.data = gamma_k->data;
            r->acct.referenced_param_bytes += bytes_of(gamma_k);
        }
        r->eps = rotary->eps;
        r->blk.heads = rotary->q_heads;
        r->blk.turned = a.R;
        r->blk.next = a.next;
        r->blk.norm = a.norm;
        if (a.R) {
            r->blk.positions = rotary->positions;
            r->blk.freq = rotary->inv_freq;
            r->acct.saved_activation_bytes += (uint64_t)a.T * sizeof(int32_t);
            r->acct.referenced_param_bytes += (uint64_t)a.R / 2 * sizeof(float);
        }
        r->acct.transient_workspace_bytes = ms::rotary_bwd_workspace(x->dtype, a, mask & (MS_RG_WEIGHT | MS_RG_BIAS)) + stand_bytes(y, false) +
                                            (keep_x ? stand_bytes(x, false) : 0) + ((mask & MS_RG_INPUT) ? stand_bytes(x, false) : 0);
    }
    int err = put_in(sx, w.base, stream);
    const ms::HeadsView vx = view(sx, w.base), vy = view(sy, w.base);
    a.x = vx.p;
    a.xts = vx.ts;
    a.xhs = vx.hs;
    a.y = vy.p;
    a.yts = vy.ts;
    a.yhs = vy.hs;
    if (!err) err = ms::launch_rotary_fwd(x->dtype, a, false, stream);
    if (!err) err = put_out(sy, w.base, stream);
    if (err) {
        delete r;
        return hip_fail(err, "forward launch");
    }
    file_record(r, rec);
    return MS_OK;
}

uint64_t ms_attention_kept_bytes(int64_t rows, int64_t heads, uint32_t mask) {
    return rows <= 0 || heads <= 0 || !(mask & 7u) ? 0 : (uint64_t)rows * (uint64_t)heads * sizeof(float);
}

ms_status ms_attention_forward(const ms_tensor *q, const ms_tensor *k, const ms_tensor *v, const int32_t *q_offsets, const int32_t *k_offsets,
                               int64_t sequences, int32_t causal, float scale, void *kept, uint32_t mask, const ms_tensor *o, ms_record **rec,
                               void *stream) {
    clear_err();
    if (!rec) return fail(MS_E_NULL, "rec is NULL");
    *rec = nullptr;
    if (mask & ~7u) return fail(MS_E_MASK, "mask 0x%x has bits outside INPUT|WEIGHT|BIAS", mask);
    ms_status st = check_tensor(q, "q", 3, true);
    if (!st) st = check_heads(q, "q", q->dtype, false);
    if (!st) st = check_heads(k, "k", q->dtype, false);
    if (!st) st = check_heads(v, "v", q->dtype, false);
    if (!st) st = check_heads(o, "o", q->dtype, true);
    if (st) return st;
    const int64_t Tq = q->shape[0], Tk = k->shape[0], Hq = q->shape[1], Hk = k->shape[1], D = q->shape[2];
    if (D < 1 || D > ms::kMaxHeadDim) return fail(MS_E_UNSUPPORTED, "heads of 1 to %d elements; got %lld", ms::kMaxHeadDim, (long long)D);
    if (Hk < 1 || Hq < 1 || Hq % Hk) return fail(MS_E_SHAPE, "%lld query heads for %lld heads of keys", (long long)Hq, (long long)Hk);
    if (k->shape[2] != D || !same_shape(k, v)) return fail(MS_E_SHAPE, "k and v must be alike, with heads of q's size");
    if (!same_shape(q, o)) return fail(MS_E_SHAPE, "o must have the shape of q");
    // (other blocks read k and v later, and the backward q)
    for (const ms_tensor *t : {q, k, v})
        if (Tk > 0 && shared(t, o) == Shared::kYes) return fail(MS_E_ARG, "o must not be q, k or v");
    // stand-ins of padded rows have 32-bit counts too
    if (capped_product({std::max(Tq * Hq, Tk * Hk), padded(D, q->dtype)}) > kMaxElems) return fail(MS_E_UNSUPPORTED, "2^31 or more padded elements");
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(MS_E_ARG, "scale must be finite and > 0");
    if (!q_offsets && k_offsets) return fail(MS_E_NULL, "k_offsets without q_offsets");
    if (q_offsets) {
        if (sequences < 0 || sequences > kMaxElems - 2) return fail(MS_E_ARG, "a number of sequences from 0 on is needed");
        if (!aligned(q_offsets, 4) || !aligned(k_offsets, 4)) return fail(MS_E_ARG, "offsets must be 4-byte aligned");
    }
    const int64_t n = q_offsets ? sequences : 0;
    // (heads are a launch's second dimension, too)
    if (Hq > 65535) return fail(MS_E_UNSUPPORTED, "more than 65535 heads");
    if (capped_product({std::max(Tq, Tk) / 128 + n + 2, Hq}) > kMaxBlocks)
        return fail(MS_E_UNSUPPORTED, "2^24 or more blocks of 128 rows");
    if (mask && Tq > 0 && !kept) return fail(MS_E_NULL, "kept is NULL but gradients are asked for");
    if (mask && !aligned(kept, 4)) return fail(MS_E_ARG, "kept must be 4-byte aligned");
    BlockState blk;
    blk.qoff = q_offsets;
    blk.koff = q_offsets && !k_offsets ? q_offsets : k_offsets;
    blk.n = n;
    blk.causal = causal != 0;
    blk.scale = scale;
    ms::AttnArgs a = attention_args(q, k, blk);
    Stands sg;
    const Stand sq = sg.add(q, true), sk = sg.add(k, true), sv = sg.add(v, true), so = sg.add(o, true);
    const size_t kb = ms::attention_fwd_workspace(q->dtype, a);
    Work w;
    if ((st = take(&w, sg.bytes + kb, stream, false))) return st;
    ms_record *r = nullptr;
    if (mask) {
        const bool both = mask & (MS_RG_INPUT | MS_RG_WEIGHT);
        const uint32_t borrowed = (uint32_t)(MS_SAVED_X | MS_SAVED_W | MS_SAVED_LSE) | (both ? (uint32_t)(MS_SAVED_B | MS_SAVED_Y) : 0u) |
                                  (q_offsets ? (uint32_t)MS_SAVED_INDEX : 0u);
        r = new_record(MS_ATTENTION, q, k, v, o, mask, borrowed, attention_backward);
        if (!r) return fail(MS_E_NOMEM, "record allocation failed");
        // (all of it activations: the keys are no parameter)
        r->acct.referenced_param_bytes = 0;
        r->acct.saved_activation_bytes = bytes_of(q) + bytes_of(k) + (both ? bytes_of(v) + bytes_of(o) : 0) +
                                         ms_attention_kept_bytes(Tq, Hq, mask) +
                                         (q_offsets ? (uint64_t)(n + 1) * sizeof(int32_t) * (k_offsets ? 2 : 1) : 0);
        if (both) {
            r->b.data = v->data;
            r->y.data = o->data;
        }
        r->blk = blk;
        r->blk.lse = static_cast<float *>(kept);
        r->acct.transient_workspace_bytes = ms::attention_bwd_workspace(q->dtype, a, mask & MS_RG_INPUT, mask & MS_RG_WEIGHT, mask & MS_RG_BIAS) +
                                            stand_bytes(q, true) + stand_bytes(k, true) + stand_bytes(o, true) +
                                            (both ? stand_bytes(v, true) + stand_bytes(o, true) : 0) +
                                            ((mask & MS_RG_INPUT) ? stand_bytes(q, true) : 0) + ((mask & MS_RG_WEIGHT) ? stand_bytes(k, true) : 0) +
                                            ((mask & MS_RG_BIAS) ? stand_bytes(v, true) : 0);
    }
    int err = 0;
    for (const Stand *s : {&sq, &sk, &sv})
        if (!err) err = put_in(*s, w.base, stream);
    a.q = view(sq, w.base);
    a.k = view(sk, w.base);
    a.v = view(sv, w.base);
    a.o = view(so, w.base);
    a.lse = mask ? static_cast<float *>(kept) : nullptr;
    if (!err) err = ms::launch_attention_fwd(q->dtype, a, kb ? w.base + sg.bytes : nullptr, stream);
    if (!err) err = put_out(so, w.base, stream);
    if (err) {
        delete r;
        return hip_fail(err, "forward launch");
    }
    file_record(r, rec);
    return MS_OK;
}

ms_status ms_cache_append(const ms_tensor *x, const ms_tensor *gamma_q, const ms_tensor *gamma_k, const ms_rotary *rotary,
                          const ms_tensor *k_pages, const ms_tensor *v_pages, const int32_t *tables, int64_t sequences, int64_t width,
                          const int32_t *rows, const ms_tensor *q, void *stream) {
    clear_err();
    ms_status st = check_tensor(x, "x", 3, true);
    if (!st) st = check_heads(x, "x", x->dtype, false);
    if (!st) st = check_pages(k_pages, "k_pages", x->dtype);
    if (!st) st = check_pages(v_pages, "v_pages", x->dtype);
    if (st) return st;
    if (!same_shape(k_pages, v_pages)) return fail(MS_E_SHAPE, "k_pages and v_pages must be alike");
    const int64_t T = x->shape[0], Hk = k_pages->shape[1], D = x->shape[2];
    if (D != k_pages->shape[3]) return fail(MS_E_SHAPE, "x has heads of %lld elements, the cache of %lld", (long long)D, (long long)k_pages->shape[3]);
    if ((st = check_rotary(rotary, gamma_q, gamma_k, T, x->shape[1], D, x->dtype, true))) return st;
    if (x->shape[1] != rotary->q_heads + 2 * Hk)
        return fail(MS_E_SHAPE, "x must have q_heads + 2 x %lld heads: queries, keys, values", (long long)Hk);
    if ((st = check_tables(tables, sequences, width))) return st;
    if (!aligned(rows, 4)) return fail(MS_E_ARG, "rows must be 4-byte aligned");
    if (!rows && T > sequences) return fail(MS_E_SHAPE, "%lld tokens for %lld sequences and no rows", (long long)T, (long long)sequences);
    if (rotary->q_heads > 0 || q) {
        if ((st = check_heads(q, "q", x->dtype, true))) return st;
        if (q->shape[0] != T || q->shape[1] != rotary->q_heads || q->shape[2] != D)
            return fail(MS_E_SHAPE, "q must be [%lld, %lld, %lld]", (long long)T, (long long)rotary->q_heads, (long long)D);
        if (crosses(x, q) == Shared::kYes) return fail(MS_E_ARG, "q may be x's first heads, but not others of x");
    }
    ms::RotaryArgs a = rotary_args(rotary, x, gamma_q, gamma_k);
    a.Hk = (int)Hk;
    a.kp = k_pages->data;
    a.vp = v_pages->data;
    a.tables = tables;
    a.rows = rows;
    a.nseq = sequences;
    a.pages = k_pages->shape[0];
    a.width = (int)width;
    a.page = (int)k_pages->shape[2];
    Stands sg;
    const Stand sx = sg.add(x, false), sq = sg.add(q, false);
    Work w;
    if ((st = take(&w, sg.bytes, stream, false))) return st;
    int err = put_in(sx, w.base, stream);
    const ms::HeadsView vx = view(sx, w.base), vq = view(sq, w.base);
    a.x = vx.p;
    a.xts = vx.ts;
    a.xhs = vx.hs;
    a.y = vq.p;
    a.yts = vq.ts;
    a.yhs = vq.hs;
    if (!err) err = ms::launch_rotary_fwd(x->dtype, a, true, stream);
    if (!err) err = put_out(sq, w.base, stream);
    return err ? hip_fail(err, "append launch") : MS_OK;
}

ms_status ms_paged_attention_forward(const ms_tensor *q, const ms_tensor *k_pages, const ms_tensor *v_pages, const int32_t *tables,
                                     int64_t sequences, int64_t width, const int32_t *lengths, float scale, const ms_tensor *o,
                                     void *stream) {
    clear_err();
    ms_status st = check_tensor(q, "q", 3, true);
    if (!st) st = check_heads(q, "q", q->dtype, false);
    if (!st) st = check_pages(k_pages, "k_pages", q->dtype);
    if (!st) st = check_pages(v_pages, "v_pages", q->dtype);
    if (!st) st = check_heads(o, "o", q->dtype, true);
    if (st) return st;
    if (!same_shape(k_pages, v_pages)) return fail(MS_E_SHAPE, "k_pages and v_pages must be alike");
    const int64_t n = q->shape[0], Hq = q->shape[1], Hk = k_pages->shape[1], D = q->shape[2];
    if (D != k_pages->shape[3]) return fail(MS_E_SHAPE, "q has heads of %lld elements, the cache of %lld", (long long)D, (long long)k_pages->shape[3]);
    if (Hq < 1 || Hq % Hk) return fail(MS_E_SHAPE, "%lld query heads for %lld heads of keys", (long long)Hq, (long long)Hk);
    if (!same_shape(q, o)) return fail(MS_E_SHAPE, "o must have the shape of q");
    if (crosses(q, o) == Shared::kYes) return fail(MS_E_ARG, "o may be q, but not other heads of q");
    if ((st = check_tables(tables, sequences, width))) return st;
    if (sequences != n) return fail(MS_E_SHAPE, "%lld queries for %lld sequences", (long long)n, (long long)sequences);
    if (n > 0 && !lengths) return fail(MS_E_NULL, "lengths is NULL");
    if (!aligned(lengths, 4)) return fail(MS_E_ARG, "lengths must be 4-byte aligned");
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(MS_E_ARG, "scale must be finite and > 0");
    // (a block's waves look up to two steps past the last place)
    if (width * k_pages->shape[2] > kMaxElems - 4096) return fail(MS_E_UNSUPPORTED, "a table of 2^31 - 2^12 or more places");
    ms::PagedArgs a{};
    a.kp = k_pages->data;
    a.vp = v_pages->data;
    a.tables = tables;
    a.lengths = lengths;
    a.pages = k_pages->shape[0];
    a.n = (int)n;
    a.Hq = (int)Hq;
    a.Hk = (int)Hk;
    a.D = (int)D;
    a.page = (int)k_pages->shape[2];
    a.width = (int)width;
    a.scale = scale;
    // (blocks of 32 query heads of a group are a launch's second dimension)
    if (Hq / Hk > 32 * 65535) return fail(MS_E_UNSUPPORTED, "more than 32 x 65535 query heads for a head of the cache");
    if (ms::paged_blocks(a) > kMaxBlocks) return fail(MS_E_UNSUPPORTED, "2^24 or more blocks");
    Stands sg;
    const Stand sq = sg.add(q, true), so = sg.add(o, false);
    const size_t kb = ms::paged_workspace(q->dtype, a);
    Work w;
    if ((st = take(&w, sg.bytes + kb, stream, false))) return st;
    int err = put_in(sq, w.base, stream);
    const ms::HeadsView vq = view(sq, w.base), vo = view(so, w.base);
    a.q = vq.p;
    a.qts = vq.ts;
    a.qhs = vq.hs;
    a.o = vo.p;
    a.ots = vo.ts;
    a.ohs = vo.hs;
    if (!err) err = ms::launch_paged(q->dtype, a, kb ? w.base + sg.bytes : nullptr, stream);
    if (!err) err = put_out(so, w.base, stream);
    return err ? hip_fail(err, "forward launch") : MS_OK;
}

}  // extern "C"
