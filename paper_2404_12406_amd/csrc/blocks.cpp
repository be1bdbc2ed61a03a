// Host runtime of the transformer layers: layer norm, the gated linear unit and
// the cross entropy of a linear head.
// Validation, the save rule and the records follow memsave.cpp: every check
// runs before the first launch, a record borrows what its mask's gradients
// need and nothing else, and all work goes to the caller's stream.
#include "runtime.h"

using namespace ms::rt;

namespace {

// Transient workspace of one call: the stream's (held until the last launch) or,
// with `fixed`, the library's static scratch.
struct Work {
    char *base = nullptr;
    ms::WorkspaceHold hold;
};

ms_status take(Work *w, size_t bytes, void *stream, bool fixed) {
    if (!bytes) return MS_OK;
    int err = 0;
    if (fixed) {
        w->base = static_cast<char *>(ms::scratch_get(bytes, &err));
        if (err)
            return err == 1 ? fail(MS_E_UNSUPPORTED, "backward needs %zu bytes of scratch; the fixed scratch holds %zu", bytes,
                                   ms::kScratchBytes)
                            : hip_fail(ms::device_last_error(), "scratch lookup");
        return MS_OK;
    }
    w->base = static_cast<char *>(ms::workspace_get(stream, bytes, &err, &w->hold));
    if (err)
        return err == 1 ? fail(MS_E_NOMEM, "workspace of %zu bytes unavailable", bytes)
                        : hip_fail(ms::device_last_error(), "workspace");
    return MS_OK;
}

ms_status check_mask(uint32_t mask, const ms_tensor *W, const ms_tensor *b) {
    if (mask & ~7u) return fail(MS_E_MASK, "mask 0x%x has bits outside INPUT|WEIGHT|BIAS", mask);
    if ((mask & MS_RG_WEIGHT) && !W) return fail(MS_E_MASK, "WEIGHT bit set but the layer has no weight");
    if ((mask & MS_RG_BIAS) && !b) return fail(MS_E_MASK, "BIAS bit set but the layer has no bias");
    return MS_OK;
}

// A 1-D parameter of n elements; null is allowed.
ms_status check_vector(const ms_tensor *t, const char *name, int64_t n, int32_t dtype) {
    if (!t) return MS_OK;
    const ms_status st = check_tensor(t, name, 1, true);
    if (st) return st;
    if (t->dtype != dtype) return fail(MS_E_DTYPE, "%s dtype differs from x", name);
    if (t->shape[0] != n) return fail(MS_E_SHAPE, "%s must have %lld elements", name, (long long)n);
    if (!is_contig1(t)) return fail(MS_E_LAYOUT, "%s must be contiguous", name);
    return MS_OK;
}

ms_status check_output(const ms_tensor *y, const char *name, int64_t rows, int64_t cols, int32_t dtype) {
    const ms_status st = check_tensor(y, name, 2, true);
    if (st) return st;
    if (y->dtype != dtype) return fail(MS_E_DTYPE, "%s dtype differs from x", name);
    if (y->shape[0] != rows || y->shape[1] != cols)
        return fail(MS_E_SHAPE, "%s must be [%lld, %lld]", name, (long long)rows, (long long)cols);
    if (!non_overlapping(y)) return fail(MS_E_LAYOUT, "%s must not overlap itself", name);
    return MS_OK;
}

using Run = ms_status (*)(ms_record *, const ms_tensor *, const ms_tensor *, const ms_tensor *, const ms_tensor *, void *, bool);

uint64_t bytes_of(const ms_tensor *t) { return t ? (uint64_t)numel(t) * elt_size(t->dtype) : 0; }

// A record with the shapes of its layer's tensors and the data of those that
// `borrowed` names; not yet in the ledger.
ms_record *new_record(int32_t kind, const ms_tensor *x, const ms_tensor *W, const ms_tensor *b, const ms_tensor *y, uint32_t mask,
                      uint32_t borrowed, Run run) {
    ms_record *r = new (std::nothrow) ms_record();
    if (!r) return nullptr;
    r->magic = kMagic;
    r->plan.kind = kind;
    r->plan.dtype = x->dtype;
    r->x = shape_only(x);
    r->y = shape_only(y);
    if (W) r->W = shape_only(W);
    if (b) r->b = shape_only(b);
    if (borrowed & MS_SAVED_X) r->x.data = x->data;
    if (borrowed & MS_SAVED_W) r->W.data = W->data;
    r->acct.mask = mask;
    r->acct.borrowed = borrowed;
    r->acct.kernels = ((mask & MS_RG_INPUT) ? (uint32_t)MS_K_DGRAD : 0u) | ((mask & MS_RG_WEIGHT) ? (uint32_t)MS_K_WGRAD : 0u) |
                      ((mask & MS_RG_BIAS) ? (uint32_t)MS_K_BGRAD : 0u);
    r->acct.saved_activation_bytes = (borrowed & MS_SAVED_X) ? bytes_of(x) : 0;
    r->acct.referenced_param_bytes = (borrowed & MS_SAVED_W) ? bytes_of(W) : 0;
    r->run = run;
    return r;
}

void file_record(ms_record *r, ms_record **rec) {
    if (!r) return;
    ledger_add(r->acct.saved_activation_bytes);
    g_records.fetch_add(1);
    *rec = r;
}

// ------------------------------------------------------------------ layer norm
// Bytes of the stand-in of a tensor in another layout.
size_t staging(const ms_tensor *a, bool used) {
    return used && numel(a) && !canonical(a) ? al256((size_t)numel(a) * elt_size(a->dtype)) : 0;
}

size_t norm_workspace(int32_t dtype, int64_t M, int64_t D, uint32_t mask) {
    if (mask & (MS_RG_INPUT | MS_RG_WEIGHT))
        return ms::layer_norm_bwd_workspace(dtype, M, D, (mask & (MS_RG_WEIGHT | MS_RG_BIAS)) != 0);
    return ms::colsum_workspace(dtype, M, (int)D);   // the shift alone
}

ms_status norm_backward(ms_record *r, const ms_tensor *gy, const ms_tensor *gx, const ms_tensor *gg, const ms_tensor *gb,
                        void *stream, bool fixed) {
    const int32_t dt = r->plan.dtype;
    const int64_t M = r->blk.M, D = r->blk.D;
    Stager sg;
    const bool read_x = gx || gg;
    const size_t oy = sg.add(gy), ox = read_x ? sg.add(&r->x) : kNoStage, ogx = gx ? sg.add(gx) : kNoStage;
    const size_t kb = norm_workspace(dt, M, D, r->acct.mask);
    Work w;
    ms_status st = take(&w, sg.bytes + kb, stream, fixed);
    if (st) return st;
    void *ws = kb ? w.base + sg.bytes : nullptr;
    int err = stage_in(gy, w.base, oy, stream);
    if (!err && read_x) err = stage_in(&r->x, w.base, ox, stream);
    const void *dy = kptr(gy, w.base, oy);
    if (!err) {
        if (read_x)
            err = ms::launch_layer_norm_bwd(dt, kptr(&r->x, w.base, ox), dy, r->W.data, r->eps, M, D, kptr(gx, w.base, ogx),
                                            gg ? gg->data : nullptr, gb ? gb->data : nullptr, ws, stream);
        else
            err = ms::launch_colsum(dt, dy, M, (int)D, gb->data, ws, stream);
    }
    if (!err) err = stage_out(gx, w.base, ogx, stream);
    return err ? hip_fail(err, "backward launch") : MS_OK;
}

// ------------------------------------------------------------------ gated linear unit
bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Where a stand-in will lie: aligned, whatever the caller's pointer is.
const void *place(const ms_tensor *t, size_t off) { return off == kNoStage ? t->data : nullptr; }

ms_status gated_backward(ms_record *r, const ms_tensor *gy, const ms_tensor *gx, const ms_tensor *gw, const ms_tensor *gb,
                         void *stream, bool fixed) {
    const int32_t dt = r->plan.dtype;
    const int64_t M = r->blk.M, D = r->blk.D, F = r->blk.F;
    const bool again = !r->blk.proj && numel(&r->x);   // z is taken again
    const bool read_x = again || gw, read_w = again || gx;
    Stager sg;
    const size_t oy = sg.add(gy), ox = read_x ? sg.add(&r->x) : kNoStage, ow = read_w ? sg.add(&r->W) : kNoStage;
    const size_t ogx = gx ? sg.add(gx) : kNoStage, ogw = gw ? sg.add(gw) : kNoStage;
    const size_t kb = ms::gated_bwd_workspace(dt, M, D, F, place(&r->x, ox), place(&r->W, ow), r->b.data, !again, gx, gw, gb);
    Work w;
    ms_status st = take(&w, sg.bytes + kb, stream, fixed);
    if (st) return st;
    int err = stage_in(gy, w.base, oy, stream);
    if (!err && read_x) err = stage_in(&r->x, w.base, ox, stream);
    if (!err && read_w) err = stage_in(&r->W, w.base, ow, stream);
    if (!err)
        err = ms::launch_gated_bwd(dt, M, D, F, r->blk.act, kptr(&r->x, w.base, ox), kptr(&r->W, w.base, ow), r->b.data, r->blk.proj,
                                   kptr(gy, w.base, oy), kptr(gx, w.base, ogx), kptr(gw, w.base, ogw), gb ? gb->data : nullptr,
                                   w.base + sg.bytes, stream);
    if (!err) err = stage_out(gx, w.base, ogx, stream);
    if (!err) err = stage_out(gw, w.base, ogw, stream);
    return err ? hip_fail(err, "backward launch") : MS_OK;
}

// ------------------------------------------------------------------ cross entropy
struct HeadPads {
    bool w, b;
};

HeadPads head_pads(int32_t dtype, int64_t D, const void *w, const void *b) {
    if (dtype != MS_BF16) return {false, false};
    return {D % 8 != 0 || !aligned(w, 16), b && !aligned(b, 4)};
}

ms_status xent_backward(ms_record *r, const ms_tensor *gloss, const ms_tensor *gx, const ms_tensor *gw, const ms_tensor *gb,
                        void *stream, bool fixed) {
    const int32_t dt = r->plan.dtype;
    const int64_t M = r->blk.M, D = r->blk.D, V = r->blk.F;
    if (r->blk.grad) {
        Stager sg;
        const size_t ogx = sg.add(gx);
        Work w;
        ms_status st = take(&w, sg.bytes, stream, fixed);
        if (st) return st;
        int err = ms::launch_xent_scale(dt, M, D, r->blk.grad, static_cast<const float *>(gloss->data), r->blk.reduction,
                                        kptr(gx, w.base, ogx), stream);
        if (!err) err = stage_out(gx, w.base, ogx, stream);
        return err ? hip_fail(err, "backward launch") : MS_OK;
    }
    Stager sg;
    const size_t ox = sg.add(&r->x), ow = sg.add(&r->W), ogx = gx ? sg.add(gx) : kNoStage, ogw = gw ? sg.add(gw) : kNoStage;
    const HeadPads p = head_pads(dt, D, place(&r->W, ow), r->b.data);
    const size_t kb = ms::xent_bwd_workspace(dt, M, D, V, p.w, p.b, gx, gw, gb);
    Work w;
    ms_status st = take(&w, sg.bytes + kb, stream, fixed);
    if (st) return st;
    int err = stage_in(&r->x, w.base, ox, stream);
    if (!err) err = stage_in(&r->W, w.base, ow, stream);
    if (!err)
        err = ms::launch_xent_bwd(dt, M, D, V, kptr(&r->x, w.base, ox), kptr(&r->W, w.base, ow), r->b.data, p.w, p.b, r->blk.target,
                                  r->blk.ignore, r->blk.reduction, static_cast<const float *>(gloss->data), r->blk.lse, kptr(gx, w.base, ogx),
                                  kptr(gw, w.base, ogw), gb ? gb->data : nullptr, w.base + sg.bytes, stream);
    if (!err) err = stage_out(gx, w.base, ogx, stream);
    if (!err) err = stage_out(gw, w.base, ogw, stream);
    return err ? hip_fail(err, "backward launch") : MS_OK;
}

}  // namespace

extern "C" {

ms_status ms_layer_norm_forward(const ms_tensor *x, const ms_tensor *gamma, const ms_tensor *beta, float eps, uint32_t mask,
                                const ms_tensor *y, ms_record **rec, void *stream) {
    clear_err();
    if (!rec) return fail(MS_E_NULL, "rec is NULL");
    *rec = nullptr;
    ms_status st = check_mask(mask, gamma, beta);
    if (!st) st = check_tensor(x, "x", 2, true);
    if (st) return st;
    const int64_t M = x->shape[0], D = x->shape[1];
    if (D < 1) return fail(MS_E_SHAPE, "layer norm needs rows of at least one element");
    if (!strides_ok(x)) return fail(MS_E_LAYOUT, "x needs non-negative strides");
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MS_E_ARG, "eps must be finite and >= 0");
    if ((st = check_vector(gamma, "gamma", D, x->dtype)) || (st = check_vector(beta, "beta", D, x->dtype)) ||
        (st = check_output(y, "y", M, D, x->dtype)))
        return st;
    Stager sg;
    const size_t ox = sg.add(x), oy = sg.add(y);
    Work w;
    if ((st = take(&w, sg.bytes, stream, false))) return st;
    ms_record *r = nullptr;
    if (mask) {
        const uint32_t borrowed = ((mask & (MS_RG_INPUT | MS_RG_WEIGHT)) ? (uint32_t)MS_SAVED_X : 0u) |
                                  ((mask & MS_RG_INPUT) && gamma ? (uint32_t)MS_SAVED_W : 0u);
        r = new_record(MS_LAYER_NORM, x, gamma, beta, y, mask, borrowed, norm_backward);
        if (!r) return fail(MS_E_NOMEM, "record allocation failed");
        r->eps = eps;
        r->blk.M = M;
        r->blk.D = D;
        // the output gradient in y's layout, the input's gradient in x's
        r->acct.transient_workspace_bytes = norm_workspace(x->dtype, M, D, mask) + staging(y, true) +
                                            staging(x, (mask & (MS_RG_INPUT | MS_RG_WEIGHT)) != 0) +
                                            staging(x, (mask & MS_RG_INPUT) != 0);
    }
    int err = stage_in(x, w.base, ox, stream);
    if (!err)
        err = ms::launch_layer_norm_fwd(x->dtype, kptr(x, w.base, ox), gamma ? gamma->data : nullptr, beta ? beta->data : nullptr,
                                        eps, M, D, kptr(y, w.base, oy), stream);
    if (!err) err = stage_out(y, w.base, oy, stream);
    if (err) {
        delete r;
        return hip_fail(err, "forward launch");
    }
    file_record(r, rec);
    return MS_OK;
}

uint64_t ms_gated_projection_bytes(int64_t rows, int64_t F, int32_t dtype) {
    if (rows <= 0 || F <= 0) return 0;
    return dtype == MS_BF16 ? (uint64_t)rows * 2u * (uint64_t)F * 3u : (uint64_t)rows * 2u * (uint64_t)((F + 15) / 16 * 16) * 4u;
}

ms_status ms_gated_linear_forward(const ms_tensor *x, const ms_tensor *W, const ms_tensor *b, int32_t activation,
                                  void *proj, uint32_t mask, const ms_tensor *y, ms_record **rec, void *stream) {
    clear_err();
    if (!rec) return fail(MS_E_NULL, "rec is NULL");
    *rec = nullptr;
    if (!W) return fail(MS_E_NULL, "a gated linear unit needs W");
    ms_status st = check_mask(mask, W, b);
    if (!st) st = check_tensor(x, "x", 2, true);
    if (!st) st = check_tensor(W, "W", 2, true);
    if (st) return st;
    const int64_t M = x->shape[0], D = x->shape[1], F = W->shape[0] / 2;
    if (x->dtype != W->dtype) return fail(MS_E_DTYPE, "x and W dtypes differ");
    if (D < 1 || F < 1 || W->shape[0] % 2) return fail(MS_E_SHAPE, "W must be [2 F, D] with F, D >= 1");
    if (W->shape[1] != D)
        return fail(MS_E_SHAPE, "W has %lld input features, x has %lld", (long long)W->shape[1], (long long)D);
    if (!strides_ok(x) || !strides_ok(W)) return fail(MS_E_LAYOUT, "x and W need non-negative strides");
    if (activation < MS_ACT_SILU || activation > MS_ACT_SIGMOID) return fail(MS_E_ARG, "unknown activation %d", activation);
    if (capped_product({M, 2 * F}) > kMaxElems) return fail(MS_E_UNSUPPORTED, "projections have more than 2^31-1 elements");
    // rows of bf16 padded to whole 16-byte vectors have 32-bit offsets too
    if (x->dtype == MS_BF16 && capped_product({std::max(M, 2 * F), (D + 7) / 8 * 8}) > kMaxElems - 16)
        return fail(MS_E_UNSUPPORTED, "operands have more than 2^31-17 elements");
    if ((st = check_vector(b, "b", 2 * F, x->dtype)) || (st = check_output(y, "y", M, F, x->dtype))) return st;
    if (proj) {
        if (!mask) return fail(MS_E_ARG, "without a mask the projections are not kept: proj must be NULL");
        if (!aligned(proj, 16)) return fail(MS_E_ARG, "proj must be 16-byte aligned");
    }
    Stager sg;
    const size_t ox = sg.add(x), ow = sg.add(W), oy = sg.add(y);
    const void *bk = b ? b->data : nullptr;
    const size_t kb = ms::gated_fwd_workspace(x->dtype, M, D, F, place(x, ox), place(W, ow), bk, proj != nullptr);
    Work w;
    if ((st = take(&w, sg.bytes + kb, stream, false))) return st;
    ms_record *r = nullptr;
    if (mask) {
        const bool again = !proj;
        const uint32_t borrowed = ((again || (mask & MS_RG_WEIGHT)) ? (uint32_t)MS_SAVED_X : 0u) |
                                  ((again || (mask & MS_RG_INPUT)) ? (uint32_t)MS_SAVED_W : 0u) |
                                  (proj ? (uint32_t)MS_SAVED_PROJ : 0u);
        r = new_record(MS_GATED_LINEAR, x, W, b, y, mask, borrowed, gated_backward);
        if (!r) return fail(MS_E_NOMEM, "record allocation failed");
        r->blk.M = M;
        r->blk.D = D;
        r->blk.F = F;
        r->blk.act = activation;
        r->blk.proj = proj;
        if (b && again) {
            r->b.data = b->data;
            r->acct.referenced_param_bytes += bytes_of(b);
        }
        if (proj) r->acct.saved_activation_bytes += ms_gated_projection_bytes(M, F, x->dtype);
        const bool dx = mask & MS_RG_INPUT, dw = mask & MS_RG_WEIGHT, db = mask & MS_RG_BIAS;
        r->acct.transient_workspace_bytes = ms::gated_bwd_workspace(x->dtype, M, D, F, place(x, ox), place(W, ow), bk, !again, dx, dw, db) +
                                            staging(y, true) + staging(x, again || dw) + staging(W, again || dx) +
                                            staging(x, dx) + staging(W, dw);
    }
    int err = stage_in(x, w.base, ox, stream);
    if (!err) err = stage_in(W, w.base, ow, stream);
    if (!err)
        err = ms::launch_gated_fwd(x->dtype, M, D, F, activation, kptr(x, w.base, ox), kptr(W, w.base, ow), bk, kptr(y, w.base, oy), proj,
                                   w.base + sg.bytes, stream);
    if (!err) err = stage_out(y, w.base, oy, stream);
    if (err) {
        delete r;
        return hip_fail(err, "forward launch");
    }
    file_record(r, rec);
    return MS_OK;
}

uint64_t ms_cross_entropy_kept_bytes(int64_t rows, int64_t D, int64_t V, int32_t dtype, uint32_t mask) {
    if (rows <= 0 || D <= 0 || V <= 0 || !(mask & 7u)) return 0;
    if (ms::xent_keeps_gradient(dtype, rows, D, V, mask & MS_RG_INPUT, mask & MS_RG_WEIGHT, mask & MS_RG_BIAS))
        return ms::xent_kept_bytes(dtype, rows, D);
    return (uint64_t)rows * sizeof(float);
}

ms_status ms_cross_entropy_forward(const ms_tensor *x, const ms_tensor *W, const ms_tensor *b, const int64_t *target,
                                   int64_t ignore_index, int32_t reduction, void *kept, uint32_t mask, const ms_tensor *loss,
                                   ms_record **rec, void *stream) {
    clear_err();
    if (!rec) return fail(MS_E_NULL, "rec is NULL");
    *rec = nullptr;
    if (!W) return fail(MS_E_NULL, "cross entropy needs W");
    ms_status st = check_mask(mask, W, b);
    if (!st) st = check_tensor(x, "x", 2, true);
    if (!st) st = check_tensor(W, "W", 2, true);
    if (st) return st;
    const int64_t M = x->shape[0], D = x->shape[1], V = W->shape[0];
    if (x->dtype != W->dtype) return fail(MS_E_DTYPE, "x and W dtypes differ");
    if (D < 1 || V < 1) return fail(MS_E_SHAPE, "W must be [V, D] with V, D >= 1");
    if (W->shape[1] != D)
        return fail(MS_E_SHAPE, "W has %lld input features, x has %lld", (long long)W->shape[1], (long long)D);
    if (!strides_ok(x) || !strides_ok(W)) return fail(MS_E_LAYOUT, "x and W need non-negative strides");
    // rows padded to whole 16-byte vectors have 32-bit offsets too
    if (capped_product({std::max(M, V), (D + 7) / 8 * 8}) > kMaxElems - 16)
        return fail(MS_E_UNSUPPORTED, "operands have more than 2^31-17 elements");
    if (M > ms::kMaxHeadRows) return fail(MS_E_UNSUPPORTED, "x has more than 2^27-8 rows");
    // one launch of bf16 tiles of 128 x 128 logits, of 256 threads each: 2^32 - 1 threads
    if (x->dtype == MS_BF16 && (M + 127) / 128 * ((V + 127) / 128) >= int64_t(1) << 24)
        return fail(MS_E_UNSUPPORTED, "2^38 or more logits");
    if ((st = check_vector(b, "b", V, x->dtype))) return st;
    if (reduction < MS_REDUCE_MEAN || reduction > MS_REDUCE_NONE) return fail(MS_E_ARG, "unknown reduction %d", reduction);
    if (M > 0 && !target) return fail(MS_E_NULL, "target is NULL");
    if (!aligned(target, 8)) return fail(MS_E_ARG, "target must be 8-byte aligned");
    if ((st = check_tensor(loss, "loss", 1, true))) return st;
    if (loss->dtype != MS_F32) return fail(MS_E_DTYPE, "loss must be fp32");
    const int64_t n = reduction == MS_REDUCE_NONE ? M : 1;
    if (loss->shape[0] != n) return fail(MS_E_SHAPE, "loss must have %lld elements", (long long)n);
    if (!is_contig1(loss)) return fail(MS_E_LAYOUT, "loss must be contiguous");
    if (mask && M > 0 && !kept) return fail(MS_E_NULL, "kept is NULL but gradients are asked for");
    if (mask && !aligned(kept, 16)) return fail(MS_E_ARG, "kept must be 16-byte aligned");
    const bool grad = ms::xent_keeps_gradient(x->dtype, M, D, V, mask & MS_RG_INPUT, mask & MS_RG_WEIGHT, mask & MS_RG_BIAS);
    float *lse = mask && !grad ? static_cast<float *>(kept) : nullptr;
    Stager sg;
    const size_t ox = sg.add(x), ow = sg.add(W);
    const HeadPads p = head_pads(x->dtype, D, place(W, ow), b ? b->data : nullptr);
    const size_t kb = ms::xent_fwd_workspace(x->dtype, M, D, V, p.w, p.b, reduction, grad);
    Work w;
    if ((st = take(&w, sg.bytes + kb, stream, false))) return st;
    ms_record *r = nullptr;
    if (mask) {
        r = new_record(MS_CROSS_ENTROPY, x, W, b, loss, mask, grad ? (uint32_t)MS_SAVED_GRAD : MS_SAVED_X | MS_SAVED_W | MS_SAVED_LSE,
                       xent_backward);
        if (!r) return fail(MS_E_NOMEM, "record allocation failed");
        r->blk.M = M;
        r->blk.D = D;
        r->blk.F = V;
        r->blk.reduction = reduction;
        if (grad) {
            r->blk.grad = kept;
            r->acct.saved_activation_bytes = ms::xent_kept_bytes(x->dtype, M, D);
            r->acct.transient_workspace_bytes = staging(x, true);
        } else {
            r->blk.ignore = ignore_index;
            r->blk.target = target;
            r->blk.lse = lse;
            if (b) {
                r->b.data = b->data;
                r->acct.referenced_param_bytes += bytes_of(b);
            }
            r->acct.saved_activation_bytes += (uint64_t)M * (sizeof(float) + sizeof(int64_t));
            const bool dx = mask & MS_RG_INPUT, dw = mask & MS_RG_WEIGHT, db = mask & MS_RG_BIAS;
            r->acct.transient_workspace_bytes = ms::xent_bwd_workspace(x->dtype, M, D, V, p.w, p.b, dx, dw, db) + staging(x, true) +
                                                staging(W, true) + staging(x, dx) + staging(W, dw);
        }
    }
    int err = stage_in(x, w.base, ox, stream);
    if (!err) err = stage_in(W, w.base, ow, stream);
    if (!err)
        err = ms::launch_xent_fwd(x->dtype, M, D, V, kptr(x, w.base, ox), kptr(W, w.base, ow), b ? b->data : nullptr, p.w, p.b, target,
                                  ignore_index, reduction, static_cast<float *>(loss->data), lse, grad ? kept : nullptr,
                                  w.base + sg.bytes, stream);
    if (err) {
        delete r;
        return hip_fail(err, "forward launch");
    }
    file_record(r, rec);
    return MS_OK;
}

}  // extern "C"
