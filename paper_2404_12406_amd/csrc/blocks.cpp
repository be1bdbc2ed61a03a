// Host runtime of the transformer layers: layer norm.
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
size_t norm_staging(const ms_tensor *a, bool used) {
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
        r->acct.transient_workspace_bytes = norm_workspace(x->dtype, M, D, mask) + norm_staging(y, true) +
                                            norm_staging(x, (mask & (MS_RG_INPUT | MS_RG_WEIGHT)) != 0) +
                                            norm_staging(x, (mask & MS_RG_INPUT) != 0);
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

}  // extern "C"
