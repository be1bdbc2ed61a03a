// Shared by the files of the layers with entry points of their own (blocks.cpp,
// attention.cpp): workspace, checks of arguments, records.
#pragma once

#include "runtime.h"

namespace ms {
namespace rt {

// Transient workspace of one call: the stream's (held until the last launch) or,
// with `fixed`, the library's static scratch.
struct Work {
    char *base = nullptr;
    ms::WorkspaceHold hold;
};

inline ms_status take(Work *w, size_t bytes, void *stream, bool fixed) {
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

inline ms_status check_mask(uint32_t mask, const ms_tensor *W, const ms_tensor *b) {
    if (mask & ~7u) return fail(MS_E_MASK, "mask 0x%x has bits outside INPUT|WEIGHT|BIAS", mask);
    if ((mask & MS_RG_WEIGHT) && !W) return fail(MS_E_MASK, "WEIGHT bit set but the layer has no weight");
    if ((mask & MS_RG_BIAS) && !b) return fail(MS_E_MASK, "BIAS bit set but the layer has no bias");
    return MS_OK;
}

// A 1-D parameter of n elements; null is allowed.
inline ms_status check_vector(const ms_tensor *t, const char *name, int64_t n, int32_t dtype) {
    if (!t) return MS_OK;
    const ms_status st = check_tensor(t, name, 1, true);
    if (st) return st;
    if (t->dtype != dtype) return fail(MS_E_DTYPE, "%s dtype differs from x", name);
    if (t->shape[0] != n) return fail(MS_E_SHAPE, "%s must have %lld elements", name, (long long)n);
    if (!is_contig1(t)) return fail(MS_E_LAYOUT, "%s must be contiguous", name);
    return MS_OK;
}

using Run = ms_status (*)(ms_record *, const ms_tensor *, const ms_tensor *, const ms_tensor *, const ms_tensor *, void *, bool);

inline uint64_t bytes_of(const ms_tensor *t) { return t ? (uint64_t)numel(t) * elt_size(t->dtype) : 0; }

// A record with the shapes of its layer's tensors and the data of those that
// `borrowed` names; not yet in the ledger.
inline ms_record *new_record(int32_t kind, const ms_tensor *x, const ms_tensor *W, const ms_tensor *b, const ms_tensor *y, uint32_t mask,
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

inline void file_record(ms_record *r, ms_record **rec) {
    if (!r) return;
    ledger_add(r->acct.saved_activation_bytes);
    g_records.fetch_add(1);
    *rec = r;
}

inline bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace rt
}  // namespace ms
