// Shared by the host runtime's files (memsave.cpp, blocks.cpp): errors, the
// byte ledger, tensor checks, layout staging and the record.  Plain C++, as
// memsave.cpp: nothing here touches the device except through device.h.
#pragma once

#include <algorithm>
#include <initializer_list>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <string>

#include "../../include/memsave.h"
#include "device.h"

namespace ms {
namespace rt {

// defined in memsave.cpp: an inline variable would be one object for every library
// in the process that holds this header
extern thread_local std::string g_err;

inline ms_status fail(ms_status s, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    g_err = buf;
    return s;
}

inline void clear_err() { g_err.clear(); }

// ------------------------------------------------------------------ ledger
extern std::atomic<uint64_t> g_live, g_peak;
extern std::atomic<int64_t> g_records;

inline void ledger_add(uint64_t n) {
    uint64_t now = g_live.fetch_add(n) + n;
    uint64_t pk = g_peak.load();
    while (now > pk && !g_peak.compare_exchange_weak(pk, now)) {
    }
}

inline void ledger_sub(uint64_t n) { g_live.fetch_sub(n); }

// ------------------------------------------------------------------ tensors
constexpr int64_t kMaxElems = (int64_t(1) << 31) - 1;
constexpr uint32_t kMagic = 0x4d53524bu;  // "MSRK"

// Product of non-negative extents, saturated just above kMaxElems (the
// limit checks below must not be fooled by an int64 overflow).
inline int64_t capped_product(std::initializer_list<int64_t> f);

inline int64_t numel(const ms_tensor *t) {
    int64_t n = 1;
    for (int i = 0; i < t->ndim; ++i) n *= t->shape[i];
    return n;
}

inline size_t elt_size(int32_t dt) { return dt == MS_BF16 ? 2 : 4; }

inline int64_t capped_product(std::initializer_list<int64_t> f) {
    int64_t p = 1;
    for (int64_t v : f) {
        if (v == 0) return 0;
        if (p > (kMaxElems + 1) / v) p = kMaxElems + 1;
        else p = std::min<int64_t>(p * v, kMaxElems + 1);
    }
    return p;
}

inline bool dtype_ok(int32_t dt) { return dt == MS_F32 || dt == MS_BF16; }

// Basic sanity: ndim, non-negative extents, element limit, dtype.
inline ms_status check_tensor(const ms_tensor *t, const char *name, int ndim, bool need_data) {
    if (!t) return fail(MS_E_NULL, "%s is NULL", name);
    if (t->ndim != ndim) return fail(MS_E_SHAPE, "%s: expected %d dims, got %d", name, ndim, t->ndim);
    if (!dtype_ok(t->dtype)) return fail(MS_E_DTYPE, "%s: unsupported dtype %d", name, t->dtype);
    int64_t n = 1;
    for (int i = 0; i < ndim; ++i) {
        if (t->shape[i] < 0) return fail(MS_E_SHAPE, "%s: negative extent", name);
        if (t->shape[i] > kMaxElems) return fail(MS_E_UNSUPPORTED, "%s: extent too large", name);
        n *= t->shape[i];
        if (n > kMaxElems) return fail(MS_E_UNSUPPORTED, "%s: more than 2^31-1 elements", name);
    }
    if (need_data && n > 0 && t->data == nullptr) return fail(MS_E_NULL, "%s.data is NULL", name);
    return MS_OK;
}

// Channels-last 4-D: memory order N, H, W, C (dims of extent 1 may carry any stride).
inline bool is_nhwc(const ms_tensor *t) {
    if (numel(t) == 0) return true;   // no element is ever addressed
    const int64_t N = t->shape[0], C = t->shape[1], H = t->shape[2], W = t->shape[3];
    (void)N;
    const int64_t want[4] = {H * W * C, 1, W * C, C};
    for (int i = 0; i < 4; ++i)
        if (t->shape[i] > 1 && t->stride[i] != want[i]) return false;
    return true;
}

// Channels-last 5-D: memory order N, D, H, W, C.
inline bool is_ndhwc(const ms_tensor *t) {
    if (numel(t) == 0) return true;
    const int64_t C = t->shape[1], D = t->shape[2], H = t->shape[3], W = t->shape[4];
    const int64_t want[5] = {D * H * W * C, 1, H * W * C, W * C, C};
    for (int i = 0; i < 5; ++i)
        if (t->shape[i] > 1 && t->stride[i] != want[i]) return false;
    return true;
}

inline bool is_rowmajor2(const ms_tensor *t) {
    if (numel(t) == 0) return true;
    if (t->shape[1] > 1 && t->stride[1] != 1) return false;
    if (t->shape[0] > 1 && t->stride[0] != t->shape[1]) return false;
    return true;
}

inline bool is_contig1(const ms_tensor *t) { return t->shape[0] <= 1 || t->stride[0] == 1; }

// Any layout of an input: strides of the varying dims must be >= 0.
inline bool strides_ok(const ms_tensor *t) {
    for (int i = 0; i < t->ndim; ++i)
        if (t->shape[i] > 1 && t->stride[i] < 0) return false;
    return true;
}

// No two elements share an address: with the varying dims sorted by stride,
// each stride is at least the span of the faster ones (a strided sub-array
// of a dense array).  Outputs must satisfy this.
inline bool non_overlapping(const ms_tensor *t) {
    if (!strides_ok(t)) return false;
    if (numel(t) == 0) return true;
    int d[5], k = 0;
    for (int i = 0; i < t->ndim; ++i)
        if (t->shape[i] > 1) d[k++] = i;
    std::sort(d, d + k, [&](int a, int b) { return t->stride[a] < t->stride[b]; });
    int64_t span = 1;
    for (int i = 0; i < k; ++i) {
        if (t->stride[d[i]] < span) return false;
        span = t->stride[d[i]] * t->shape[d[i]];
    }
    return true;
}

// Every element of a dense block of numel(t) elements, in some order of the
// dims (channels-last, NCHW, a transposed matrix, ...).
inline bool dense_any_order(const ms_tensor *t) {
    if (!non_overlapping(t)) return false;
    if (numel(t) == 0) return true;
    int64_t lo_span = 1;
    int d[5], k = 0;
    for (int i = 0; i < t->ndim; ++i)
        if (t->shape[i] > 1) d[k++] = i;
    std::sort(d, d + k, [&](int a, int b) { return t->stride[a] < t->stride[b]; });
    for (int i = 0; i < k; ++i) {
        if (t->stride[d[i]] != lo_span) return false;
        lo_span *= t->shape[d[i]];
    }
    return true;
}

// Plain row-major [N, C, H, W] (PyTorch's default contiguous layout).
inline bool is_nchw(const ms_tensor *t) {
    if (t->ndim != 4) return false;
    const int64_t C = t->shape[1], H = t->shape[2], W = t->shape[3];
    const int64_t want[4] = {C * H * W, H * W, W, 1};
    for (int i = 0; i < 4; ++i)
        if (t->shape[i] > 1 && t->stride[i] != want[i]) return false;
    return true;
}

inline bool same_strides(const ms_tensor *a, const ms_tensor *b) {
    for (int i = 0; i < a->ndim; ++i)
        if (a->shape[i] > 1 && a->stride[i] != b->stride[i]) return false;
    return true;
}

// The dense layout the kernels read and write: channels-last for 4-D
// tensors (NHWC activations, KRSC filters), row-major for matrices.
inline bool canonical(const ms_tensor *t) {
    if (t->ndim == 4) return is_nhwc(t);
    if (t->ndim == 2) return is_rowmajor2(t);
    if (t->ndim == 5) return is_ndhwc(t);
    return is_contig1(t);
}

inline bool same_shape(const ms_tensor *a, const ms_tensor *b) {
    if (a->ndim != b->ndim) return false;
    for (int i = 0; i < a->ndim; ++i)
        if (a->shape[i] != b->shape[i]) return false;
    return true;
}

inline ms_tensor shape_only(const ms_tensor *t) {
    ms_tensor s = *t;
    s.data = nullptr;
    return s;
}

// ------------------------------------------------------------------ layer plan
struct Plan {
    int32_t kind = 0;
    int32_t dtype = 0;
    ms::ConvGeom g{};      // conv / linear; transposed conv: the convolution it is the adjoint of
    ms::Conv3dGeom q{};    // 3-D kinds: the (adjoint) 3-D convolution; g = q.g
    int64_t rows = 0;      // BN / avgpool: pixels; conv/linear bias grad rows
    int C = 0;             // BN / avgpool channels
    int L = 0;             // avgpool pixels per sample
    int Nb = 0;            // avgpool batch
    bool has_w = false, has_b = false;
    uint64_t x_bytes = 0, w_bytes = 0, stat_bytes = 0;
    int64_t n = 0;                           // ReLU / dropout: elements
    uint64_t bits_bytes = 0, y_bytes = 0;    // ReLU: 1-bit mask, output
    uint64_t mask8_bytes = 0;                // dropout: stock PyTorch's one-byte mask
    // layouts that are not the kernels' (staged through transient workspace)
    bool st_x = false, st_w = false, st_y = false;
    uint64_t out_bytes = 0;                  // bytes of y
    bool bn_nchw = false;                    // BN-eval on plain NCHW tensors: its sweeps run in place
    int64_t hw = 0;                          // BN-eval: H * W of a 4-D x
};

inline ms_status hip_fail(int err, const char *what) {
    return fail(MS_E_HIP, "%s failed with HIP error %d", what, err);
}

// ------------------------------------------------------------------ layout staging
// A caller tensor that is not in the kernels' layout (NCHW, a strided
// slice, a transposed matrix) is copied into a dense channels-last (or
// row-major) stand-in in transient workspace before the launch, and an
// output is written to such a stand-in and copied out after it.  The record
// still borrows the caller's own tensor.
constexpr size_t kNoStage = ~size_t(0);

inline size_t al256(size_t n) { return (n + 255) / 256 * 256; }

struct Stager {
    size_t bytes = 0;
    // Offset of t's stand-in, or kNoStage when t is used in place.
    size_t add(const ms_tensor *t) {
        if (!t || !t->data || numel(t) == 0 || canonical(t)) return kNoStage;
        const size_t off = bytes;
        bytes += al256((size_t)numel(t) * elt_size(t->dtype));
        return off;
    }
};

// The copy between t's layout and its dense stand-in, over (n, h, w, c) for
// 4-D tensors and (m, -, -, k) for matrices.
inline void copy_desc(const ms_tensor *t, int64_t ext[4], int64_t s[4], int64_t dense[4]) {
    if (t->ndim == 4) {
        const int64_t N = t->shape[0], C = t->shape[1], H = t->shape[2], W = t->shape[3];
        const int64_t e[4] = {N, H, W, C}, st[4] = {t->stride[0], t->stride[2], t->stride[3], t->stride[1]},
                      d[4] = {H * W * C, W * C, C, 1};
        for (int i = 0; i < 4; ++i) ext[i] = e[i], s[i] = st[i], dense[i] = d[i];
    } else {
        const int64_t e[4] = {t->shape[0], 1, 1, t->shape[1]}, st[4] = {t->stride[0], 0, 0, t->stride[1]},
                      d[4] = {t->shape[1], 0, 0, 1};
        for (int i = 0; i < 4; ++i) ext[i] = e[i], s[i] = st[i], dense[i] = d[i];
    }
}

inline int stage_in(const ms_tensor *t, char *base, size_t off, void *stream) {
    if (off == kNoStage) return 0;
    int64_t ext[4], s[4], d[4];
    copy_desc(t, ext, s, d);
    return ms::launch_copy4(t->dtype, t->data, ext, s, base + off, d, stream);
}

inline int stage_out(const ms_tensor *t, char *base, size_t off, void *stream) {
    if (off == kNoStage) return 0;
    int64_t ext[4], s[4], d[4];
    copy_desc(t, ext, s, d);
    return ms::launch_copy4(t->dtype, base + off, ext, d, t->data, s, stream);
}

// Data pointer the kernels use for t: its stand-in or the caller's memory.
inline void *kptr(const ms_tensor *t, char *base, size_t off) {
    if (!t) return nullptr;
    return off == kNoStage ? t->data : base + off;
}

// What the backward of a block layer (blocks.cpp) needs besides the borrowed tensors.
struct BlockState {
    int64_t M = 0, D = 0;        // rows and input width
    int64_t F = 0;               // gated linear: output width; cross entropy: vocabulary
    int32_t act = 0, keep = 0, reduction = 0;
    int64_t ignore = 0;
    const int64_t *target = nullptr;
    void *proj = nullptr;        // gated linear: the kept projections
    float *lse = nullptr;        // cross entropy: log-sum-exp of each row without its target,
    const void *grad = nullptr;  // or the kept gradient
};

}  // namespace rt
}  // namespace ms

struct ms_record {
    uint32_t magic;
    ms::rt::Plan plan;
    float eps;
    ms_tensor x, W, b, mean, var, y;   // data non-NULL only for borrowed tensors
    void *bits;                         // ReLU: the borrowed 1-bit mask
    uint64_t seed, offset;              // dropout: generator key and first block
    uint32_t thresh;                    // dropout: keep iff word >= thresh
    float scale;                        // dropout: 1 / (1 - p) (0 when p = 1)
    int drop_all;                       // dropout: p = 1
    ms_account acct;
    // the backward of a layer that runs outside the linear kinds' switch (null: none)
    ms_status (*run)(ms_record *r, const ms_tensor *grad_y, const ms_tensor *grad_x, const ms_tensor *grad_W,
                     const ms_tensor *grad_b, void *stream, bool fixed_scratch) = nullptr;
    ms::rt::BlockState blk;             // its state
    bool consumed;
    bool released;
};

namespace ms {
namespace rt {

inline void release(ms_record *r) {
    if (!r->released) {
        ledger_sub(r->acct.saved_activation_bytes);
        r->released = true;
        r->x.data = nullptr;
        r->W.data = nullptr;
        r->b.data = nullptr;
        r->mean.data = nullptr;
        r->var.data = nullptr;
        r->bits = nullptr;
        r->blk.target = nullptr;
        r->blk.proj = nullptr;
        r->blk.lse = nullptr;
    }
}

inline ms_status check_grad(const ms_tensor *g, const ms_tensor *primal, const char *name, int32_t kind, bool output) {
    ms_status st = check_tensor(g, name, primal->ndim, true);
    if (st) return st;
    if (g->dtype != primal->dtype) return fail(MS_E_DTYPE, "%s dtype must match its primal", name);
    if (!same_shape(g, primal)) return fail(MS_E_SHAPE, "%s shape must match its primal", name);
    if (g->ndim == 5 && !is_ndhwc(g)) return fail(MS_E_LAYOUT, "%s must be channels-last", name);
    if (g->ndim == 1 && !is_contig1(g)) return fail(MS_E_LAYOUT, "%s must be contiguous", name);
    if (kind == MS_RELU || kind == MS_DROPOUT) {
        // elementwise in memory order: the layout of the forward's tensors
        if (!dense_any_order(g) || !same_strides(g, primal)) return fail(MS_E_LAYOUT, "%s must be in the layout of x", name);
    } else if (output ? !non_overlapping(g) : !strides_ok(g)) {
        return fail(MS_E_LAYOUT, output ? "%s must not overlap itself" : "%s needs non-negative strides", name);
    }
    return MS_OK;
}

}  // namespace rt
}  // namespace ms
