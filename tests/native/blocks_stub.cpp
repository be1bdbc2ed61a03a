// Stub launchers of the transformer layers for host-only tests of their entry
// points (blocks.cpp), beside host_stub.cpp: each checks that it was handed every
// pointer that its kernel would read or write, notes the call and launches nothing.
#include <mutex>
#include <string>

#include "../../paper_2404_12406_amd/csrc/device.h"

namespace {
std::mutex g_mu;
std::string g_log, g_violation;

void note(const std::string &s) {
    std::lock_guard<std::mutex> lk(g_mu);
    g_log += s + ";";
}

int need(bool ok, const char *what) {
    if (ok) return 0;
    std::lock_guard<std::mutex> lk(g_mu);
    g_violation += std::string(what) + ";";
    return 77;
}
}  // namespace

extern "C" {
const char *blocks_log() { return g_log.c_str(); }
const char *blocks_violations() { return g_violation.c_str(); }
void blocks_reset() {
    std::lock_guard<std::mutex> lk(g_mu);
    g_log.clear();
    g_violation.clear();
}
}

namespace ms {

int launch_layer_norm_fwd(int, const void *x, const void *, const void *, float, int64_t M, int64_t, void *y, void *) {
    note("norm");
    return M > 0 ? need(x && y, "norm:x,y") : 0;
}

size_t layer_norm_bwd_workspace(int, int64_t, int64_t D, bool params) { return params ? (size_t)D * 8 * 4 : 0; }

int launch_layer_norm_bwd(int, const void *x, const void *dy, const void *, float, int64_t M, int64_t, void *dx, void *dg, void *db,
                          void *ws, void *) {
    note(std::string("norm_bwd") + (dx ? "+dx" : "") + (dg ? "+dg" : "") + (db ? "+db" : ""));
    return (M > 0 ? need(x && dy, "norm_bwd:x,dy") : 0) | (dg || db ? need(ws, "norm_bwd:ws") : 0);
}

size_t gated_fwd_workspace(int, int64_t, int64_t, int64_t, const void *, const void *, const void *, bool) { return 256; }

int launch_gated_fwd(int, int64_t M, int64_t, int64_t, int, const void *x, const void *w, const void *, void *y, void *proj, void *ws,
                     void *) {
    note(proj ? "gated+proj" : "gated");
    return (M > 0 ? need(x && w && y, "gated:x,w,y") : 0) | need(ws, "gated:ws");
}

size_t gated_bwd_workspace(int, int64_t, int64_t, int64_t, const void *, const void *, const void *, bool, bool, bool, bool) {
    return 512;
}

int launch_gated_bwd(int, int64_t M, int64_t, int64_t, int, const void *x, const void *w, const void *, const void *proj, const void *dy,
                     void *dx, void *dw, void *db, void *ws, void *) {
    note(std::string("gated_bwd") + (dx ? "+dx" : "") + (dw ? "+dw" : "") + (db ? "+db" : ""));
    int e = need(ws, "gated_bwd:ws");
    if (M > 0) {
        e |= need(dy, "gated_bwd:dy");
        e |= need(proj || (x && w), "gated_bwd:x,w of z");
        if (dx) e |= need(w, "gated_bwd:w");
        if (dw) e |= need(x, "gated_bwd:x");
    }
    return e;
}

// (the rule's form; its sizes are the library's own business)
bool xent_keeps_gradient(int, int64_t M, int64_t, int64_t, bool dx, bool dw, bool db) { return dx && !dw && !db && M >= 1000; }
size_t xent_kept_bytes(int dtype, int64_t M, int64_t D) { return (size_t)M * D * (dtype == kBF16 ? 3 : 4); }
size_t xent_fwd_workspace(int, int64_t, int64_t, int64_t, bool, bool, int, bool keep) { return keep ? 1024 : 256; }

int launch_xent_fwd(int, int64_t M, int64_t, int64_t, const void *x, const void *w, const void *, bool, bool, const int64_t *target,
                    int64_t, int, float *loss, float *lse, void *kept, void *ws, void *) {
    note(kept ? "xent+dx" : lse ? "xent+lse" : "xent");
    if (kept && lse) return need(false, "xent:both");
    return (M > 0 ? need(x && w && target && loss, "xent:x,w,target,loss") : 0) | need(ws, "xent:ws");
}

size_t xent_bwd_workspace(int, int64_t, int64_t, int64_t, bool, bool, bool, bool, bool) { return 512; }

int launch_xent_bwd(int, int64_t M, int64_t, int64_t, const void *x, const void *w, const void *, bool, bool, const int64_t *target,
                    int64_t, int, const float *gloss, const float *lse, void *dx, void *dw, void *db, void *ws, void *) {
    note(std::string("xent_bwd") + (dx ? "+dx" : "") + (dw ? "+dw" : "") + (db ? "+db" : ""));
    return (M > 0 ? need(x && w && target && gloss && lse, "xent_bwd:x,w,target,gloss,lse") : 0) | need(ws, "xent_bwd:ws");
}

int launch_xent_scale(int, int64_t, int64_t, const void *kept, const float *gloss, int, void *dx, void *) {
    note("xent_scale");
    return need(kept && gloss && dx, "xent_scale:kept,gloss,dx");
}

}  // namespace ms
