// Stub launchers of attention and its cache for host-only tests of their entry points
// (attention.cpp), beside host_stub.cpp: each checks that it was handed every pointer that
// its kernels would read or write, in the layout they need, notes the call and launches nothing.
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

int need(bool ok, const std::string &what) {
    if (ok) return 0;
    std::lock_guard<std::mutex> lk(g_mu);
    g_violation += what + ";";
    return 77;
}

// rows and heads that start at whole 16-byte vectors
int whole(int dtype, const ms::HeadsView &v, int64_t rows, int heads, int D, const std::string &what) {
    if (rows == 0) return 0;
    const int64_t e = dtype == ms::kBF16 ? 2 : 4;
    return need(v.p && reinterpret_cast<uintptr_t>(v.p) % 16 == 0, what + ":pointer") |
           need(v.ts * e % 16 == 0 && v.ts >= D && v.ts * e <= (int64_t(1) << 24), what + ":rows") |
           need(heads <= 1 || v.hs * e % 16 == 0, what + ":heads") | need(D * e % 16 == 0, what + ":D");
}
}  // namespace

extern "C" {
const char *attention_log() { return g_log.c_str(); }
const char *attention_violations() { return g_violation.c_str(); }
void attention_reset() {
    std::lock_guard<std::mutex> lk(g_mu);
    g_log.clear();
    g_violation.clear();
}
}

namespace ms {

int launch_rotary_fwd(int, const RotaryArgs &a, bool append, void *) {
    note(append ? "append" : "rotary");
    if (a.T == 0 || a.Hq + a.Hk == 0) return 0;
    int e = need(a.x, "rotary:x") | need(a.R == 0 || (a.freq && a.pos), "rotary:positions");
    if (append) return e | need(a.pos && (a.pages == 0 || (a.kp && a.vp)) && (a.y || a.Hq == 0), "append:pointers");
    return e | need(a.y, "rotary:y");
}

size_t rotary_bwd_workspace(int, const RotaryArgs &a, bool params) { return params ? (size_t)a.D * 8 * 4 : 0; }

int launch_rotary_bwd(int, const RotaryArgs &a, const void *dy, const int64_t *, void *dx, const int64_t *, void *dgq, void *dgk, void *ws,
                      void *) {
    note(std::string("rotary_bwd") + (dx ? "+dx" : "") + (dgq ? "+dgq" : "") + (dgk ? "+dgk" : ""));
    int e = need(!(dgq || dgk) || ws, "rotary_bwd:ws");
    if (a.T == 0 || a.Hq + a.Hk == 0) return e;
    return e | need(dy, "rotary_bwd:dy") | need(!a.norm || a.x, "rotary_bwd:x") | need(a.R == 0 || (a.freq && a.pos), "rotary_bwd:positions");
}

size_t attention_fwd_workspace(int, const AttnArgs &) { return 256; }

int launch_attention_fwd(int dtype, const AttnArgs &a, void *ws, void *) {
    note(a.lse ? "attention+lse" : "attention");
    return whole(dtype, a.q, a.Tq, a.Hq, a.D, "q") | whole(dtype, a.k, a.Tk, a.Hk, a.D, "k") | whole(dtype, a.v, a.Tk, a.Hk, a.D, "v") |
           whole(dtype, a.o, a.Tq, a.Hq, a.D, "o") | need(ws, "attention:ws") | need(!a.qoff == !a.koff, "attention:offsets");
}

size_t attention_bwd_workspace(int, const AttnArgs &, bool, bool, bool) { return 512; }

int launch_attention_bwd(int dtype, const AttnArgs &a, void *ws, void *) {
    const bool dq = a.dq.p, dk = a.dk.p, dv = a.dv.p;
    note(std::string("attention_bwd") + (dq ? "+dq" : "") + (dk ? "+dk" : "") + (dv ? "+dv" : ""));
    int e = whole(dtype, a.q, a.Tq, a.Hq, a.D, "q") | whole(dtype, a.k, a.Tk, a.Hk, a.D, "k") | whole(dtype, a.go, a.Tq, a.Hq, a.D, "go") |
            need(ws, "attention_bwd:ws") | need(a.lse || a.Tq == 0, "attention_bwd:lse") | need(!a.qoff == !a.koff, "attention_bwd:offsets");
    if (dq || dk) e |= whole(dtype, a.v, a.Tk, a.Hk, a.D, "v") | whole(dtype, a.o, a.Tq, a.Hq, a.D, "o");
    if (dq) e |= whole(dtype, a.dq, a.Tq, a.Hq, a.D, "dq");
    if (dk) e |= whole(dtype, a.dk, a.Tk, a.Hk, a.D, "dk");
    if (dv) e |= whole(dtype, a.dv, a.Tk, a.Hk, a.D, "dv");
    return e;
}

int launch_pack_heads(int, const void *src, int64_t, int64_t, int64_t, int64_t, int, int D, void *dst, int Dp, void *) {
    note("pack");
    return need(src && dst && Dp >= D, "pack:pointers");
}

int64_t paged_blocks(const PagedArgs &a) { return (int64_t)a.n * a.Hk; }
size_t paged_workspace(int, const PagedArgs &) { return 256; }

int launch_paged(int dtype, const PagedArgs &a, void *ws, void *) {
    note("paged");
    const int D = dtype == kBF16 ? (a.D + 7) / 8 * 8 : (a.D + 3) / 4 * 4;
    return whole(dtype, {const_cast<void *>(a.q), a.qts, a.qhs}, a.n, a.Hq, D, "paged:q") |
           need(a.n == 0 || (a.o && a.lengths), "paged:o,lengths") | need(a.width == 0 || a.n == 0 || a.tables, "paged:tables") |
           need(ws, "paged:ws");
}

}  // namespace ms
