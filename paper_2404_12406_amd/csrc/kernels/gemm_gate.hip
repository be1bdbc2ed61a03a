// The gated linear unit's bf16 contractions (gemm_fused.h).
#include "gemm_fused.h"

namespace ms {
namespace g2 {

namespace {
bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <int EPI>
int go_act(int act, int tile, const FusedArgs &a, hipStream_t st) {
    switch (act) {
    case kActSilu: return go_rows<EPI, kActSilu>(tile, kProfFwd, a, st);
    case kActGelu: return go_rows<EPI, kActGelu>(tile, kProfFwd, a, st);
    case kActGeluTanh: return go_rows<EPI, kActGeluTanh>(tile, kProfFwd, a, st);
    case kActRelu: return go_rows<EPI, kActRelu>(tile, kProfFwd, a, st);
    default: return go_rows<EPI, kActSigmoid>(tile, kProfFwd, a, st);
    }
}
}  // namespace

// Operands: D a multiple of 8, x and w 16-byte aligned, the bias 4-byte aligned.
bool rows_ok(int64_t M, int64_t N, int64_t D, const void *x, const void *w) {
    return D % 8 == 0 && al16(x) && al16(w) && operand_fits(M * D) && operand_fits(N * D);
}

int gate_fwd(int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *bias, void *y, void *proj,
             hipStream_t st) {
    const FusedPlan p = plan(kRowTiles, 3, M, 2 * F, D, 1);
    const Tile &t = kRowTiles[p.tile];
    FusedArgs a = rows_args(t, M, 2 * F, D, x, w, 2 * F);
    a.ntn = (int)((F + t.bn / 2 - 1) / (t.bn / 2));
    a.F = (int)F;
    a.fbias = (const bf16 *)bias;
    a.c = (bf16 *)y;
    a.proj = (uint16_t *)proj;
    a.proj_lo = proj ? static_cast<uint8_t *>(proj) + M * 4 * F : nullptr;
    return go_act<kEpiGate>(act, p.tile, a, st);
}

int gate_grad(int64_t M, int64_t D, int64_t F, int act, const void *x, const void *w, const void *bias, const void *dy, void *dz,
              hipStream_t st) {
    const FusedPlan p = plan(kRowTiles, 3, M, 2 * F, D, 1);
    const Tile &t = kRowTiles[p.tile];
    FusedArgs a = rows_args(t, M, 2 * F, D, x, w, 2 * F);
    a.ntn = (int)((F + t.bn / 2 - 1) / (t.bn / 2));
    a.F = (int)F;
    a.fbias = (const bf16 *)bias;
    a.dh = (const bf16 *)dy;
    a.c = (bf16 *)dz;
    return go_act<kEpiGateGrad>(act, p.tile, a, st);
}

}  // namespace g2
}  // namespace ms
