// overlap.h for host tests, and attention's backward with a launcher that notes whether it was told to
// write its gradients after the last read.
#include "../../paper_2404_12406_amd/csrc/overlap.h"

#define launch_attention_bwd stub_launch_attention_bwd
#include "attention_stub.cpp"
#undef launch_attention_bwd

namespace {
int g_shared = -1;
}

namespace ms {
int launch_attention_bwd(int dtype, const AttnArgs &a, void *ws, void *stream) {
    g_shared = a.shared;
    return stub_launch_attention_bwd(dtype, a, ws, stream);
}
}  // namespace ms

extern "C" {
int overlap_shared(const ms_tensor *a, const ms_tensor *b) { return (int)ms::rt::shared(a, b); }
int overlap_noted() { return g_shared; }
}
