// The plan of a paged attention for host tests.
#include "../../paper_2404_12406_amd/csrc/paged_plan.h"

extern "C" void paged_plan(int n, int Hq, int Hk, int page, int width, int64_t *out) {
    ms::PagedArgs a{};
    a.n = n;
    a.Hq = Hq;
    a.Hk = Hk;
    a.page = page;
    a.width = width;
    const ms::att::PagedPlan p = ms::att::paged_plan(a);
    out[0] = p.splits;
    out[1] = p.per;
}
