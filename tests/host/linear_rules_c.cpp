// The rules of linear_rules.h for ctypes.
#include "linear_rules.h"

extern "C" void plan_of_product(const size_t* shape, const int* flags, size_t* out)
{
    const mics::ProductShape s{shape[0], shape[1], shape[2], shape[3], flags[0] != 0, flags[1] != 0, flags[2] != 0, flags[3] != 0,
                               flags[4] != 0, flags[5] != 0};
    const mics::ProductPlan p = mics::plan_product(s);
    const size_t v[] = {(size_t)p.few, p.bm, p.bn, p.whole, p.shared, p.splits, p.depth, p.a_copy, p.b_copy, mics::workspace_of(p),
                        mics::most_workspace(s.m, s.n, s.k, s.a_turned, s.b_turned)};
    for (int i = 0; i < 11; ++i) out[i] = v[i];
}
