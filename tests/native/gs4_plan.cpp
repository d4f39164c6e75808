// The plans of the group-scaled products, callable from a test: what a shape is launched with.
#include "../../paper_2111_00153_b200/csrc/gs4_plan.h"

using namespace rmsmp;

namespace {
Gs4Sizes sizes(int64_t R, int E, int M, int K, int group, int zero, int x_type, int experts, int in_order, int x_vec, int sms)
{
    const int sums = group % 128 == 0 ? 1 : group % 64 == 0 ? 2 : 4;
    return {R, E, (M + 31) / 32, (K + 127) / 128 * 128, sums, 2048 + 64 * sums + (zero ? 16 * sums : 0), x_type, experts != 0, in_order != 0, x_vec != 0, sms};
}
}  // namespace

#define SHAPE int64_t R, int E, int M, int K, int group, int zero, int x_type, int experts, int in_order, int x_vec, int sms
#define GIVEN R, E, M, K, group, zero, x_type, experts, in_order, x_vec, sms

extern "C" {

int gs4_is_many(SHAPE) { (void)M, (void)K, (void)group, (void)zero, (void)in_order, (void)x_vec, (void)sms; return gs4_many_tokens(R, E, x_type, experts != 0); }

void gs4_few(SHAPE, int64_t* out)
{
    const Gs4FewPlan p = gs4_plan_few(sizes(GIVEN));
    const int64_t all[] = {p.nt, p.wr, p.wk, p.split, p.per, p.groups, p.slice, p.slab, p.alone, p.single, p.tokens, p.parts, (int64_t)p.smem, p.grid};
    for (int i = 0; i < 14; ++i) out[i] = all[i];
}

void gs4_many(SHAPE, int64_t* out)
{
    const Gs4ManyPlan p = gs4_plan_many(sizes(GIVEN));
    const int64_t all[] = {p.bn, p.split, p.units, p.mtiles, p.ntiles};
    for (int i = 0; i < 5; ++i) out[i] = all[i];
}

}
