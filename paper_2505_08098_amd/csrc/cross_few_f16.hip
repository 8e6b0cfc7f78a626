// Cross attention of few query rows, f16 (see few_rows.h).
#include "cross_few.h"

namespace f3s {

hipError_t launch_cross_few_f16(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s)
{
#define F3S_CALL(D) launch_cross_few_d<D, kInF16>(p, a, s)
    F3S_FOR_D(p.d, F3S_CALL)
#undef F3S_CALL
}

hipError_t launch_cross_merge_f16(const f3s_cross_plan_s &p, const CrossMergeArgs &a,
                                  hipStream_t s)
{
#define F3S_CALL(D) launch_cross_merge_d<D, kInF16>(p, a, s)
    F3S_FOR_D(p.d, F3S_CALL)
#undef F3S_CALL
}

}  // namespace f3s
