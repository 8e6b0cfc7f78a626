// Backward of cross attention, bf16 (see cross_backward.h).
#include "cross_backward.h"
#include "cross_few.h"

namespace f3s {

hipError_t launch_cross_backward_bf16(const f3s_cross_plan_s &p, const CrossBwdArgs &a,
                                     hipStream_t s)
{
#define F3S_CALL(D) launch_cross_backward_d<D, kInBF16>(p, a, s)
    F3S_FOR_D(p.d, F3S_CALL)
#undef F3S_CALL
}

}  // namespace f3s
