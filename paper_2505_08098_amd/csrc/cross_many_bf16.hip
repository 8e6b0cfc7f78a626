// Forward of cross attention for many query rows, bf16 (see many_rows.h).
#include "cross_few.h"
#include "many_rows.h"

namespace f3s {

hipError_t launch_cross_many_bf16(const f3s_cross_plan_s &p, const FewArgs &a, hipStream_t s)
{
#define F3S_CALL(D) launch_cross_many_d<D, kInBF16>(p, a, s)
    F3S_FOR_D(p.d, F3S_CALL)
#undef F3S_CALL
}

}  // namespace f3s
