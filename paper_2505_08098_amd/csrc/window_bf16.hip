// Forward of window attention, bf16 (see window.h).
#include "cross_few.h"
#include "window.h"

namespace f3s {

hipError_t launch_window_bf16(const f3s_window_plan_s &p, const FewArgs &a, hipStream_t s)
{
#define F3S_CALL(D) launch_window_d<D, kInBF16>(p, a, s)
    F3S_FOR_D(p.d, F3S_CALL)
#undef F3S_CALL
}

}  // namespace f3s
