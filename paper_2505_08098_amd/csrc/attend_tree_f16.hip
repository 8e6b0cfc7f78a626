// Attention over the 8-bit cache with a mask (tree), f16 queries (see attend_masked.h).
#include "attend_masked.h"
#include "cross_few.h"

namespace f3s {

hipError_t launch_attend_tree_f16(const AttendArgs &a, int d, hipStream_t s)
{
#define F3S_CALL(D) launch_attend_tree_d<D, kInF16>(a, s)
    F3S_FOR_D(d, F3S_CALL)
#undef F3S_CALL
}

}  // namespace f3s
