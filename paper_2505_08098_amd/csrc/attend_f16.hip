// Attention over the 8-bit cache, f16 queries (see few_rows.h, attend_many.h).
#include "attend_many.h"
#include "cross_few.h"

namespace f3s {

hipError_t launch_attend_f16(const AttendArgs &a, int d, hipStream_t s)
{
#define F3S_CALL(D) launch_attend_d<D, kInF16>(a, s)
    F3S_FOR_D(d, F3S_CALL)
#undef F3S_CALL
}

}  // namespace f3s
