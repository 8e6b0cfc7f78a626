// Attention over the 8-bit cache, f16 queries (see few_rows.h).
#include "attend.h"

namespace f3s {

hipError_t launch_attend_f16(const AttendArgs &a, int d, hipStream_t s)
{
    return launch_attend_type<kInF16>(a, d, s);
}

}  // namespace f3s
