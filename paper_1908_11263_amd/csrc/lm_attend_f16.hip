// The attention kernel for f16 queries.
#include "lm_attend_impl.h"

namespace qnn_lm {

hipError_t launch_attend_f16(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int bits, int dim,
                              hipStream_t s)
{
    return launch_attend_typed<F16>(a, c, p, bits, dim, s);
}

}  // namespace qnn_lm
