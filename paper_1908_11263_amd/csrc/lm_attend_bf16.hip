// The attention kernel for bf16 queries.
#include "lm_attend_impl.h"

namespace qnn_lm {

hipError_t launch_attend_bf16(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int bits, int dim,
                              hipStream_t s)
{
    return launch_attend_typed<Bf16>(a, c, p, bits, dim, s);
}

}  // namespace qnn_lm
