// The linear layer for one type of numbers and one width of weights.
#pragma once

#include "lm_matmul_rows.h"
#include "lm_matmul_tile.h"

namespace qnn_lm {

template <class N, int BITS>
hipError_t launch_matmul_one(const MatmulArgs &a, void *ws, hipStream_t s)
{
    const TilePlan p = plan_matmul(a, BITS);
    return p.tf ? launch_tile_bits<N, BITS>(a, p, ws, s) : launch_rows_bits<N, BITS>(a, s);
}

}  // namespace qnn_lm
