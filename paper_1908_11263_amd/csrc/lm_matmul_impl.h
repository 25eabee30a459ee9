// The linear layer for one type of numbers and one width of weights.
#pragma once

#include "lm_matmul_rows.h"
#include "lm_matmul_tile.h"

namespace qnn_lm {

template <class N, int BITS>
hipError_t launch_matmul_one(const MatmulArgs &a, hipStream_t s)
{
    // the tile kernel's offsets within a tile are 32 bits
    const bool near = a.x_pitch < 1 << 23 && a.w_row < 1 << 23;
    return a.r > 64 && near ? launch_tile_bits<N, BITS>(a, s) : launch_rows_bits<N, BITS>(a, s);
}

}  // namespace qnn_lm
