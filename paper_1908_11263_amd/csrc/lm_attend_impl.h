// Instances of the attention kernel for one type of queries.
#pragma once

#include "lm_attend.h"
#include "qnn_internal.h"

namespace qnn_lm {

template <class N, int BITS, int DIM, int NR>
hipError_t launch_attend_one(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, hipStream_t s)
{
    constexpr size_t join = (4 * 16 * (DIM + 4) + 128) * sizeof(float);
    constexpr size_t stage = 4 * KvShape<BITS, DIM>::kWaveLds;
    constexpr size_t lds = join > stage ? join : stage;
    const void *kernel = (const void *)attend_kernel<N, BITS, DIM, NR>;
    if constexpr (lds > 64 * 1024) {
        static std::atomic<uint64_t> devices{0};
        qnn::allow_large_lds(kernel, devices);
    }
    hipLaunchKernelGGL((attend_kernel<N, BITS, DIM, NR>), dim3(p.row_tiles * p.splits, c.heads, c.b), dim3(256), lds, s,
                       a, c, p);
    return hipGetLastError();
}

template <class N, int BITS, int DIM>
hipError_t launch_attend_dim(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int nr, hipStream_t s)
{
    switch (nr) {
    case 1: return launch_attend_one<N, BITS, DIM, 1>(a, c, p, s);
    case 2: return launch_attend_one<N, BITS, DIM, 2>(a, c, p, s);
    case 4:
        if constexpr (DIM <= 128)
            return launch_attend_one<N, BITS, DIM, 4>(a, c, p, s);
    }
    return hipErrorInvalidValue;
}

template <class N, int BITS>
hipError_t launch_attend_bits(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int dim, int nr, hipStream_t s)
{
    switch (dim) {
    case 64: return launch_attend_dim<N, BITS, 64>(a, c, p, nr, s);
    case 128: return launch_attend_dim<N, BITS, 128>(a, c, p, nr, s);
    case 256: return launch_attend_dim<N, BITS, 256>(a, c, p, nr, s);
    }
    return hipErrorInvalidValue;
}

template <class N>
hipError_t launch_attend_typed(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int bits, int dim, int nr,
                               hipStream_t s)
{
    switch (bits) {
    case 16: return launch_attend_bits<N, 16>(a, c, p, dim, nr, s);
    case 8: return launch_attend_bits<N, 8>(a, c, p, dim, nr, s);
    case 4: return launch_attend_bits<N, 4>(a, c, p, dim, nr, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace qnn_lm
