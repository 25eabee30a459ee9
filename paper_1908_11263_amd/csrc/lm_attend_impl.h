// Instances of the attention kernel for one type of queries.
#pragma once

#include "lm_attend_few.h"
#include "lm_attend_many.h"

namespace qnn_lm {

template <class Kernel>
void attend_lds(Kernel kernel, size_t lds, std::atomic<uint64_t> &devices)
{
    if (lds > 64 * 1024)
        qnn::allow_large_lds((const void *)kernel, devices);
}

template <class N, int BITS, int DIM, int NR>
hipError_t launch_few(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, hipStream_t s)
{
    constexpr size_t join = (4 * 16 * (DIM + 4) + 128) * sizeof(float);
    constexpr size_t stage = 4 * KvShape<BITS, DIM>::kWaveLds;
    constexpr size_t lds = join > stage ? join : stage;
    static std::atomic<uint64_t> devices{0};
    attend_lds(attend_kernel<N, BITS, DIM, NR>, lds, devices);
    hipLaunchKernelGGL((attend_kernel<N, BITS, DIM, NR>), dim3(p.row_tiles * p.splits, c.heads, c.b), dim3(256), lds, s,
                       a, c, p);
    return hipGetLastError();
}

template <class N, int BITS, int DIM, int NR>
hipError_t launch_many(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, hipStream_t s)
{
    constexpr size_t lds = 2 * ManyShape<BITS, DIM>::kBuffer;
    static std::atomic<uint64_t> devices{0};
    attend_lds(attend_many_kernel<N, BITS, DIM, NR>, lds, devices);
    const int64_t units = ((int64_t)p.splits * c.heads * c.b + 7) / 8 * 8;
    hipLaunchKernelGGL((attend_many_kernel<N, BITS, DIM, NR>), grid_of(units * p.row_tiles), dim3(256), lds, s, a, c, p);
    return hipGetLastError();
}

template <class N, int BITS, int DIM>
hipError_t launch_attend_dim(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, hipStream_t s)
{
    if (p.many) {
        if constexpr (DIM < 256)
            if (p.nr == 2)
                return launch_many<N, BITS, DIM, 2>(a, c, p, s);
        return launch_many<N, BITS, DIM, 1>(a, c, p, s);
    }
    if constexpr (DIM < 256)
        if (p.nr == 2)
            return launch_few<N, BITS, DIM, 2>(a, c, p, s);
    return launch_few<N, BITS, DIM, 1>(a, c, p, s);
}

template <class N, int BITS>
hipError_t launch_attend_bits(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int dim, hipStream_t s)
{
    switch (dim) {
    case 64: return launch_attend_dim<N, BITS, 64>(a, c, p, s);
    case 128: return launch_attend_dim<N, BITS, 128>(a, c, p, s);
    case 256: return launch_attend_dim<N, BITS, 256>(a, c, p, s);
    }
    return hipErrorInvalidValue;
}

template <class N>
hipError_t launch_attend_typed(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int bits, int dim,
                               hipStream_t s)
{
    switch (bits) {
    case 16: return launch_attend_bits<N, 16>(a, c, p, dim, s);
    case 8: return launch_attend_bits<N, 8>(a, c, p, dim, s);
    case 4: return launch_attend_bits<N, 4>(a, c, p, dim, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace qnn_lm
