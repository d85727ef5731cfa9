// After a wait of k_fp4_few ran out: its copies in flight.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

namespace moara {

// Every stage's last copies are waited for.  A phase of a stage ends with the producer's
// copies and one arrival of each of WARPS warps; a warp that filled fewer stages than the producer
// (by no more than there are stages) owes the arrivals, which arrive(stage) makes up for;
// wait(stage, parity) waits for the phase.
template <int WARPS, class Arrive, class Wait>
__host__ __device__ void settle_few(int copied, const int* filled, int stages, Arrive arrive, Wait wait) {
    for (int w = 0; w < WARPS; ++w)
        for (int k = filled[w]; k < copied; ++k) arrive(k % stages);
    for (int s = 0; s < stages && s < copied; ++s) wait(s, static_cast<uint32_t>((copied - 1 - s) / stages) & 1u);
}

}  // namespace moara
