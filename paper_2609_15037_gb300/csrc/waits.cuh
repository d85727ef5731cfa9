// What the tensor-core kernels do when a bounded wait runs out: wait, with the default
// bound, for their own work in flight.
#pragma once

#include "tc_ptx.cuh"

namespace moara {

constexpr long long kWaitLimit = 1LL << 32;   // ~2 s of SM clocks

__device__ __forceinline__ bool wait_drain(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!ptx::mbar_try_wait(bar, parity)) {
        if (clock64() - t0 > kWaitLimit) return false;
    }
    return true;
}

// A pair whose waits may run out while copies are in flight (a wait limit below
// a copy's latency).  A copy of either CTA completes on the even CTA's barrier,
// and a stage's phase ends when both CTAs' copies have landed; the two producers
// may have given up a different number of stages in.
//
// pair_abort, by every warp before the last cluster barrier: if its CTA gave up,
// the peer knows behind that barrier.  pair_settle, by one thread of each CTA
// behind it: the CTA that filled fewer stages fills the missing ones (the MMAs
// are done, what lands there is not used), and the even CTA waits for every
// stage's last phase.  Another cluster barrier, and no copy is left in flight.
template <class Ctl> __device__ __forceinline__ void pair_abort(Ctl* ctl, int crank) {
    if ((threadIdx.x & 31) == 0 && *const_cast<volatile int*>(&ctl->abort) != 0)
        ptx::st_cluster_u32(ptx::mapa(ptx::smem_u32(&ctl->abort), crank ^ 1), 1);
}

template <int STAGES, class Ctl, class Fill>
__device__ __forceinline__ void pair_settle(Ctl* ctl, int crank, Fill fill) {
    const uint32_t own = ctl->steps, peer = ptx::ld_cluster_u32(ptx::mapa(ptx::smem_u32(&ctl->steps), crank ^ 1));
    const uint32_t all = own > peer ? own : peer;
    for (uint32_t k = own; k < all; ++k) fill(static_cast<int>(k), static_cast<int>(k % STAGES));
    if (crank == 0)
        for (uint32_t q = 0; q < STAGES && q < all; ++q)
            wait_drain(ptx::smem_u32(&ctl->full[q]), ((all - 1 - q) / STAGES) & 1);
}

}  // namespace moara
