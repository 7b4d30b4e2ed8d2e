// Bounded waits on mbarriers and the driver's tensor-map encoder: what every TMA kernel of the library shares.
#pragma once

#include <atomic>

#include "dybit_common.cuh"
#include "dybit_sm100.cuh"

namespace dybit {

using namespace sm100;

constexpr unsigned long long kWaitLimitNs = 4000000000ull;

// Waits for the phase with the given parity; gives up after `limit_ns` (kWaitLimitNs in every kernel of the
// library), records the site in the device status word and raises the CTA-wide abort flag.
__device__ __forceinline__ bool wait_bounded(uint64_t *bar, uint32_t parity, volatile uint32_t *abort_flag,
                                             unsigned site, unsigned long long limit_ns = kWaitLimitNs) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    unsigned spins = 0;
    for (;;) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((++spins & 63u) == 0u) {
            if (*abort_flag) return false;
            if (global_timer_ns() - t0 > limit_ns) {
                atomicOr(&g_device_status, (site << 8) | 1u);
                *abort_flag = 1u;
                return false;
            }
        }
    }
}

// The same wait for the MMA-issuing thread: the barrier is named by its shared-memory address and only the first
// probe is inlined, so the common case (the stage is there already) costs three instructions.
static __device__ __noinline__ bool wait_bounded_slow(uint32_t bar_addr, uint32_t parity, volatile uint32_t *abort_flag, unsigned site) {
    const uint64_t t0 = global_timer_ns();
    unsigned spins = 0;
    for (;;) {
        if (mbar_try_wait_addr(bar_addr, parity)) return true;
        if ((++spins & 63u) == 0u) {
            if (*abort_flag) return false;
            if (global_timer_ns() - t0 > kWaitLimitNs) {
                atomicOr(&g_device_status, (site << 8) | 1u);
                *abort_flag = 1u;
                return false;
            }
        }
    }
}

__device__ __forceinline__ bool wait_bounded_addr(uint32_t bar_addr, uint32_t parity, volatile uint32_t *abort_flag,
                                                  unsigned site) {
    if (mbar_try_wait_addr(bar_addr, parity)) return true;
    return wait_bounded_slow(bar_addr, parity, abort_flag, site);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiledFn encode_tiled_fn() {
    static std::atomic<EncodeTiledFn> fn{nullptr};
    EncodeTiledFn f = fn.load(std::memory_order_acquire);
    if (f == nullptr) {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess) {
            f = reinterpret_cast<EncodeTiledFn>(ptr);
            fn.store(f, std::memory_order_release);
        } else {
            (void)cudaGetLastError();
        }
    }
    return f;
}

}  // namespace dybit
