// Time on the device, for the limits of waits.
#pragma once

#include <stdint.h>

namespace dendsn {

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// What a block does before it gives memory back after a wait has run out: 10 ms, thousands of
// times what a copy, a product or a store that is still on its way takes. At most 4096 naps of up
// to 0.2 ms.
__device__ __forceinline__ void let_land() {
    const uint64_t began = now_ns();
    for (int i = 0; i < 4096 && now_ns() - began < 10000000; ++i) __nanosleep(100000);
}

}  // namespace dendsn
