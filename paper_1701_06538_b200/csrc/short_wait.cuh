// For kernels whose waits are short and whose products are many and small: waits that do not look at the clock at once, products issued by a warp that stays together
#pragma once

#include "tc.cuh"

namespace moe {

namespace {

// As mbar_wait, which reads the clock as soon as its first try fails: here only after many tries
__device__ __forceinline__ bool short_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int32_t *status) {
    for (int i = 0; i < 64; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait(bar, parity, abort_flag, status);
}

// tc_mma_bf16, tc_mma2_bf16, tc_commit and tc_commit2 for all lanes of a warp together, one of which (always the same, so that a commit is of this warp's products) does it: the loop
// around them stays without branches of single lanes.
__device__ __forceinline__ void warp_mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p, q;\n elect.sync _|q, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void warp_mma2(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p, q;\n elect.sync _|q, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
        " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(0u)
        : "memory");
}
__device__ __forceinline__ void warp_commit(uint32_t bar) {
    asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void warp_commit2(uint32_t bar) {  // arrives at this offset in both CTAs of the pair
    asm volatile(
        "{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}"
        ::"r"(bar), "h"((uint16_t)3)
        : "memory");
}

}  // namespace

}  // namespace moe
