// What the two block forms of linear attention share (wpp_linear_chunk.cu, wpp_linear_tc.cu).
#pragma once
#include "wpp_device.h"

namespace wpp {

// Logarithm of a token's decay, base 2.  One below -256 is taken for that: it leaves nothing of an fp32 state, and sums of logarithms stay
// finite.  A NaN stays one (fmaxf would take it for -256).
__device__ __forceinline__ float decay_log2(const LinearParams& p, int64_t token, int head) {
    const float x = p.log_decay[token * p.decay_token_stride + head] * 1.4426950408889634f;
    return x < -256.f ? -256.f : x;
}

// Whether one of the numbers is a NaN or an infinity: `zero` stays +0 while they are finite.
__device__ __forceinline__ void probe_bf16x2(uint32_t& zero, uint32_t x) { asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(zero) : "r"(x), "r"(0u)); }

}  // namespace wpp
