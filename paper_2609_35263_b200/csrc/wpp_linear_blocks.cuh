// What the forms of linear attention share (wpp_linear.cu, wpp_linear_chunk.cu, wpp_linear_tc.cu).
#pragma once
#include "wpp_device.h"

namespace wpp {

// Slot of the pool that holds a state, or -1; a slot id outside the pool is reported and taken for -1.
__device__ __forceinline__ int64_t linear_slot(const LinearParams& p, int slot) {
    if (slot >= -1 && slot < p.num_slots) return slot;
    if (p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
    return -1;
}

// The request and segment of number `index` in the second pass, where request r's are numbered from row_offsets[r] / seg_tokens + r on;
// in the first pass, where all but the last ones of a chain count, from row_offsets[r] / seg_tokens on.  A warp finds it together.
struct LinearSegment {
    int req;
    int64_t row0, tokens;              // of the request
    int64_t index0, seg, segs;         // number of its first segment in the first pass; this one of them, and how many there are
    bool work;                         // false: no such segment, another form's, or (first pass) a last one, whose state is nobody's before
};
template <bool kFirst>
__device__ __forceinline__ LinearSegment linear_segment(const LinearChunkParams& p, int64_t index) {
    LinearSegment s;
    const int lane = threadIdx.x & 31;
    s.req = 0;
    int hi = p.num_requests;
    while (hi - s.req > 1) {
        const int width = (hi - s.req + 31) / 32, i = s.req + lane * width;
        const unsigned le = __ballot_sync(0xffffffffu, i < hi && p.row_offsets[i] / p.seg_tokens + (kFirst ? 0 : i) <= index) | 1u;
        const int last = 31 - __clz((int)le);
        hi = min(hi, s.req + (last + 1) * width);
        s.req += last * width;
    }
    s.row0 = p.row_offsets[s.req];
    s.tokens = p.row_offsets[s.req + 1] - s.row0;
    s.index0 = s.row0 / p.seg_tokens;
    s.seg = index - s.index0 - (kFirst ? 0 : s.req);
    s.segs = s.tokens > 0 ? (s.tokens + p.seg_tokens - 1) / p.seg_tokens : 1;
    s.work = s.tokens > p.few_tokens && s.seg < s.segs && !(kFirst && s.seg == s.segs - 1);
    return s;
}

// Logarithm of a token's decay, base 2.  One below -256 is taken for that: it leaves nothing of an fp32 state, and sums of logarithms stay
// finite.  A NaN stays one (fmaxf would take it for -256).
__device__ __forceinline__ float decay_log2(const LinearParams& p, int64_t token, int head) {
    const float x = p.log_decay[token * p.decay_token_stride + head] * 1.4426950408889634f;
    return x < -256.f ? -256.f : x;
}

// Whether one of the numbers is a NaN or an infinity: `zero` stays +0 while they are finite.
__device__ __forceinline__ void probe_bf16x2(uint32_t& zero, uint32_t x) { asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(zero) : "r"(x), "r"(0u)); }

}  // namespace wpp
