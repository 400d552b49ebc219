// KV append into a cache held in 8 bits with a scale per page and head.
//
// The rows that a request's chunk has in one page (K or V of one head) share a scale: the least power of two 2^e with which their largest
// finite value is within 448, but no less than the scale of prefix rows that stand in the page.  A code is x / 2^e rounded to e4m3; the
// division is a product with 2^-e, exact (what it would make a subnormal number is far below the least code).  Where the scale
// of standing rows rises by 2^n, their codes are taken down by 2^n.
//
// A (touched page, head, K or V) is a CTA, of as many warps as the page has 16 slots, each of which holds its rows in registers
// between the search for the largest value and the conversion: the rows are read once.  The plan lists the touched pages, so that a CTA
// knows its rows after one load, and asks for rows, lengths and page id at once.
//
// 38,839 tokens of 8 heads of 128 take 44 to 45 us, 5.3 TB/s (the bytes at the measured copy rate 37); with 8 warps in every CTA 3 more, with a record
// that leads to the rows over the plan's offsets 1.  64 single tokens 3.3 us, the launch and a chain of two loads; over the plan's
// offsets 3.6, found by bisection over the requests 7.2.
#include <cuda_runtime.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_kv8.cuh"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace wpp {

__device__ __forceinline__ uint32_t abs_max(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7fff7fffu); }

// the exponent of the least scale for values of which `top` (bf16 bits, finite) is the largest: 448 = 1.75 * 2^8
__device__ __forceinline__ int scale_exponent(uint32_t top) {
    const int e = (int)(top >> 7) - 135 + ((top & 0x7fu) > 0x60u);
    return top == 0u ? kKv8LeastExp : min(max(e, kKv8LeastExp), kKv8MostExp);
}

template <int D>
__global__ void __launch_bounds__(256) wpp_kv8_append_kernel(const Kv4AppendParams p) {
    constexpr int kVecs = D / 8, kTurns = 16 * kVecs / 32, kApart = 32 / kVecs;      // 16-byte vectors of a row; of a lane; rows between them
    __shared__ uint32_t s_top[8];
    if (!p.few) grid_launch_dependents();
    grid_dependency_wait();
    const char* plan = static_cast<const char*>(p.plan);
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, page_shift = 31 - __clz(p.page_size), parts = p.page_size / 16;      // warps; which this is
    const uint32_t heads = (uint32_t)p.num_kv_heads, pair = blockIdx.x / heads, head = blockIdx.x - pair * heads;
    const bool is_v = (pair & 1u) != 0u;
    // ---- the rows, from the plan: slots [slot0, slot1) of the page; those before slot0 stand
    const int2 page_of = reinterpret_cast<const int2*>(plan + p.off_touched)[pair >> 1], rows = reinterpret_cast<const int2*>(plan + p.off_touched)[p.num_touched + (pair >> 1)];
    const WppTouched at = {page_of.x, page_of.y};
    const int slot0 = (int16_t)rows.y, slot1 = rows.y >> 16, stand = slot0;
    const int32_t* q_offsets = reinterpret_cast<const int32_t*>(plan + p.off_q_offsets) + at.request;
    const int P = reinterpret_cast<const int32_t*>(plan + p.off_prefix)[at.request], C = q_offsets[1] - q_offsets[0];
    const int P_now = p.prefix_lens[at.request], C_now = p.chunk_lens[at.request];
    const int page = at.block < p.max_blocks ? p.block_tables[(int64_t)at.request * p.max_blocks + at.block] : -1;

    // ---- the warp's rows, and the largest finite value of the CTA's
    const int col = lane % kVecs, row = 16 * part + lane / kVecs;      // rows row, row + kApart, ..
    const __nv_bfloat16* src = (is_v ? p.v_new : p.k_new) + (int64_t)head * p.kvnew_head_stride + col * 8;
    uint4 x[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int slot = row + i * kApart;
        x[i] = make_uint4(0, 0, 0, 0);
        if (slot >= slot0 && slot < slot1) x[i] = *reinterpret_cast<const uint4*>(src + (int64_t)(rows.x + slot) * p.kvnew_token_stride);
    }
    uint8_t* block = nullptr;
    if (P_now != P || C_now != C) {
        if (lane == 0 && p.status) atomicCAS(p.status, 0, WPP_ERR_PLAN_MISMATCH);
    } else if (page < 0 || page >= p.num_pages) {
        if (lane == 0 && p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
    } else {
        block = (is_v ? p.v_cache : p.k_cache) + page * p.page_bytes + head * p.head_bytes;
    }
    float* const scale_at = reinterpret_cast<float*>(block + (D << page_shift));
    int e_old = kKv8LeastExp;
    if (block && stand > 0) e_old = min(max(exponent_of(*scale_at), kKv8LeastExp), kKv8MostExp);
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) m = abs_max(abs_max(abs_max(abs_max(m, x[i].x), x[i].y), x[i].z), x[i].w);
    uint32_t top = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
    const bool odd = top >= 0x7f80u;          // a NaN or an infinity is among them: the largest of the others
    if (odd) {
        m = 0u;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = w[j] & 0x7fffu, b = w[j] >> 16 & 0x7fffu;
                m = max(m, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
            }
        }
        top = __reduce_max_sync(0xffffffffu, m);
    }
    if (parts > 1) {
        if (lane == 0) s_top[part] = top;
        __syncthreads();                      // (every warp has read the standing scale before one of them replaces it, too)
        for (int i = 0; i < parts; ++i) top = max(top, s_top[i]);
    }
    if (!block) return;
    const int e = max(scale_exponent(top), e_old);
    __syncwarp();                             // (so has every lane of a CTA of one warp)
    if (part == 0 && lane == 0 && (stand == 0 || e != e_old)) *scale_at = power_of_two(e);

    // ---- codes
    const float inverse = power_of_two(-e);
    uint8_t* const dst = block + col * 8;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int slot = row + i * kApart;
        if (slot < slot0 || slot >= slot1) continue;
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        uint32_t c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float a = __uint_as_float(w[j] << 16), b = __uint_as_float(w[j] & 0xffff0000u);
            if (odd) {                        // (an infinity would be rounded to 448)
                a = (w[j] & 0x7f80u) == 0x7f80u ? __uint_as_float(0x7fffffffu) : a;
                b = (w[j] & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fffffffu) : b;
            }
            c[j] = codes_of(a * inverse, b * inverse);
        }
        *reinterpret_cast<uint2*>(dst + slot * D) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
    }
    if (stand > 0 && e != e_old) {
        const float down = power_of_two(e_old - e);
#pragma unroll 1
        for (int slot = row; slot < min(stand, 16 * part + 16); slot += kApart) {
            const uint2 old = *reinterpret_cast<const uint2*>(dst + slot * D);
            const uint32_t f[4] = {codes_f16x2_low(old.x), codes_f16x2_high(old.x), codes_f16x2_low(old.y), codes_f16x2_high(old.y)};
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = codes_of(f16_low(f[j]) * down, f16_high(f[j]) * down);
            *reinterpret_cast<uint2*>(dst + slot * D) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
        }
    }
}

}  // namespace wpp

extern "C" int wpp_launch_kv8_append(int head_dim, const wpp::Kv4AppendParams* p, int num_sms, void* stream) {
    if (p->total_new_tokens == 0) return 0;
    const int64_t blocks = (int64_t)p->num_touched * 2 * p->num_kv_heads;
    const int warps = p->page_size / 16;
    if (blocks > 0x7fffffff) return (int)cudaErrorInvalidValue;
    wpp::Kv4AppendParams q = *p;
    q.few = blocks * warps <= 32 * (int64_t)num_sms;      // (see wpp_launch_kv4_append)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)(32 * warps));
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = q.few ? 1 : 0;
    return (int)cudaLaunchKernelEx(&cfg, head_dim == 128 ? wpp::wpp_kv8_append_kernel<128> : wpp::wpp_kv8_append_kernel<64>, q);
}
