// KV append into a cache held in 4 bits.
//
// A row x (one token, KV head, K or V; d bf16 values) is kept as
//     least = min x (a least value of -0 as +0),  scale = bf16((max x - least) / 15),  code_e = round((x_e - least) / scale) in 0..15
// and stands for least + scale * code.  The quotient is the correctly rounded one and is rounded to even halves, so that the result
// is defined to the bit.  scale < 2^-100 (equal values, or nearly): scale and codes are 0.  A row with a NaN or an infinity, or
// whose extent is more than a float holds, has the quiet NaN 0x7fc0 as its least value, and scale and codes 0.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr float kLeastScale = 7.888609052210118e-31f;      // 2^-100

// The row of which this lane has 16 values, the kLanes lanes beside it the others: its codes (two words) and its number pair.
template <int kLanes>
__device__ __forceinline__ void kv4_row(const uint4 (&x)[2], uint2& codes, uint32_t& pair) {
    const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    float f[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    float lo = f[0], hi = f[0];
    bool nan = f[0] != f[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) {
        lo = fminf(lo, f[i]);
        hi = fmaxf(hi, f[i]);
        nan |= f[i] != f[i];
    }
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        nan |= __shfl_xor_sync(0xffffffffu, (int)nan, o) != 0;
    }
    lo += 0.f;
    const float extent = hi - lo;
    const bool fine = !nan && extent <= 3.402823466e+38f;
    float scale = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(extent, 15.f)));
    const bool zero = !fine || !(scale >= kLeastScale);
    if (zero) scale = 0.f;
    // The quotient d / scale from the correctly rounded reciprocal r: q = d r, then q + (d - q scale) r with fused operations is
    // the correctly rounded quotient (Markstein 1990).  d / scale <= 15.03 and scale >= 2^-100: nothing over- or underflows that
    // could reach the next integer's half.
    const float r = zero ? 0.f : __frcp_rn(scale);
    uint32_t c[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float d = f[i] - lo, q0 = d * r, q = fmaf(fmaf(-q0, scale, d), r, q0);
        // + 2^23: rounded to an integer, halves to even, which the low bits hold
        const uint32_t n = __float_as_uint(q + 8388608.f) & 15u;
        c[i >> 3] |= n << (4 * (i & 7));
    }
    codes = zero ? make_uint2(0u, 0u) : make_uint2(c[0], c[1]);
    pair = fine ? (__float_as_uint(lo) >> 16) | (__float_as_uint(scale) & 0xffff0000u) : 0x00007fc0u;
}

// D / 16 lanes take a row of K and the matching one of V.  A request whose span on the device is not the span the plan was made for
// is refused, as in wpp_append_kernel.
constexpr int kKv4AppendCtas = 4;          // per SM
template <int D>
__global__ void __launch_bounds__(256, kKv4AppendCtas) wpp_kv4_append_kernel(const Kv4AppendParams p) {
    constexpr int kLanes = D / 16, kRows = 32 / kLanes;       // rows of a warp
    grid_dependency_wait();
    grid_launch_dependents();
    const char* plan = static_cast<const char*>(p.plan);
    const int32_t* q_offsets = reinterpret_cast<const int32_t*>(plan + p.off_q_offsets);
    const int32_t* plan_prefix = reinterpret_cast<const int32_t*>(plan + p.off_prefix);
    const int lane = threadIdx.x & 31, sub = lane % kLanes;
    const int64_t total = p.total_new_tokens * p.num_kv_heads, stride = (int64_t)gridDim.x * (blockDim.x / 32) * kRows;
    for (int64_t first = ((int64_t)blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5)) * kRows; first < total; first += stride) {
        const int64_t tok0 = first / p.num_kv_heads;
        const int r = (int)(first - tok0 * p.num_kv_heads) + lane / kLanes, ahead = r / p.num_kv_heads, h = r - ahead * p.num_kv_heads;
        const bool there = first + lane / kLanes < total;
        const int tok = (int)tok0 + ahead;
        uint4 xk[2] = {}, xv[2] = {};
        if (there) {
            const int64_t src = (int64_t)tok * p.kvnew_token_stride + (int64_t)h * p.kvnew_head_stride + sub * 16;
            const uint4* k = reinterpret_cast<const uint4*>(p.k_new + src);
            const uint4* v = reinterpret_cast<const uint4*>(p.v_new + src);
            xk[0] = k[0]; xk[1] = k[1];
            xv[0] = v[0]; xv[1] = v[1];
        }
        int lo = 0, hi = p.num_requests;          // largest i with q_offsets[i] <= tok0
        while (hi - lo > 1) {
            const int width = (hi - lo + 31) / 32, i = lo + lane * width;
            const unsigned le = __ballot_sync(0xffffffffu, i < hi && q_offsets[i] <= tok0) | 1u;
            const int last = 31 - __clz((int)le);
            hi = min(hi, lo + (last + 1) * width);
            lo += last * width;
        }
        int64_t block = -1;                       // of the row's page and head, in bytes
        int slot = 0;
        if (there) {
            // (strides that double, then halve: empty requests may lie between)
            if (lo + 1 < p.num_requests && q_offsets[lo + 1] <= tok) {
                int width = 1;
                for (++lo; lo + width < p.num_requests && q_offsets[lo + width] <= tok; width *= 2) lo += width;
                while ((width /= 2) > 0)
                    if (lo + width < p.num_requests && q_offsets[lo + width] <= tok) lo += width;
            }
            const int P = p.prefix_lens[lo], from = q_offsets[lo];
            if (P != plan_prefix[lo] || p.chunk_lens[lo] != q_offsets[lo + 1] - from) {
                if (p.status) atomicCAS(p.status, 0, WPP_ERR_PLAN_MISMATCH);
            } else {
                const int pos = P + (tok - from), blk = pos / p.page_size;
                slot = pos - blk * p.page_size;
                const int page = blk < p.max_blocks ? p.block_tables[(int64_t)lo * p.max_blocks + blk] : -1;
                if (page < 0 || page >= p.num_pages) {
                    if (p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
                } else {
                    block = page * p.page_bytes + h * p.head_bytes;
                }
            }
        }
        uint2 ck, cv;
        uint32_t pk, pv;
        kv4_row<kLanes>(xk, ck, pk);
        kv4_row<kLanes>(xv, cv, pv);
        if (block < 0) continue;
        const int64_t codes = block + slot * (D / 2) + sub * 8, pairs = block + p.page_size * (D / 2) + slot * 4;
        *reinterpret_cast<uint2*>(p.k_cache + codes) = ck;
        *reinterpret_cast<uint2*>(p.v_cache + codes) = cv;
        if (sub == 0) *reinterpret_cast<uint32_t*>(p.k_cache + pairs) = pk;
        if (sub == 1) *reinterpret_cast<uint32_t*>(p.v_cache + pairs) = pv;
    }
}

}  // namespace wpp

extern "C" int wpp_launch_kv4_append(int head_dim, const wpp::Kv4AppendParams* p, int num_sms, void* stream) {
    const int64_t rows = p->total_new_tokens * p->num_kv_heads, per_block = 8 * (32 / (head_dim / 16));
    if (rows == 0) return 0;
    int64_t blocks = (rows + per_block - 1) / per_block;
    const int64_t cap = (int64_t)num_sms * wpp::kKv4AppendCtas;
    if (blocks > cap) blocks = cap;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(256);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return (int)cudaLaunchKernelEx(&cfg, head_dim == 128 ? wpp::wpp_kv4_append_kernel<128> : wpp::wpp_kv4_append_kernel<64>, *p);
}
