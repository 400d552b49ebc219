// KV append into a cache held in 4 bits.
//
// A row x (one token, KV head, K or V; d bf16 values) is kept as
//     least = min x (a least value of -0 as +0),  scale = bf16((max x - least) / 15),  code_e = round((x_e - least) / scale) in 0..15
// and stands for least + scale * code.  The quotient is the correctly rounded one and is rounded to even halves, so that the result
// is defined to the bit.  scale < 2^-100 (equal values, or nearly): scale and codes are 0.  A row with a NaN or an infinity, or
// whose extent is more than a float holds, has the quiet NaN 0x7fc0 as its least value, and scale and codes 0.
//
// A large grid is bound by instructions: 32 x 256..2,048 tokens of 8 heads of 128 take 49 us, a copy of the rows to the same addresses 33, the
// bytes at the measured copy bandwidth 29.  64 single tokens take 4.1 us, a launch and a chain of dependent loads.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr float kLeastScale = 7.888609052210118e-31f;      // 2^-100

// least and greatest that are NaN if one of the numbers is
__device__ __forceinline__ float min3_nan(float a, float b, float c) {
    float r;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min2_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max2_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// n / d rounded correctly, r being 1 / d rounded correctly: q = n r, then q + (n - q d) r with fused operations (Markstein 1990).  Nothing
// over- or underflows here that could reach a result: quotients are at most 15.03, divisors at least 2^-100, or the divisor is 15 and
// a quotient below 2^-100 counts as zero.
__device__ __forceinline__ float quotient(float n, float d, float r) {
    const float q = n * r;
    return fmaf(fmaf(-q, d, n), r, q);
}

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
    float lo = min2_nan(f[0], f[1]), hi = max2_nan(f[0], f[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) {
        lo = min3_nan(lo, f[i], f[i + 1]);
        hi = max3_nan(hi, f[i], f[i + 1]);
    }
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) {
        lo = min2_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max2_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    lo += 0.f;
    const float extent = hi - lo;
    const bool fine = extent <= 3.402823466e+38f;                      // (not if it is NaN)
    float scale = __bfloat162float(__float2bfloat16_rn(quotient(extent, 15.f, 1.f / 15.f)));
    const bool zero = !fine || !(scale >= kLeastScale);
    if (zero) scale = 0.f;
    const float r = zero ? 0.f : __frcp_rn(scale);
    const uint64_t least2 = pack2(-lo, -lo), r2 = pack2(r, r), minus2 = pack2(-scale, -scale), whole2 = pack2(8388608.f, 8388608.f);
    uint32_t c[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t n[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t d = fadd2(pack2(f[8 * half + 2 * i], f[8 * half + 2 * i + 1]), least2), q = fmul2(d, r2);
            // + 2^23: rounded to an integer, halves to even, which the low bits hold
            float a, b;
            unpack2(fadd2(ffma2(ffma2(q, minus2, d), r2, q), whole2), a, b);
            n[2 * i] = __float_as_uint(a);
            n[2 * i + 1] = __float_as_uint(b);
        }
        // (2^23 itself stands above them in every one: 4b000000, shifted by 0, 4, .. 28 and added up)
        uint32_t sum = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += n[i] << (4 * i);
        c[half] = sum - 0xfb000000u;
    }
    codes = zero ? make_uint2(0u, 0u) : make_uint2(c[0], c[1]);
    pair = fine ? (__float_as_uint(lo) >> 16) | (__float_as_uint(scale) & 0xffff0000u) : 0x00007fc0u;
}

// D / 16 lanes take a row of K and the matching one of V; a warp takes kUnroll such groups of rows behind one search for its first
// row's request, and asks for all their values first.  A request whose span on the device is not the span the plan was made for
// is refused, as in wpp_append_kernel.
constexpr int kKv4AppendCtas = 4;          // per SM
constexpr int kKv4AppendUnroll = 2;      // of a large grid (32 x 256..2,048 tokens: 1 51.4 us, 2 49.4, 4 with half the CTAs 55.5)
template <int D, int kUnroll>
__global__ void __launch_bounds__(256, kKv4AppendCtas) wpp_kv4_append_kernel(const Kv4AppendParams p) {
    constexpr int kLanes = D / 16, kRows = 32 / kLanes;       // rows of a warp at a time
    if (!p.few) grid_launch_dependents();
    grid_dependency_wait();
    const char* plan = static_cast<const char*>(p.plan);
    const int32_t* q_offsets = reinterpret_cast<const int32_t*>(plan + p.off_q_offsets);
    const int32_t* plan_prefix = reinterpret_cast<const int32_t*>(plan + p.off_prefix);
    const int lane = threadIdx.x & 31, sub = lane % kLanes, page_shift = 31 - __clz(p.page_size);
    const uint32_t heads = (uint32_t)p.num_kv_heads;
    const int64_t total = p.total_new_tokens * heads, stride = (int64_t)gridDim.x * (blockDim.x / 32) * (kRows * kUnroll);
    for (int64_t first = ((int64_t)blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5)) * (kRows * kUnroll); first < total; first += stride) {
        const int64_t tok0 = first >> 32 ? first / heads : (int64_t)((uint32_t)first / heads);      // (a 64-bit division takes seventy operations)
        const uint32_t rem0 = (uint32_t)(first - tok0 * heads) + lane / kLanes;
        uint4 xk[kUnroll][2] = {}, xv[kUnroll][2] = {};
        int tok[kUnroll];
        uint32_t h[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const uint32_t r = rem0 + u * kRows, ahead = r / heads;
            h[u] = r - ahead * heads;
            tok[u] = first + u * kRows + lane / kLanes < total ? (int)(tok0 + ahead) : -1;
            if (tok[u] < 0) continue;
            const int64_t src = (int64_t)tok[u] * p.kvnew_token_stride + (int64_t)h[u] * p.kvnew_head_stride + sub * 16;
            const uint4* k = reinterpret_cast<const uint4*>(p.k_new + src);
            const uint4* v = reinterpret_cast<const uint4*>(p.v_new + src);
            xk[u][0] = k[0]; xk[u][1] = k[1];
            xv[u][0] = v[0]; xv[u][1] = v[1];
        }
        int lo = 0, hi = p.num_requests;          // largest i with q_offsets[i] <= tok0
        while (hi - lo > 1) {
            const int width = (hi - lo + 31) / 32, i = lo + lane * width;
            const unsigned le = __ballot_sync(0xffffffffu, i < hi && q_offsets[i] <= tok0) | 1u;
            const int last = 31 - __clz((int)le);
            hi = min(hi, lo + (last + 1) * width);
            lo += last * width;
        }
        int P = 0, from = 0, next = -1;           // of request lo; next: its rows end here (-1: not looked at yet)
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            int64_t block = -1;                   // of the row's page and head, in bytes
            int slot = 0;
            if (tok[u] >= 0) {
                if (next < 0 || tok[u] >= next) {
                    // (strides that double, then halve: empty requests may lie between)
                    if (lo + 1 < p.num_requests && q_offsets[lo + 1] <= tok[u]) {
                        int width = 1;
                        for (++lo; lo + width < p.num_requests && q_offsets[lo + width] <= tok[u]; width *= 2) lo += width;
                        while ((width /= 2) > 0)
                            if (lo + width < p.num_requests && q_offsets[lo + width] <= tok[u]) lo += width;
                    }
                    P = p.prefix_lens[lo];
                    from = q_offsets[lo];
                    next = q_offsets[lo + 1];
                    if (P != plan_prefix[lo] || p.chunk_lens[lo] != next - from) {
                        if (p.status) atomicCAS(p.status, 0, WPP_ERR_PLAN_MISMATCH);
                        P = -1;
                    }
                }
                if (P >= 0) {
                    const int pos = P + (tok[u] - from), blk = pos >> page_shift;
                    slot = pos & (p.page_size - 1);
                    const int page = blk < p.max_blocks ? p.block_tables[(int64_t)lo * p.max_blocks + blk] : -1;
                    if (page < 0 || page >= p.num_pages) {
                        if (p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
                    } else {
                        block = page * p.page_bytes + h[u] * p.head_bytes;
                    }
                }
            }
            uint2 ck, cv;
            uint32_t pk, pv;
            kv4_row<kLanes>(xk[u], ck, pk);
            kv4_row<kLanes>(xv[u], cv, pv);
            if (block >= 0) {
                const int64_t codes = block + slot * (D / 2) + sub * 8, pairs = block + p.page_size * (D / 2) + slot * 4;
                *reinterpret_cast<uint2*>(p.k_cache + codes) = ck;
                *reinterpret_cast<uint2*>(p.v_cache + codes) = cv;
                if (sub == 0) *reinterpret_cast<uint32_t*>(p.k_cache + pairs) = pk;
                if (sub == 1) *reinterpret_cast<uint32_t*>(p.v_cache + pairs) = pv;
            }
        }
    }
}

}  // namespace wpp

extern "C" int wpp_launch_kv4_append(int head_dim, const wpp::Kv4AppendParams* p, int num_sms, void* stream) {
    const int64_t rows = p->total_new_tokens * p->num_kv_heads, per_block = 8 * (32 / (head_dim / 16));
    if (rows == 0) return 0;
    // a grid that the SMs hold at once is set up while the kernel before it runs and lets the one behind it in as its CTAs end; a
    // larger one lets it in once its last CTAs have started (see wpp_launch_append)
    const int64_t cap = (int64_t)num_sms * wpp::kKv4AppendCtas;
    wpp::Kv4AppendParams q = *p;
    q.few = rows <= cap * per_block;
    const int unroll = q.few ? 1 : wpp::kKv4AppendUnroll;
    int64_t blocks = (rows + per_block * unroll - 1) / (per_block * unroll);
    if (blocks > cap) blocks = cap;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(256);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = q.few ? 1 : 0;
    if (head_dim == 128)
        return (int)cudaLaunchKernelEx(&cfg, q.few ? wpp::wpp_kv4_append_kernel<128, 1> : wpp::wpp_kv4_append_kernel<128, wpp::kKv4AppendUnroll>, q);
    return (int)cudaLaunchKernelEx(&cfg, q.few ? wpp::wpp_kv4_append_kernel<64, 1> : wpp::wpp_kv4_append_kernel<64, wpp::kKv4AppendUnroll>, q);
}
