// Linear attention with a decay per head, token by token:  S_t = e^(g_t) S_(t-1) + k_t v_t^T,  o_t = scale S_t^T q_t.
//
// One CTA has kCols columns of a (request, head)'s state in registers: kCols / 4 lanes hold a row's columns, four each, the CTA's 256
// threads rows kRowsAtOnce apart.  For a chunk of one token the state's bytes bound it, read once and written once; all of a
// thread's rows are asked for before the first is used.  Outputs are sums over the rows, of a lane's own first, then over the
// threads with the same columns by shuffles and shared memory.  64 requests of one token, 32 heads of 128: 45 us, 6.0 TB/s (92 % of the
// measured copy); with fewer than two chains per SM a CTA takes 32 columns, for the latency.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_linear_blocks.cuh"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr int kLinThreads = 256;

template <int D, int kCols>
__global__ void __launch_bounds__(kLinThreads) wpp_linear_token_kernel(const LinearParams p) {
    constexpr int kLanes = kCols / 4, kRowsAtOnce = kLinThreads / kLanes, kRows = D / kRowsAtOnce, kWarps = kLinThreads / 32;
    __shared__ float s_q[D], s_k[D];
    __shared__ float4 s_o[kWarps][kLanes];
    grid_launch_dependents();
    grid_dependency_wait();
    const int slices = D / kCols, head = blockIdx.x / slices, col = blockIdx.x % slices * kCols + threadIdx.x % kLanes * 4;
    const int req = blockIdx.y, row0 = threadIdx.x / kLanes, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = p.row_offsets[req], n = p.row_offsets[req + 1] - first;
    if (p.few_tokens >= 0 && n > p.few_tokens) return;
    const int64_t in = linear_slot(p, p.state_in[req]), out = linear_slot(p, p.state_out[req]);
    const int64_t state = ((int64_t)head * D + row0) * D + col, slot_size = (int64_t)p.num_heads * D * D;
    float4 s[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        s[i] = in >= 0 ? *reinterpret_cast<const float4*>(p.state_pool + in * slot_size + state + (int64_t)i * kRowsAtOnce * D) : make_float4(0.f, 0.f, 0.f, 0.f);
    auto store = [&](int64_t slot) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) *reinterpret_cast<float4*>(p.state_pool + slot * slot_size + state + (int64_t)i * kRowsAtOnce * D) = s[i];
    };
    const int64_t prefix = p.snap_interval > 0 ? p.prefix_lens[req] : 0;
    int snap = 0;
    for (int64_t t = 0; t < n; ++t) {
        const int64_t tok = first + t;
        if (threadIdx.x < D) s_q[threadIdx.x] = p.scale * __bfloat162float(p.q[tok * p.q_token_stride + (int64_t)head * D + threadIdx.x]);
        else if (threadIdx.x < 2 * D) s_k[threadIdx.x - D] = __bfloat162float(p.k[tok * p.k_token_stride + (int64_t)head * D + threadIdx.x - D]);
        const uint2 vb = *reinterpret_cast<const uint2*>(p.v + tok * p.v_token_stride + (int64_t)head * D + col);
        const float4 v = make_float4(__uint_as_float(vb.x << 16), __uint_as_float(vb.x & 0xffff0000u), __uint_as_float(vb.y << 16), __uint_as_float(vb.y & 0xffff0000u));
        const float a = expf(p.log_decay[tok * p.decay_token_stride + head]);
        __syncthreads();
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const float k = s_k[row0 + i * kRowsAtOnce], q = s_q[row0 + i * kRowsAtOnce];
            s[i].x = fmaf(a, s[i].x, k * v.x); s[i].y = fmaf(a, s[i].y, k * v.y);
            s[i].z = fmaf(a, s[i].z, k * v.z); s[i].w = fmaf(a, s[i].w, k * v.w);
            o.x = fmaf(q, s[i].x, o.x); o.y = fmaf(q, s[i].y, o.y); o.z = fmaf(q, s[i].z, o.z); o.w = fmaf(q, s[i].w, o.w);
        }
#pragma unroll
        for (int w = kLanes; w < 32; w *= 2) {
            o.x += __shfl_xor_sync(0xffffffffu, o.x, w);
            o.y += __shfl_xor_sync(0xffffffffu, o.y, w);
            o.z += __shfl_xor_sync(0xffffffffu, o.z, w);
            o.w += __shfl_xor_sync(0xffffffffu, o.w, w);
        }
        if (lane < kLanes) s_o[warp][lane] = o;
        __syncthreads();
        if (threadIdx.x < kLanes) {
            o = s_o[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) {
                const float4 x = s_o[w][threadIdx.x];
                o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
            }
            *reinterpret_cast<uint2*>(p.out + tok * p.o_token_stride + (int64_t)head * D + col) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
        }
        if (p.snap_interval > 0 && (prefix + t + 1) % p.snap_interval == 0) {
            const int64_t slot = p.snap_slots && snap < p.max_snaps ? linear_slot(p, p.snap_slots[(int64_t)req * p.max_snaps + snap]) : -1;
            if (slot >= 0) store(slot);
            ++snap;
        }
    }
    if (out >= 0) store(out);
}

template <int D, int kCols>
static cudaError_t launch_token(const LinearParams& p, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.num_heads * (D / kCols)), (unsigned)p.num_requests);
    cfg.blockDim = dim3(kLinThreads);
    cfg.stream = stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, wpp_linear_token_kernel<D, kCols>, p);
}

}  // namespace wpp

extern "C" int wpp_launch_linear_token(const wpp::LinearParams* p, int head_dim, int num_sms, void* stream) {
    cudaStream_t st = (cudaStream_t)stream;
    // few chains: columns of a state go to CTAs of their own
    const bool few = (int64_t)p->num_requests * p->num_heads < 2 * (int64_t)num_sms;
    if (head_dim == 128) return (int)(few ? wpp::launch_token<128, 32>(*p, st) : wpp::launch_token<128, 128>(*p, st));
    return (int)(few ? wpp::launch_token<64, 32>(*p, st) : wpp::launch_token<64, 64>(*p, st));
}
