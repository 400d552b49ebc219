// The pages of a wave's new tokens, out of a list of free ones, from the requests' lengths: block tables, row offsets, positions, slots.
//
// Request i holds ceil(P_i / B) pages and needs ceil((P_i + C_i) / B): its new ones stand in the list behind those of the requests
// before it, so that everything follows from two running sums over the requests, which every CTA works out for itself (R lengths
// from L2 cost less than a second launch or a wait for another CTA).  Then a token, and a new page, finds its request by bisection in
// shared memory.  A step's sizes leave nothing but latency: the launch, the lengths, the sums, one dependent load and a store, 3.8 us for 256
// requests of one token each in a graph of such calls.
// The CTA that is done last moves the list's cursor on, when all have read it.
#include <cuda_runtime.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr int kPagesThreads = 512;

struct PageSpan {
    int64_t P, C, there, blocks;       // lengths; pages held and needed (as far as the table goes)
    bool bad, short_row;               // a negative length (the request counts as empty); new tokens, and a table's row that ends before them
};
__device__ __forceinline__ PageSpan span_of(const PagesParams& p, int i) {
    PageSpan s;
    s.P = p.prefix_lens[i];
    s.C = p.chunk_lens[i];
    s.bad = s.P < 0 || s.C < 0;
    if (s.bad) s.P = s.C = 0;
    const int64_t round = ((int64_t)1 << p.page_shift) - 1, need = (s.P + s.C + round) >> p.page_shift;
    s.there = min((s.P + round) >> p.page_shift, (int64_t)p.max_blocks);
    s.blocks = min(need, (int64_t)p.max_blocks);
    s.short_row = s.C > 0 && need > p.max_blocks;
    return s;
}
// the last i of [0, n) with at[i] <= x, if at[0] <= x; of equal ones the last: the one that has something
__device__ __forceinline__ int last_not_above(const int32_t* at, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kPagesThreads) wpp_pages_kernel(const PagesParams p) {
    extern __shared__ int32_t s_sums[];       // tokens, then new pages, before each request: [R + 1] each, at most 2^31 - 1
    __shared__ int64_t s_tokens[kPagesThreads / 32];
    __shared__ int64_t s_pages[kPagesThreads / 32];
    grid_launch_dependents();
    grid_dependency_wait();
    const int R = p.num_requests, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t* const s_tok = s_sums;
    int32_t* const s_new = s_sums + R + 1;
    const int32_t cursor = p.cursor[0];
    const int32_t taken = min(max(cursor, 0), p.num_free);
    int error = cursor != taken ? WPP_ERR_BOUNDS : 0;

    // ---- running sums
    int64_t tokens = 0, pages = 0;            // of the requests so far
    for (int base = 0; base < R; base += kPagesThreads) {
        const int i = base + tid;
        PageSpan s = {0, 0, 0, 0, false, false};
        if (i < R) {
            s = span_of(p, i);
            if (s.bad) error = WPP_ERR_INVALID_ARG;
            if (s.short_row) error = WPP_ERR_BOUNDS;
            if (!p.slots && blockIdx.x == 0 && s.C > 0 && !s.short_row && s.there > s.P >> p.page_shift) {
                // the page that the first new token goes to, which the slots' makers look at otherwise
                const int32_t page = p.block_tables[(int64_t)i * p.max_blocks + (s.P >> p.page_shift)];
                if (page < 0 || page >= p.num_pages) error = WPP_ERR_BOUNDS;
            }
        }
        int64_t t = s.C;
        int64_t n = s.blocks - s.there;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t tt = __shfl_up_sync(0xffffffffu, t, d);
            const int64_t nn = __shfl_up_sync(0xffffffffu, n, d);
            if (lane >= d) { t += tt; n += nn; }
        }
        if (lane == 31) { s_tokens[warp] = t; s_pages[warp] = n; }
        __syncthreads();
        int64_t t0 = tokens, n0 = pages;
        for (int w = 0; w < kPagesThreads / 32; ++w) {
            if (w < warp) { t0 += s_tokens[w]; n0 += s_pages[w]; }
            tokens += s_tokens[w];
            pages += s_pages[w];
        }
        const int64_t before = t0 + t - s.C;
        if (i < R) {
            s_tok[i] = (int32_t)min(before, (int64_t)0x7fffffff);
            s_new[i] = (int32_t)min(n0 + n - (s.blocks - s.there), (int64_t)0x7fffffff);
            if (blockIdx.x == 0) p.row_offsets[i] = before;
        }
        __syncthreads();
    }
    if (tid == 0) {
        s_tok[R] = (int32_t)min(tokens, (int64_t)0x7fffffff);
        s_new[R] = (int32_t)min(pages, (int64_t)0x7fffffff);
        if (blockIdx.x == 0) p.row_offsets[R] = tokens;
    }
    __syncthreads();
    if (tokens > p.max_tokens && p.max_tokens >= 0 && (p.positions || p.slots)) error = WPP_ERR_BOUNDS;

    auto new_page = [&](int64_t k) -> int32_t {               // the wave's k-th new page, -1: there is none
        const int64_t at = taken + k;
        const int32_t page = at < p.num_free ? p.free_pages[at] : -1;
        if (page >= 0 && page < p.num_pages) return page;
        error = WPP_ERR_BOUNDS;
        return -1;
    };
    const int64_t thread = (int64_t)blockIdx.x * kPagesThreads + tid, threads = (int64_t)gridDim.x * kPagesThreads;
    // ---- positions and slots
    for (int64_t t = thread; t < p.max_tokens; t += threads) {
        int32_t pos = 0;
        int64_t slot = -1;
        if (t < s_tok[R]) {
            const int i = last_not_above(s_tok, R, (int32_t)t);
            const PageSpan s = span_of(p, i);
            const int64_t at = s.P + (t - s_tok[i]), blk = at >> p.page_shift;
            pos = (int32_t)min(at, (int64_t)0x7fffffff);
            if (p.slots) {
                int32_t page = -1;
                if (blk >= p.max_blocks) {
                    error = WPP_ERR_BOUNDS;
                } else if (blk >= s.there) {
                    page = new_page(s_new[i] + (blk - s.there));
                } else {
                    page = p.block_tables[(int64_t)i * p.max_blocks + blk];
                    if (page < 0 || page >= p.num_pages) {
                        error = WPP_ERR_BOUNDS;
                        page = -1;
                    }
                }
                if (page >= 0) slot = ((int64_t)page << p.page_shift) + (at & (((int64_t)1 << p.page_shift) - 1));
            }
        }
        if (p.positions) p.positions[t] = pos;
        if (p.slots) p.slots[t] = slot;
    }
    // ---- block tables
    for (int64_t k = thread; k < s_new[R]; k += threads) {
        const int i = last_not_above(s_new, R, (int32_t)k);
        p.block_tables[(int64_t)i * p.max_blocks + span_of(p, i).there + (k - s_new[i])] = new_page(k);
    }
    if (error && p.status) atomicCAS(p.status, 0, error);
    // ---- the list's cursor
    __syncthreads();
    if (tid == 0) {
        bool last = blockIdx.x == 0;          // (another word than the one that is read: any CTA may write it)
        if (gridDim.x > 1 && p.cursor_out == p.cursor) last = atomicAdd(reinterpret_cast<uint32_t*>(p.cursor_out) + 1, 1u) == gridDim.x - 1;
        if (last) {
            p.cursor_out[0] = (int32_t)min((int64_t)taken + pages, (int64_t)p.num_free);
            p.cursor_out[1] = 0;
        }
    }
}

}  // namespace wpp

extern "C" int wpp_launch_pages(const wpp::PagesParams* p, int num_sms, void* stream) {
    // a CTA for every 512 tokens, and no more than the SMs (62,000 tokens of 64 requests: 99 us on one CTA, 10.2 on 16, 5.4 so)
    int64_t blocks = ((int64_t)p->max_tokens + wpp::kPagesThreads - 1) / wpp::kPagesThreads;
    blocks = blocks < 1 ? 1 : blocks > num_sms ? num_sms : blocks;
    const size_t smem = 2 * ((size_t)p->num_requests + 1) * sizeof(int32_t);
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(wpp::wpp_pages_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(2 * (wpp::kPagesMostRequests + 1) * sizeof(int32_t)));
        if (e != cudaSuccess) return (int)e;
        attr_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(wpp::kPagesThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return (int)cudaLaunchKernelEx(&cfg, wpp::wpp_pages_kernel, *p);
}
