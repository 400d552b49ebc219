// Linear attention with a decay per head, heads of 128, in blocks of up to 128 tokens on the 5th-generation tensor cores (the algebra is
// wpp_linear_chunk.cu's).  One CTA per SM walks a chain (request, head), or a segment of one, with the fp32 state S (128 x 128) in
// tensor memory.  Per block, with w_j = e^(G_L - G_j):
//     (1) S1 = Q K^T          (2) O2 = P V, P_ij = scale e^(G_i - G_j) S1_ij for j <= i, as bf16 where S1 was
//     (3) O1 = Q bf16(S)      (4) S = e^(G_L) S + (w K)^T V, the weighted K in two bf16 terms (16 bits of every product's factor)
//     o_i = scale e^(G_i) O1_i + O2_i
// (2) has zeros for j > i, and zero times what is no number is none either: outputs that are not finite are looked into and, where V is
// the reason, made again without the products (outputs_again; the look costs 1.5 % of a block).
// 16 warps, by warpgroup:
//   warps 0-3    thread = token: P, and at the block's end the outputs
//   warps 4-7    thread = row of S: bf16(S) into shared memory for (3), e^(G_L) S back, snapshots, first and last states
//   warps 8-11   thread = token: w K in two terms, one of them in K's place; zeros in the rows of V behind the block
//   warp 12      issues all products (one thread), warp 13 loads Q, K, V by TMA into a ring of four tiles, in the order in which
//                their places come free, warp 15 sums the logarithms of the decays
// What bounds it: memory wants 44 clocks a token (1,032 bytes at 6.5 TB/s on 148 SMs), the products 28; the chains
// S1 -> P -> O2 -> outputs -> S1 and (4) -> bf16(S) -> (3), with all their hand-overs, take about 60.  Measured: 8 x 2,048 tokens of 32 heads
// 138 us back to back and 158 on inputs that are not in L2, where the memory would take 87 (256 chains on 148 SMs are two rounds, the
// second not full), 1 x 32,768 of 16 in segments 214 us; products of 16 x 8 x 16 (wpp_linear_chunk.cu) 365 us for the former.
// Tensor memory: S1, then P [0,128)  O1 [128,256)  O2 [256,384)  S [384,512).
// All mbarrier waits are bounded; on expiry the CTA raises its abort flag, every role drains, TMEM is freed and WPP_ERR_TIMEOUT is
// written to the status word.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_linear_blocks.cuh"
#include "wpp_ptx.cuh"

namespace lintc {
using namespace wpp;

constexpr int kD = 128, kL = 128, kThreads = 512, kSlots = 4;
constexpr int kTile = kL * kD * 2, kHalf = kL * 128;                   // a tile: two 64-column halves of 128-byte rows
constexpr uint32_t kColS1 = 0, kColO1 = 128, kColO2 = 256, kColS = 384, kTmemCols = 512;

struct Smem {
    static constexpr int kOffLow = kSlots * kTile;                     // the second term of w K
    static constexpr int kOffS = kOffLow + kTile;                      // bf16(S)
    static constexpr int kOffStage = kOffS + kTile;                    // 4 x 2 KB: the output warps' store staging
    // [2] of float [2][kL + 4]: G, a multiple of 1/64 and the rest, [kL] being G_L; and float [kL]: e^(G_e - G_j), e the last token of j's 32
    static constexpr int kOffG = kOffStage + 4 * 2048;
    static constexpr int kGates = (2 * (kL + 4) + kL) * 4;
    static constexpr int kOffBars = kOffG + 2 * kGates;
    static constexpr int kNumBars = 2 * kSlots + 4 + 8;
    static constexpr int kOffMisc = kOffBars + 8 * kNumBars;
    static constexpr int kBytes = kOffMisc + 8 + 1024;
};
static_assert(Smem::kBytes <= 232448, "more shared memory than a CTA can have");

struct Walk {
    int64_t at, end, left, interval;                   // left: tokens up to the next boundary
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ __forceinline__ int len() const { return (int)min(min((int64_t)kL, end - at), left); }
    __device__ __forceinline__ void next() {
        const int n = len();
        at += n;
        left = left == n ? interval : left - n;
    }
    __device__ __forceinline__ bool at_boundary() const { return left == interval; }
};

// A row of the state (this thread's) between tensor memory and global memory, `apart` float4s between its pieces: rarely called, and
// apart from the loops for the same reason.
__device__ __noinline__ void state_to_memory(uint32_t taddr, float4* to, int apart) {
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
        float x[32];
        tmem_ld32(taddr + 32 * q, reinterpret_cast<uint32_t*>(x));
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 8; ++c) to[(8 * q + c) * apart] = make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
    }
}

// Outputs of a block in which there is something that is no number.  If that is in V, it stands in (2) beside the zeros above P's diagonal
// too, and reaches the tokens before it.  Then the warp's outputs are made once more, in fp32 and from tokens j <= i alone.  row0: the
// block's first row; e1: scale e^(G_i) of this thread's token r.  Rarely called, and slow: about a millisecond for a block.
__device__ __noinline__ void outputs_again(const LinearChunkParams& p, int64_t row0, int len, int r, int head, float e1, uint32_t t_o1) {
    const int lane = r & 31;
    uint32_t zero = 0u;
    for (int j = lane; j < len; j += 32) {
        const uint4* v = reinterpret_cast<const uint4*>(p.v + (row0 + j) * p.v_token_stride + (int64_t)head * kD);
#pragma unroll 4
        for (int c = 0; c < 16; ++c) {
            const uint4 x = v[c];
            probe_bf16x2(zero, x.x); probe_bf16x2(zero, x.y); probe_bf16x2(zero, x.z); probe_bf16x2(zero, x.w);
        }
    }
    if (!__any_sync(0xffffffffu, zero != 0u)) return;
    const int row = min(r, len - 1), last = min(r | 31, len - 1);
    const uint4* q = reinterpret_cast<const uint4*>(p.q + (row0 + row) * p.q_token_stride + (int64_t)head * kD);
#pragma unroll 1
    for (int part = 0; part < 4; ++part) {             // 32 columns at a time
        float y[32];
        __syncwarp();
        tmem_ld32(t_o1 + 32 * part, reinterpret_cast<uint32_t*>(y));
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 32; ++c) y[c] *= e1;
        double fall = 0.0;                             // logarithm of what token j's term has left at token `row`
#pragma unroll 1
        for (int j = last; j >= 0; --j) {
            if (j > row) continue;
            const uint4* k = reinterpret_cast<const uint4*>(p.k + (row0 + j) * p.k_token_stride + (int64_t)head * kD);
            const uint4* v = reinterpret_cast<const uint4*>(p.v + (row0 + j) * p.v_token_stride + (int64_t)head * kD + 32 * part);
            float dot = 0.f;
#pragma unroll 2
            for (int c = 0; c < 16; ++c) {
                const uint4 a = q[c], b = k[c];
                const uint32_t aa[4] = {a.x, a.y, a.z, a.w}, bb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    dot = fmaf(__uint_as_float(aa[i] << 16), __uint_as_float(bb[i] << 16), dot);
                    dot = fmaf(__uint_as_float(aa[i] & 0xffff0000u), __uint_as_float(bb[i] & 0xffff0000u), dot);
                }
            }
            const float w = p.scale * fast_exp2((float)fall) * dot;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 b = v[c];
                const uint32_t bb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[8 * c + 2 * i] = fmaf(w, __uint_as_float(bb[i] << 16), y[8 * c + 2 * i]);
                    y[8 * c + 2 * i + 1] = fmaf(w, __uint_as_float(bb[i] & 0xffff0000u), y[8 * c + 2 * i + 1]);
                }
            }
            fall += (double)decay_log2(p, row0 + j, head);
        }
        __syncwarp();
        if (r < len) {
            uint4* to = reinterpret_cast<uint4*>(p.out + (row0 + r) * p.o_token_stride + (int64_t)head * kD + 32 * part);
#pragma unroll
            for (int c = 0; c < 4; ++c)
                to[c] = make_uint4(pack_bf16x2(y[8 * c], y[8 * c + 1]), pack_bf16x2(y[8 * c + 2], y[8 * c + 3]),
                                   pack_bf16x2(y[8 * c + 4], y[8 * c + 5]), pack_bf16x2(y[8 * c + 6], y[8 * c + 7]));
        }
    }
}

// kFirst: the pass that leaves the segments' own states (no outputs: (4) alone)
template <bool kFirst>
__global__ void __launch_bounds__(kThreads, 1)
wpp_linear_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const __grid_constant__ LinearChunkParams p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t bars = base + Smem::kOffBars;
    const uint32_t bFull = bars, bEmpty = bFull + 8 * kSlots, bGFull = bEmpty + 8 * kSlots, bGEmpty = bGFull + 16, bRest = bGEmpty + 16;
    // S1 landed; P written; O1 and O2 landed; outputs read out of them; bf16(S) written and S scaled; (4) done; w K written
    const uint32_t bS1 = bRest, bP = bRest + 8, bO = bRest + 16, bOFree = bRest + 24, bState = bRest + 32, bDone = bRest + 40, bK = bRest + 48;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + Smem::kOffMisc);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wg = warp >> 2, r = threadIdx.x & 127;
    constexpr int kGateUsers = kFirst ? 256 : 384;

    const int head = blockIdx.y;
    const int64_t index = blockIdx.x;
    int req = 0;
    int64_t row0 = 0, n = 0, index0 = 0, seg = 0, segs = 0;
    auto find = [&] {                                  // false: nothing to do
        grid_dependency_wait();
        const LinearSegment s = linear_segment<kFirst>(p, index);
        req = s.req, row0 = s.row0, n = s.tokens, index0 = s.index0, seg = s.seg, segs = s.segs;
        return s.work;
    };
    // Where many CTAs may have nothing to do they see it before anything is set up: 62 requests of 1 token and 2 of 2,048 with 32 heads
    // 172 us | 157.  Elsewhere the kernel before may still run while they are set up: 8 x 2,048 tokens 134 us | 141.
    bool mine = true;
    if (p.few_tokens >= 0 && !find()) return;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kSlots; ++i) { mbar_init(bFull + 8 * i, 1); mbar_init(bEmpty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(bGFull + 8 * i, 1); mbar_init(bGEmpty + 8 * i, kGateUsers); }
        mbar_init(bS1, 1); mbar_init(bP, 128); mbar_init(bO, 1); mbar_init(bOFree, 128); mbar_init(bState, 128); mbar_init(bDone, 1); mbar_init(bK, 128);
        *abort_flag = 0u;
        fence_barrier_init();
    }
    if (warp == 12) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
        tmem_relinquish();
    }
    if (warp == 13 && lane == 0) { prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_launch_dependents();
    if (p.few_tokens < 0) mine = find();
    const int64_t begin = seg * p.seg_tokens, end = mine ? min(n, begin + p.seg_tokens) : begin;
    const int64_t prefix = p.snap_interval > 0 ? p.prefix_lens[req] : 0;
    // Blocks end at the next boundary of the snapshots.  (Every role walks them by itself: with a 64-bit remainder per block in the
    // roles' loops the instructions of so many roles no longer fit where an SM fetches them fast; 151 us for 8 x 2,048 tokens | 142.)
    const int64_t interval = p.snap_interval > 0 ? p.snap_interval : (int64_t)1 << 60;
    const Walk blocks = {begin, end, p.snap_interval > 0 ? interval - (prefix + begin) % interval : interval, interval};

    if (mine && wg == 3) {
        if (warp == 13 && lane == 0) {
            // ================================================================ loads
            uint32_t slot = 0, phase = 0;
            bool ok = true;
            for (Walk w = blocks; w.more() && ok; w.next()) {
#pragma unroll
                for (int x = kFirst ? 1 : 0; x < 3; ++x) {
                    if (!mbar_wait(bEmpty + 8 * slot, phase ^ 1u, abort_flag)) { ok = false; break; }
                    mbar_arrive_expect_tx(bFull + 8 * slot, kTile);
                    const CUtensorMap* m = x == 0 ? &tm_q : x == 1 ? &tm_k : &tm_v;
                    tma_load_3d(base + slot * kTile, m, bFull + 8 * slot, 0, head, (int)(row0 + w.at));
                    tma_load_3d(base + slot * kTile + kHalf, m, bFull + 8 * slot, 64, head, (int)(row0 + w.at));
                    if (++slot == kSlots) { slot = 0; phase ^= 1u; }
                }
            }
        } else if (warp == 12 && lane == 0) {
            // ================================================================ products
            constexpr uint32_t id_qk = idesc_bf16(128, 0, 0), id_o = idesc_bf16(128, 0, 1), id_s = idesc_bf16(128, 1, 1);
            uint32_t slot = 0, phase = 0, b = 0;       // b: blocks so far
            const uint64_t d_s = smem_desc_sw128(base + Smem::kOffS, kHalf, 1024), d_low = smem_desc_sw128(base + Smem::kOffLow, kHalf, 1024);
            auto take = [&](uint32_t& at) {            // the ring's next tile
                const bool ok = mbar_wait(bFull + 8 * slot, phase, abort_flag);
                at = slot;
                if (++slot == kSlots) { slot = 0; phase ^= 1u; }
                return ok;
            };
            for (Walk w = blocks; w.more(); w.next(), ++b) {
                const int len = w.len();
                const uint32_t par = b & 1u;
                uint32_t sq = 0, sk = 0, sv = 0;
                bool k_waited = false;
                if (!kFirst) {
                    if (!take(sq) || !take(sk)) break;
                    if (b > 0 && !mbar_wait(bO, par ^ 1u, abort_flag)) break;       // P, which stands where S1 goes, has been read
                    tc_fence_after();
                    const uint64_t dq = smem_desc_sw128(base + sq * kTile, 16, 1024), dk = smem_desc_sw128(base + sk * kTile, 16, 1024);
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {
                        const uint64_t off = (uint64_t)(((kk >> 2) * kHalf + (kk & 3) * 32) >> 4);
                        mma_ss(tmem + kColS1, dq + off, dk + off, id_qk, kk > 0);
                    }
                    mma_commit(bS1);
                    if (!mbar_wait(bState, par, abort_flag)) break;
                    if (!mbar_wait(bOFree, par ^ 1u, abort_flag)) break;
                    tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        mma_ss(tmem + kColO1, dq + (uint64_t)(((kk >> 2) * kHalf + (kk & 3) * 32) >> 4), d_s + (uint64_t)(kk * 128), id_o, kk > 0);
                    mma_commit(bEmpty + 8 * sq);
                    if (!take(sv)) break;
                    if (len < kL) {                    // rows of V behind the block have been zeroed
                        if (!mbar_wait(bK, par, abort_flag)) break;
                        k_waited = true;
                    }
                    if (!mbar_wait(bP, par, abort_flag)) break;
                    tc_fence_after();
                    const uint64_t dv = smem_desc_sw128(base + sv * kTile, kHalf, 1024);
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {
                        if (kk == 0) mma_ts_overwrite(tmem + kColO2, tmem + kColS1, dv, id_o);
                        else mma_ts_accumulate(tmem + kColO2, tmem + kColS1 + kk * 8, dv + (uint64_t)(kk * 128), id_o);
                    }
                    mma_commit(bO);
                } else {
                    if (!take(sk) || !take(sv)) break;
                    if (!mbar_wait(bState, par, abort_flag)) break;
                }
                if (!k_waited && !mbar_wait(bK, par, abort_flag)) break;
                tc_fence_after();
                const uint64_t dk = smem_desc_sw128(base + sk * kTile, kHalf, 1024), dv = smem_desc_sw128(base + sv * kTile, kHalf, 1024);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) mma_ss(tmem + kColS, dk + (uint64_t)(kk * 128), dv + (uint64_t)(kk * 128), id_s, 1);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) mma_ss(tmem + kColS, d_low + (uint64_t)(kk * 128), dv + (uint64_t)(kk * 128), id_s, 1);
                mma_commit(bEmpty + 8 * sk);
                mma_commit(bEmpty + 8 * sv);
                mma_commit(bDone);
            }
        } else if (warp == 15) {
            // ================================================================ sums of the decays' logarithms, base 2, in 64 bits
            uint32_t b = 0;
            float g[4] = {0.f, 0.f, 0.f, 0.f};
            auto load = [&](int64_t at, int len) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 4 * lane + i;
                    g[i] = t < len ? decay_log2(p, row0 + at + t, head) : 0.f;
                }
            };
            double all = 0.0;
            Walk w = blocks;
            if (w.more()) load(w.at, w.len());
            for (; w.more(); ++b) {
                double s[4], sum = 0.0;
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = sum += (double)g[i];
                double before = sum;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const double x = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += x;
                }
                const double total = __shfl_sync(0xffffffffu, before, 31), behind = __shfl_up_sync(0xffffffffu, before, 1);
                before = lane > 0 ? behind : 0.0;      // (not before - sum: sum may be no number)
                w.next();
                if (w.more()) load(w.at, w.len());
                if (!__all_sync(0xffffffffu, mbar_wait(bGEmpty + 8 * (b & 1u), ((b >> 1) & 1u) ^ 1u, abort_flag))) break;
                float* whole = reinterpret_cast<float*>(gen + Smem::kOffG + (b & 1u) * Smem::kGates);
                float* rest = whole + kL + 4;
                auto put = [&](int i, double x) {
                    const float y = rintf((float)x * 64.f) * 0.015625f;
                    whole[i] = y;
                    rest[i] = (float)(x - (double)y);
                };
#pragma unroll
                for (int i = 0; i < 4; ++i) put(4 * lane + i, before + s[i]);
                const double at_end = __shfl_sync(0xffffffffu, before + s[3], lane | 7);
#pragma unroll
                for (int i = 0; i < 4; ++i) rest[kL + 4 + 4 * lane + i] = fast_exp2((float)(at_end - (before + s[i])));
                if (lane == 0) put(kL, total);
                all += total;
                __syncwarp();
                if (lane == 0) mbar_arrive(bGFull + 8 * (b & 1u));
            }
            if (kFirst && lane == 0) p.ws_log[index * p.num_heads + head] = (float)all;
        }
    } else if (mine && wg == 2) {
        // ================================================================ w K in two terms (thread = token)
        uint32_t slot = 0, phase = 0, b = 0;
        auto skip = [&] { if (++slot == kSlots) { slot = 0; phase ^= 1u; } };
        bool ok = true;
        for (Walk walk = blocks; walk.more() && ok; walk.next(), ++b) {
            const int len = walk.len();
            if (!kFirst) skip();
            const uint32_t sk = slot;
            ok = mbar_wait(bFull + 8 * sk, phase, abort_flag);
            skip();
            const uint32_t sv = slot, v_phase = phase;
            skip();
            ok = ok && mbar_wait(bGFull + 8 * (b & 1u), (b >> 1) & 1u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const float* whole = reinterpret_cast<const float*>(gen + Smem::kOffG + (b & 1u) * Smem::kGates);
            const float* rest = whole + kL + 4;
            const float w = r < len ? fast_exp2((whole[kL] - whole[r]) + (rest[kL] - rest[r])) : 0.f;
            mbar_arrive(bGEmpty + 8 * (b & 1u));
            // K's place is free to be written once (1) has read it, the second term's once the (4) before has
            if (!kFirst) ok = mbar_wait(bS1, b & 1u, abort_flag);
            if (b > 0) ok = ok && mbar_wait(bDone, (b - 1) & 1u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const uint64_t w2 = pack2(w, w), minus = pack2(-1.f, -1.f);
#pragma unroll 2
            for (int ch = 0; ch < 16; ++ch) {
                const int off = (ch >> 3) * kHalf + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                uint4* at_k = reinterpret_cast<uint4*>(gen + sk * kTile + off);
                const uint4 z = *at_k;
                const uint32_t x[4] = {z.x, z.y, z.z, z.w};
                uint32_t h[4], l[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t xi = r < len ? x[i] : 0u;           // (a row of something else may hold anything)
                    const uint64_t y = fmul2(pack2(__uint_as_float(xi << 16), __uint_as_float(xi & 0xffff0000u)), w2);
                    float y0, y1;
                    unpack2(y, y0, y1);
                    h[i] = pack_bf16x2(y0, y1);
                    unpack2(ffma2(pack2(__uint_as_float(h[i] << 16), __uint_as_float(h[i] & 0xffff0000u)), minus, y), y0, y1);
                    l[i] = pack_bf16x2(y0, y1);
                }
                *at_k = make_uint4(h[0], h[1], h[2], h[3]);
                *reinterpret_cast<uint4*>(gen + Smem::kOffLow + off) = make_uint4(l[0], l[1], l[2], l[3]);
            }
            if (len < kL) {
                ok = __all_sync(0xffffffffu, mbar_wait(bFull + 8 * sv, v_phase, abort_flag));
                if (!ok) break;
                if (r >= len)
                    for (int ch = 0; ch < 16; ++ch)
                        *reinterpret_cast<uint4*>(gen + sv * kTile + (ch >> 3) * kHalf + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();
            mbar_arrive(bK);
        }
    } else if (mine && wg == 1) {
        // ================================================================ the state (thread = row of S)
        const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + kColS;
        const int64_t slot_size = (int64_t)p.num_heads * kD * kD, row_at = (int64_t)head * kD * kD + (int64_t)r * kD;
        // workspace: segments' own states, four columns of all rows after one another
        auto ws = [&](int64_t i, int c4) { return reinterpret_cast<float4*>(p.ws_state + (i * p.num_heads + head) * kD * kD) + c4 * kD + r; };
        const bool from_pool = seg == 0 && (kFirst || segs == 1);
        const int64_t in = from_pool ? linear_slot(p, p.state_in[req]) : -1;
        // the state before the segment into tensor memory
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
            float x[32];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                if (from_pool) {
                    if (in >= 0) y = *reinterpret_cast<const float4*>(p.state_pool + in * slot_size + row_at + 32 * q + 4 * c);
                    if (kFirst) *ws(p.ws_segments + index0, 8 * q + c) = y;         // (state_out may be the same slot, and its segment done first)
                } else if (!kFirst) {
                    y = *ws(seg == 0 ? p.ws_segments + index0 : index0, 8 * q + c);
                }
                x[4 * c] = y.x; x[4 * c + 1] = y.y; x[4 * c + 2] = y.z; x[4 * c + 3] = y.w;
            }
            if (!kFirst) {
#pragma unroll 1
                for (int64_t i = 1; i < seg; ++i) {
                    const float a = fast_exp2(p.ws_log[(index0 + i) * p.num_heads + head]);
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float4 y = *ws(index0 + i, 8 * q + c);
                        x[4 * c] = fmaf(a, x[4 * c], y.x); x[4 * c + 1] = fmaf(a, x[4 * c + 1], y.y);
                        x[4 * c + 2] = fmaf(a, x[4 * c + 2], y.z); x[4 * c + 3] = fmaf(a, x[4 * c + 3], y.w);
                    }
                }
            }
            tmem_st32(lane_addr + 32 * q, reinterpret_cast<const uint32_t*>(x));
        }
        tmem_wait_st();
        int64_t snap = p.snap_interval > 0 ? (prefix + begin) / p.snap_interval - prefix / p.snap_interval : 0;
        auto snapshot = [&] {                          // of the state as it is, at a boundary
            const int64_t slot = p.snap_slots && snap < p.max_snaps ? linear_slot(p, p.snap_slots[(int64_t)req * p.max_snaps + snap]) : -1;
            ++snap;
            if (slot >= 0) state_to_memory(lane_addr, reinterpret_cast<float4*>(p.state_pool + slot * slot_size + row_at), 1);
        };
        uint32_t b = 0;
        bool ok = true;
        Walk walk = blocks;
        for (; walk.more(); walk.next(), ++b) {
            ok = mbar_wait(bGFull + 8 * (b & 1u), (b >> 1) & 1u, abort_flag);
            if (b > 0) ok = ok && mbar_wait(bDone, (b - 1) & 1u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const float* whole = reinterpret_cast<const float*>(gen + Smem::kOffG + (b & 1u) * Smem::kGates);
            const float a = fast_exp2(whole[kL] + whole[2 * kL + 4]);
            mbar_arrive(bGEmpty + 8 * (b & 1u));
            tc_fence_after();
            if (!kFirst && b > 0 && walk.at_boundary()) snapshot();
            const uint64_t a2 = pack2(a, a);
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                float x[32];
                tmem_ld32(lane_addr + 32 * q, reinterpret_cast<uint32_t*>(x));
                tmem_wait_ld();
                if (!kFirst) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        *reinterpret_cast<uint4*>(gen + Smem::kOffS + (q >> 1) * kHalf + r * 128 + ((((q & 1) * 4 + c) ^ (r & 7)) << 4)) =
                            make_uint4(pack_bf16x2(x[8 * c], x[8 * c + 1]), pack_bf16x2(x[8 * c + 2], x[8 * c + 3]),
                                       pack_bf16x2(x[8 * c + 4], x[8 * c + 5]), pack_bf16x2(x[8 * c + 6], x[8 * c + 7]));
                }
#pragma unroll
                for (int i = 0; i < 32; i += 2) unpack2(fmul2(pack2(x[i], x[i + 1]), a2), x[i], x[i + 1]);
                tmem_st32(lane_addr + 32 * q, reinterpret_cast<const uint32_t*>(x));
            }
            tmem_wait_st();
            if (!kFirst) fence_proxy_async_smem();
            tc_fence_before();
            mbar_arrive(bState);
        }
        // ---- the state behind the segment
        if (ok && b > 0) ok = __all_sync(0xffffffffu, mbar_wait(bDone, (b - 1) & 1u, abort_flag));
        if (ok) {
            tc_fence_after();
            if (kFirst) {
                state_to_memory(lane_addr, ws(index, 0), kD);
            } else {
                if (b > 0 && walk.at_boundary() && p.snap_interval > 0) snapshot();
                const int64_t out = seg == segs - 1 ? linear_slot(p, p.state_out[req]) : -1;
                if (out >= 0) state_to_memory(lane_addr, reinterpret_cast<float4*>(p.state_pool + out * slot_size + row_at), 1);
            }
        }
    } else if (mine && wg == 0 && !kFirst) {
        // ================================================================ P and the outputs (thread = token)
        const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        uint32_t b = 0;
        for (Walk walk = blocks; walk.more(); walk.next(), ++b) {
            const int len = walk.len();
            bool ok = mbar_wait(bGFull + 8 * (b & 1u), (b >> 1) & 1u, abort_flag);
            ok = ok && mbar_wait(bS1, b & 1u, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const float* whole = reinterpret_cast<const float*>(gen + Smem::kOffG + (b & 1u) * Smem::kGates);
            const float* rest = whole + kL + 4;
            const float* to_end = rest + kL + 4;
            const float gh = whole[r], gl = rest[r];
            // (column pair i of P stands where columns 2 i, 2 i + 1 of S1, or some before them, have been read)
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                uint32_t y[16];
                if (q > warp) {                        // columns beyond the warp's last row
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = 0u;
                } else {
                    float x[32];
                    tmem_ld32(lane_addr + kColS1 + 32 * q, reinterpret_cast<uint32_t*>(x));
                    if (q < warp) {
                        // e^(G_i - G_j) = e^(G_i - G_e) e^(G_e - G_j), e the last of the 32 columns: neither factor is above 1 if no g is above 0
                        const float f = p.scale * fast_exp2((gh - whole[32 * q + 31]) + (gl - rest[32 * q + 31]));
                        const uint64_t f2 = pack2(f, f);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const float4 c = *reinterpret_cast<const float4*>(to_end + 32 * q + 2 * i);
                            float v[4];
                            unpack2(fmul2(pack2(x[2 * i], x[2 * i + 1]), fmul2(pack2(c.x, c.y), f2)), v[0], v[1]);
                            unpack2(fmul2(pack2(x[2 * i + 2], x[2 * i + 3]), fmul2(pack2(c.z, c.w), f2)), v[2], v[3]);
                            y[i] = pack_bf16x2(v[0], v[1]);
                            y[i + 1] = pack_bf16x2(v[2], v[3]);
                        }
                    } else {
                        const uint64_t gh2 = pack2(gh, gh), gl2 = pack2(gl, gl), minus = pack2(-1.f, -1.f);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const float4 h4 = *reinterpret_cast<const float4*>(whole + 32 * q + 2 * i), l4 = *reinterpret_cast<const float4*>(rest + 32 * q + 2 * i);
                            float e[4];
                            unpack2(fadd2(ffma2(pack2(h4.x, h4.y), minus, gh2), ffma2(pack2(l4.x, l4.y), minus, gl2)), e[0], e[1]);
                            unpack2(fadd2(ffma2(pack2(h4.z, h4.w), minus, gh2), ffma2(pack2(l4.z, l4.w), minus, gl2)), e[2], e[3]);
#pragma unroll
                            for (int c = 0; c < 4; ++c) e[c] = 2 * i + c <= lane ? p.scale * fast_exp2(e[c]) * x[2 * i + c] : 0.f;
                            y[i] = pack_bf16x2(e[0], e[1]);
                            y[i + 1] = pack_bf16x2(e[2], e[3]);
                        }
                    }
                }
                tmem_st8(lane_addr + kColS1 + 16 * q, y);
                tmem_st8(lane_addr + kColS1 + 16 * q + 8, y + 8);
            }
            mbar_arrive(bGEmpty + 8 * (b & 1u));
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(bP);
            const float e1 = p.scale * fast_exp2(gh + gl);
            const uint64_t e2 = pack2(e1, e1);
            if (!__all_sync(0xffffffffu, mbar_wait(bO, b & 1u, abort_flag))) break;
            tc_fence_after();
            const __nv_bfloat16* dst = p.out + (row0 + walk.at + r) * p.o_token_stride + (int64_t)head * kD;
            uint64_t finite = 0ull;                    // two numbers, as long as the outputs are (or numbers whose products are none)
            bool again = false;
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                float x[32], z[32];
                tmem_ld32(lane_addr + kColO1 + 32 * q, reinterpret_cast<uint32_t*>(x));
                tmem_ld32(lane_addr + kColO2 + 32 * q, reinterpret_cast<uint32_t*>(z));
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const uint64_t a = ffma2(pack2(x[i], x[i + 1]), e2, pack2(z[i], z[i + 1])), b = ffma2(pack2(x[i + 2], x[i + 3]), e2, pack2(z[i + 2], z[i + 3]));
                    finite = ffma2(a, b, finite);
                    unpack2(a, x[i], x[i + 1]);
                    unpack2(b, x[i + 2], x[i + 3]);
                }
                uint4 w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = make_uint4(pack_bf16x2(x[8 * i], x[8 * i + 1]), pack_bf16x2(x[8 * i + 2], x[8 * i + 3]),
                                      pack_bf16x2(x[8 * i + 4], x[8 * i + 5]), pack_bf16x2(x[8 * i + 6], x[8 * i + 7]));
                if (q == 3) {
                    float f0, f1;
                    unpack2(finite, f0, f1);
                    again = __any_sync(0xffffffffu, r < len && !(fabsf(f0) + fabsf(f1) <= 3.402823466e+38f));
                    if (!again) {
                        tc_fence_before();
                        mbar_arrive(bOFree);
                    }
                }
                warp_store_rows64(gen + Smem::kOffStage + warp * 2048, lane, w, dst, r < len, q * 64);
            }
            if (__builtin_expect(again, 0)) {
                __syncwarp();
                outputs_again(p, row0 + walk.at, len, r, head, e1, lane_addr + kColO1);
                tc_fence_before();
                mbar_arrive(bOFree);
            }
        }
    }

    // ---- teardown: every loop above is bounded, so every thread gets here
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        const long long t0 = clock64();
        while (clock64() - t0 < 400000) { }            // let copies and tensor-core work in flight land
        if (threadIdx.x == 0 && p.status) atomicCAS(p.status, 0, WPP_ERR_TIMEOUT);
        __syncthreads();
    }
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

template <bool kFirst>
static cudaError_t launch(const CUtensorMap* maps, const LinearChunkParams& p, int64_t segments, cudaStream_t stream) {
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(wpp_linear_tc_kernel<kFirst>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem::kBytes);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)segments, (unsigned)p.num_heads);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Smem::kBytes;
    cfg.stream = stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, wpp_linear_tc_kernel<kFirst>, maps[0], maps[1], maps[2], p);
}

}  // namespace lintc

// maps: q, k, v with boxes of 64 columns of 128 rows; segments: an upper bound of all requests' segments; two_passes: some chain may
// have several
extern "C" int wpp_launch_linear_tc(const wpp::LinearChunkParams* p, const CUtensorMap* maps, int64_t segments, int two_passes, void* stream) {
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    if (two_passes) e = lintc::launch<true>(maps, *p, p->ws_segments, st);
    if (e == cudaSuccess) e = lintc::launch<false>(maps, *p, segments, st);
    return (int)e;
}
