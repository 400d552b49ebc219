// Linear attention with a decay per head, in blocks of up to 64 tokens on the tensor cores.
//
// Inside a block, with G_i the sum of the logarithms g up to token i (of the block) and S the state before it,
//     o_i = scale (e^(G_i) S^T q_i + sum_(j <= i) e^(G_i - G_j) <q_i, k_j> v_j),
//     S'  = e^(G_L) S + sum_j e^(G_L - G_j) k_j v_j^T.
// One CTA walks a chain (request, head), or a segment of one, with S in registers: a warp has 16 columns of it, S^T as the
// accumulators of its products, which turn into the factors of S^T Q^T without a move.  Products per block and warp: its
// part of Q K^T; S^T Q^T and V^T P^T into the same accumulators (the first scaled by e^(G_i) before the second); V^T K into the
// state, V weighted and split into two bf16 terms, so that the state's terms have 16 bits.  For the outputs, which are rounded
// to bf16, P and S are rounded to bf16 once.
//
// What bounds it are the products (1,856 of 16 x 8 x 16 for 64 tokens at 128 columns, half a one per clock: 58 clocks a token where
// the memory needs 44; heads of 128 come here with few chains of short chunks only, see kLinTcTokens, the others to
// wpp_linear_tc.cu: 8 x 2,048 tokens of 32 heads 365 us | 138 there).  Heads of 64: 8 x 2,048 of 32 heads 137 us, half the bytes
// and a quarter of the products.  The sums G are made in 64 bits and kept as a multiple of 1/64 and a rest, so that differences of long
// sums are exact to fp32.
//
// Few long chains are cut into segments (`seg_tokens`): a first pass leaves every segment's own state but the last one's, starting
// at zero (the first one's at the chain's), and its decay; in the second pass a CTA makes its segment's state before from those.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_linear_blocks.cuh"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr int kLinBlock = 64;              // tokens

__device__ __forceinline__ void lin_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm_4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_4_trans(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void stsm_4_trans(uint32_t at, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r0), "r"(r1), "r"(r2), "r"(r3) : "memory");
}
__device__ __forceinline__ void copy_16_or_zero(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

template <int D>
struct LinCfg {
    static constexpr int kWarps = D / 16, kThreads = 32 * kWarps;
    static constexpr int kTile = kLinBlock * D * 2;                    // 64 rows of q, k or v
    static constexpr int kOffP = 2 * 3 * kTile, kRowP = 2 * kLinBlock + 16;
    static constexpr int kOffG = kOffP + kLinBlock * kRowP;            // float2 [64]: G as (multiple of 1/64, rest), base 2
    static constexpr int kOffE = kOffG + kLinBlock * 8;                // float [64]: scale e^(G_i)
    static constexpr int kOffW = kOffE + kLinBlock * 4;                // float [64]: e^(G_L - G_j)
    static constexpr int kOffA = kOffW + kLinBlock * 4;                // float: e^(G_L); double: G_L
    static constexpr int kOffSpoilt = kOffA + 16;                      // int [D]: see spoilt
    static constexpr int kBytes = kOffSpoilt + D * 4;
};

// kFirst: the pass that leaves the segments' own states (no outputs)
template <int D, bool kFirst>
__global__ void __launch_bounds__(LinCfg<D>::kThreads, 2) wpp_linear_chunk_kernel(const LinearChunkParams p) {
    using Cf = LinCfg<D>;
    constexpr int kN = D / 8;                          // 8-column tiles of a warp's S^T
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sm = smem_u32(smem);
    float2* s_g = reinterpret_cast<float2*>(smem + Cf::kOffG);
    float* s_e = reinterpret_cast<float*>(smem + Cf::kOffE);
    float* s_w = reinterpret_cast<float*>(smem + Cf::kOffW);
    float* s_a = reinterpret_cast<float*>(smem + Cf::kOffA);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // Of the warp's 16 columns: the block's first token whose value is no number (written and read where there is one)
    volatile int* spoilt = reinterpret_cast<volatile int*>(smem + Cf::kOffSpoilt) + 16 * warp;
    grid_launch_dependents();
    grid_dependency_wait();

    const int head = blockIdx.y;
    const int64_t index = blockIdx.x;
    const LinearSegment found = linear_segment<kFirst>(p, index);
    if (!found.work) return;
    const int req = found.req;
    const int64_t row0 = found.row0, n = found.tokens, index0 = found.index0, seg = found.seg, segs = found.segs;
    const int64_t begin = seg * p.seg_tokens, end = min(n, begin + p.seg_tokens);

    // ---- the state before the segment.  Workspace: a segment's own state is at ws_state, thread by thread.
    float s[kN][4];                                    // S^T: rows (columns of S) 16 warp + g, + 8; columns 8 nt + 2 t, + 1
    const int64_t slot_size = (int64_t)p.num_heads * D * D;
    const int64_t mine = (int64_t)head * D * D + (int64_t)(2 * t) * D + 16 * warp + g;     // of S[2 t][16 warp + g]
    auto ws_at = [&](int64_t i) { return p.ws_state + ((i * p.num_heads + head) * D * D) + threadIdx.x * 4; };
    auto ws_load = [&](int64_t i, float (&x)[kN][4]) {
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) *reinterpret_cast<float4*>(x[nt]) = *reinterpret_cast<const float4*>(ws_at(i) + nt * Cf::kThreads * 4);
    };
    auto ws_store = [&](int64_t i) {
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) *reinterpret_cast<float4*>(ws_at(i) + nt * Cf::kThreads * 4) = *reinterpret_cast<const float4*>(s[nt]);
    };
    auto pool_store = [&](int64_t slot) {
        float* at = p.state_pool + slot * slot_size + mine;
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) {
            at[(8 * nt) * D] = s[nt][0];
            at[(8 * nt + 1) * D] = s[nt][1];
            at[(8 * nt) * D + 8] = s[nt][2];
            at[(8 * nt + 1) * D + 8] = s[nt][3];
        }
    };
    if (seg == 0 && (kFirst || segs == 1)) {
        const int64_t in = linear_slot(p, p.state_in[req]);
        const float* at = p.state_pool + in * slot_size + mine;
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) {
            s[nt][0] = in >= 0 ? at[(8 * nt) * D] : 0.f;
            s[nt][1] = in >= 0 ? at[(8 * nt + 1) * D] : 0.f;
            s[nt][2] = in >= 0 ? at[(8 * nt) * D + 8] : 0.f;
            s[nt][3] = in >= 0 ? at[(8 * nt + 1) * D + 8] : 0.f;
        }
        if (kFirst) ws_store(p.ws_segments + index0);       // (state_out may be the same slot, and its last segment done first)
    } else if (kFirst) {
#pragma unroll
        for (int nt = 0; nt < kN; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = 0.f;
    } else if (seg == 0) {
        ws_load(p.ws_segments + index0, s);
    } else {
        ws_load(index0, s);
        for (int64_t i = 1; i < seg; ++i) {
            const float a = exp2f(p.ws_log[(index0 + i) * p.num_heads + head]);
            float x[kN][4];
            ws_load(index0 + i, x);
#pragma unroll
            for (int nt = 0; nt < kN; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[nt][c] = fmaf(a, s[nt][c], x[nt][c]);
        }
    }

    const int64_t prefix = p.snap_interval > 0 ? p.prefix_lens[req] : 0;
    // a block ends at the next boundary of the snapshots
    auto block_len = [&](int64_t at) {
        int64_t len = min((int64_t)kLinBlock, end - at);
        if (p.snap_interval > 0) len = min(len, p.snap_interval - (prefix + at) % p.snap_interval);
        return (int)len;
    };
    auto load = [&](int64_t at, int len, int buf) {
        constexpr int kChunks = D / 8;
        const uint32_t to = sm + buf * 3 * Cf::kTile;
        for (int i = threadIdx.x; i < kLinBlock * kChunks; i += Cf::kThreads) {
            const int r = i / kChunks, c = i % kChunks;
            const bool there = r < len;
            const int64_t tok = row0 + at + (there ? r : 0), col = (int64_t)head * D + c * 8;
            const uint32_t dst = to + r * (2 * D) + ((c ^ (r & 7)) << 4);
            if (!kFirst) copy_16_or_zero(dst, p.q + tok * p.q_token_stride + col, there);
            copy_16_or_zero(dst + Cf::kTile, p.k + tok * p.k_token_stride + col, there);
            copy_16_or_zero(dst + 2 * Cf::kTile, p.v + tok * p.v_token_stride + col, there);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // the logarithms of a block's decays, base 2, of tokens 2 lane and 2 lane + 1
    float g0 = 0.f, g1 = 0.f;
    auto load_decay = [&](int64_t at, int len) {
        auto one = [&](int r) {
            return r < len ? decay_log2(p, row0 + at + r, head) : 0.f;
        };
        g0 = one(2 * lane);
        g1 = one(2 * lane + 1);
    };
    int64_t at = begin;
    int len = at < end ? block_len(at) : 0, buf = 0;
    int64_t snap = p.snap_interval > 0 ? (prefix + begin) / p.snap_interval - prefix / p.snap_interval : 0;
    double all = 0.0;                                  // logarithm of the segment's decay
    if (len > 0) {
        load(at, len, 0);
        if (warp == 0) load_decay(at, len);
    }
    while (at < end) {
        if (warp == 0) {
            // sums of the logarithms in 64 bits
            double a = g0, b = (double)g0 + g1;
            double sum = b;
#pragma unroll
            for (int w = 1; w < 32; w *= 2) {
                const double x = __shfl_up_sync(0xffffffffu, sum, w);
                if (lane >= w) sum += x;
            }
            const double total = __shfl_sync(0xffffffffu, sum, 31), before = __shfl_up_sync(0xffffffffu, sum, 1);
            a += lane > 0 ? before : 0.0;              // (not sum - b: b may be no number)
            b = sum;
            auto put = [&](int i, double x) {
                const float whole = rintf((float)x * 64.f) * 0.015625f;
                s_g[i] = make_float2(whole, (float)(x - (double)whole));
                s_e[i] = p.scale * exp2f((float)x);
                s_w[i] = exp2f((float)(total - x));
            };
            put(2 * lane, a);
            put(2 * lane + 1, b);
            if (lane == 0) s_a[0] = exp2f((float)total);
            all += total;
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        const int64_t next = at + len;
        const int next_len = next < end ? block_len(next) : 0;
        if (next_len > 0) {
            load(next, next_len, buf ^ 1);
            if (warp == 0) load_decay(next, next_len);
        }
        const uint32_t sq = sm + buf * 3 * Cf::kTile, sk = sq + Cf::kTile, sv = sk + Cf::kTile, sp = sm + Cf::kOffP;
        auto tile_at = [&](uint32_t base, int r, int c) { return base + r * (2 * D) + ((c ^ (r & 7)) << 4); };

        if (!kFirst) {
            // ---- P = scale e^(G_i - G_j) <q_i, k_j>: rows of 16 by the warp, 32 columns at a time, none of them beyond the diagonal
            const int mi = warp & 3;
#pragma unroll
            for (int pass = 0; pass < (D == 128 ? 1 : 2); ++pass) {
                const int jh = D == 128 ? warp >> 2 : pass;
                if (32 * jh > 16 * mi + 15) continue;
                float x[4][4] = {};
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t a[4];
                    ldsm_4(a, tile_at(sq, 16 * mi + (lane & 15), 2 * ks + (lane >> 4)));
#pragma unroll
                    for (int nn = 0; nn < 2; ++nn) {
                        uint32_t b[4];
                        ldsm_4(b, tile_at(sk, 32 * jh + 16 * nn + (lane & 7) + ((lane >> 4) << 3), 2 * ks + ((lane >> 3) & 1)));
                        lin_mma(x[2 * nn], a, b[0], b[1]);
                        lin_mma(x[2 * nn + 1], a, b[2], b[3]);
                    }
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int i = 16 * mi + g + 8 * half;
                    const float2 gi = s_g[i];
#pragma unroll
                    for (int nt = 0; nt < 4; ++nt) {
                        const int j = 32 * jh + 8 * nt + 2 * t;
                        const float4 gj = *reinterpret_cast<const float4*>(&s_g[j]);
                        const float y0 = j <= i ? x[nt][2 * half] * p.scale * fast_exp2((gi.x - gj.x) + (gi.y - gj.y)) : 0.f;
                        const float y1 = j + 1 <= i ? x[nt][2 * half + 1] * p.scale * fast_exp2((gi.x - gj.z) + (gi.y - gj.w)) : 0.f;
                        *reinterpret_cast<uint32_t*>(smem + Cf::kOffP + i * Cf::kRowP + j * 2) = pack_bf16x2(y0, y1);
                    }
                }
            }
            __syncthreads();
        }
        // ---- V^T: rows are the warp's 16 columns, columns the block's tokens
        uint32_t v[4][4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
            ldsm_4_trans(v[ks], tile_at(sv, 16 * ks + (lane & 7) + ((lane >> 4) << 3), 2 * warp + ((lane >> 3) & 1)));
        // Values that are no numbers stand in P's product beside zeros as well, and would reach the tokens before them.  They are zeros
        // for the products; the outputs and the state of their columns are NaN from their tokens on.
        bool any_spoilt = false;
        if (!kFirst) {
            uint32_t zero = 0u;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int c = 0; c < 4; ++c) probe_bf16x2(zero, v[ks][c]);
            any_spoilt = __any_sync(0xffffffffu, zero != 0u);
            if (__builtin_expect(any_spoilt, 0)) {
                int first[2] = {kLinBlock, kLinBlock};  // of rows g and g + 8
#pragma unroll
                for (int ks = 3; ks >= 0; --ks)
#pragma unroll
                    for (int c = 3; c >= 0; --c)
#pragma unroll
                        for (int h = 1; h >= 0; --h)
                            if ((v[ks][c] >> (16 * h) & 0x7f80u) == 0x7f80u) {
                                first[c & 1] = 16 * ks + 8 * (c >> 1) + 2 * t + h;
                                v[ks][c] &= h ? 0x0000ffffu : 0xffff0000u;
                            }
#pragma unroll
                for (int w = 1; w < 4; w *= 2) {
                    first[0] = min(first[0], __shfl_xor_sync(0xffffffffu, first[0], w));
                    first[1] = min(first[1], __shfl_xor_sync(0xffffffffu, first[1], w));
                }
                if (t == 0) {
                    spoilt[g] = first[0];
                    spoilt[g + 8] = first[1];
                }
                __syncwarp();
            }
        }
        if (!kFirst) {
            // ---- O^T = e^(G_i) S^T Q^T + V^T P^T, 32 tokens at a time
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float o[4][4] = {};
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t a[4] = {pack_bf16x2(s[2 * ks][0], s[2 * ks][1]), pack_bf16x2(s[2 * ks][2], s[2 * ks][3]),
                                           pack_bf16x2(s[2 * ks + 1][0], s[2 * ks + 1][1]), pack_bf16x2(s[2 * ks + 1][2], s[2 * ks + 1][3])};
#pragma unroll
                    for (int nn = 0; nn < 2; ++nn) {
                        uint32_t b[4];
                        ldsm_4(b, tile_at(sq, 32 * half + 16 * nn + (lane & 7) + ((lane >> 4) << 3), 2 * ks + ((lane >> 3) & 1)));
                        lin_mma(o[2 * nn], a, b[0], b[1]);
                        lin_mma(o[2 * nn + 1], a, b[2], b[3]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < 4; ++nt) {
                    const float2 e = *reinterpret_cast<const float2*>(&s_e[32 * half + 8 * nt + 2 * t]);
                    o[nt][0] *= e.x;
                    o[nt][1] *= e.y;
                    o[nt][2] *= e.x;
                    o[nt][3] *= e.y;
                }
#pragma unroll
                for (int ks = 0; ks < 2 * (half + 1); ++ks)
#pragma unroll
                    for (int nn = 0; nn < 2; ++nn) {
                        uint32_t b[4];
                        ldsm_4(b, sp + (32 * half + 16 * nn + (lane & 7) + ((lane >> 4) << 3)) * Cf::kRowP + (16 * ks + 8 * ((lane >> 3) & 1)) * 2);
                        lin_mma(o[2 * nn], v[ks], b[0], b[1]);
                        lin_mma(o[2 * nn + 1], v[ks], b[2], b[3]);
                    }
                if (__builtin_expect(any_spoilt, 0)) {
#pragma unroll
                    for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (32 * half + 8 * nt + 2 * t + (c & 1) >= spoilt[g + 8 * (c >> 1)]) o[nt][c] = NAN;
                }
                // two 8 x 8 pieces turned round in registers: the thread has columns 2 t, 2 t + 1 of token g
#pragma unroll
                for (int nt = 0; nt < 4; ++nt) {
                    uint32_t lo = pack_bf16x2(o[nt][0], o[nt][1]), hi2 = pack_bf16x2(o[nt][2], o[nt][3]);
                    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(lo));
                    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(hi2));
                    const int tok = 32 * half + 8 * nt + g;
                    if (tok < len) {
                        __nv_bfloat16* dst = p.out + (row0 + at + tok) * p.o_token_stride + (int64_t)head * D + 16 * warp + 2 * t;
                        *reinterpret_cast<uint32_t*>(dst) = lo;
                        *reinterpret_cast<uint32_t*>(dst + 8) = hi2;
                    }
                }
            }
        }
        if (__builtin_expect(any_spoilt, 0)) {                              // the state's columns are NaN from here on: the first such value is one again
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int ahead = spoilt[g + 8 * (c & 1)] - (16 * ks + 8 * (c >> 1) + 2 * t);
                    if (ahead == 0 || ahead == 1) v[ks][c] |= 0x7fc0u << (16 * ahead);
                }
        }
        // ---- S^T = e^(G_L) S^T + (e^(G_L - G_j) V)^T K, the weighted V in two bf16 terms
        {
            const float a = s_a[0];
#pragma unroll
            for (int nt = 0; nt < kN; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[nt][c] *= a;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                uint32_t vh[4], vl[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float2 w = *reinterpret_cast<const float2*>(&s_w[16 * ks + 8 * (c >> 1) + 2 * t]);
                    const float x0 = __uint_as_float(v[ks][c] << 16) * w.x, x1 = __uint_as_float(v[ks][c] & 0xffff0000u) * w.y;
                    vh[c] = pack_bf16x2(x0, x1);
                    vl[c] = pack_bf16x2(x0 - __uint_as_float(vh[c] << 16), x1 - __uint_as_float(vh[c] & 0xffff0000u));
                }
#pragma unroll
                for (int nn = 0; nn < kN / 2; ++nn) {
                    uint32_t b[4];
                    ldsm_4_trans(b, tile_at(sk, 16 * ks + (lane & 15), 2 * nn + (lane >> 4)));
                    lin_mma(s[2 * nn], vh, b[0], b[1]);
                    lin_mma(s[2 * nn], vl, b[0], b[1]);
                    lin_mma(s[2 * nn + 1], vh, b[2], b[3]);
                    lin_mma(s[2 * nn + 1], vl, b[2], b[3]);
                }
            }
        }
        at = next;
        if (!kFirst && p.snap_interval > 0 && (prefix + at) % p.snap_interval == 0) {
            const int64_t slot = p.snap_slots && snap < p.max_snaps ? linear_slot(p, p.snap_slots[(int64_t)req * p.max_snaps + snap]) : -1;
            if (slot >= 0) pool_store(slot);
            ++snap;
        }
        len = next_len;
        buf ^= 1;
        __syncthreads();                               // the sums and the tiles of this block are done with
    }
    if (kFirst) {
        ws_store(index);
        if (threadIdx.x == 0) p.ws_log[index * p.num_heads + head] = (float)all;
    } else if (seg == segs - 1) {
        const int64_t out = linear_slot(p, p.state_out[req]);
        if (out >= 0) pool_store(out);
    }
}

template <int D, bool kFirst>
static cudaError_t launch_chunk(const LinearChunkParams& p, int64_t segments, cudaStream_t stream) {
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(wpp_linear_chunk_kernel<D, kFirst>, cudaFuncAttributeMaxDynamicSharedMemorySize, LinCfg<D>::kBytes);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)segments, (unsigned)p.num_heads);
    cfg.blockDim = dim3(LinCfg<D>::kThreads);
    cfg.dynamicSmemBytes = LinCfg<D>::kBytes;
    cfg.stream = stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, wpp_linear_chunk_kernel<D, kFirst>, p);
}

}  // namespace wpp

// segments: an upper bound of all requests' segments; two_passes: some chain may have several
extern "C" int wpp_launch_linear_chunk(const wpp::LinearChunkParams* p, int head_dim, int64_t segments, int two_passes, void* stream) {
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    if (two_passes) e = head_dim == 128 ? wpp::launch_chunk<128, true>(*p, p->ws_segments, st) : wpp::launch_chunk<64, true>(*p, p->ws_segments, st);
    if (e == cudaSuccess) e = head_dim == 128 ? wpp::launch_chunk<128, false>(*p, segments, st) : wpp::launch_chunk<64, false>(*p, segments, st);
    return (int)e;
}
