// Attention of few query rows over a cache held in 4 bits: single new tokens, and chunks' row blocks of at most WPP_FEW_ROWS rows
// (tokens x heads of a KV group).
//
// With k_j = least_j + scale_j c_j (c_j the codes), the score of key j for row n is
//     sm_scale (scale_j <q_n, c_j> + least_j sum q_n),
// so the tensor cores multiply the codes themselves, which f16 holds exactly, and two numbers per key finish the score in fp32;
// in the same way sum_j p_j v_j = sum_j (p_j scale_j) c_j + sum_j p_j least_j, of which only p_j scale_j is rounded to f16.
//
// What bounds it is the cache's bytes, and close behind them the ALU's instructions that turn codes into numbers a product takes.  So
// nothing else is done per code: a warp takes 32 keys at a time straight from global memory in the order the tensor cores' fragments
// want (which element of a row stands at which place of a product does not matter as long as both factors agree); keys are the
// rows and query rows the columns of the products (S^T = K Q^T, O^T = V^T P^T: eight columns, of which the group's heads fill all);
// the two products share no data but P, which a transposing move turns round in registers.
// A mask makes the codes f16 numbers 1024 + c or 1024 + 16 c, a packed f16 operation c - 8, both exact.  (As e4m3 numbers, which
// bytes below 16 are with no operation at all, they come to more: the products of 8-bit numbers take them apart into f16 ones by
// themselves.)  V's codes of two keys first stand above one another by a byte permutation.  Q is taken as f16 times a power of two
// per row.  p_j scale_j is rounded to f16 times a power of two per row and warp that puts the largest one so far between 2^6 and 2^15: it
// is off by 2^-11 of itself or by 2^-31 of that largest one, of which a million keys of a warp make 2^-11, however wide the rows of V.
//
// Measured: 64 requests of one token behind 255 to 16,383 keys, 64/8 heads of 128, 130 us back to back and 132 to 135 on a cache that is not
// in L2 (the copies alone 93, the bytes at the measured copy bandwidth 82); four behind 131,071 125 and 132 to 135 us (87).  No unit is
// full (issue 58 %, ALU 51, DRAM 51, products 25): a warp goes through a step as one chain, and twelve warps an SM do not hide all of it.
// Three CTAs an SM of blocks of at most 8 rows: with four, which leaves the products 128 registers, 8 % more.

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr int kFewWarps = 4;
constexpr int kFewKeys = 32;               // a warp's keys at a time
constexpr float kFewSlack = 8.f;           // a row keeps its reference while its scores stay below reference + 8 (log2)
constexpr float kFewMostProduct = 32768.f; // p scale times a row's power of two stays within f16's range; moved, it is in [2^6, 2^7)
constexpr float kFewMostPower = 120.f;     // log2 of that power at most (there is no scale below 2^-100)

// D += A B, 16 x 8 x 16, f16 in, fp32 out
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two codes, one at bits 0 to 3 or 4 to 7 of either half of a word, as f16 numbers code - 8 (exact).  `k1024` is 1024 in both halves, a
// kernel parameter: of two constants the compiler makes two operations (167 us for the 64 requests' tokens when this was tried, so 150).
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t b) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(mask), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t codes_low(uint32_t u, uint32_t k1024) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(and_or(u, 0x000f000fu, k1024)), "r"(0x64086408u));                   // - 1032
    return r;
}
__device__ __forceinline__ uint32_t codes_high(uint32_t u, uint32_t k1024) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(and_or(u, 0x00f000f0u, k1024)), "r"(0x2c002c00u), "r"(0xd480d480u));   // / 16 - 72
    return r;
}
// The same as 64 + code, for K: Q's product with the 64 is what the sums begin at, with the other sign.  (V's sums run over all keys:
// there an offset of eight times the codes would stand above a result that averages out, and its roundings with it.)
__device__ __forceinline__ uint32_t codes_high_64(uint32_t u, uint32_t k64) { return and_or(u, 0x00f000f0u, k64); }
template <int kWords>
__device__ __forceinline__ void load_words(uint32_t (&w)[kWords], uint32_t at) {
    if constexpr (kWords == 4) {
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
    } else if constexpr (kWords == 2) {
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    } else {
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
    }
}

// A warp's ring of stages in shared memory, kFewKeys keys each: K's rows, V's rows, K's pairs, V's pairs.  The warp copies them
// itself, asynchronously, 16 bytes a lane: no thread's registers are spent on what is under way, and warps wait for nobody else.
// (Bulk copies took some thirty instructions each to set up, for the 64 requests' tokens 142 us with stages of a warp's own, 144
// with a CTA's common ones, which couple the warps besides.)
template <int D, int NT>
struct FewSmem {
    static constexpr int kRows = kFewKeys * (D / 2), kPairs = kFewKeys * 4, kStage = 2 * kRows + 2 * kPairs;
    static constexpr int kDepth = NT == 1 ? 4 : 5;
    // in the stages' place, once a unit's are done with: float [warps][8 NT][D + 4], float2 [warps][8 NT]
    static constexpr int kOffMl = kFewWarps * 8 * NT * (D + 4) * 4;
    static constexpr int kBytes = kFewWarps * kDepth * kStage;
    static_assert(kOffMl + kFewWarps * 8 * NT * 8 <= kBytes, "a unit's results fit the stages");
};
__device__ __forceinline__ void copy_16(uint32_t dst, const uint8_t* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Which key stands in row r of a 16-key tile of the products: rows 2 and 3, 6 and 7, ... are exchanged, so that the four keys whose V
// a quarter of the lanes reads at once do not all begin at one bank (64 bytes a row: every second one does).
__device__ __forceinline__ int key_of_row(int r) { return r ^ ((r >> 1) & 1); }

__device__ __forceinline__ float pair_least(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float pair_scale(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

// The running state of a warp's columns (query rows): lane 4 g + t has columns 2 t and 2 t + 1 of every eight.
template <int D, int NT>
struct FewState {
    float o[NT][D / 16][4];            // O^T power
    float m[NT][2], l[NT][2], off[NT][2];            // off: sum of p (least + 8 scale) over this lane's keys
    float power[NT][2];                // of two, that makes p scale an f16 number
};

// 32 keys, at shared-memory address `at`.  Lane 4 g + t takes, of a tile's rows g and g + 8, columns [t D / 4, (t + 1) D / 4) of K; of
// rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9, columns [g D / 8, (g + 1) D / 8) of V; and the number pairs of rows g and g + 8.
template <int D, int NT, bool kMasked>
__device__ __forceinline__ void few_step(FewState<D, NT>& st, const uint32_t at, const uint32_t (&qf)[NT][D / 16][2],
                                         const float (&q_sum)[NT][2], const float (&q_scale)[NT][2], const float (&q_64)[NT][2], int key0, int first_pos, int toks, int last, bool first,
                                         uint32_t k1024, uint32_t k64, int g, int t) {
    using M = FewSmem<D, NT>;
    const int kg = key_of_row(g), kt = key_of_row(2 * t);
    int limit[NT][2];                                                  // last key that the column's row sees
    if (kMasked) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) limit[nt][c] = first_pos + (8 * nt + 2 * t + c) % toks;
    }
    // ---- S^T = codes Q^T (q_64 makes up for codes less 8 and 64 + codes), then the scores in log2 units (q_scale and q_sum have the scale) above m
    float s[2][NT][4];
    float vs[2][2], vo[2][2];
    const uint32_t k_at = at + kg * (D / 2) + t * (D / 8), p_at = at + 2 * M::kRows + kg * 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t k[2][D / 32];
#pragma unroll
        for (int i = 0; i < 2; ++i) load_words<D / 32>(k[i], k_at + (16 * h + 8 * i) * (D / 2));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[h][nt][i] = q_64[nt][i & 1];
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            uint32_t wa = k[0][w], wb = k[1][w];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t a0 = codes_low(wa, k1024), a1 = codes_low(wb, k1024), a2 = codes_high_64(wa, k64), a3 = codes_high_64(wb, k64);
                wa >>= 8;
                wb >>= 8;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(s[h][nt], a0, a1, a2, a3, qf[nt][2 * w + u][0], qf[nt][2 * w + u][1]);
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int key = key0 + 16 * h + 8 * i + kg;
            uint32_t kp[1], vp[1];
            load_words<1>(kp, p_at + (16 * h + 8 * i) * 4);
            load_words<1>(vp, p_at + M::kPairs + (16 * h + 8 * i) * 4);
            const float ks = pair_scale(kp[0]), ko = pair_least(kp[0]);
            vs[h][i] = pair_scale(vp[0]);
            if (kMasked && key > last) vs[h][i] = 0.f;                 // (no row sees it: its pair may be anything)
            vo[h][i] = fmaf(8.f, vs[h][i], pair_least(vp[0]));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float& y = s[h][nt][2 * i + c];
                    y = fmaf(y, ks * q_scale[nt][c], fmaf(ko, q_sum[nt][c], -st.m[nt][c]));
                    if (kMasked && key > limit[nt][c]) y = -INFINITY;
                }
        }
    // ---- references move only where a score or a scale is far above them
    bool move = first;
    float mx[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            mx[nt][c] = fmaxf(fmaxf(s[0][nt][c], s[0][nt][2 + c]), fmaxf(s[1][nt][c], s[1][nt][2 + c]));
            move |= mx[nt][c] > kFewSlack;
        }
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                // how far the reference goes up; the first one may go down as well, and stays where the row sees nothing
                float y = first ? mx[nt][c] : fmaxf(mx[nt][c], 0.f);
#pragma unroll
                for (int w = 4; w < 32; w *= 2) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, w));
                if (kMasked && y == -INFINITY) y = 0.f;
                y = ceilf(y);
                const float a = first ? 1.f : fast_exp2(-y);
                // (scores and power move together: what is summed up keeps its size, unless the power is the largest already)
                float shrink = 1.f;
                if (!first) {
                    const float e = (float)((int)(__float_as_uint(st.power[nt][c]) >> 23) - 127), e1 = fminf(e + y, kFewMostPower);
                    st.power[nt][c] = __uint_as_float((uint32_t)((int)e1 + 127) << 23);
                    shrink = fast_exp2((e1 - e) - y);
                }
                st.m[nt][c] += y;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[h][nt][c] -= y;
                    s[h][nt][2 + c] -= y;
                }
                st.l[nt][c] *= a;
                st.off[nt][c] *= a;
#pragma unroll
                for (int mt = 0; mt < D / 16; ++mt) {
                    st.o[nt][mt][c] *= shrink;
                    st.o[nt][mt][2 + c] *= shrink;
                }
            }
    }
    // ---- P^T, its rows times the keys' V scales and the columns' powers, turned round into the second factor of O^T = V^T P^T
    float top[NT][2];
    bool above = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float& y = s[h][nt][2 * i + c];
                    const bool out = kMasked && key0 + 16 * h + 8 * i + kg > limit[nt][c];
                    const float e = out ? 0.f : fast_exp2(y);
                    st.l[nt][c] += e;
                    st.off[nt][c] = out ? st.off[nt][c] : fmaf(e, vo[h][i], st.off[nt][c]);
                    y = e * vs[h][i];
                }
            top[nt][c] = fmaxf(fmaxf(s[0][nt][c], s[0][nt][2 + c]), fmaxf(s[1][nt][c], s[1][nt][2 + c]));
            above |= top[nt][c] * st.power[nt][c] > kFewMostProduct;
        }
    }
    if (__any_sync(0xffffffffu, above)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float x = top[nt][c];
#pragma unroll
                for (int w = 4; w < 32; w *= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
                // 2^(6 - e) where x is in [2^e, 2^(e + 1)), and never more than it was
                const int e = 260 - (int)(__float_as_uint(x) >> 23 & 0xffu);
                const float power = fminf(st.power[nt][c], __uint_as_float((uint32_t)min(e, 254) << 23)), shrink = power * __frcp_rn(st.power[nt][c]);
                st.power[nt][c] = power;
#pragma unroll
                for (int mt = 0; mt < D / 16; ++mt) {
                    st.o[nt][mt][c] *= shrink;
                    st.o[nt][mt][2 + c] *= shrink;
                }
            }
    }
    uint32_t pb[2][NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                pb[h][nt][i] = transpose_8x8(pack_f16x2(s[h][nt][2 * i] * st.power[nt][0], s[h][nt][2 * i + 1] * st.power[nt][1]));
    // ---- O^T += (codes - 8)^T P^T: a word holds four codes of one key and of the next, one above the other
    const uint32_t v_at = at + M::kRows + g * (D / 16);
    const int flip = kt & 1 ? -(D / 2) : D / 2;                        // from row 2 t's key to row 2 t + 1's
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v[4][D / 64];
#pragma unroll
        for (int i = 0; i < 4; ++i) load_words<D / 64>(v[i], v_at + (16 * h + kt) * (D / 2) + (i & 1) * flip + 8 * (i >> 1) * (D / 2));
#pragma unroll
        for (int w = 0; w < D / 64; ++w)
#pragma unroll
            for (int hw = 0; hw < 2; ++hw) {
                uint32_t lo = __byte_perm(v[0][w], v[1][w], hw ? 0x7632 : 0x5410);
                uint32_t hi = __byte_perm(v[2][w], v[3][w], hw ? 0x7632 : 0x5410);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t a0 = codes_low(lo, k1024), a1 = codes_high(lo, k1024), a2 = codes_low(hi, k1024), a3 = codes_high(hi, k1024);
                    lo >>= 8;
                    hi >>= 8;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(st.o[nt][4 * w + 2 * hw + u], a0, a1, a2, a3, pb[h][nt][0], pb[h][nt][1]);
                }
            }
    }
}

template <int D, int NT>
__device__ __forceinline__ void few_unit(const Kv4AttnParams& p, const int unit, uint8_t* smem) {
    using M = FewSmem<D, NT>;
    constexpr int kSteps = D / 16;             // 16-wide pieces of a row
    float (*s_o)[8 * NT][D + 4] = reinterpret_cast<float (*)[8 * NT][D + 4]>(smem);
    float2 (*s_ml)[8 * NT] = reinterpret_cast<float2 (*)[8 * NT]>(smem + M::kOffMl);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const char* plan = static_cast<const char*>(p.plan);
    const WppUnit un = reinterpret_cast<const WppUnit*>(plan + p.off_units)[unit];
    const int32_t* q_offsets = reinterpret_cast<const int32_t*>(plan + p.off_q_offsets);
    const int q_off = q_offsets[un.request], P = p.prefix_lens[un.request], C = p.chunk_lens[un.request];
    if (P != reinterpret_cast<const int32_t*>(plan + p.off_prefix)[un.request] || C != q_offsets[un.request + 1] - q_off) {
        if (threadIdx.x == 0 && p.status) atomicCAS(p.status, 0, WPP_ERR_PLAN_MISMATCH);
        // (the combine pass reads the parts of a refused request too: none of them has seen a key)
        if (un.split_slot >= 0 && threadIdx.x < un.rows[0] * un.rows[1])
            p.ws_lse[((int64_t)un.split_slot * 2 + un.row0[1]) * 128 + un.head[1] + threadIdx.x] = -INFINITY;
        return;
    }
    const int toks = un.rows[0], rows = toks * un.rows[1], first_pos = P + un.row0[0];     // first_pos: last key that token 0 sees
    const int key_begin = un.kv_begin * WPP_TILE_N;
    const int seen = min(min(P + C, un.kv_end * WPP_TILE_N), first_pos + toks);            // keys that some row sees end here
    const int kvh = un.head[0] / p.group, page_shift = 31 - __clz(p.page_size), in_page = p.page_size - 1;
    const int32_t* table = p.block_tables + (int64_t)un.request * p.max_blocks;

    // ---- the warp's keys: 32 at a time, every kFewWarps-th
    constexpr int kStride = kFewKeys * kFewWarps, kRow = D / 2;
    const uint32_t ring = smem_u32(smem) + warp * M::kDepth * M::kStage;
    const uint8_t* const kc = p.k_cache + kvh * p.head_bytes;
    const uint8_t* const vc = p.v_cache + kvh * p.head_bytes;
    int bad = 0;
    auto request16 = [&](int key, int keys, uint32_t dst, int at) {    // `keys` (16 or 32) keys of one page, `at` keys into the stage
        int page = table[key >> page_shift];
        if (page < 0 || page >= p.num_pages) {
            bad = 1;
            page = 0;
        }
        const int64_t block = page * p.page_bytes;
        const int slot = key & in_page;
        const uint8_t* k = kc + block + slot * kRow + lane * 16;
        const uint8_t* v = vc + block + slot * kRow + lane * 16;
        const uint32_t to = dst + at * kRow + lane * 16;
#pragma unroll
        for (int i = 0; i < kFewKeys * kRow / 512; ++i)
            if (i * 512 + lane * 16 < keys * kRow) {
                copy_16(to + i * 512, k + i * 512);
                copy_16(to + M::kRows + i * 512, v + i * 512);
            }
        const int l = lane & 7;                                        // lanes 0 to 7: K's pairs, 8 to 15: V's
        if (lane < 16 && l * 4 < keys)
            copy_16(dst + 2 * M::kRows + (lane >> 3) * M::kPairs + at * 4 + l * 16, (lane & 8 ? vc : kc) + block + p.page_size * kRow + slot * 4 + l * 16);
    };
    auto request = [&](int key, uint32_t dst) {
        if (key < seen) {
            if (p.page_size > 16) {
                request16(key, min((seen - key + 15) & ~15, kFewKeys), dst, 0);
            } else {
                request16(key, 16, dst, 0);
                if (key + 16 < seen) request16(key + 16, 16, dst, 16);
            }
        }
        copies_commit();                                               // (an empty group where there is nothing: groups are counted)
    };
    int key = key_begin + warp * kFewKeys;
#pragma unroll
    for (int i = 0; i < M::kDepth - 1; ++i) request(key + i * kStride, ring + i * M::kStage);

    // ---- Q as the first product's second factor: f16 numbers q 2^e, e so that the row's largest is in [2^7, 2^8) (what is less than
    //      2^-21 of that may be off by 2^-32 of it); and the sums of its rows
    uint32_t qf[NT][D / 16][2];
    float q_sum[NT][2], q_scale[NT][2], q_64[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = 8 * nt + g;
        uint4 z[D / 32];
        float sum = 0.f, even = 0.f, top = 0.f;                  // even: of the elements whose codes are taken less 8
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            z[w] = make_uint4(0, 0, 0, 0);
            if (n < rows) {
                const int head = un.head[0] + n / toks, tok = q_off + un.row0[0] + n % toks;
                z[w] = *reinterpret_cast<const uint4*>(p.q + (int64_t)tok * p.q_token_stride + (int64_t)head * p.q_head_stride + t * (D / 4) + 8 * w);
            }
            const uint32_t zz[4] = {z[w].x, z[w].y, z[w].z, z[w].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = __uint_as_float(zz[i] << 16), b = __uint_as_float(zz[i] & 0xffff0000u);
                sum += a + b;
                even += a;
                top = fmaxf(top, fmaxf(fabsf(a), fabsf(b)));
            }
        }
#pragma unroll
        for (int w = 1; w < 4; w *= 2) {
            sum += __shfl_xor_sync(0xffffffffu, sum, w);
            even += __shfl_xor_sync(0xffffffffu, even, w);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        }
        // 2^e and 2^-e, both normal numbers
        const int e = min(max(134 - (int)(__float_as_uint(top) >> 23), -119), 126);
        const float up = __uint_as_float((uint32_t)(127 + e) << 23), down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            const uint32_t zz[4] = {z[w].x, z[w].y, z[w].z, z[w].w};
            float y[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[2 * i] = __uint_as_float(zz[i] << 16) * up;
                y[2 * i + 1] = __uint_as_float(zz[i] & 0xffff0000u) * up;
            }
            // elements i and i + 4 of the eight stand side by side, as the codes of a word do
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[nt][2 * w + (i >> 1)][i & 1] = pack_f16x2(y[i], y[i + 4]);
        }
        // of the columns this thread has of S^T: 2 t, 2 t + 1
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            q_sum[nt][c] = p.scale_log2 * __shfl_sync(0xffffffffu, sum, 8 * t + 4 * c);
            q_64[nt][c] = __shfl_sync(0xffffffffu, up * (8.f * even - 64.f * (sum - even)), 8 * t + 4 * c);
            q_scale[nt][c] = p.scale_log2 * __shfl_sync(0xffffffffu, down, 8 * t + 4 * c);
        }
    }
    FewState<D, NT> st;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int mt = 0; mt < kSteps; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[nt][mt][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            st.m[nt][i] = 0.f;
            st.power[nt][i] = 1.329227996e36f;         // 2^120
            st.l[nt][i] = st.off[nt][i] = 0.f;
        }
    }

    bool first = true;
    uint32_t at = 0, fill = (M::kDepth - 1) * M::kStage;               // offsets in the ring: of the keys, and of the next ones to be asked for
    for (; key < seen; key += kStride) {
        copies_wait<M::kDepth - 2>();
        __syncwarp();                          // every lane's copies are here, and every lane has read the stage before
        request(key + (M::kDepth - 1) * kStride, ring + fill);
        fill = at;
        if (key + kFewKeys - 1 <= first_pos && key + kFewKeys <= seen)
            few_step<D, NT, false>(st, ring + at, qf, q_sum, q_scale, q_64, key, first_pos, toks, seen - 1, first, p.f16_1024, p.f16_64, g, t);
        else
            few_step<D, NT, true>(st, ring + at, qf, q_sum, q_scale, q_64, key, first_pos, toks, seen - 1, first, p.f16_1024, p.f16_64, g, t);
        first = false;
        at = at == (M::kDepth - 1) * M::kStage ? 0u : at + M::kStage;
    }
    if (bad && p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
    copies_wait<0>();
    __syncthreads();                           // the warps' results take the stages' place

    // ---- the warps' parts joined
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float l = st.l[nt][c], off = st.off[nt][c];
            const float inverse = __frcp_rn(st.power[nt][c]);
#pragma unroll
            for (int w = 4; w < 32; w *= 2) {
                l += __shfl_xor_sync(0xffffffffu, l, w);
                off += __shfl_xor_sync(0xffffffffu, off, w);
            }
            const int n = 8 * nt + 2 * t + c;
            if (g == 0) s_ml[warp][n] = make_float2(l == 0.f ? -INFINITY : st.m[nt][c], l);
#pragma unroll
            for (int mt = 0; mt < kSteps; ++mt) {
                const int d0 = g * (D / 8) + 2 * mt;       // element 8 w + 4 hw + 2 u of the thread's columns, mt = 4 w + 2 hw + u
                *reinterpret_cast<float2*>(&s_o[warp][n][d0]) =
                    make_float2(fmaf(st.o[nt][mt][c], inverse, off), fmaf(st.o[nt][mt][2 + c], inverse, off));
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * (D / 4); i += 32 * kFewWarps) {
        const int n = i / (D / 4), c = i % (D / 4) * 4;
        float mm = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) mm = fmaxf(mm, s_ml[w][n].x);
        const float ref = mm == -INFINITY ? 0.f : mm;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) {
            const float2 ml = s_ml[w][n];
            if (ml.y == 0.f) continue;                     // saw no key of this row
            const float a = fast_exp2(ml.x - ref);
            const float4 x = *reinterpret_cast<const float4*>(&s_o[w][n][c]);
            sum = fmaf(a, ml.y, sum);
            acc.x = fmaf(a, x.x, acc.x);
            acc.y = fmaf(a, x.y, acc.y);
            acc.z = fmaf(a, x.z, acc.z);
            acc.w = fmaf(a, x.w, acc.w);
        }
        const bool nan = sum != sum;
        const float inv = nan ? NAN : sum > 0.f ? 1.f / sum : 0.f;
        acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
        const float lse2 = nan ? NAN : sum > 0.f ? mm + log2f(sum) : -INFINITY;
        if (un.split_slot < 0) {
            const int64_t tok = (int64_t)q_off + un.row0[0] + n % toks, head = un.head[0] + n / toks;
            *reinterpret_cast<uint2*>(p.out + tok * p.o_token_stride + head * p.o_head_stride + c) =
                make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
            if (p.lse && c == 0) p.lse[tok * p.num_q_heads + head] = fmaxf(lse2 * 0.6931471805599453f, -INFINITY);
        } else {
            const int64_t row = ((int64_t)un.split_slot * 2 + un.row0[1]) * 128 + un.head[1] + n;
            *reinterpret_cast<float4*>(p.ws_o + row * D + c) = acc;
            if (c == 0) p.ws_lse[row] = lse2;
        }
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(32 * kFewWarps, NT == 1 ? 3 : 2) wpp_kv4_few_kernel(const Kv4AttnParams p) {
    extern __shared__ __align__(128) uint8_t smem[];
    grid_launch_dependents();
    grid_dependency_wait();
    const int32_t* first = reinterpret_cast<const int32_t*>(static_cast<const char*>(p.plan) + p.off_few_ctas) + blockIdx.x;
    const int end = first[1];
    for (int u = first[0]; u < end; ++u) {
        few_unit<D, NT>(p, u, smem);
        __syncthreads();                       // (the next unit's keys take the place of this one's results)
    }
}

template <int D, int NT>
static cudaError_t launch_few_nt(const Kv4AttnParams& p, int num_ctas, cudaStream_t stream) {
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(wpp_kv4_few_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewSmem<D, NT>::kBytes);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)num_ctas);
    cfg.blockDim = dim3(32 * kFewWarps);
    cfg.dynamicSmemBytes = FewSmem<D, NT>::kBytes;
    cfg.stream = stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, wpp_kv4_few_kernel<D, NT>, p);
}

template <int D>
static cudaError_t launch_few(const Kv4AttnParams& p, int num_ctas, int max_rows, cudaStream_t stream) {
    return max_rows <= 8 ? launch_few_nt<D, 1>(p, num_ctas, stream) : launch_few_nt<D, 2>(p, num_ctas, stream);
}

}  // namespace wpp

extern "C" int wpp_launch_kv4_few(int head_dim, const wpp::Kv4AttnParams* p, int num_ctas, int max_rows, void* stream) {
    return (int)(head_dim == 128 ? wpp::launch_few<128>(*p, num_ctas, max_rows, (cudaStream_t)stream)
                                 : wpp::launch_few<64>(*p, num_ctas, max_rows, (cudaStream_t)stream));
}
