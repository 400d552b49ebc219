// Attention of many query rows over a cache held in 8 bits: persistent, one CTA per SM, tiles of two 128-row halves against key steps
// of 128 keys, as wpp_attention.cu has them.
//   warps 0-3   softmax of half A: thread r owns query row r; at a tile's end it writes its row
//   warps 4-7   softmax of half B
//   warps 8-11  at a tile's start Q's rows as two e4m3 terms; then, for every step, V's codes as f16
//   warp 12     issuer of S = Q K^T, warp 14 issuer of O += P V (one thread each), warp 13 takes tiles and loads Q, K and V by TMA,
//               warp 15 the scales of the steps' pages
// S = Q K^T is a product of 8-bit numbers: K's codes go from the pages to the tensor cores as they are.  A row of Q is taken as hi + lo, times a
// power of two that puts its largest element into [128, 256): hi is q rounded to e4m3, four significant bits, lo what is left, of which a
// bf16 number has no more than e4m3 holds; elements below 2^-9 of the row's largest are off by up to 2^-18 of it, the others exact.  Two products of
// 8-bit numbers take as long as one of bf16.
// O += P V is a product of f16 numbers, because P as two e4m3 terms would cost the softmax warps, which are what everybody waits for,
// several operations a score, and four other warps turn two of V's codes into f16 by one.  V's tiles hold code * vs / v, vs the scale of
// the code's page and v the largest of the tile's first 128 keys (of a part's own first ones): exact, being a power of two, while vs / v is from
// 2^-12 to 2^4.  A step with a page outside of that (wide) is a product of bf16 numbers, whose exponents do for any two scales; it takes three
// times as long: with the first 128 keys' pages 2^6 narrower than all others 4,096 tokens behind 32,768, 64/8 heads of 128, 12.2 ms instead of 4.0,
// 16 ragged prompts 5.07 instead of 1.85.  So P is the softmax's own, 2^(y - m), m at least 7
// and at most 15 below the row's largest score y so far in log2 units: off by 2^-11 of itself or by 2^-32 of the largest (2^-8 of itself in bf16).
// Where not all rows see all of a step's keys, and in every step done in bf16 (whose conversion knows no NaN), a NaN code of V is 0 for the
// product; the first key that has one is kept per element, and the epilogue makes the element of the rows that see it NaN.
// What bounds it is the power limit: 4,096 tokens behind 32,768, 64/8 heads of 128, 3.5 ms by itself (1,340 TFLOP/s), 4.1 ms one call after the
// other (1,140; the bf16 cache's kernel 3.25 and 3.7; the operations at the measured rates 2.75 and 3.3).  16 ragged prompts, 32/8 heads: 1.92 ms
// against 1.69 (1.98 on a GPU that keeps lower clocks, and 4.24 for the 4.1).
// Up to there it was the fetching of instructions: an SM's scheduler runs the softmax's loop of some 480
// instructions, the conversion's and an issuer's side by side, and what does not fit its instruction cache comes late.  So the issuers' loops,
// the conversion's and the producer's are rolled up and have one place each for what they do (issuers 2,700 -> 2,040 us for half as many tokens, the
// producer 2,010, warp 15 1,985), and steps that want bf16 take their scores in short loops.  What a tile does once is late in any case: Q's
// conversion took 4 to 7 us as straight code and takes 2 a half as a loop, the last step's mask 3 (in tensor memory, in a loop, it would take
// 1, but that code costs every step 3 %), the epilogue 3.
// Tensor memory: S [0,128)  P_A [128,192)  P_B [192,256)  O_A [256,256+D)  O_B [384,384+D).
// All mbarrier waits are bounded; on expiry the CTA raises its abort flag, every role drains, TMEM is freed and
// WPP_ERR_TIMEOUT is written to the status word.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_kv8.cuh"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace kv8tiles {
using namespace wpp;

constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512, kColS = 0;
__host__ __device__ constexpr uint32_t col_p(int hf) { return 128u + 64u * hf; }
__host__ __device__ constexpr uint32_t col_o(int hf) { return 256u + 128u * hf; }
// Registers of a thread by role.  4,096 tokens behind 32,768, one call after the other, and 16 ragged prompts, us: 184, 96, 48 4,178 and 1,925;
// 192, 80, 48 4,164 and 1,905; so 4,101 and 1,885; 208, 56, 40 4,112 and 1,917 (kTop 0).
constexpr int kRegsSoftmax = 200, kRegsCodes = 64, kRegsUtil = 48;
static_assert(8 * kRegsSoftmax + 4 * kRegsCodes + 4 * kRegsUtil <= 2048, "register file exceeded");
// log2 of a row's largest p when its reference is moved, and when it has to be.  (Moves are dear: all 32 rows of a warp wait for the product
// before and take O through registers.  16 ragged prompts with scores of deviation 1.3: kTop 7 1,920 us, 4 1,899, 0 1,892.  But f16 numbers end
// 2^25 below 1, and what a key far above all others leaves to them, each less than that, may be all that its own value does not outweigh.)
constexpr float kTop = 7.f, kMost = 15.f;
constexpr int kScaleDown = -12, kScaleUp = 4;      // log2 of vs / v that f16 numbers take
constexpr int kPar = 4;                    // key steps of a half whose scales are held
constexpr int kNan = 8;                    // tiles whose first NaN codes of V are held

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = 128 * D * 2, kHalfBytes = 128 * 128;     // bf16: a half of Q, a step of V
    static constexpr int kCodeBytes = 128 * D;                                 // a step of K or V as codes
    static constexpr int kStages = D == 128 ? 2 : 4;                           // of K's ring and of that of V's codes
    static constexpr int kOffV = 2 * kTileBytes, kOffK = kOffV + 2 * kTileBytes, kOffRaw = kOffK + kStages * kCodeBytes;
    static constexpr int kOffStage = kOffRaw + kStages * kCodeBytes;           // 8 x 2 KB
    static constexpr int kOffPar = kOffStage + 8 * 2048;               // float [2][kPar][12], a ring for each half: of 16 keys each: K's scale; whether P is bf16; log2 v
    static constexpr int kOffVPar = kOffPar + 2 * kPar * 48;           // int [kStages][12]: log2 of vs / v of 16 keys each, whether that wants bf16; int [2]: so of V's tiles
    static constexpr int kOffDown = kOffVPar + kStages * 48 + 16;      // float [2][2][128]: what Q's rows were multiplied by, inverse, by tile parity and half
    static constexpr int kOffNan = kOffDown + 2 * 2 * 128 * 4;         // int [kNan][D]: first key whose code of V is NaN; int [kNan]: first of all
    static constexpr int kOffBars = kOffNan + kNan * (D + 1) * 4;
    static constexpr int kTileQ = 2;
    static constexpr int kNumBars = 3 + 4 * kStages + 4 + 2 * kPar + 1 + 5 * 2 + 2 * kTileQ;
    static constexpr int kOffMisc = kOffBars + 8 * kNumBars;           // tmem address, abort flag, tile ids
    static constexpr int kSmemBytes = kOffMisc + 8 + 4 * kTileQ + 1024;
    static_assert(kOffBars % 8 == 0, "barriers");
    static_assert(kSmemBytes <= 232448, "more shared memory than a CTA can have");
};

struct Ring {
    uint32_t stage, phase;
    __device__ __forceinline__ void advance(uint32_t n) {
        if (++stage == n) { stage = 0; phase ^= 1u; }
    }
};

struct UnitView {
    int request, kv_begin, n_steps, n[2], P, kv_len, q_off;
    bool mismatch;
};
__device__ __forceinline__ UnitView view_of(const WppUnit& un, const Kv4AttnParams& p, const int32_t* q_offsets, const int32_t* plan_prefix) {
    UnitView v;
    v.request = un.request;
    v.kv_begin = un.kv_begin;
    v.P = p.prefix_lens[un.request];
    const int C = p.chunk_lens[un.request];
    v.kv_len = v.P + C;
    v.q_off = q_offsets[un.request];
    v.mismatch = (v.P != plan_prefix[un.request]) || (C != q_offsets[un.request + 1] - v.q_off);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int end = (un.rows[h] > 0 && !v.mismatch) ? (v.P + un.row0[h] + un.rows[h] + 127) / 128 : 0;
        v.n[h] = max(0, min(un.kv_end, end) - un.kv_begin);
    }
    v.n_steps = max(v.n[0], v.n[1]);
    return v;
}

// Two codes of a word (bytes 0 and 1, or 2 and 3) as bf16 numbers, exact; a NaN code comes out as 480.  An e4m3 number's bits, its sign
// apart, are a bf16 number's of 2^-120 times its size.
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t codes_bf16x2(uint32_t w, bool high) {
    const uint32_t x = __byte_perm(w, 0u, high ? 0x3322 : 0x1100);
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "r"(0x80008000u), "r"((x >> 4) & 0x07f007f0u));
    return mul_bf16x2(r, 0x7b807b80u);                                 // 2^120
}
// bits 7, 15, 23, 31: which of the four codes are NaN
__device__ __forceinline__ uint32_t nan_bits(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

__device__ __forceinline__ void st_shared_16(uint32_t at, uint4 y) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w) : "memory");
}

// D[tmem] (+)= A[smem] * B[smem], 128 x 128 x 32, e4m3 in, fp32 out
__device__ __forceinline__ void mma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Eight scores from tensor memory, a x - m, those above the limit -infinity; returns the largest
__device__ __forceinline__ float wide_scores(uint32_t taddr, float a, int limit, float m, float* y) {
    tmem_ld8(taddr, reinterpret_cast<uint32_t*>(y));
    tmem_wait_ld();
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = i > limit ? -INFINITY : fmaf(a, y[i], -m);
        most = fmaxf(most, y[i]);
    }
    return most;
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

// Instruction descriptor: e4m3 x e4m3 -> fp32, M = 128, both factors K-major (types 0 are e4m3; see idesc_bf16)
constexpr uint32_t kIdescE4m3 = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
// K's tiles: rows of 128 bytes with the 128-byte swizzle, or of 64 with the 64-byte one (layout 4; groups of 8 rows are 512 bytes apart)
template <int D>
__device__ __forceinline__ uint64_t k_desc(uint32_t saddr) {
    if constexpr (D == 128) return smem_desc_sw128(saddr, 16, 1024);
    return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (1ull << 16) | (static_cast<uint64_t>(512 >> 4) << 32) | (1ull << 46) | (4ull << 61);
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
wpp_kv8_tiles_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_q64, const __grid_constant__ CUtensorMap tm_q32,
                     const __grid_constant__ CUtensorMap tm_q16, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const Kv4AttnParams p) {
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    const uint32_t sQ = smem_base, sV = smem_base + C::kOffV, sK = smem_base + C::kOffK, sRaw = smem_base + C::kOffRaw, bars = smem_base + C::kOffBars;
    const uint32_t bQFull = bars, bQReady = bars + 8, bQEmpty = bars + 16;
    // k_full, raw_full: the codes of K and of V by TMA and their scales by warp 15; v: V's numbers
    const uint32_t bKFull = bars + 24, bKEmpty = bKFull + 8 * C::kStages, bRawFull = bKEmpty + 8 * C::kStages, bRawEmpty = bRawFull + 8 * C::kStages;
    const uint32_t bVFull = bRawEmpty + 8 * C::kStages, bVEmpty = bVFull + 16, bParEmpty = bVEmpty + 16;
    const uint32_t bSFree = bParEmpty + 16 * kPar, bHalf = bSFree + 8;
    auto bSFull = [&](int h) { return bHalf + 40 * h; };
    auto bPReady = [&](int h) { return bHalf + 40 * h + 8; };
    auto bPFree = [&](int h) { return bHalf + 40 * h + 16; };
    auto bOFinal = [&](int h) { return bHalf + 40 * h + 24; };
    auto bOFree = [&](int h) { return bHalf + 40 * h + 32; };
    const uint32_t bTileFull = bHalf + 80, bTileEmpty = bTileFull + 8 * C::kTileQ;
    float* s_par = reinterpret_cast<float*>(smem_gen + C::kOffPar);
    int32_t* s_vpar = reinterpret_cast<int32_t*>(smem_gen + C::kOffVPar);
    volatile int32_t* s_wide = s_vpar + C::kStages * 12;
    float* s_down = reinterpret_cast<float*>(smem_gen + C::kOffDown);
    int32_t* s_nan = reinterpret_cast<int32_t*>(smem_gen + C::kOffNan);
    int32_t* s_nan_any = s_nan + kNan * D;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_gen + C::kOffMisc);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    volatile int32_t* tile_ids = reinterpret_cast<volatile int32_t*>(tmem_slot + 2);
    constexpr uint32_t kTileConsumers = 2 + 256 + 128 + 32;      // two issuing threads, softmax, codes, scales
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wg = warp >> 2;

    if (threadIdx.x == 0) {
        mbar_init(bQFull, 1); mbar_init(bQReady, 128); mbar_init(bQEmpty, 1);
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(bKFull + 8 * s, 2); mbar_init(bKEmpty + 8 * s, 1); mbar_init(bRawFull + 8 * s, 2); mbar_init(bRawEmpty + 8 * s, 128);
        }
        for (int s = 0; s < 2; ++s) { mbar_init(bVFull + 8 * s, 128); mbar_init(bVEmpty + 8 * s, 1); }
        for (int s = 0; s < 2 * kPar; ++s) mbar_init(bParEmpty + 8 * s, 4);
        mbar_init(bSFree, 128);
        for (int h = 0; h < 2; ++h) {
            mbar_init(bSFull(h), 1); mbar_init(bPReady(h), 128); mbar_init(bPFree(h), 1); mbar_init(bOFinal(h), 1); mbar_init(bOFree(h), 128);
        }
        for (int i = 0; i < C::kTileQ; ++i) { mbar_init(bTileFull + 8 * i, 1); mbar_init(bTileEmpty + 8 * i, kTileConsumers); }
        *abort_flag = 0u;
        fence_barrier_init();
    }
    for (int i = threadIdx.x; i < kNan * (D + 1); i += kThreads) s_nan[i] = 0x7fffffff;
    if (warp == 12) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
        tmem_relinquish();
    }
    if (warp == 13 && lane == 0) {
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_q64); prefetch_tensormap(&tm_q32); prefetch_tensormap(&tm_q16);
        prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_launch_dependents();
    grid_dependency_wait();

    const char* plan = static_cast<const char*>(p.plan);
    const int32_t* q_offsets = reinterpret_cast<const int32_t*>(plan + p.off_q_offsets);
    const int32_t* plan_prefix = reinterpret_cast<const int32_t*>(plan + p.off_prefix);
    const WppUnit* units = reinterpret_cast<const WppUnit*>(plan + p.off_units) + p.first_tile;
    const int num_units = p.num_tiles;
    Ring tile_ring = {0, 0};
    auto next_tile = [&]() -> int {        // -1 = no more tiles, -2 = the wait was abandoned
        if (!mbar_wait(bTileFull + 8 * tile_ring.stage, tile_ring.phase, abort_flag)) return -2;
        const int id = tile_ids[tile_ring.stage];
        mbar_arrive(bTileEmpty + 8 * tile_ring.stage);
        tile_ring.advance(C::kTileQ);
        return id;
    };
    const int page_shift = 31 - __clz(p.page_size), ppt = 128 >> page_shift;       // ppt: pages of a key step

    if (wg == 3) {
        setmaxnreg_dec<kRegsUtil>();
        if (warp == 13) {
            // ================================================================ tiles, Q, and the codes of K and V
            Ring ring_k = {0, 0}, ring_v = {0, 0};
            uint32_t q_phase = 0;
            bool first = true, dead = false;
            while (!dead) {
                int u = (int)blockIdx.x;
                if (!first) {
                    if (lane == 0) u = p.tile_counter ? (int)(gridDim.x + atomicAdd(p.tile_counter, 1u)) : num_units;
                    u = __shfl_sync(0xffffffffu, u, 0);
                }
                first = false;
                if (u >= num_units) u = -1;
                {
                    const bool ok = mbar_wait(bTileEmpty + 8 * tile_ring.stage, tile_ring.phase ^ 1u, abort_flag);
                    if (!__all_sync(0xffffffffu, ok)) break;
                    if (lane == 0) {
                        tile_ids[tile_ring.stage] = u;
                        mbar_arrive(bTileFull + 8 * tile_ring.stage);
                    }
                    tile_ring.advance(C::kTileQ);
                }
                if (u < 0) break;
                const WppUnit un = units[u];
                const UnitView v = view_of(un, p, q_offsets, plan_prefix);
                if (v.mismatch && lane == 0 && p.status) atomicCAS(p.status, 0, WPP_ERR_PLAN_MISMATCH);
                if (v.n_steps == 0) continue;
                const int kvh = un.head[0] / p.group, n_pages = (v.kv_len + p.page_size - 1) >> page_shift;
                const int32_t* bt = p.block_tables + (int64_t)un.request * p.max_blocks;
                // K(0) (only needs a place in the ring, which is free before the tile before's Q is), Q, K(1), V(0), K(2), V(1), ..: one place in the
                // code for them all
                bool ok = true;
                for (int i = 0; i < 2 * v.n_steps && ok; ++i) {
                    const bool is_v = i == 2 * v.n_steps - 1 || (i > 0 && (i & 1) == 0);
                    const int step = is_v ? i == 2 * v.n_steps - 1 ? v.n_steps - 1 : i / 2 - 1 : (i + 1) / 2;
                    if (i == 1) {
                        ok = __all_sync(0xffffffffu, mbar_wait(bQEmpty, q_phase ^ 1u, abort_flag));
                        if (!ok) break;
                        q_phase ^= 1u;
                        if (lane == 0) mbar_arrive_expect_tx(bQFull, ((v.n[0] > 0) + (v.n[1] > 0)) * C::kTileBytes);
                        __syncwarp();
                        const int rph = 128 / un.pack;
                        const CUtensorMap* qm = un.pack == 1 ? &tm_q : un.pack == 2 ? &tm_q64 : un.pack == 4 ? &tm_q32 : &tm_q16;
                        const int per_half = un.pack * C::kHalves;
#pragma unroll 1
                        for (int b = lane; b < 2 * per_half; b += 32) {
                            const int hf = b / per_half, k = (b % per_half) / C::kHalves, h = b % C::kHalves;
                            if ((hf ? v.n[1] : v.n[0]) == 0) continue;
                            // (more places than heads in the group: the last head again, into rows that nobody stores)
                            tma_load_3d(sQ + hf * C::kTileBytes + h * C::kHalfBytes + k * rph * 128, qm, bQFull, h * 64,
                                        (hf ? un.head[1] : un.head[0]) + min(k, p.group - 1), v.q_off + (hf ? un.row0[1] : un.row0[0]));
                        }
                        __syncwarp();
                    }
                    // a step's codes of K or of V: a lane for each page
                    const int page0 = (v.kv_begin + step) * ppt, cnt = min(ppt, n_pages - page0);
                    int pid = 0;
                    if (lane < cnt) pid = bt[page0 + lane];
                    if (pid < 0 || pid >= p.num_pages) {
                        if (p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
                        pid = 0;
                    }
                    const Ring ring = is_v ? ring_v : ring_k;
                    const uint32_t full = (is_v ? bRawFull : bKFull) + 8 * ring.stage, empty = (is_v ? bRawEmpty : bKEmpty) + 8 * ring.stage;
                    ok = __all_sync(0xffffffffu, mbar_wait(empty, ring.phase ^ 1u, abort_flag));
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(full, (uint32_t)(cnt * p.page_size * D));
                    __syncwarp();
                    if (lane < cnt)
                        tma_load_4d((is_v ? sRaw : sK) + ring.stage * C::kCodeBytes + lane * p.page_size * D, is_v ? &tm_v : &tm_k, full, 0, 0, kvh, pid);
                    if (is_v) ring_v.advance(C::kStages);
                    else ring_k.advance(C::kStages);
                }
                dead = !ok;
            }
        } else if (warp == 15) {
            // ================================================================ the scales of a step's pages, asked for a step ahead
            Ring ring_k = {0, 0}, ring_v = {0, 0}, ring_p[2] = {{0, 0}, {0, 0}};
            bool dead = false;
            while (!dead) {
                const int u = next_tile();
                if (!__all_sync(0xffffffffu, u != -2) || u < 0) break;
                const WppUnit un = units[u];
                const UnitView v = view_of(un, p, q_offsets, plan_prefix);
                if (v.n_steps == 0) continue;
                const int kvh = un.head[0] / p.group, group = lane & 7;
                const int32_t* bt = p.block_tables + (int64_t)un.request * p.max_blocks;
                const uint8_t* pool = (lane & 8 ? p.v_cache : p.k_cache) + kvh * p.head_bytes + p.page_size * D;
                auto scale_of = [&](int k) -> float {                  // lanes 0 to 7: K's, of the step's groups of 16 keys; 8 to 15: V's; 0: no such key
                    const int key = (v.kv_begin + k) * 128 + group * 16;
                    if (lane >= 16 || k >= v.n_steps || key >= v.kv_len) return 0.f;
                    const int pid = bt[key >> page_shift];
                    return *reinterpret_cast<const float*>(pool + (pid < 0 || pid >= p.num_pages ? 0 : pid) * p.page_bytes);
                };
                // K(0), then K(k + 1) and V(k), the order in which the codes are asked for
                float next = scale_of(0), after = scale_of(1);
                int v_exp = 0, apart = 0, wide = 0, apart_v = 0, wide_v = 0;       // log2 v; log2 vs / v, and whether that wants bf16; the same of the step before
                for (int k = 0; k <= v.n_steps; ++k) {
                    bool ok = true;
                    apart_v = apart;
                    wide_v = wide;
                    if (k < v.n_steps) {
                        const float mine = next, vs = __shfl_sync(0xffffffffu, mine, 8 + group);
                        next = after;
                        after = scale_of(k + 2);
                        if (k == 0) v_exp = (int)__reduce_max_sync(0xffffffffu, (uint32_t)(vs == 0.f ? 0 : exponent_of(vs) + 128)) - 128;
                        apart = vs == 0.f ? 0 : min(max(exponent_of(vs) - v_exp, -100), 100);
                        wide = __any_sync(0xffffffffu, apart < kScaleDown || apart > kScaleUp);
                        ok = mbar_wait(bKEmpty + 8 * ring_k.stage, ring_k.phase ^ 1u, abort_flag);
#pragma unroll 1
                        for (int h = 0; h < 2; ++h) {
                            if (k >= (h ? v.n[1] : v.n[0])) continue;
                            const Ring ring = h ? ring_p[1] : ring_p[0];
                            const int at = h * kPar + (int)ring.stage;
                            ok = ok && mbar_wait(bParEmpty + 8 * at, ring.phase ^ 1u, abort_flag);
                            if (ok && lane < 10) s_par[at * 12 + lane] = lane < 8 ? (mine == 0.f ? 1.f : mine) : (float)(lane == 8 ? wide : v_exp);
                            if (h) ring_p[1].advance(kPar);
                            else ring_p[0].advance(kPar);
                        }
                        if (!__all_sync(0xffffffffu, ok)) { dead = true; break; }
                        __syncwarp();                                  // (a vote orders no memory: all lanes' entries before lane 0's arrival)
                        if (lane == 0) mbar_arrive(bKFull + 8 * ring_k.stage);
                        ring_k.advance(C::kStages);
                    }
                    if (k > 0) {
                        ok = mbar_wait(bRawEmpty + 8 * ring_v.stage, ring_v.phase ^ 1u, abort_flag);
                        if (ok && lane < 8) s_vpar[ring_v.stage * 12 + lane] = apart_v;
                        if (ok && lane == 8) s_vpar[ring_v.stage * 12 + 8] = wide_v;
                        if (!__all_sync(0xffffffffu, ok)) { dead = true; break; }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bRawFull + 8 * ring_v.stage);
                        ring_v.advance(C::kStages);
                    }
                }
            }
        } else if (warp == 12 && lane == 0) {
            // ================================================================ issuer of S = Q K^T
            Ring ring = {0, 0};
            uint32_t q_phase = 0, sfree_phase = 0;
            const uint64_t q_desc0 = smem_desc_sw128(sQ, 16, 1024), k_desc0 = k_desc<D>(sK);
            const uint32_t tS = tmem + kColS;
            bool dead = false;
            while (!dead) {
                const int u = next_tile();
                if (u < 0) break;
                const WppUnit un = units[u];
                const UnitView v = view_of(un, p, q_offsets, plan_prefix);
                if (v.n_steps == 0) continue;
                if (!mbar_wait(bQReady, q_phase, abort_flag)) break;
                q_phase ^= 1u;
                for (int k = 0; k < v.n_steps && !dead; ++k) {
                    if (!mbar_wait(bKFull + 8 * ring.stage, ring.phase, abort_flag)) { dead = true; break; }
                    const uint64_t kd = k_desc0 + (uint64_t)(ring.stage * (C::kCodeBytes >> 4));
#pragma unroll 1
                    for (int hf = 0; hf < 2; ++hf) {
                        if (k >= (hf ? v.n[1] : v.n[0])) continue;
                        if (!mbar_wait(bSFree, sfree_phase ^ 1u, abort_flag)) { dead = true; break; }
                        sfree_phase ^= 1u;
                        tc_fence_after();
                        const uint64_t qd = q_desc0 + (uint64_t)(hf * (C::kTileBytes >> 4));
#pragma unroll 1
                        for (int kk = 0; kk < D / 32; ++kk) {
                            const uint64_t hi = qd + (uint64_t)((kk >> 1) * (C::kHalfBytes >> 4) + (kk & 1) * 4);
                            mma_e4m3(tS, hi, kd + kk * 2, kIdescE4m3, kk > 0);
                            mma_e4m3(tS, hi + 2, kd + kk * 2, kIdescE4m3, 1u);
                        }
                        mma_commit(bSFull(hf));
                    }
                    if (dead) break;
                    mma_commit(bKEmpty + 8 * ring.stage);
                    ring.advance(C::kStages);
                }
                if (!dead) mma_commit(bQEmpty);
            }
        } else if (warp == 14 && lane == 0) {
            // ================================================================ issuer of O += P V
            Ring ring = {0, 0};
            uint32_t p_phase[2] = {0, 0}, of_phase[2] = {0, 0};
            constexpr uint32_t kIdescBf16 = idesc_bf16(D, 0, 1), kIdescF16 = kIdescBf16 & ~((1u << 7) | (1u << 10));       // (types 0 are f16)
            const uint64_t v_desc0 = smem_desc_sw128(sV, C::kHalfBytes, 1024);
            bool dead = false;
            while (!dead) {
                const int u = next_tile();
                if (u < 0) break;
                const WppUnit un = units[u];
                const UnitView v = view_of(un, p, q_offsets, plan_prefix);
                if (v.n_steps == 0) continue;
                for (int k = 0; k < v.n_steps && !dead; ++k) {
                    if (!mbar_wait(bVFull + 8 * ring.stage, ring.phase, abort_flag)) { dead = true; break; }
                    const uint64_t vd = v_desc0 + (uint64_t)(ring.stage * (C::kTileBytes >> 4));
                    const uint32_t idesc_pv = s_wide[ring.stage] ? kIdescBf16 : kIdescF16;
#pragma unroll 1
                    for (int hf = 0; hf < 2; ++hf) {
                        const int n = hf ? v.n[1] : v.n[0];
                        if (k >= n) continue;
                        if (!mbar_wait(bPReady(hf), hf ? p_phase[1] : p_phase[0], abort_flag)) { dead = true; break; }
                        if (hf) p_phase[1] ^= 1u; else p_phase[0] ^= 1u;
                        if (k == 0) {          // the tile before's O has been read
                            if (!mbar_wait(bOFree(hf), (hf ? of_phase[1] : of_phase[0]) ^ 1u, abort_flag)) { dead = true; break; }
                            if (hf) of_phase[1] ^= 1u; else of_phase[0] ^= 1u;
                        }
                        tc_fence_after();
                        const uint32_t tP = tmem + col_p(hf), tO = tmem + col_o(hf);
#pragma unroll 1
                        for (int kk = 0; kk < 8; ++kk) mma_ts(tO, tP + kk * 8, vd + (uint64_t)(kk * 128), idesc_pv, (k | kk) > 0);
                        mma_commit(bPFree(hf));
                        if (k + 1 == n) mma_commit(bOFinal(hf));
                    }
                    if (dead) break;
                    mma_commit(bVEmpty + 8 * ring.stage);
                    ring.advance(2);
                }
            }
        }
    } else if (wg == 2) {
        // ================================================================ Q as two terms, V's codes as f16 (in wide steps as bf16)
        setmaxnreg_dec<kRegsCodes>();
        constexpr int kChunks = D / 16, kApart = 32 / kChunks;         // 16-byte pieces of a row of codes; rows of a warp at a time
        const int r = threadIdx.x & 127, c = lane % kChunks, row0 = (warp & 3) * 32 + lane / kChunks;
        const bool swap = D == 128 && (c & 4);         // of lanes 4 apart, whose numbers would meet in a bank, one begins with its second half
        // where the two pieces of 8 numbers go in the tile's first row of this thread; kApart rows on it is the same place but for a turned bit
        uint32_t place[2];
#pragma unroll
        for (int q = 0; q < 2; ++q)
            place[q] = (uint32_t)((c >> 2) * C::kHalfBytes + row0 * 128 + ((((c & 3) * 2 + (q ^ (swap ? 1 : 0))) ^ (row0 & 7)) << 4));
        Ring ring_raw = {0, 0}, ring_v = {0, 0};
        uint32_t q_phase = 0, tiles = 0;               // tiles: with work, so far
        bool dead = false;
        while (!dead) {
            const int u = next_tile();
            if (!__all_sync(0xffffffffu, u != -2) || u < 0) break;
            const WppUnit un = units[u];
            const UnitView v = view_of(un, p, q_offsets, plan_prefix);
            if (v.n_steps == 0) continue;
            const int nan_slot = tiles % kNan;
            // the place of four tiles on: nobody is so far behind that it reads the one of four tiles ago, nor so far ahead
            if (r < D) s_nan[(tiles + kNan / 2) % kNan * D + r] = 0x7fffffff;
            if (r == 0) s_nan_any[(tiles + kNan / 2) % kNan] = 0x7fffffff;
            // ---- Q (thread = row): hi into the places of the row's first elements, lo behind it, once all have been read
            if (!__all_sync(0xffffffffu, mbar_wait(bQFull, q_phase, abort_flag))) break;
            q_phase ^= 1u;
#pragma unroll 1
            for (int hf = 0; hf < 2; ++hf) {
                if (v.n[hf] == 0) continue;
                uint8_t* const row = smem_gen + hf * C::kTileBytes + r * 128;
                auto numbers = [&](int ch) { return *reinterpret_cast<const uint4*>(row + (ch >> 3) * C::kHalfBytes + (((ch & 7) ^ (r & 7)) << 4)); };
                float top = 0.f;
#pragma unroll 4
                for (int ch = 0; ch < D / 8; ++ch) {
                    const uint4 z = numbers(ch);
                    const uint32_t w[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
                }
                // 2^e and 2^-e, both normal numbers; an infinity makes the row NaN
                const int biased = (int)(__float_as_uint(top) >> 23), e = min(max(134 - biased, -119), 126);
                const float up = biased == 255 ? NAN : power_of_two(e);
                s_down[((tiles & 1) * 2 + hf) * 128 + r] = power_of_two(-e);
                // 32 elements at a time, whose two terms take the place of their numbers (a short loop: see above)
#pragma unroll 1
                for (int b = 0; b < D / 32; ++b) {
                    uint8_t* const part = row + (b >> 1) * C::kHalfBytes;
                    const int piece = 4 * (b & 1);
                    uint4 z0 = numbers(4 * b), z1 = numbers(4 * b + 1);
                    const uint4 z2 = numbers(4 * b + 2), z3 = numbers(4 * b + 3);
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint4 z = k < 2 ? z0 : z1;
                            const uint32_t w0 = k & 1 ? z.z : z.x, w1 = k & 1 ? z.w : z.y;
                            const float x0 = __uint_as_float(w0 << 16) * up, x1 = __uint_as_float(w0 & 0xffff0000u) * up;
                            const float x2 = __uint_as_float(w1 << 16) * up, x3 = __uint_as_float(w1 & 0xffff0000u) * up;
                            const uint16_t c0 = codes_of(x0, x1), c1 = codes_of(x2, x3);
                            const uint32_t f0 = codes_f16x2(c0), f1 = codes_f16x2(c1);
                            hi[k] = (uint32_t)c0 | (uint32_t)c1 << 16;
                            lo[k] = (uint32_t)codes_of(x0 - f16_low(f0), x1 - f16_high(f0)) | (uint32_t)codes_of(x2 - f16_low(f1), x3 - f16_high(f1)) << 16;
                        }
                        *reinterpret_cast<uint4*>(part + (((piece + i) ^ (r & 7)) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        *reinterpret_cast<uint4*>(part + (((piece + 2 + i) ^ (r & 7)) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                        z0 = z2;
                        z1 = z3;
                    }
                }
            }
            fence_proxy_async_smem();
            mbar_arrive(bQReady);
            ++tiles;
            // ---- V.  Where some rows do not see all keys: NaN codes, and rows behind the sequence, which are zeros.  NaN codes in wide steps too,
            //      whoever sees them: their conversion would make numbers of them
            const int all_see = min(v.n[0] > 0 ? v.P + un.row0[0] : 0x7fffffff, v.n[1] > 0 ? v.P + un.row0[1] : 0x7fffffff);       // the last key that every row sees
            for (int k = 0; k < v.n_steps; ++k) {
                bool ok = mbar_wait(bRawFull + 8 * ring_raw.stage, ring_raw.phase, abort_flag);
                ok = ok && mbar_wait(bVEmpty + 8 * ring_v.stage, ring_v.phase ^ 1u, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { dead = true; break; }
                uint8_t* const from = smem_gen + C::kOffRaw + ring_raw.stage * C::kCodeBytes + row0 * D + c * 16;
                const uint32_t to = sV + ring_v.stage * C::kTileBytes;
                const int key0 = (v.kv_begin + k) * 128;
                const int32_t* vp = s_vpar + ring_raw.stage * 12;
                const int apart[2] = {vp[2 * (warp & 3)], vp[2 * (warp & 3) + 1]};      // of the warp's first and last 16 rows
                const bool wide = vp[8] != 0;
                if (r == 0) s_wide[ring_v.stage] = wide;
                if (__builtin_expect(wide || key0 + 127 > all_see, 0)) {
                    const int rows = v.kv_len - key0;
#pragma unroll 1
                    for (int i = 0; i < kChunks; ++i) {
                        const int row = row0 + i * kApart;
                        uint4* const at = reinterpret_cast<uint4*>(from + i * kApart * D);
                        const uint4 x = *at;
                        uint32_t w[4] = {x.x, x.y, x.z, x.w};
                        if (row >= rows) {
                            *at = make_uint4(0, 0, 0, 0);
                        } else if (nan_bits(w[0]) | nan_bits(w[1]) | nan_bits(w[2]) | nan_bits(w[3])) {
#pragma unroll 1
                            for (int b = 0; b < 16; ++b) {
                                const uint32_t word = b < 4 ? w[0] : b < 8 ? w[1] : b < 12 ? w[2] : w[3];
                                if ((word >> (8 * (b & 3)) & 0x7fu) == 0x7fu) {
                                    atomicMin(&s_nan[nan_slot * D + c * 16 + b], key0 + row);
                                    atomicMin(&s_nan_any[nan_slot], key0 + row);
                                }
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) w[j] &= ~((nan_bits(w[j]) >> 7) * 0xffu);
                            *at = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                }
                if (__builtin_expect(!wide, 1)) {
                    // (a row at a time, the next one's codes under way, and the loop short: see above)
                    const uint8_t* const first = from + (swap ? 8 : 0);
                    const uint8_t* const second = from + (swap ? 0 : 8);
                    uint2 x0 = *reinterpret_cast<const uint2*>(first), x1 = *reinterpret_cast<const uint2*>(second);
                    uint32_t turned = 0u, times = (uint32_t)(15 + apart[0]) * 0x04000400u;                 // a power of two, as f16, twice
                    uint32_t at0 = to + place[0], at1 = to + place[1];
#pragma unroll 1
                    for (int i = 0; i < kChunks; ++i) {
                        const uint32_t w[4] = {x0.x, x0.y, x1.x, x1.y};
                        if (i + 1 < kChunks) {
                            x0 = *reinterpret_cast<const uint2*>(first + (i + 1) * kApart * D);
                            x1 = *reinterpret_cast<const uint2*>(second + (i + 1) * kApart * D);
                        }
                        if (i == kChunks / 2) times = (uint32_t)(15 + apart[1]) * 0x04000400u;
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = mul_f16x2(j & 1 ? codes_f16x2_high(w[j >> 1]) : codes_f16x2_low(w[j >> 1]), times);
                        st_shared_16(at0 ^ turned, make_uint4(y[0], y[1], y[2], y[3]));
                        st_shared_16(at1 ^ turned, make_uint4(y[4], y[5], y[6], y[7]));
                        at0 += kApart * 128;
                        at1 += kApart * 128;
                        if (kApart == 4) turned ^= 64u;
                    }
                } else {
#pragma unroll 1
                    for (int i = 0; i < 2 * kChunks; ++i) {            // (half a piece at a time)
                        const int row = i >> 1, q = i & 1;
                        const uint32_t up = (uint32_t)(127 + (row < kChunks / 2 ? apart[0] : apart[1])) * 0x00800080u;
                        const uint2 x = *reinterpret_cast<const uint2*>(from + row * kApart * D + ((q != 0) != swap ? 8 : 0));
                        st_shared_16(to + ((place[q] + row * kApart * 128) ^ (kApart == 4 ? (uint32_t)(row & 1) << 6 : 0u)),
                                     make_uint4(mul_bf16x2(codes_bf16x2(x.x, false), up), mul_bf16x2(codes_bf16x2(x.x, true), up),
                                                mul_bf16x2(codes_bf16x2(x.y, false), up), mul_bf16x2(codes_bf16x2(x.y, true), up)));
                    }
                }
                fence_proxy_async_smem();
                mbar_arrive(bVFull + 8 * ring_v.stage);
                mbar_arrive(bRawEmpty + 8 * ring_raw.stage);
                ring_raw.advance(C::kStages);
                ring_v.advance(2);
            }
        }
    } else {
        // ================================================================ softmax (thread = query row of half `hf`) and epilogue
        setmaxnreg_inc<kRegsSoftmax>();
        const int hf = wg, r = threadIdx.x & 127;
        const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        uint32_t s_phase = 0, pf_phase = 0, of_phase = 0, par = 0, tiles = 0;
        bool dead = false;
        while (!dead) {
            const int u = next_tile();
            if (!__all_sync(0xffffffffu, u != -2) || u < 0) break;
            const WppUnit un = units[u];
            const UnitView v = view_of(un, p, q_offsets, plan_prefix);
            const int n = v.n[hf];
            const int rph = 128 / un.pack, rr = r & (rph - 1);         // row inside its head's block
            const bool row_ok = un.rows[hf] > 0 && rr < un.rows[hf] && r / rph < p.group;
            const int64_t prow = ((int64_t)un.split_slot * 2 + hf) * 128 + r;
            if (n == 0) {
                // a split part that lies wholly above this half's diagonal, or a refused request's: no key is visible
                if (un.split_slot >= 0 && row_ok) p.ws_lse[prow] = -INFINITY;
            }
            if (v.n_steps == 0) continue;
            const int first_pos = v.P + un.row0[hf], row_last = min(first_pos + rr, v.kv_len - 1);
            float m_ref = 0.f, l_run = 0.f, down = 0.f, unit = 0.f;       // down: of the row, scores in log2 units; unit: v, of the sums
            // the row's reference, where a score is `above` it by too much; O is rescaled once the product before has landed
            auto settle = [&](float above, int j, bool& waited) -> bool {
                const bool move = j == 0 || above > kMost;
                if (__builtin_expect(!__any_sync(0xffffffffu, move), 1)) return true;
                // how far it goes up (the first one may go down; a row that sees nothing keeps its)
                float y = j == 0 ? above - kTop : fmaxf(above - kTop, 0.f);
                if (y == -INFINITY) y = 0.f;
                const float alpha = j == 0 ? 1.f : fast_exp2(-y);
                m_ref += y;
                l_run *= alpha;
                if (j == 0) return true;
                if (!__all_sync(0xffffffffu, mbar_wait(bPFree(hf), pf_phase ^ 1u, abort_flag))) return false;
                pf_phase ^= 1u;
                waited = true;
                tc_fence_after();
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
                    for (int q0 = 0; q0 < D; q0 += 16) {
                        float o[16];
                        tmem_ld8(lane_addr + col_o(hf) + q0, reinterpret_cast<uint32_t*>(o));
                        tmem_ld8(lane_addr + col_o(hf) + q0 + 8, reinterpret_cast<uint32_t*>(o) + 8);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] *= alpha;
                        tmem_st8(lane_addr + col_o(hf) + q0, reinterpret_cast<uint32_t*>(o));
                        tmem_st8(lane_addr + col_o(hf) + q0 + 8, reinterpret_cast<uint32_t*>(o) + 8);
                    }
                }
                return true;
            };
            auto p_is_free = [&]() -> bool {           // P(j - 1) has been consumed
                if (!__all_sync(0xffffffffu, mbar_wait(bPFree(hf), pf_phase ^ 1u, abort_flag))) return false;
                pf_phase ^= 1u;
                tc_fence_after();
                return true;
            };
            for (int j = 0; j < n; ++j) {
                if (!__all_sync(0xffffffffu, mbar_wait(bSFull(hf), s_phase, abort_flag))) { dead = true; break; }
                s_phase ^= 1u;
                tc_fence_after();
                const float* pr = s_par + (hf * kPar + par) * 12;      // of 16 keys each: K's scale
                if (j == 0) {
                    // (at least 2^-90: no product of an infinity and 0, whatever K's scale, and below it all scores are 0 to fp32)
                    down = fmaxf(s_down[((tiles & 1) * 2 + hf) * 128 + r] * p.scale_log2, 8.077936e-28f);
                    unit = fast_exp2(pr[9]);
                }
                const int key0 = (v.kv_begin + j) * 128;
                bool waited = false;
                if (__builtin_expect(pr[8] != 0.f, 0)) {
                    // P as bf16: such steps are few, and take their scores twice, 8 at a time, in loops that cost no registers and little code
                    const int limit = row_last - key0;
                    float most = -INFINITY;
#pragma unroll 1
                    for (int i = 0; i < 128; i += 8) {
                        float y[8];
                        most = fmaxf(most, wide_scores(lane_addr + kColS + i, pr[i >> 4] * down, limit - i, 0.f, y));
                    }
                    if (!settle(most - m_ref, j, waited) || (!waited && !p_is_free())) { dead = true; break; }
#pragma unroll 1
                    for (int i = 0; i < 128; i += 8) {
                        float y[8];
                        wide_scores(lane_addr + kColS + i, pr[i >> 4] * down, limit - i, m_ref, y);
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = fast_exp2(y[k]);
                        l_run += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
                        const uint32_t two[4] = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
                        tmem_st4(lane_addr + col_p(hf) + i / 2, two);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bSFree);
                } else {
                    float s[128], most = -INFINITY;
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) tmem_ld32(lane_addr + kColS + q4 * 32, reinterpret_cast<uint32_t*>(s) + q4 * 32);
                    tmem_wait_ld();
                    tc_fence_before();
                    mbar_arrive(bSFree);
                    if (__builtin_expect(key0 + 127 > first_pos, 0)) {      // only steps that touch the diagonal are masked
                        const int limit = row_last - key0;
#pragma unroll
                        for (int i = 0; i < 128; ++i) s[i] = (i > limit) ? -INFINITY : s[i];
                    }
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const float* x = s + 16 * g;
                        const float m0 = fmax3(x[0], x[1], x[2]), m1 = fmax3(x[3], x[4], x[5]), m2 = fmax3(x[6], x[7], x[8]), m3 = fmax3(x[9], x[10], x[11]);
                        most = fmaxf(most, pr[g] * fmaxf(fmax3(fmax3(m0, m1, m2), fmax3(m3, x[12], x[13]), x[14]), x[15]));
                    }
                    if (!settle(fmaf(most, down, -m_ref), j, waited)) { dead = true; break; }
                    uint32_t* pk = reinterpret_cast<uint32_t*>(s);
                    const uint64_t nm2 = pack2(-m_ref, -m_ref);
                    uint64_t sum2a = pack2(0.f, 0.f), sum2b = pack2(0.f, 0.f);
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const float a = pr[g] * down;
                        const uint64_t a2 = pack2(a, a);
                        float e[16];
#pragma unroll
                        for (int k = 0; k < 8; ++k) unpack2(ffma2(pack2(s[16 * g + 2 * k], s[16 * g + 2 * k + 1]), a2, nm2), e[2 * k], e[2 * k + 1]);
#pragma unroll
                        for (int k = 0; k < 16; ++k) e[k] = fast_exp2(e[k]);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            if (k & 1) sum2b = fadd2(sum2b, pack2(e[2 * k], e[2 * k + 1]));
                            else sum2a = fadd2(sum2a, pack2(e[2 * k], e[2 * k + 1]));
                            pk[8 * g + k] = pack_f16x2(e[2 * k], e[2 * k + 1]);
                        }
                    }
                    float t0, t1;
                    unpack2(fadd2(sum2a, sum2b), t0, t1);
                    l_run += t0 + t1;
                    if (!waited && !p_is_free()) { dead = true; break; }
#pragma unroll
                    for (int c8 = 0; c8 < 64; c8 += 8) tmem_st8(lane_addr + col_p(hf) + c8, pk + c8);
                    tmem_wait_st();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bParEmpty + 8 * (hf * kPar + par));
                par = (par + 1) % kPar;
                mbar_arrive(bPReady(hf));
            }
            if (dead) break;
            const int nan_slot = tiles % kNan;
            ++tiles;
            if (n == 0) continue;
            // ---- epilogue
            if (!__all_sync(0xffffffffu, mbar_wait(bOFinal(hf), of_phase, abort_flag))) break;
            of_phase ^= 1u;
            tc_fence_after();
            const int64_t tok = (int64_t)v.q_off + un.row0[hf] + rr;
            const int head = un.head[hf] + r / rph;
            const bool nans = s_nan_any[nan_slot] <= row_last;         // of V: some elements of the row may be NaN
            const float inv_l = l_run > 0.f ? 1.f / l_run : l_run != l_run ? l_run : 0.f;
            const float lse2 = (l_run <= 0.f) ? -INFINITY : (m_ref + log2f(l_run));
            uint8_t* stage = smem_gen + C::kOffStage + warp * 2048;
            const bool split = un.split_slot >= 0;
            const __nv_bfloat16* dst = p.out + tok * p.o_token_stride + (int64_t)head * p.o_head_stride;
            const float* part = p.ws_o + prow * D;
#pragma unroll 1
            for (int q4 = 0; q4 < D / 32; ++q4) {
                float o[32];
                tmem_ld32(lane_addr + col_o(hf) + q4 * 32, reinterpret_cast<uint32_t*>(o));
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] *= inv_l * unit;
                uint4 w[4];
                if (!split) {
#pragma unroll
                    for (int w4 = 0; w4 < 4; ++w4)
                        w[w4] = make_uint4(pack_bf16x2(o[8 * w4], o[8 * w4 + 1]), pack_bf16x2(o[8 * w4 + 2], o[8 * w4 + 3]),
                                           pack_bf16x2(o[8 * w4 + 4], o[8 * w4 + 5]), pack_bf16x2(o[8 * w4 + 6], o[8 * w4 + 7]));
                    warp_store_rows64(stage, lane, w, dst, row_ok, q4 * 64);
                } else {
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
#pragma unroll
                        for (int w4 = 0; w4 < 4; ++w4)
                            w[w4] = make_uint4(__float_as_uint(o[16 * h2 + 4 * w4]), __float_as_uint(o[16 * h2 + 4 * w4 + 1]),
                                               __float_as_uint(o[16 * h2 + 4 * w4 + 2]), __float_as_uint(o[16 * h2 + 4 * w4 + 3]));
                        warp_store_rows64(stage, lane, w, part, row_ok, q4 * 128 + h2 * 64);
                    }
                }
            }
            tc_fence_before();
            mbar_arrive(bOFree(hf));
            if (__builtin_expect(__any_sync(0xffffffffu, nans), 0)) {         // (over what has just been written, and apart from it: see above)
                __syncwarp();
#pragma unroll 1
                for (int i = 0; i < D; ++i)
                    if (row_ok && s_nan[nan_slot * D + i] <= row_last) {
                        if (split) const_cast<float*>(part)[i] = NAN;
                        else const_cast<__nv_bfloat16*>(dst)[i] = __ushort_as_bfloat16(0x7fffu);
                    }
            }
            if (row_ok && split) p.ws_lse[prow] = lse2;
            else if (row_ok && p.lse) p.lse[tok * p.num_q_heads + head] = fmaxf(lse2 * 0.6931471805599453f, -INFINITY);
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

template <int D>
static cudaError_t launch(const CUtensorMap* tq, const CUtensorMap* tk, const CUtensorMap* tv, const Kv4AttnParams& p, int num_ctas, cudaStream_t stream) {
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(wpp_kv8_tiles_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kSmemBytes);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)num_ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<D>::kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, wpp_kv8_tiles_kernel<D>, tq[0], tq[1], tq[2], tq[3], *tk, *tv, p);
}

}  // namespace kv8tiles

// tq: four maps of q with boxes of 128, 64, 32 and 16 rows; tk, tv: of the pools' codes, boxes of a page's rows
extern "C" int wpp_launch_kv8_tiles(int head_dim, const CUtensorMap* tq, const CUtensorMap* tk, const CUtensorMap* tv, const wpp::Kv4AttnParams* p,
                                    int num_ctas, void* stream) {
    return (int)(head_dim == 128 ? kv8tiles::launch<128>(tq, tk, tv, *p, num_ctas, (cudaStream_t)stream)
                                 : kv8tiles::launch<64>(tq, tk, tv, *p, num_ctas, (cudaStream_t)stream));
}
