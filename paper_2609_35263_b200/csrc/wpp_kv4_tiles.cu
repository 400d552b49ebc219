// Attention of many query rows over a cache held in 4 bits: persistent, one CTA per SM, tiles of two 128-row halves against key steps
// of 128 keys, as wpp_attention.cu has them.  What differs is where K and V come from, and where the epilogue is done:
//   warps 0-3   softmax of half A: thread r owns query row r; at a tile's end it writes its row
//   warps 4-7   softmax of half B
//   warps 8-11  codes -> bf16: they read rows of codes from global memory into registers, an item (the K or the V of a key step)
//               ahead, and write what the products read into a ring of two K and two V tiles in shared memory
//   warp 12     issuer of S = Q K^T, warp 14 issuer of O += P V (one thread each), warp 13 takes tiles and loads Q by TMA
// K's tiles hold code - 8, exactly; the softmax makes the score of it with two numbers per key and the sum of the query row
// (see wpp_kv4_few.cu), so that scores have no more error than the bf16 cache's.  V's tiles hold least + scale code rounded to bf16
// once (the probabilities are rounded too): folding V's scales into the probabilities as well would cost the softmax warps,
// which are what everybody waits for, three more operations for every two scores, and the conversion saves only one.
// Codes s and s + 4 of a word's eight come out side by side.  The tiles keep that order (it saves four permutations for eight
// codes): Q's rows are put in the same order once per tile, which also gives their sums, and the epilogue puts O's columns back.
// What bounds it is that conversion, four warps' packed operations for every K and V item, and the softmax beside it: 4,096 tokens behind
// 32,768, 64/8 heads of 128, 5.95 ms (785 TFLOP/s; the operations at the measured rate 2.9 ms), 16 ragged prompts, 32/8 heads, 2.9 ms
// (1.14). The instructions of the conversion are few enough to stay where an SM fetches them fast: with two items under way
// by unrolling it took 7.5 ms, with one code for K and V and a choice inside 6.8.
// Tensor memory: S [0,128)  P_A [128,192)  P_B [192,256)  O_A [256,256+D)  O_B [384,384+D).
// All mbarrier waits are bounded; on expiry the CTA raises its abort flag, every role drains, TMEM is freed and
// WPP_ERR_TIMEOUT is written to the status word.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace kv4tiles {
using namespace wpp;

constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512, kColS = 0;
__host__ __device__ constexpr uint32_t col_p(int hf) { return 128u + 64u * hf; }
__host__ __device__ constexpr uint32_t col_o(int hf) { return 256u + 128u * hf; }
constexpr int kRegsSoftmax = 184, kRegsCodes = 96, kRegsUtil = 48;
static_assert(8 * kRegsSoftmax + 4 * kRegsCodes + 4 * kRegsUtil <= 2048, "register file exceeded");
constexpr float kRefSlack = 16.f;
constexpr int kPar = 4;                    // key steps of a half whose number pairs are held
constexpr int kNan = 8;                    // tiles whose first NaN row of V is held

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = 128 * D * 2, kHalfBytes = 128 * 128;
    static constexpr int kOffK = 2 * kTileBytes, kOffV = kOffK + 2 * kTileBytes;
    static constexpr int kOffPar = kOffV + 2 * kTileBytes;             // float4 [2][kPar][64], a ring for each half: of keys 2 i, 2 i + 1: a, a, b, b; score = a S + b sum q
    static constexpr int kOffStage = kOffPar + 2 * kPar * 1024;            // 8 x 2 KB
    static constexpr int kOffSum = kOffStage + 8 * 2048;               // float [2][2][128]: sums of Q's rows, by tile parity and half
    static constexpr int kOffBars = kOffSum + 2 * 2 * 128 * 4;
    static constexpr int kTileQ = 2;
    static constexpr int kNumBars = 3 + 8 + 2 * kPar + 1 + 5 * 2 + 2 * kTileQ;
    static constexpr int kOffMisc = kOffBars + 8 * kNumBars;           // tmem address, abort flag, tile ids, first NaN rows
    static constexpr int kSmemBytes = kOffMisc + 8 + 4 * kTileQ + 4 * kNan + 1024;
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

// Codes s and s + 4 of a word (16 bits apart) as bf16 numbers 128 + code; `k128` is 128 in both halves (a kernel parameter, so that mask
// and number take one operation)
__device__ __forceinline__ uint32_t codes_128(uint32_t w, uint32_t k128) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "r"(0x000f000fu), "r"(k128));
    return r;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

__device__ __forceinline__ void st_shared_16(uint32_t at, const uint32_t (&y)[4]) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
}

// What a conversion thread holds of a K or V tile: 16 bytes of each of kRows rows, and their number pairs (0: no such key).
template <int D>
struct Raw {
    static constexpr int kChunks = D / 32, kRows = kChunks;            // 16-byte pieces of a row; rows of a thread
    uint4 x[kRows];
    uint32_t pair[kRows];
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
wpp_kv4_tiles_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_q64, const __grid_constant__ CUtensorMap tm_q32,
                     const __grid_constant__ CUtensorMap tm_q16, const Kv4AttnParams p) {
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    const uint32_t sQ = smem_base, sK = smem_base + C::kOffK, sV = smem_base + C::kOffV, bars = smem_base + C::kOffBars;
    const uint32_t bQFull = bars, bQReady = bars + 8, bQEmpty = bars + 16;
    const uint32_t bKFull = bars + 24, bKEmpty = bKFull + 16, bVFull = bKEmpty + 16, bVEmpty = bVFull + 16, bParEmpty = bVEmpty + 16;
    const uint32_t bSFree = bParEmpty + 16 * kPar, bHalf = bSFree + 8;
    auto bSFull = [&](int h) { return bHalf + 40 * h; };
    auto bPReady = [&](int h) { return bHalf + 40 * h + 8; };
    auto bPFree = [&](int h) { return bHalf + 40 * h + 16; };
    auto bOFinal = [&](int h) { return bHalf + 40 * h + 24; };
    auto bOFree = [&](int h) { return bHalf + 40 * h + 32; };
    const uint32_t bTileFull = bHalf + 80, bTileEmpty = bTileFull + 8 * C::kTileQ;
    float* s_sum = reinterpret_cast<float*>(smem_gen + C::kOffSum);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_gen + C::kOffMisc);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    volatile int32_t* tile_ids = reinterpret_cast<volatile int32_t*>(tmem_slot + 2);
    int32_t* s_nan = reinterpret_cast<int32_t*>(smem_gen + C::kOffMisc + 8 + 4 * C::kTileQ);
    constexpr uint32_t kTileConsumers = 2 + 256 + 128;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wg = warp >> 2;

    if (threadIdx.x == 0) {
        mbar_init(bQFull, 1); mbar_init(bQReady, 128); mbar_init(bQEmpty, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bKFull + 8 * s, 128); mbar_init(bKEmpty + 8 * s, 1); mbar_init(bVFull + 8 * s, 128); mbar_init(bVEmpty + 8 * s, 1);
        }
        for (int s = 0; s < 2 * kPar; ++s) mbar_init(bParEmpty + 8 * s, 4);
        for (int s = 0; s < kNan; ++s) s_nan[s] = 0x7fffffff;
        mbar_init(bSFree, 128);
        for (int h = 0; h < 2; ++h) {
            mbar_init(bSFull(h), 1); mbar_init(bPReady(h), 128); mbar_init(bPFree(h), 1); mbar_init(bOFinal(h), 1); mbar_init(bOFree(h), 128);
        }
        for (int i = 0; i < C::kTileQ; ++i) { mbar_init(bTileFull + 8 * i, 1); mbar_init(bTileEmpty + 8 * i, kTileConsumers); }
        *abort_flag = 0u;
        fence_barrier_init();
    }
    if (warp == 12) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols);
        tmem_relinquish();
    }
    if (warp == 13 && lane == 0) {
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_q64); prefetch_tensormap(&tm_q32); prefetch_tensormap(&tm_q16);
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

    if (wg == 3) {
        setmaxnreg_dec<kRegsUtil>();
        if (warp == 13) {
            // ================================================================ tiles and Q
            uint32_t q_phase = 0;
            bool first = true;
            while (true) {
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
                const bool ok = mbar_wait(bQEmpty, q_phase ^ 1u, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) break;
                q_phase ^= 1u;
                if (lane == 0) mbar_arrive_expect_tx(bQFull, ((v.n[0] > 0) + (v.n[1] > 0)) * C::kTileBytes);
                __syncwarp();
                const int rph = 128 / un.pack;
                const CUtensorMap* qm = un.pack == 1 ? &tm_q : un.pack == 2 ? &tm_q64 : un.pack == 4 ? &tm_q32 : &tm_q16;
                const int per_half = un.pack * C::kHalves;
                for (int b = lane; b < 2 * per_half; b += 32) {
                    const int hf = b / per_half, k = (b % per_half) / C::kHalves, h = b % C::kHalves;
                    if ((hf ? v.n[1] : v.n[0]) == 0) continue;
                    // (more places than heads in the group: the last head again, into rows that nobody stores)
                    tma_load_3d(sQ + hf * C::kTileBytes + h * C::kHalfBytes + k * rph * 128, qm, bQFull, h * 64,
                                (hf ? un.head[1] : un.head[0]) + min(k, p.group - 1), v.q_off + (hf ? un.row0[1] : un.row0[0]));
                }
                __syncwarp();
            }
        } else if (warp == 12 && lane == 0) {
            // ================================================================ issuer of S = Q K^T
            Ring ring = {0, 0};
            uint32_t q_phase = 0, sfree_phase = 0;
            constexpr uint32_t idesc_qk = idesc_bf16(128, 0, 0);
            const uint64_t q_desc0 = smem_desc_sw128(sQ, 16, 1024), k_desc0 = smem_desc_sw128(sK, 16, 1024);
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
                    const uint64_t kd = k_desc0 + (uint64_t)(ring.stage * (C::kTileBytes >> 4));
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        if (k >= v.n[hf]) continue;
                        if (!mbar_wait(bSFree, sfree_phase ^ 1u, abort_flag)) { dead = true; break; }
                        sfree_phase ^= 1u;
                        tc_fence_after();
                        const uint64_t qd = q_desc0 + (uint64_t)(hf * (C::kTileBytes >> 4));
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint64_t off = (uint64_t)(((kk >> 2) * C::kHalfBytes + (kk & 3) * 32) >> 4);
                            if (kk == 0) mma_ss_overwrite(tS, qd + off, kd + off, idesc_qk);
                            else mma_ss_accumulate(tS, qd + off, kd + off, idesc_qk);
                        }
                        mma_commit(bSFull(hf));
                    }
                    if (dead) break;
                    mma_commit(bKEmpty + 8 * ring.stage);
                    ring.advance(2);
                }
                if (!dead) mma_commit(bQEmpty);
            }
        } else if (warp == 14 && lane == 0) {
            // ================================================================ issuer of O += P V
            Ring ring = {0, 0};
            uint32_t p_phase[2] = {0, 0}, of_phase[2] = {0, 0};
            constexpr uint32_t idesc_pv = idesc_bf16(D, 0, 1);
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
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const int n = v.n[hf];
                        if (k >= n) continue;
                        if (!mbar_wait(bPReady(hf), p_phase[hf], abort_flag)) { dead = true; break; }
                        p_phase[hf] ^= 1u;
                        if (k == 0) {          // the tile before's O has been read
                            if (!mbar_wait(bOFree(hf), of_phase[hf] ^ 1u, abort_flag)) { dead = true; break; }
                            of_phase[hf] ^= 1u;
                        }
                        tc_fence_after();
                        const uint32_t tP = tmem + col_p(hf), tO = tmem + col_o(hf);
                        if (k > 0) mma_ts_accumulate(tO, tP, vd, idesc_pv); else mma_ts_overwrite(tO, tP, vd, idesc_pv);
#pragma unroll
                        for (int kk = 1; kk < 8; ++kk) mma_ts_accumulate(tO, tP + kk * 8, vd + (uint64_t)(kk * 128), idesc_pv);
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
        // ================================================================ codes -> bf16
        setmaxnreg_dec<kRegsCodes>();
        using R = Raw<D>;
        const int dw = warp & 3, c = lane % R::kChunks, rr = lane / R::kChunks, r = threadIdx.x & 127;
        const int page_shift = 31 - __clz(p.page_size);
        const bool swap = D == 128 && (c & 2);         // of lanes 2 apart, whose pieces would meet in a bank, one begins with its second half
        // what of a row's place does not change from key step to key step: the row in the tile, its page, its bytes in the block
        constexpr int kApart = 32 / R::kChunks;        // rows from one of the thread's rows to the next
        const int row0 = dw * 32 + rr, ppt = 128 >> page_shift;
        // (the thread's rows are in one group of 32 keys: one page, or two where pages have 16)
        const int page_of[2] = {row0 >> page_shift, (row0 + 16) >> page_shift};
        int bytes_of[R::kRows], pair_of[R::kRows];
#pragma unroll
        for (int i = 0; i < R::kRows; ++i) {
            const int row = row0 + i * kApart, slot = row & (p.page_size - 1);
            bytes_of[i] = slot * (D / 2) + c * 16;
            pair_of[i] = p.page_size * (D / 2) + slot * 4;
        }
        uint32_t piece[4];                             // where the four pieces of 8 numbers go in the tile's first row of this thread
#pragma unroll
        for (int q = 0; q < 4; ++q)
            piece[q] = (uint32_t)((c >> 1) * C::kHalfBytes + row0 * 128 + ((((c & 1) * 4 + (q ^ (swap ? 2 : 0))) ^ (row0 & 7)) << 4));
        Ring ring_k = {0, 0}, ring_v = {0, 0}, ring_p[2] = {{0, 0}, {0, 0}};
        uint32_t q_phase = 0, tiles = 0;               // tiles: with work, so far
        int bad = 0;
        bool dead = false;
        while (!dead) {
            const int u = next_tile();
            if (!__all_sync(0xffffffffu, u != -2) || u < 0) break;
            const WppUnit un = units[u];
            const UnitView v = view_of(un, p, q_offsets, plan_prefix);
            if (v.n_steps == 0) continue;
            const int kvh = un.head[0] / p.group;
            const int32_t* bt = p.block_tables + (int64_t)un.request * p.max_blocks;
            const uint8_t* const kc = p.k_cache + kvh * p.head_bytes;
            const uint8_t* const vc = p.v_cache + kvh * p.head_bytes;
            int32_t* nan_at = s_nan + tiles % kNan;
            // the place of four tiles on: nobody is so far behind that it reads the one of four tiles ago, nor so far ahead
            if (r == 0) s_nan[(tiles + kNan / 2) % kNan] = 0x7fffffff;
            const int last_page = (v.kv_len - 1) >> page_shift;
            // page ids are asked for an item before the rows they lead to, rows an item before their use
            int page[2];
            auto look_up = [&](int step) {
                const int at = (v.kv_begin + step) * ppt;
                page[0] = bt[min(at + page_of[0], last_page)];
                if (p.page_size == 16) page[1] = bt[min(at + page_of[1], last_page)];
            };
            auto fetch = [&](R& x, const uint8_t* pool, int step) {
                const int step_at = v.kv_begin + step;
                const uint8_t* block[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h == 1 && p.page_size != 16) { block[1] = block[0]; break; }
                    const bool there = (uint32_t)page[h] < (uint32_t)p.num_pages;
                    bad |= !there;
                    block[h] = pool + (there ? page[h] : 0) * p.page_bytes;
                }
                // (coherent loads: the append before may still write the pool while this kernel is set up)
#pragma unroll
                for (int i = 0; i < R::kRows; ++i) {
                    const uint8_t* from = block[i * kApart / 16];
                    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(x.x[i].x), "=r"(x.x[i].y), "=r"(x.x[i].z), "=r"(x.x[i].w) : "l"(from + bytes_of[i]));
                    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(x.pair[i]) : "l"(from + pair_of[i]));
                }
                if ((step_at + 1) * 128 > v.kv_len) {  // what lies behind the sequence counts as zeros
#pragma unroll
                    for (int i = 0; i < R::kRows; ++i)
                        if (step_at * 128 + row0 + i * kApart >= v.kv_len) x.pair[i] = 0u;
                }
            };
            int nk = 0, nv = 0;                        // fetched so far
            auto next_is_k = [&]() { return nk < v.n_steps && nk <= nv + 1; };      // K(0) K(1) V(0) K(2) V(1) ...
            R cur, next;
            look_up(0);
            fetch(cur, kc, 0);
            nk = 1;
            look_up(next_is_k() ? nk : nv);
            bool cur_k = true;
            // ---- Q in the codes' order, and the sums of its rows (thread = row)
            if (!__all_sync(0xffffffffu, mbar_wait(bQFull, q_phase, abort_flag))) { dead = true; break; }
            q_phase ^= 1u;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                if (v.n[hf] == 0) continue;
                float sum = 0.f;
#pragma unroll 4
                for (int ch = 0; ch < D / 8; ++ch) {
                    uint4* at = reinterpret_cast<uint4*>(smem_gen + hf * C::kTileBytes + (ch >> 3) * C::kHalfBytes + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
                    const uint4 z = *at;
                    *at = make_uint4(__byte_perm(z.x, z.z, 0x5410), __byte_perm(z.x, z.z, 0x7632), __byte_perm(z.y, z.w, 0x5410), __byte_perm(z.y, z.w, 0x7632));
                    sum += (__uint_as_float(z.x << 16) + __uint_as_float(z.x & 0xffff0000u)) + (__uint_as_float(z.y << 16) + __uint_as_float(z.y & 0xffff0000u)) +
                           (__uint_as_float(z.z << 16) + __uint_as_float(z.z & 0xffff0000u)) + (__uint_as_float(z.w << 16) + __uint_as_float(z.w & 0xffff0000u));
                }
                s_sum[((tiles & 1) * 2 + hf) * 128 + r] = sum;
            }
            fence_proxy_async_smem();
            mbar_arrive(bQReady);
            ++tiles;
            int done_k = 0, done_v = 0;
            while (done_v < v.n_steps) {
                bool next_k = false;
                if (nk < v.n_steps || nv < v.n_steps) {
                    next_k = next_is_k();
                    fetch(next, next_k ? kc : vc, next_k ? nk : nv);
                    if (next_k) ++nk; else ++nv;
                    if (nv < v.n_steps) look_up(next_is_k() ? nk : nv);
                }
                const uint32_t slot = cur_k ? ring_k.stage : ring_v.stage;
                if (!__all_sync(0xffffffffu, mbar_wait((cur_k ? bKEmpty : bVEmpty) + 8 * slot, (cur_k ? ring_k.phase : ring_v.phase) ^ 1u, abort_flag))) {
                    dead = true;
                    break;
                }
                const bool par_of[2] = {cur_k && done_k < v.n[0], cur_k && done_k < v.n[1]};
                bool ok = true;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (par_of[h]) ok = ok && mbar_wait(bParEmpty + 8 * (h * kPar + ring_p[h].stage), ring_p[h].phase ^ 1u, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) {
                    dead = true;
                    break;
                }
                const uint32_t to = (cur_k ? sK : sV) + slot * C::kTileBytes;
                if (cur_k) {
#pragma unroll
                    for (int i = 0; i < R::kRows; ++i) {
                        const uint32_t w[4] = {swap ? cur.x[i].z : cur.x[i].x, swap ? cur.x[i].w : cur.x[i].y, swap ? cur.x[i].x : cur.x[i].z,
                                               swap ? cur.x[i].y : cur.x[i].w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint32_t y[4];
#pragma unroll
                            for (int s = 0; s < 4; ++s) y[s] = sub_bf16x2(codes_128(w[q] >> (4 * s), p.bf16_128), 0x43084308u);          // - 136
                            st_shared_16(to + piece[q] + i * kApart * 128, y);
                        }
                        if (c == 0) {
                            const float scale = __uint_as_float(cur.pair[i] & 0xffff0000u) * p.scale_log2, least = __uint_as_float(cur.pair[i] << 16) * p.scale_log2;
                            const int row = row0 + i * kApart;
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                if (par_of[h]) {
                                    float* par = reinterpret_cast<float*>(smem_gen + C::kOffPar + (h * kPar + ring_p[h].stage) * 1024) + (row >> 1) * 4 + (row & 1);
                                    par[0] = scale;
                                    par[2] = fmaf(8.f, scale, least);
                                }
                        }
                    }
                } else {
                    bool nan = false;
#pragma unroll
                    for (int i = 0; i < R::kRows; ++i) nan |= (cur.pair[i] & 0x7f80u) == 0x7f80u;
                    if (nan) {                         // rows that stand for NaN: zero for the product, see the epilogue
#pragma unroll
                        for (int i = 0; i < R::kRows; ++i)
                            if ((cur.pair[i] & 0x7f80u) == 0x7f80u) {
                                if (c == 0) atomicMin(nan_at, (v.kv_begin + done_v) * 128 + row0 + i * kApart);
                                cur.pair[i] = 0u;
                            }
                    }
#pragma unroll
                    for (int i = 0; i < R::kRows; ++i) {
                        const uint32_t least2 = __byte_perm(cur.pair[i], 0u, 0x1010), scale2 = __byte_perm(cur.pair[i], 0u, 0x3232);
                        const uint32_t w[4] = {swap ? cur.x[i].z : cur.x[i].x, swap ? cur.x[i].w : cur.x[i].y, swap ? cur.x[i].x : cur.x[i].z,
                                               swap ? cur.x[i].y : cur.x[i].w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint32_t y[4];
#pragma unroll
                            for (int s = 0; s < 4; ++s) y[s] = fma_bf16x2(sub_bf16x2(codes_128(w[q] >> (4 * s), p.bf16_128), 0x43004300u), scale2, least2);
                            st_shared_16(to + piece[q] + i * kApart * 128, y);
                        }
                    }
                }
                fence_proxy_async_smem();
                if (cur_k) {
                    mbar_arrive(bKFull + 8 * slot);
                    ring_k.advance(2);
                    if (par_of[0]) ring_p[0].advance(kPar);
                    if (par_of[1]) ring_p[1].advance(kPar);
                    ++done_k;
                } else {
                    mbar_arrive(bVFull + 8 * slot);
                    ring_v.advance(2);
                    ++done_v;
                }
                cur = next;
                cur_k = next_k;
            }
        }
        if (bad && p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
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
            float m_ref = 0.f, l_run = 0.f, qs = 0.f;
            for (int j = 0; j < n; ++j) {
                if (!__all_sync(0xffffffffu, mbar_wait(bSFull(hf), s_phase, abort_flag))) { dead = true; break; }
                s_phase ^= 1u;
                tc_fence_after();
                if (j == 0) qs = s_sum[((tiles & 1) * 2 + hf) * 128 + r];
                float s[128];
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) tmem_ld32(lane_addr + kColS + q4 * 32, reinterpret_cast<uint32_t*>(s) + q4 * 32);
                tmem_wait_ld();
                tc_fence_before();
                mbar_arrive(bSFree);
                {
                    const float4* pr = reinterpret_cast<const float4*>(smem_gen + C::kOffPar + (hf * kPar + par) * 1024);
                    const uint64_t qs2 = pack2(qs, qs), nm2 = pack2(-m_ref, -m_ref);
#pragma unroll
                    for (int i = 0; i < 64; ++i) {
                        const float4 f = pr[i];
                        unpack2(ffma2(pack2(s[2 * i], s[2 * i + 1]), pack2(f.x, f.y), ffma2(pack2(f.z, f.w), qs2, nm2)), s[2 * i], s[2 * i + 1]);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bParEmpty + 8 * (hf * kPar + par));
                    par = (par + 1) % kPar;
                }
                const int key0 = (v.kv_begin + j) * 128;
                if (key0 + 127 > first_pos) {          // only steps that touch the diagonal are masked
                    const int limit = row_last - key0;
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i] = (i > limit) ? -INFINITY : s[i];
                }
                float mx[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) mx[k] = fmaxf(s[2 * k], s[2 * k + 1]);
#pragma unroll
                for (int i = 16; i < 128; i += 16) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) mx[k] = fmax3(mx[k], s[i + 2 * k], s[i + 2 * k + 1]);
                }
                const float mxx = fmaxf(fmax3(mx[0], mx[1], mx[2]), fmaxf(fmax3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])));
                bool waited = false;
                const bool move = j == 0 || mxx > kRefSlack;
                if (__any_sync(0xffffffffu, move)) {
                    // how far the reference goes up (the first one may go down; a row that sees nothing keeps its)
                    float y = j == 0 ? mxx : fmaxf(mxx, 0.f);
                    if (y == -INFINITY) y = 0.f;
                    const float alpha = j == 0 ? 1.f : fast_exp2(-y);
                    m_ref += y;
                    l_run *= alpha;
                    const uint64_t ny2 = pack2(-y, -y);
#pragma unroll
                    for (int i = 0; i < 64; ++i) unpack2(fadd2(pack2(s[2 * i], s[2 * i + 1]), ny2), s[2 * i], s[2 * i + 1]);
                    if (j > 0) {
                        if (!__all_sync(0xffffffffu, mbar_wait(bPFree(hf), pf_phase ^ 1u, abort_flag))) { dead = true; break; }
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
                    }
                }
                uint32_t* pk = reinterpret_cast<uint32_t*>(s);
                {
                    uint64_t sum2a = pack2(0.f, 0.f), sum2b = pack2(0.f, 0.f);
#pragma unroll
                    for (int i0 = 0; i0 < 64; i0 += 8) {
                        float e[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) e[k] = fast_exp2(s[2 * i0 + k]);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            if (k & 1) sum2b = fadd2(sum2b, pack2(e[2 * k], e[2 * k + 1]));
                            else sum2a = fadd2(sum2a, pack2(e[2 * k], e[2 * k + 1]));
                            pk[i0 + k] = pack_bf16x2(e[2 * k], e[2 * k + 1]);
                        }
                    }
                    float t0, t1;
                    unpack2(fadd2(sum2a, sum2b), t0, t1);
                    l_run += t0 + t1;
                }
                if (!waited) {                         // P(j - 1) has been consumed
                    if (!__all_sync(0xffffffffu, mbar_wait(bPFree(hf), pf_phase ^ 1u, abort_flag))) { dead = true; break; }
                    pf_phase ^= 1u;
                    tc_fence_after();
                }
#pragma unroll
                for (int c8 = 0; c8 < 64; c8 += 8) tmem_st8(lane_addr + col_p(hf) + c8, pk + c8);
                tmem_wait_st();
                tc_fence_before();
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
            // a row that sees a NaN row of V is NaN
            const float inv_l = s_nan[nan_slot] <= row_last ? NAN : l_run > 0.f ? 1.f / l_run : l_run != l_run ? l_run : 0.f;
            const float lse2 = (l_run <= 0.f) ? -INFINITY : (m_ref + log2f(l_run));
            uint8_t* stage = smem_gen + C::kOffStage + warp * 2048;
            const bool split = un.split_slot >= 0;
            const __nv_bfloat16* dst = p.out + tok * p.o_token_stride + (int64_t)head * p.o_head_stride;
            const float* part = p.ws_o + prow * D;
#pragma unroll 1
            for (int q4 = 0; q4 < D / 32; ++q4) {
                float x[32], o[32];
                tmem_ld32(lane_addr + col_o(hf) + q4 * 32, reinterpret_cast<uint32_t*>(x));
                tmem_wait_ld();
                // columns 0 to 7 of every eight hold elements 0 4 1 5 2 6 3 7
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = x[(i & ~7) + ((i & 3) << 1) + ((i >> 2) & 1)] * inv_l;
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
static cudaError_t launch(const CUtensorMap* tq, const Kv4AttnParams& p, int num_ctas, cudaStream_t stream) {
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(wpp_kv4_tiles_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kSmemBytes);
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
    return cudaLaunchKernelEx(&cfg, wpp_kv4_tiles_kernel<D>, tq[0], tq[1], tq[2], tq[3], p);
}

}  // namespace kv4tiles

// tq: four maps of q with boxes of 128, 64, 32 and 16 rows
extern "C" int wpp_launch_kv4_tiles(int head_dim, const CUtensorMap* tq, const wpp::Kv4AttnParams* p, int num_ctas, void* stream) {
    return (int)(head_dim == 128 ? kv4tiles::launch<128>(tq, *p, num_ctas, (cudaStream_t)stream)
                                 : kv4tiles::launch<64>(tq, *p, num_ctas, (cudaStream_t)stream));
}
