// Attention of few query rows over a cache held in 8 bits: single new tokens, and chunks' row blocks of at most WPP_FEW_ROWS rows
// (tokens x heads of a KV group).
//
// With K_j = ks c_j and V_j = vs c'_j (c, c' the codes, ks and vs the powers of two of key j's page), y_j = sm_scale log2(e) ks <q, c_j>:
//     out = sum_j 2^y_j vs c'_j / sum_j 2^y_j,
// and the products are taken of the codes themselves, which f16 holds exactly: S^T = C Q^T, O^T = C'^T P^T by mma.sync, eight columns of
// query rows that the group's heads fill (a product of 128 rows on the 5th-generation tensor cores would be nearly empty).
// The sums O are in units of the largest vs so far, v: p_j = 2^(y_j - m + log2(vs / v)), so that V's scales cost no operation of their own
// beyond a factor v / vs per 16 keys (a page has at least so many) for the sum of 2^(y_j - m).  The reference m, a whole number, is put 6 to 7
// below a row's largest y_j and moved when one comes 15 above: p lies within f16's range, off by 2^-11 of itself or by 2^-25, which is 2^-31 of
// the row's largest where vs is v, and 2^-23 of the largest that its page's keys can have where vs is 2^-8 v.  Pages whose scale is more than
// 2^8 below v would be pushed out of that range, by others that may have a large scale for one row's sake: their product is taken by
// itself, without vs / v, and added with it in fp32.
//
// What bounds it is the cache's bytes.  A warp takes 32 keys at a time, copied asynchronously into a ring of its own and read in the
// order the fragments want: which element of a row stands at which place of a product does not matter as long as both factors agree,
// so that a lane's codes of K and of V are 16-byte pieces; the pieces of a row change places, by the row's number, so that lanes do not
// meet in a bank.  V's codes of two keys first stand side by side by a byte permutation.
//
// Measured: 64 requests of one token behind 255 to 16,383 keys, 64/8 heads of 128, on a cache that is not in L2 181 to 200 us, from GPU
// to GPU (the bytes at the measured copy rate 158), combine pass included; four behind 131,071 199 (167).  The loop needs 40 % of the issue slots at that rate.
// One behind 8,191, 32/8 heads: 11.5 us in a graph, of which the copies under way are 0.4, the chain from the page id to the first keys 1.4,
// four stages a warp 2.5, the joins of warps and of a cluster's CTAs 2.  That leaves 5.2, of which a launch is 2 to 3 (the whole call of a
// small kernel takes as much); the rest has not been taken apart.

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_kv8.cuh"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace wpp {
namespace kv8few {

constexpr int kWarps = 4;
constexpr int kKeys = 32;                  // a warp's keys at a time
constexpr float kTop = 7.f, kMost = 15.f;  // log2 of a row's largest 2^(y - m) when its reference is moved, and when it has to be
constexpr float kLow = -8.f;               // log2 of vs / v down to which p holds it

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
template <int kWords>
__device__ __forceinline__ void load_words(uint32_t* w, uint32_t at) {
    if constexpr (kWords == 4) {
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
    } else if constexpr (kWords == 2) {
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    } else {
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
    }
}
__device__ __forceinline__ void copy_16(uint32_t dst, const uint8_t* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A warp's ring of stages in shared memory, kKeys keys each: K's rows, V's rows, and the 16 bytes behind the rows of the two groups of 16
// keys, of K and of V.
template <int D, int NT, bool kCluster>
struct Smem {
    static constexpr int kRows = kKeys * D, kStage = 2 * kRows + 64;
    // (as many as leave three CTAs an SM of blocks of at most 8 rows, else two, which clusters make do with: where each CTA has a few
    // stages in all, what counts is how many are under way)
    static constexpr int kDepth = D == 128 ? (NT == 1 && !kCluster ? 2 : 3) : (NT == 1 && !kCluster ? 4 : 5);
    // in the stages' place, once a unit's are done with: float [warps][8 NT][D + 4], float2 [warps][8 NT]
    static constexpr int kOffMl = kWarps * 8 * NT * (D + 4) * 4;
    // and, of a CTA of a cluster, behind them: float [8 NT][D], the part's rows, and float [8 NT], their log-sums
    static constexpr int kOffPart = kOffMl + kWarps * 8 * NT * 8, kOffPartLse = kOffPart + 8 * NT * D * 4;
    static constexpr int kBytes = kWarps * kDepth * kStage;
    static_assert(kOffPartLse + 8 * NT * 4 <= kBytes, "a unit's results fit the stages");
};

// Which key stands in row r of a 16-key tile of the products (rows 2 and 3, 6 and 7, ... are exchanged), and by how much the 16-byte
// pieces of a key's row of K and of V are displaced (exclusive or): lanes that read at once are rows g and g + 1 of K, 0, 2, 4 and 6 of V.
__device__ __forceinline__ int key_of_row(int r) { return r ^ ((r >> 1) & 1); }
template <int D>
__device__ __forceinline__ int shift_k(int key) { return D == 128 ? key & 1 : 0; }
template <int D>
__device__ __forceinline__ int shift_v(int key) { return D == 128 ? (key >> 1 & 3) << 1 : (key >> 2 & 1) << 1; }

// The running state of a warp's columns (query rows): lane 4 g + t has columns 2 t and 2 t + 1 of every eight.
template <int D, int NT>
struct State {
    float o[NT][D / 16][4];
    float m[NT][2], l[NT][2];
    float v_exp;                           // log2 of the sums' unit (the warp's)
};

// A byte of ones for every code that is NaN
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu); }

// 32 keys, at shared-memory address `at`.  Lane 4 g + t takes, of a tile's rows g and g + 8, columns [t D / 4, (t + 1) D / 4) of K; of
// rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9, columns [g D / 8, (g + 1) D / 8) of V.
template <int D, int NT, bool kCluster, bool kMasked>
__device__ __forceinline__ void step(State<D, NT>& st, const uint32_t at, const uint32_t (&qf)[NT][D / 16][2], const float (&q_scale)[NT][2],
                                     int key0, int first_pos, int toks, int last, bool first, int g, int t) {
    using M = Smem<D, NT, kCluster>;
    const int kg = key_of_row(g), kt = key_of_row(2 * t);
    int limit[NT][2];                                                  // last key that the column's row sees
    if (kMasked) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) limit[nt][c] = first_pos + (8 * nt + 2 * t + c) % toks;
    }
    // ---- S^T = codes Q^T
    float s[2][NT][4];
    const uint32_t k_at = at + kg * D;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t k[2][D / 16];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int w = 0; w < D / 64; ++w)                           // (keys 8 apart have their pieces at the same places)
                load_words<4>(&k[i][4 * w], k_at + (16 * h + 8 * i) * D + (((t * (D / 64) + w) ^ shift_k<D>(kg)) << 4));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[h][nt][i] = 0.f;
#pragma unroll
        for (int w = 0; w < D / 16; ++w) {
            const uint32_t a0 = codes_f16x2_low(k[0][w]), a1 = codes_f16x2_low(k[1][w]), a2 = codes_f16x2_high(k[0][w]), a3 = codes_f16x2_high(k[1][w]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(s[h][nt], a0, a1, a2, a3, qf[nt][w][0], qf[nt][w][1]);
        }
    }
    // ---- V's scales, in the sums' unit
    float below[2];                                                    // log2 of vs / v
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t vs[1];
        load_words<1>(vs, at + 2 * M::kRows + 32 + 16 * h);
        below[h] = kMasked && key0 + 16 * h > last ? -1e9f : (float)exponent_of(__uint_as_float(vs[0]));      // (no row sees these keys: there may be anything)
    }
    const float v_most = fmaxf(below[0], below[1]);
    if (first || v_most > st.v_exp) {
        const float a = first ? 1.f : fast_exp2(st.v_exp - v_most);
        st.v_exp = v_most;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[nt][mt][i] *= a;
    }
    float apart[2];                                                    // what the group's own product is multiplied by; 0: it is in p
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        below[h] -= st.v_exp;
        apart[h] = 0.f;
        if (below[h] < kLow) {
            apart[h] = fast_exp2(below[h]);
            below[h] = 0.f;
        }
    }
    // ---- scores in log2 units, above m
    bool move = first;
    float mx[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) mx[nt][c] = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t ks[1];
        load_words<1>(ks, at + 2 * M::kRows + 16 * h);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float a = __uint_as_float(ks[0]) * q_scale[nt][c], b = below[h] - st.m[nt][c];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float& y = s[h][nt][2 * i + c];
                    y = fmaf(y, a, b);
                    if (kMasked && key0 + 16 * h + 8 * i + kg > limit[nt][c]) y = -INFINITY;
                }
                mx[nt][c] = fmaxf(mx[nt][c], fmaxf(s[h][nt][c], s[h][nt][2 + c]) - below[h]);
                move |= mx[nt][c] > kMost;
            }
    }
    // ---- references move only where a score is far above them
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                // how far the reference goes up; the first one may go down as well, and stays where the row sees nothing
                float y = mx[nt][c];
#pragma unroll
                for (int w = 4; w < 32; w *= 2) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, w));
                y = ceilf(y - kTop);
                y = first ? (y == -INFINITY ? 0.f : y) : fmaxf(y, 0.f);
                const float a = first ? 1.f : fast_exp2(-y);
                st.m[nt][c] += y;
                st.l[nt][c] *= a;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[h][nt][c] -= y;
                    s[h][nt][2 + c] -= y;
                }
#pragma unroll
                for (int mt = 0; mt < D / 16; ++mt) {
                    st.o[nt][mt][c] *= a;
                    st.o[nt][mt][2 + c] *= a;
                }
            }
    }
    // ---- P^T, turned round into the second factor of O^T = V^T P^T
    uint32_t pb[2][NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float less = fast_exp2(-below[h]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[h][nt][i] = fast_exp2(s[h][nt][i]);
#pragma unroll
            for (int c = 0; c < 2; ++c) st.l[nt][c] = fmaf(s[h][nt][c] + s[h][nt][2 + c], less, st.l[nt][c]);
#pragma unroll
            for (int i = 0; i < 2; ++i) pb[h][nt][i] = transpose_8x8(pack_f16x2(s[h][nt][2 * i], s[h][nt][2 * i + 1]));
        }
    }
    // ---- O^T += codes^T P^T
    const uint32_t v_at = at + M::kRows, piece = D == 128 ? (uint32_t)((g ^ shift_v<D>(kt)) << 4) : (uint32_t)((((g >> 1) ^ shift_v<D>(kt)) << 4) + (g & 1) * 8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v[4][D / 32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = 16 * h + (kt ^ (i & 1)) + 8 * (i >> 1);    // (row 2 t + 1's key is row 2 t's with the last bit turned: pieces at the same places)
            load_words<D / 32>(v[i], v_at + key * D + piece);
            if (kMasked && key0 + key > last) {
#pragma unroll
                for (int w = 0; w < D / 32; ++w) v[i][w] = 0u;
            }
        }
        if (kMasked) {
            // a NaN that not all columns see must not reach the others as 0 * NaN: it counts where it is seen, and is 0 for the product
            uint32_t nan = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < D / 32; ++w) nan |= nan_bytes(v[i][w]);
            if (__any_sync(0xffffffffu, nan != 0u)) {
#pragma unroll
                for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {                      // element 2 mt + e of the lane's columns, as in the sums' rows g and g + 8
                        uint32_t keys = 0u;                            // whose code of it is NaN
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t code = v[i][mt / 2] >> (8 * (2 * (mt & 1) + e)) & 0x7fu;
                            if (code == 0x7fu) keys |= 1u << ((kt ^ (i & 1)) + 8 * (i >> 1));
                        }
                        keys |= __shfl_xor_sync(0xffffffffu, keys, 1);
                        keys |= __shfl_xor_sync(0xffffffffu, keys, 2);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                const int sees = min(max(limit[nt][c] - key0 - 16 * h + 1, 0), 16);
                                if (keys & ((1u << sees) - 1u)) st.o[nt][mt][2 * e + c] = NAN;
                            }
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int w = 0; w < D / 32; ++w) v[i][w] &= ~nan_bytes(v[i][w]);
            }
        }
        auto product = [&](bool own) {
#pragma unroll
            for (int w = 0; w < D / 32; ++w)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t lo = __byte_perm(v[0][w], v[1][w], u ? 0x7362 : 0x5140), hi = __byte_perm(v[2][w], v[3][w], u ? 0x7362 : 0x5140);
                    const uint32_t a0 = codes_f16x2_low(lo), a1 = codes_f16x2_high(lo), a2 = codes_f16x2_low(hi), a3 = codes_f16x2_high(hi);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float (&o)[4] = st.o[nt][2 * w + u];
                        if (!own) {
                            mma_f16(o, a0, a1, a2, a3, pb[h][nt][0], pb[h][nt][1]);
                        } else {
                            float x[4] = {0.f, 0.f, 0.f, 0.f};
                            mma_f16(x, a0, a1, a2, a3, pb[h][nt][0], pb[h][nt][1]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[i] = fmaf(apart[h], x[i], o[i]);
                        }
                    }
                }
        };
        if (apart[h] == 0.f) product(false);
        else product(true);
    }
}

// A unit with what the plan says of its request.  (Behind the wait for the kernel before, which may have written the plan.)
struct Unit {
    WppUnit un;
    int q_off, P, C;
};
__device__ __forceinline__ Unit unit_at(const Kv4AttnParams& p, int unit) {
    const char* plan = static_cast<const char*>(p.plan);
    Unit x;
    x.un = reinterpret_cast<const WppUnit*>(plan + p.off_units)[unit];
    const int32_t* q_offsets = reinterpret_cast<const int32_t*>(plan + p.off_q_offsets) + x.un.request;
    x.q_off = q_offsets[0];
    x.C = q_offsets[1] - x.q_off;
    x.P = reinterpret_cast<const int32_t*>(plan + p.off_prefix)[x.un.request];
    return x;
}

// kCluster: the unit is a part of a block whose other parts the other CTAs of the cluster have; its rows are left in shared memory
template <int D, int NT, bool kCluster>
__device__ __forceinline__ void run_unit(const Kv4AttnParams& p, const Unit& unit, uint8_t* smem) {
    using M = Smem<D, NT, kCluster>;
    constexpr int kSteps = D / 16;             // 16-wide pieces of a row
    float (*s_o)[8 * NT][D + 4] = reinterpret_cast<float (*)[8 * NT][D + 4]>(smem);
    float2 (*s_ml)[8 * NT] = reinterpret_cast<float2 (*)[8 * NT]>(smem + M::kOffMl);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const WppUnit& un = unit.un;
    const int q_off = unit.q_off, P = unit.P, C = unit.C;
    // (what the launch has is compared with the plan while the first keys are under way)
    const int P_now = p.prefix_lens[un.request], C_now = p.chunk_lens[un.request];
    const int toks = un.rows[0], rows = toks * un.rows[1], first_pos = P + un.row0[0];     // first_pos: last key that token 0 sees
    const int key_begin = un.kv_begin * WPP_TILE_N;
    const int seen = min(min(P + C, un.kv_end * WPP_TILE_N), first_pos + toks);            // keys that some row sees end here
    const int kvh = un.head[0] / p.group, page_shift = 31 - __clz(p.page_size), in_page = p.page_size - 1;
    const int32_t* table = p.block_tables + (int64_t)un.request * p.max_blocks;

    // ---- the warp's keys: 32 at a time, every kWarps-th; page ids are asked for a stage ahead of the rows they lead to
    constexpr int kStride = kKeys * kWarps, kChunks = D / 16;          // kChunks: 16-byte pieces of a row
    const uint32_t ring = smem_u32(smem) + warp * M::kDepth * M::kStage;
    const uint8_t* const kc = p.k_cache + kvh * p.head_bytes;
    const uint8_t* const vc = p.v_cache + kvh * p.head_bytes;
    const int row = lane / kChunks, piece = lane % kChunks;
    int bad = 0, page[2] = {0, 0};
    auto look_up = [&](int key) {
        if (key >= seen) return;
        page[0] = table[key >> page_shift];
        if (p.page_size == 16 && key + 16 < seen) page[1] = table[(key >> page_shift) + 1];
    };
    auto request16 = [&](int key, int keys, uint32_t dst, int at, int id) {      // `keys` (16 or 32) keys of one page, `at` keys into the stage
        if (id < 0 || id >= p.num_pages) {
            bad = 1;
            id = 0;
        }
        const int64_t block = id * p.page_bytes;
        const int64_t from = block + (key & in_page) * D + lane * 16;
#pragma unroll
        for (int i = 0; i < kKeys * kChunks / 32; ++i) {
            const int r = i * (32 / kChunks) + row;
            if (r < keys) {
                copy_16(dst + (at + r) * D + ((piece ^ shift_k<D>(r)) << 4), kc + from + i * 512);
                copy_16(dst + M::kRows + (at + r) * D + ((piece ^ shift_v<D>(r)) << 4), vc + from + i * 512);
            }
        }
        // lanes 0 and 1: K's scale for the groups of 16 keys, 2 and 3: V's
        if (lane < 4 && (lane & 1) * 16 < keys)
            copy_16(dst + 2 * M::kRows + (lane >> 1) * 32 + at + (lane & 1) * 16, (lane & 2 ? vc : kc) + block + p.page_size * D);
    };
    auto request = [&](int key, uint32_t dst) {
        if (key < seen) {
            if (p.page_size > 16) {
                request16(key, min((seen - key + 15) & ~15, kKeys), dst, 0, page[0]);
            } else {
                request16(key, 16, dst, 0, page[0]);
                if (key + 16 < seen) request16(key + 16, 16, dst, 16, page[1]);
            }
            look_up(key + kStride);
        }
        copies_commit();                                               // (an empty group where there is nothing: groups are counted)
    };
    int key = key_begin + warp * kKeys;
    look_up(key);
    uint4 q_rows[NT][D / 32];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = 8 * nt + g;
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            q_rows[nt][w] = make_uint4(0, 0, 0, 0);
            if (n < rows) {
                const int head = un.head[0] + n / toks, tok = q_off + un.row0[0] + n % toks;
                q_rows[nt][w] = *reinterpret_cast<const uint4*>(p.q + (int64_t)tok * p.q_token_stride + (int64_t)head * p.q_head_stride + t * (D / 4) + 8 * w);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < M::kDepth - 1; ++i) request(key + i * kStride, ring + i * M::kStage);

    // ---- Q as the first product's second factor: f16 numbers q 2^e, e so that the row's largest is in [2^7, 2^8) (what is less than
    //      2^-21 of that may be off by 2^-32 of it)
    uint32_t qf[NT][D / 16][2];
    float q_scale[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const uint4 (&z)[D / 32] = q_rows[nt];
        float top = 0.f;
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            const uint32_t zz[4] = {z[w].x, z[w].y, z[w].z, z[w].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(zz[i] << 16)), fabsf(__uint_as_float(zz[i] & 0xffff0000u))));
        }
#pragma unroll
        for (int w = 1; w < 4; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        // 2^e and 2^-e, both normal numbers
        const int e = min(max(134 - (int)(__float_as_uint(top) >> 23), -119), 126);
        const float up = power_of_two(e), down = power_of_two(-e);
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            const uint32_t zz[4] = {z[w].x, z[w].y, z[w].z, z[w].w};
            // a word of four codes, and the four elements beside them: two for either half of the product's 16
#pragma unroll
            for (int i = 0; i < 4; ++i)
                qf[nt][2 * w + (i >> 1)][i & 1] = pack_f16x2(__uint_as_float(zz[i] << 16) * up, __uint_as_float(zz[i] & 0xffff0000u) * up);
        }
        // of the columns this thread has of S^T: 2 t, 2 t + 1
#pragma unroll
        for (int c = 0; c < 2; ++c) q_scale[nt][c] = p.scale_log2 * __shfl_sync(0xffffffffu, down, 8 * t + 4 * c);
    }
    if (P_now != P || C_now != C) {
        if (threadIdx.x == 0 && p.status) atomicCAS(p.status, 0, WPP_ERR_PLAN_MISMATCH);
        // (the combine pass reads the parts of a refused request too: none of them has seen a key)
        if (un.split_slot >= 0 && threadIdx.x < rows) p.ws_lse[((int64_t)un.split_slot * 2 + un.row0[1]) * 128 + un.head[1] + threadIdx.x] = -INFINITY;
        copies_wait<0>();
        if (kCluster) {
            __syncthreads();
            if (threadIdx.x < rows) reinterpret_cast<float*>(smem + M::kOffPartLse)[threadIdx.x] = -INFINITY;
        }
        return;
    }
    State<D, NT> st;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int mt = 0; mt < kSteps; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[nt][mt][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) st.m[nt][i] = st.l[nt][i] = 0.f;
    }
    st.v_exp = 0.f;

    bool first = true;
    uint32_t at = 0, fill = (M::kDepth - 1) * M::kStage;               // offsets in the ring: of the keys, and of the next ones to be asked for
    for (; key < seen; key += kStride) {
        copies_wait<M::kDepth - 2>();
        __syncwarp();                          // every lane's copies are here, and every lane has read the stage before
        request(key + (M::kDepth - 1) * kStride, ring + fill);
        fill = at;
        if (key + kKeys - 1 <= first_pos && key + kKeys <= seen)
            step<D, NT, kCluster, false>(st, ring + at, qf, q_scale, key, first_pos, toks, seen - 1, first, g, t);
        else
            step<D, NT, kCluster, true>(st, ring + at, qf, q_scale, key, first_pos, toks, seen - 1, first, g, t);
        first = false;
        at = at == (M::kDepth - 1) * M::kStage ? 0u : at + M::kStage;
    }
    if (bad && p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
    copies_wait<0>();
    __syncthreads();                           // the warps' results take the stages' place

    // ---- the warps' parts joined
    const float unit_of_sums = fast_exp2(st.v_exp);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float l = st.l[nt][c];
#pragma unroll
            for (int w = 4; w < 32; w *= 2) l += __shfl_xor_sync(0xffffffffu, l, w);
            const int n = 8 * nt + 2 * t + c;
            if (g == 0) s_ml[warp][n] = make_float2(l == 0.f ? -INFINITY : st.m[nt][c], l);
#pragma unroll
            for (int mt = 0; mt < kSteps; ++mt)
                *reinterpret_cast<float2*>(&s_o[warp][n][g * (D / 8) + 2 * mt]) = make_float2(st.o[nt][mt][c] * unit_of_sums, st.o[nt][mt][2 + c] * unit_of_sums);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * (D / 4); i += 32 * kWarps) {
        const int n = i / (D / 4), c = i % (D / 4) * 4;
        float mm = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, s_ml[w][n].x);
        const float ref = mm == -INFINITY ? 0.f : mm;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
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
        if (kCluster) {
            *reinterpret_cast<float4*>(smem + M::kOffPart + (n * D + c) * 4) = acc;
            if (c == 0) reinterpret_cast<float*>(smem + M::kOffPartLse)[n] = lse2;
        } else if (un.split_slot < 0) {
            const int64_t tok = (int64_t)q_off + un.row0[0] + n % toks, head = un.head[0] + n / toks;
            *reinterpret_cast<uint2*>(p.out + tok * p.o_token_stride + head * p.o_head_stride + c) =
                make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
            if (p.lse && c == 0) p.lse[tok * p.num_q_heads + head] = fmaxf(lse2 * 0.6931471805599453f, -INFINITY);
        } else {
            const int64_t at_row = ((int64_t)un.split_slot * 2 + un.row0[1]) * 128 + un.head[1] + n;
            *reinterpret_cast<float4*>(p.ws_o + at_row * D + c) = acc;
            if (c == 0) p.ws_lse[at_row] = lse2;
        }
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(32 * kWarps, NT == 1 ? 3 : 2) wpp_kv8_few_kernel(const Kv4AttnParams p) {
    extern __shared__ __align__(128) uint8_t smem[];
    grid_launch_dependents();
    grid_dependency_wait();
    // units: those that the plan says, or (few_counter) the CTA's own and then whichever is next
    __shared__ int s_next;
    const bool taken = p.few_counter != nullptr, one_each = p.num_few == (int)gridDim.x;
    int u = blockIdx.x, end = taken ? p.num_few : u + 1;
    if (!taken && !one_each) {
        const int32_t* range = reinterpret_cast<const int32_t*>(static_cast<const char*>(p.plan) + p.off_few_ctas) + blockIdx.x;
        u = range[0];
        end = range[1];
    }
    Unit unit = unit_at(p, u);
    while (true) {
        if (taken && threadIdx.x == 0) s_next = end > (int)gridDim.x ? (int)(gridDim.x + atomicAdd(p.few_counter, 1u)) : end;      // (while the unit is under way)
        run_unit<D, NT, false>(p, unit, smem);
        if (!taken && u + 1 >= end) break;
        __syncthreads();                       // (the next unit's keys take the place of this one's results)
        u = taken ? s_next : u + 1;
        if (u >= end) break;
        unit = unit_at(p, u);
        if (taken) __syncthreads();            // (read by all before it is written again)
    }
}

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {       // the same place in another CTA's shared memory
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// A wave of few blocks: a cluster has a block's parts and joins them in shared memory, so that there is no combine pass, and no
// partial result in global memory.  Each of its 2^log_parts CTAs takes as many of the rows' pieces of four elements, one lane for each part.
template <int D, int NT>
__global__ void __launch_bounds__(32 * kWarps, 2) wpp_kv8_cluster_kernel(const Kv4AttnParams p, const int log_parts) {
    using M = Smem<D, NT, true>;
    extern __shared__ __align__(128) uint8_t smem[];
    grid_launch_dependents();
    grid_dependency_wait();
    const Unit unit = unit_at(p, blockIdx.x);
    run_unit<D, NT, true>(p, unit, smem);
    cluster_barrier();
    const WppUnit& un = unit.un;
    const int parts = 1 << log_parts, rank = blockIdx.x & (parts - 1), part = threadIdx.x & (parts - 1), toks = un.rows[0], rows = toks * un.rows[1];
    const uint32_t rows_at = in_cta(smem_u32(smem) + M::kOffPart, (uint32_t)part), lse_at = in_cta(smem_u32(smem) + M::kOffPartLse, (uint32_t)part);
    const int groups = 32 * kWarps >> log_parts;                // pieces that the CTA's lanes take at a time
    for (int i0 = rank * groups; i0 < rows * (D / 4); i0 += groups << log_parts) {
        const int i = i0 + (int)(threadIdx.x >> log_parts), n = min(i / (D / 4), rows - 1), c = i % (D / 4) * 4;
        float z;
        float4 x;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(z) : "r"(lse_at + n * 4));
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(rows_at + (n * D + c) * 4));
        float top = z;
        for (int w = 1; w < parts; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        const bool seen = z != -INFINITY;                              // (what a part that saw no key of the row left is not looked at)
        const float a = seen ? fast_exp2(z - top) : 0.f;
        float sum = a;
        x = seen ? make_float4(a * x.x, a * x.y, a * x.z, a * x.w) : make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 1; w < parts; w *= 2) {
            sum += __shfl_xor_sync(0xffffffffu, sum, w);
            x.x += __shfl_xor_sync(0xffffffffu, x.x, w);
            x.y += __shfl_xor_sync(0xffffffffu, x.y, w);
            x.z += __shfl_xor_sync(0xffffffffu, x.z, w);
            x.w += __shfl_xor_sync(0xffffffffu, x.w, w);
        }
        if (part != 0 || i >= rows * (D / 4)) continue;
        const bool nan = sum != sum;
        const float inv = nan ? NAN : sum > 0.f ? 1.f / sum : 0.f;
        const int64_t tok = (int64_t)unit.q_off + un.row0[0] + n % toks, head = un.head[0] + n / toks;
        *reinterpret_cast<uint2*>(p.out + tok * p.o_token_stride + head * p.o_head_stride + c) =
            make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
        if (p.lse && c == 0) p.lse[tok * p.num_q_heads + head] = sum > 0.f && !nan ? (top + log2f(sum)) * 0.6931471805599453f : -INFINITY;
    }
    cluster_barrier();                         // (nobody leaves while another one reads its shared memory)
}

template <class Kernel, class... Args>
static cudaError_t launch_kernel(Kernel kernel, bool (&attr_set)[64], int num_ctas, int threads, int smem, int cluster, cudaStream_t stream, Args... args) {
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e == cudaSuccess && cluster > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)num_ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = (unsigned)cluster;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D, int NT>
static cudaError_t launch_nt(const Kv4AttnParams& p, int num_ctas, int log_parts, cudaStream_t stream) {
    static bool attr_set[64] = {}, attr_set_cluster[64] = {};
    if (log_parts > 0)
        return launch_kernel(wpp_kv8_cluster_kernel<D, NT>, attr_set_cluster, num_ctas, 32 * kWarps, Smem<D, NT, true>::kBytes,
                             1 << log_parts, stream, p, log_parts);
    return launch_kernel(wpp_kv8_few_kernel<D, NT>, attr_set, num_ctas, 32 * kWarps, Smem<D, NT, false>::kBytes, 0, stream, p);
}

}  // namespace kv8few
}  // namespace wpp

// log_parts > 0: the units are parts of blocks, 2^log_parts of each, that clusters of as many CTAs join
extern "C" int wpp_launch_kv8_few(int head_dim, const wpp::Kv4AttnParams* p, int num_ctas, int max_rows, int log_parts, void* stream) {
    using namespace wpp::kv8few;
    const cudaStream_t s = (cudaStream_t)stream;
    if (head_dim == 128) return (int)(max_rows <= 8 ? launch_nt<128, 1>(*p, num_ctas, log_parts, s) : launch_nt<128, 2>(*p, num_ctas, log_parts, s));
    return (int)(max_rows <= 8 ? launch_nt<64, 1>(*p, num_ctas, log_parts, s) : launch_nt<64, 2>(*p, num_ctas, log_parts, s));
}
