// Attention of few query rows over a cache held in 4 bits: single new tokens, and chunks' row blocks of at most WPP_FEW_ROWS rows
// (tokens x heads of a KV group).
//
// With k_j = least_j + scale_j c_j (c_j the codes), the score of key j for row n is
//     sm_scale (scale_j <q_n, c_j> + least_j sum q_n),
// so the tensor cores multiply the codes themselves, which bf16 holds exactly, and two numbers per key finish the score in fp32;
// in the same way sum_j p_j v_j = sum_j (p_j scale_j) c_j + sum_j p_j least_j, of which only p_j scale_j is rounded to bf16.
//
// What bounds it is the cache's bytes, and next to them the instructions that make bf16 numbers of codes: about one per code.  So
// nothing else is done per code: a warp takes 16 keys at a time straight from global memory in the order the tensor cores' fragments
// want (which element of a row stands at which place of a product does not matter as long as both factors agree), keys are the
// rows and query rows the columns of the products (S^T = K Q^T, O^T = V^T P^T: eight columns, of which the group's heads fill all),
// and the two products share no data but P, which a transposing move turns round in registers.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_plan_format.h"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr int kFewWarps = 4;
constexpr float kFewSlack = 16.f;          // a row keeps its reference while its scores stay below reference + 16 (log2)

// D += A B, 16 x 8 x 16, bf16 in, fp32 out
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// Two codes of a word, four bits each at bits s and s + 16, as the bf16 numbers 128 + code (exact).
__device__ __forceinline__ uint32_t codes_128(uint32_t w, int s) { return ((w >> s) & 0x000f000fu) | 0x43004300u; }
// The same as code - 8 (exact).
__device__ __forceinline__ uint32_t codes_8(uint32_t w, int s) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(codes_128(w, s)), "r"(0x43084308u));
    return r;
}
template <int kWords>
__device__ __forceinline__ void load_words(uint32_t (&w)[kWords], const uint8_t* at) {
    if constexpr (kWords == 4) {
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(at));
    } else if constexpr (kWords == 2) {
        asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(at));
    } else {
        asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(at));
    }
}

// What a thread holds of 16 keys: lane 4 g + t has, of keys g and g + 8, columns [t D / 4, (t + 1) D / 4) of K; of keys 2 t, 2 t + 1,
// 2 t + 8, 2 t + 9, columns [g D / 8, (g + 1) D / 8) of V; and the number pairs of keys g and g + 8.
template <int D>
struct FewKeys {
    uint32_t k[2][D / 32];
    uint32_t v[4][D / 64];
    uint32_t kp[2], vp[2];
    __device__ __forceinline__ void load(const uint8_t* kb, const uint8_t* vb, int slot, int page_size, int g, int t) {
        const uint8_t* pairs = kb + page_size * (D / 2);
        const uint8_t* vpairs = vb + page_size * (D / 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) load_words<D / 32>(k[i], kb + (slot + g + 8 * i) * (D / 2) + t * (D / 8));
#pragma unroll
        for (int i = 0; i < 4; ++i) load_words<D / 64>(v[i], vb + (slot + 2 * t + (i & 1) + 8 * (i >> 1)) * (D / 2) + g * (D / 16));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            kp[i] = *reinterpret_cast<const uint32_t*>(pairs + (slot + g + 8 * i) * 4);
            vp[i] = *reinterpret_cast<const uint32_t*>(vpairs + (slot + g + 8 * i) * 4);
        }
    }
};
__device__ __forceinline__ float pair_least(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float pair_scale(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

template <int D, int NT>
__global__ void __launch_bounds__(32 * kFewWarps) wpp_kv4_few_kernel(const Kv4AttnParams p) {
    constexpr int kSteps = D / 16;             // 16-wide pieces of a row
    __shared__ float s_o[kFewWarps][8 * NT][D + 4];
    __shared__ float2 s_ml[kFewWarps][8 * NT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    grid_dependency_wait();
    const char* plan = static_cast<const char*>(p.plan);
    const WppUnit un = reinterpret_cast<const WppUnit*>(plan + p.off_units)[blockIdx.x];
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
    const int kv_len = min(P + C, un.kv_end * WPP_TILE_N), key_begin = un.kv_begin * WPP_TILE_N;
    const int seen = min(kv_len, first_pos + toks);                                        // keys that some row sees end here
    const int tiles = (max(seen - key_begin, 0) + 15) / 16;
    const int kvh = un.head[0] / p.group, page_shift = 31 - __clz(p.page_size);
    const int32_t* table = p.block_tables + (int64_t)un.request * p.max_blocks;

    // ---- Q as the products' second factor, and the sums of its rows
    uint32_t qf[NT][kSteps][2];
    float q_sum[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = 8 * nt + g;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kSteps / 2; ++w) {
            uint4 z = make_uint4(0, 0, 0, 0);
            if (n < rows) {
                const int head = un.head[0] + n / toks, tok = q_off + un.row0[0] + n % toks;
                z = *reinterpret_cast<const uint4*>(p.q + (int64_t)tok * p.q_token_stride + (int64_t)head * p.q_head_stride + t * (D / 4) + 8 * w);
            }
            // elements s and s + 4 of the eight stand side by side, as the codes of a word do
            qf[nt][2 * w][0] = __byte_perm(z.x, z.z, 0x5410);
            qf[nt][2 * w][1] = __byte_perm(z.x, z.z, 0x7632);
            qf[nt][2 * w + 1][0] = __byte_perm(z.y, z.w, 0x5410);
            qf[nt][2 * w + 1][1] = __byte_perm(z.y, z.w, 0x7632);
            const uint32_t zz[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += __uint_as_float(zz[i] << 16) + __uint_as_float(zz[i] & 0xffff0000u);
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        q_sum[nt][0] = __shfl_sync(0xffffffffu, sum, 8 * t);            // of the columns this thread has of S^T: 2 t, 2 t + 1
        q_sum[nt][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
    }
    int limit[NT][2];                                                  // last key that the column's row sees
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        limit[nt][0] = first_pos + (8 * nt + 2 * t) % toks;
        limit[nt][1] = first_pos + (8 * nt + 2 * t + 1) % toks;
    }

    float o[NT][kSteps][4], m[NT][2], l[NT][2], off[NT][2];            // off: sum of p (least + 8 scale)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int mt = 0; mt < kSteps; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[nt][mt][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            m[nt][i] = -INFINITY;
            l[nt][i] = off[nt][i] = 0.f;
        }
    }

    int bad = 0;
    auto page_of = [&](int tile) -> int {                              // physical page of a 16-key tile, 0 if the table has none
        if (tile >= tiles) return 0;
        const int page = table[(key_begin + tile * 16) >> page_shift];
        if (page >= 0 && page < p.num_pages) return page;
        bad = 1;
        return 0;
    };
    auto load = [&](FewKeys<D>& x, int tile, int page) {
        if (tile >= tiles) return;
        const int64_t block = page * p.page_bytes + kvh * p.head_bytes;
        x.load(p.k_cache + block, p.v_cache + block, (key_begin + tile * 16) & (p.page_size - 1), p.page_size, g, t);
    };
    FewKeys<D> next;
    int next_page = page_of(warp);
    load(next, warp, next_page);
    next_page = page_of(warp + kFewWarps);
    for (int tile = warp; tile < tiles; tile += kFewWarps) {
        FewKeys<D> x = next;
        load(next, tile + kFewWarps, next_page);
        next_page = page_of(tile + 2 * kFewWarps);
        const int key0 = key_begin + tile * 16;

        // ---- S^T = (128 + codes) Q^T, then the scores in log2 units
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            const uint32_t wa = x.k[0][ks >> 1], wb = x.k[1][ks >> 1];
            const int sh = 8 * (ks & 1);
            const uint32_t a0 = codes_128(wa, sh), a1 = codes_128(wb, sh), a2 = codes_128(wa, sh + 4), a3 = codes_128(wb, sh + 4);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_16816(s[nt], a0, a1, a2, a3, qf[nt][ks][0], qf[nt][ks][1]);
        }
        float vs[2], vo[2];
        const bool masked = key0 + 15 > first_pos;                     // some row does not see every key of the tile
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float ks = pair_scale(x.kp[i]) * p.scale_log2, ko = fmaf(-128.f, ks, pair_least(x.kp[i]) * p.scale_log2);
            vs[i] = pair_scale(x.vp[i]);
            vo[i] = fmaf(8.f, vs[i], pair_least(x.vp[i]));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) s[nt][2 * i + c] = fmaf(s[nt][2 * i + c], ks, ko * q_sum[nt][c]);
        }
        if (masked) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key0 + g + 8 * (i >> 1) > limit[nt][i & 1]) s[nt][i] = -INFINITY;
        }
        // ---- references move only where a score is far above them
        bool move = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) move |= fmaxf(s[nt][c], s[nt][2 + c]) > m[nt][c] + kFewSlack;
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float mx = fmaxf(m[nt][c], fmaxf(s[nt][c], s[nt][2 + c]));
#pragma unroll
                    for (int w = 4; w < 32; w *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                    const float a = m[nt][c] == -INFINITY ? 0.f : fast_exp2(m[nt][c] - mx);
                    m[nt][c] = mx;
                    l[nt][c] *= a;
                    off[nt][c] *= a;
#pragma unroll
                    for (int mt = 0; mt < kSteps; ++mt) {
                        o[nt][mt][c] *= a;
                        o[nt][mt][2 + c] *= a;
                    }
                }
        }
        // ---- P^T, its rows times the keys' V scales, turned round into the second factor of O^T = V^T P^T
        uint32_t pb[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float e[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float ref = m[nt][c] == -INFINITY ? 0.f : m[nt][c];
                    const bool out = masked && key0 + g + 8 * i > limit[nt][c];
                    e[c] = out ? 0.f : fast_exp2(s[nt][2 * i + c] - ref);
                    l[nt][c] += e[c];
                    off[nt][c] = out ? off[nt][c] : fmaf(e[c], vo[i], off[nt][c]);
                    e[c] = out ? 0.f : e[c] * vs[i];
                }
                pb[nt][i] = transpose_8x8(pack_bf16x2(e[0], e[1]));
            }
        // ---- O^T += (codes - 8)^T P^T: a word holds two codes of one key and two of the next, one above the other
#pragma unroll
        for (int w = 0; w < D / 64; ++w)
#pragma unroll
            for (int hw = 0; hw < 2; ++hw) {
                const uint32_t lo = __byte_perm(x.v[0][w], x.v[1][w], hw ? 0x7632 : 0x5410);
                const uint32_t hi = __byte_perm(x.v[2][w], x.v[3][w], hw ? 0x7632 : 0x5410);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t a0 = codes_8(lo, 8 * u), a1 = codes_8(lo, 8 * u + 4), a2 = codes_8(hi, 8 * u), a3 = codes_8(hi, 8 * u + 4);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_16816(o[nt][4 * w + 2 * hw + u], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
                }
            }
    }
    if (bad && p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);

    // ---- the warps' parts joined
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int w = 4; w < 32; w *= 2) {
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], w);
                off[nt][c] += __shfl_xor_sync(0xffffffffu, off[nt][c], w);
            }
            const int n = 8 * nt + 2 * t + c;
            if (g == 0) s_ml[warp][n] = make_float2(m[nt][c], l[nt][c]);
#pragma unroll
            for (int mt = 0; mt < kSteps; ++mt) {
                const int d0 = g * (D / 8) + 2 * mt;       // element 8 w + 4 hw + 2 u of the thread's columns, mt = 4 w + 2 hw + u
                *reinterpret_cast<float2*>(&s_o[warp][n][d0]) = make_float2(o[nt][mt][c] + off[nt][c], o[nt][mt][2 + c] + off[nt][c]);
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
            const float a = ml.x == -INFINITY ? 1.f : fast_exp2(ml.x - ref);
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

template <int D>
static cudaError_t launch_few(const Kv4AttnParams& p, int num_units, int max_rows, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)num_units);
    cfg.blockDim = dim3(32 * kFewWarps);
    cfg.stream = stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, max_rows <= 8 ? wpp_kv4_few_kernel<D, 1> : wpp_kv4_few_kernel<D, 2>, p);
}

}  // namespace wpp

extern "C" int wpp_launch_kv4_few(int head_dim, const wpp::Kv4AttnParams* p, int num_units, int max_rows, void* stream) {
    return (int)(head_dim == 128 ? wpp::launch_few<128>(*p, num_units, max_rows, (cudaStream_t)stream)
                                 : wpp::launch_few<64>(*p, num_units, max_rows, (cudaStream_t)stream));
}
