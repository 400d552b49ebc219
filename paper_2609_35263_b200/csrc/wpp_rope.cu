// Rotary positions of queries and keys, alone and on the way into the pages of a bf16 cache.
//
// A pair (a, b) of a row's elements becomes magnitude (a cos x - b sin x, a sin x + b cos x), x = position * frequency.  A frequency comes as a
// 64-bit fraction of a turn per position: position * turns modulo 2^64 is the position's fraction of a turn, with no error but the
// frequency's own 2^-65 a position, however far the position.  32 bits of it, as fp32 and times 2 pi, are the angle within 2^-21 (from -pi to pi
// a half step of each rounding is 2^-23 or less); with the errors of sin.approx and cos.approx there, about 2^-21, the factors are within
// 2^-20, far below the results' rounding to bf16.
//
// The rows' bytes bound it.  A warp takes a token and some of its heads, D / 16 lanes a head: a lane has the pairs that two 16-byte vectors
// of a head hold, the same ones in every head, and so works out its eight angles once.  The two vectors are rot_dim / 2 elements apart,
// whichever elements are paired.  The loads of four passes' rows go out before the first is used.  Few tokens are spread over more warps,
// down to one row for each group of lanes: then the launch is what it takes (64 tokens of 32/8 heads of 128 2.1 us, of one warp each 4.0).
// 8,192 tokens, 32/8 heads of 128, 64 elements of each turned: 28.8 us, 5.8 TB/s (90 % of the measured copy); 16,742 tokens of 64/8 heads into
// the cache 109 us, 6.3 TB/s.  CTAs of two warps, because a large grid ends as they do: of eight 31.1 and 111 us.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "wpp_device.h"
#include "wpp_ptx.cuh"

namespace wpp {

constexpr int kRopeWarps = 2, kRopeAhead = 4;      // of a CTA; passes whose loads are out at a time
constexpr int64_t kRopeWarpsPerSm = 32;            // as many before a warp takes more than one pass

__device__ __forceinline__ void rotate(uint32_t& wa, uint32_t& wb, const float (&c)[2], const float (&s)[2]) {
    const float a0 = __uint_as_float(wa << 16), a1 = __uint_as_float(wa & 0xffff0000u), b0 = __uint_as_float(wb << 16), b1 = __uint_as_float(wb & 0xffff0000u);
    wa = pack_bf16x2(fmaf(a0, c[0], -(b0 * s[0])), fmaf(a1, c[1], -(b1 * s[1])));
    wb = pack_bf16x2(fmaf(a0, s[0], b0 * c[0]), fmaf(a1, s[1], b1 * c[1]));
}
__device__ __forceinline__ void rotate_neighbours(uint32_t& w, float c, float s) {
    const float a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u);
    w = pack_bf16x2(fmaf(a, c, -(b * s)), fmaf(a, s, b * c));
}

// kWrite: keys and values go to their slots of the cache
template <int D, bool kNeighbours, bool kWrite>
__global__ void __launch_bounds__(32 * kRopeWarps, 24 / kRopeWarps) wpp_rope_kernel(const RopeParams p) {
    constexpr int kLanes = D / 16, kHeads = 32 / kLanes;       // of a head; of a warp at a time
    if (!p.few) grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, sub = lane % kLanes;
    const int64_t unit = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
    const int64_t tok = unit >> 32 ? unit / p.units_per_token : (int64_t)((uint32_t)unit / (uint32_t)p.units_per_token);      // (a 64-bit division takes seventy operations)
    if (tok >= p.total_tokens) return;
    const int pass0 = (int)(unit - tok * p.units_per_token) * p.passes, heads = p.num_q_heads + p.num_k_heads + (kWrite ? p.num_k_heads : 0);
    const int pass1 = min(pass0 + p.passes, (heads + kHeads - 1) / kHeads);
    const int n = p.rot_vecs;                                  // lanes of a head that turn: vectors sub and n + sub; the others: 2 n + .. as they are
    const bool turns = sub < n;
    const int at_a = turns ? sub * 8 : n * 16 + (sub - n) * 8, apart = (turns ? n : kLanes - n) * 8;

    int64_t slot = -1, cache_at = 0;
    if (kWrite) {
        slot = p.slots[tok];
        if (slot >= p.num_slots || slot < -1) {
            if (lane == 0 && p.status) atomicCAS(p.status, 0, WPP_ERR_BOUNDS);
            slot = -1;
        }
        if (slot >= 0) cache_at = (slot >> p.page_shift) * p.kv_page_stride + (slot & ((1 << p.page_shift) - 1)) * p.kv_token_stride;
    }
    // where head h of the token is read and written; null: not at all
    auto row_of = [&](int h, const __nv_bfloat16*& src, __nv_bfloat16*& dst, bool& turned) {
        turned = turns;
        if (h < p.num_q_heads) {
            src = p.q + tok * p.q_token_stride + h * p.q_head_stride;
            dst = !turns && p.q_in_place ? nullptr : p.q_out + tok * p.qo_token_stride + h * p.qo_head_stride;
        } else if (h < p.num_q_heads + p.num_k_heads) {
            h -= p.num_q_heads;
            src = p.k + tok * p.k_token_stride + h * p.k_head_stride;
            if (kWrite) dst = slot < 0 ? nullptr : p.k_out + cache_at + h * p.kv_head_stride;
            else dst = !turns && p.k_in_place ? nullptr : p.k_out + tok * p.ko_token_stride + h * p.ko_head_stride;
        } else {
            h -= p.num_q_heads + p.num_k_heads;
            src = p.v + tok * p.v_token_stride + h * p.v_head_stride;
            dst = h < p.num_k_heads && slot >= 0 ? p.v_out + cache_at + h * p.kv_head_stride : nullptr;
            turned = false;
        }
    };

    float c[8], s[8];
    bool angles = false;
    for (int pass = pass0; pass < pass1; pass += kRopeAhead) {
        uint4 a[kRopeAhead], b[kRopeAhead];
        __nv_bfloat16* dst[kRopeAhead];
        bool turned[kRopeAhead];
#pragma unroll
        for (int i = 0; i < kRopeAhead; ++i) {
            const int h = (pass + i) * kHeads + lane / kLanes;
            const __nv_bfloat16* src = nullptr;
            dst[i] = nullptr;
            turned[i] = false;
            a[i] = b[i] = make_uint4(0, 0, 0, 0);
            if (pass + i < pass1 && h < heads) row_of(h, src, dst[i], turned[i]);
            if (dst[i]) {
                a[i] = *reinterpret_cast<const uint4*>(src + at_a);
                b[i] = *reinterpret_cast<const uint4*>(src + at_a + apart);
            }
        }
        if (!angles) {                                         // (under way meanwhile: the first rows)
            angles = true;
            const int64_t pos = p.positions[tok];
            uint64_t turn[8] = {};
            if (turns) {
                // the pairs of the lane's two vectors, four elements or pairs each
                const ulonglong2* t0 = reinterpret_cast<const ulonglong2*>(p.turns + (kNeighbours ? 4 : 8) * sub);
                const ulonglong2* t1 = reinterpret_cast<const ulonglong2*>(p.turns + (kNeighbours ? 4 * (n + sub) : 8 * sub + 4));
                const ulonglong2 t[4] = {t0[0], t0[1], t1[0], t1[1]};
#pragma unroll
                for (int i = 0; i < 4; ++i) { turn[2 * i] = t[i].x; turn[2 * i + 1] = t[i].y; }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t part = (int32_t)(uint32_t)((turn[i] * (uint64_t)pos) >> 32);     // of a turn, in 2^-32, from minus a half
                const float x = (float)part * 1.4629180792671596e-9f;                           // 2 pi 2^-32
                c[i] = __cosf(x) * p.magnitude;
                s[i] = __sinf(x) * p.magnitude;
            }
        }
#pragma unroll
        for (int i = 0; i < kRopeAhead; ++i) {
            if (!dst[i]) continue;
            if (turned[i]) {
                uint32_t wa[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, wb[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (kNeighbours) {
                        rotate_neighbours(wa[j], c[j], s[j]);
                        rotate_neighbours(wb[j], c[4 + j], s[4 + j]);
                    } else {
                        const float cc[2] = {c[2 * j], c[2 * j + 1]}, ss[2] = {s[2 * j], s[2 * j + 1]};
                        rotate(wa[j], wb[j], cc, ss);
                    }
                }
                a[i] = make_uint4(wa[0], wa[1], wa[2], wa[3]);
                b[i] = make_uint4(wb[0], wb[1], wb[2], wb[3]);
            }
            *reinterpret_cast<uint4*>(dst[i] + at_a) = a[i];
            *reinterpret_cast<uint4*>(dst[i] + at_a + apart) = b[i];
        }
    }
}

template <int D>
static cudaError_t launch_rope(const RopeParams& in, int neighbours, int write, int num_sms, cudaStream_t stream) {
    constexpr int kHeads = 512 / D;
    RopeParams p = in;
    const int64_t heads = p.num_q_heads + (int64_t)p.num_k_heads * (write ? 2 : 1), passes = (heads + kHeads - 1) / kHeads;
    const int64_t want = num_sms * kRopeWarpsPerSm;
    p.passes = (int32_t)(p.total_tokens * passes <= want ? 1 : p.total_tokens >= want ? passes : (p.total_tokens * passes + want - 1) / want);
    p.units_per_token = (int32_t)((passes + p.passes - 1) / p.passes);
    const int64_t blocks = (p.total_tokens * p.units_per_token + kRopeWarps - 1) / kRopeWarps;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    p.few = blocks * kRopeWarps <= 24 * (int64_t)num_sms;      // (see wpp_launch_kv4_append)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(32 * kRopeWarps);
    cfg.stream = stream;
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &overlap;
    cfg.numAttrs = p.few ? 1 : 0;
    if (write) return cudaLaunchKernelEx(&cfg, neighbours ? wpp_rope_kernel<D, true, true> : wpp_rope_kernel<D, false, true>, p);
    return cudaLaunchKernelEx(&cfg, neighbours ? wpp_rope_kernel<D, true, false> : wpp_rope_kernel<D, false, false>, p);
}

}  // namespace wpp

extern "C" int wpp_launch_rope(const wpp::RopeParams* p, int head_dim, int neighbours, int write, int num_sms, void* stream) {
    if (p->total_tokens == 0) return 0;
    return (int)(head_dim == 128 ? wpp::launch_rope<128>(*p, neighbours, write, num_sms, (cudaStream_t)stream)
                                 : wpp::launch_rope<64>(*p, neighbours, write, num_sms, (cudaStream_t)stream));
}

// Host only: the pairs' frequencies as turns per position, in 64 bits behind the point.
extern "C" int wpp_rope_frequencies(const wpp_rope_scaling* sc, uint64_t* turns, float* magnitude) {
    if (!sc || !turns || !magnitude) return WPP_ERR_INVALID_ARG;
    const int n = sc->rot_dim;
    if (n < 16 || n > 128 || n % 16 != 0 || sc->kind < WPP_ROPE_PLAIN || sc->kind > WPP_ROPE_TURNS) return WPP_ERR_UNSUPPORTED;
    if (!(sc->base > 1.0) || !(sc->base <= 1e30)) return WPP_ERR_INVALID_ARG;
    if (sc->kind != WPP_ROPE_PLAIN && (!(sc->factor >= 1.0) || !(sc->factor <= 1e9))) return WPP_ERR_INVALID_ARG;
    const bool bands = sc->kind == WPP_ROPE_WAVELENGTH || sc->kind == WPP_ROPE_TURNS;
    const double low = sc->low != 0.0 ? sc->low : 1.0, high = sc->high != 0.0 ? sc->high : sc->kind == WPP_ROPE_TURNS ? 32.0 : 4.0;
    if (bands && (!(sc->original_context >= 1.0) || !(sc->original_context <= 1e12) || !(low > 0.0) || !(high > low) || !(high <= 1e12)))
        return WPP_ERR_INVALID_ARG;
    const long double two_pi = 6.283185307179586476925286766559L;
    long double base = sc->base;
    if (sc->kind == WPP_ROPE_BASE) base *= powl((long double)sc->factor, (long double)n / (n - 2));
    // the pairs of WPP_ROPE_TURNS between which the factor comes in
    const double log_base = 2.0 * log(sc->base), ctx = sc->original_context;
    const double from = bands ? fmax(floor(n * log(ctx / (6.283185307179586 * high)) / log_base), 0.0) : 0.0;
    const double to = bands ? fmin(ceil(n * log(ctx / (6.283185307179586 * low)) / log_base), n - 1.0) : 0.0;
    for (int i = 0; i < n / 2; ++i) {
        long double f = powl(base, -2.0L * i / n), stretched = f;          // radians per position
        if (sc->kind != WPP_ROPE_PLAIN && sc->kind != WPP_ROPE_BASE) stretched = f / sc->factor;
        if (sc->kind == WPP_ROPE_LINEAR) {
            f = stretched;
        } else if (bands) {
            const long double share = sc->kind == WPP_ROPE_WAVELENGTH ? (ctx * f / two_pi - low) / ((long double)high - low)
                                                                       : 1.0L - (i - from) / (to != from ? (long double)to - from : 0.001L);
            const long double kept = share < 0.0L ? 0.0L : share > 1.0L ? 1.0L : share;
            f = stretched * (1.0L - kept) + f * kept;
        }
        turns[i] = (uint64_t)(f / two_pi * 18446744073709551616.0L + 0.5L);
    }
    *magnitude = sc->kind == WPP_ROPE_TURNS ? (float)(0.1 * log(sc->factor) + 1.0) : 1.0f;
    return WPP_OK;
}
