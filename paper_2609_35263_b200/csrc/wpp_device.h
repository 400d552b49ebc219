// Kernel parameter blocks and launch entry points shared by the launch code and the kernel files.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <stdint.h>

#include "../../include/wpp.h"

namespace wpp {

// Counters of the SM-wide attention kernel, per context: key steps of the softmax warps and those that rescaled O, added up in
// device memory; a launch leaves the totals in one of the context's kCounterSlots pairs of words in mapped host memory.
constexpr int kCounterContexts = 256, kCounterSlots = 16;
constexpr int kCounterBytes = kCounterContexts * kCounterSlots * 16;      // of the host side, which is aligned to its size

struct AttnParams {
    const void* plan;                // device copy of the plan
    const int32_t* block_tables;     // [R][max_blocks]
    const int32_t* prefix_lens;      // [R]
    const int32_t* chunk_lens;       // [R]
    __nv_bfloat16* out;              // [T][Hq][d]
    float* lse;                      // [T][Hq] or null
    float* ws_o;                     // split partials: [slots][2][128][d]
    float* ws_lse;                   // [slots][2][128], log2 units
    int32_t* status;                 // sticky device status word or null
    uint32_t* tile_counter;          // zeroed before the launch: how many tiles have been taken beyond the first one per CTA;
                                     // or null: every CTA has one tile; (small shape) round k of the CTAs takes tiles k gridDim ..,
                                     // rotated by k
    unsigned long long* totals;      // or null: the launch's slot of the counters' host side (see kCounterContexts)
    int64_t o_token_stride, o_head_stride;
    int32_t num_q_heads, group, page_size, max_blocks, num_pages;
    float scale_log2;                // sm_scale * log2(e)
};

// The small shape's parameters (apart from AttnParams: with more members there the SM-wide kernel, at its register limit,
// spills twice as much).
struct SmallAttnParams : AttnParams {
    uint32_t off_q_offsets, off_prefix, off_units;   // of the plan's arrays (as in its header: one dependent read less)
    int32_t num_units;
    int32_t item_shift;              // 1 if an item is half a unit, 0 if no unit has a second half
};

struct AppendParams {
    const void* plan;
    const uint4* k_new;
    const uint4* v_new;
    uint4* k_cache;
    uint4* v_cache;
    const int32_t* block_tables;
    const int32_t* prefix_lens;
    const int32_t* chunk_lens;
    int32_t* status;
    int64_t kvnew_token_stride, kvnew_head_stride;       // in 16-byte units
    int64_t kv_page_stride, kv_head_stride, kv_token_stride;
    int32_t num_requests, num_kv_heads, vec_per_row, page_size, max_blocks, num_pages;
    int32_t few;                     // the SMs hold the whole grid at once
    uint32_t off_q_offsets, off_prefix;                  // of the plan's arrays (as in its header: one dependent read less)
    int64_t total_new_tokens;
};

// 4- and 8-bit caches.  Pools in bytes; a block (page, KV head) is page_size rows of head_dim / 2 bytes and, behind them, as many pairs of
// bf16 numbers (least value, scale); or page_size rows of head_dim bytes and, behind them, an fp32 scale.
struct Kv4AppendParams {
    const void* plan;
    const __nv_bfloat16* k_new;
    const __nv_bfloat16* v_new;
    uint8_t* k_cache;
    uint8_t* v_cache;
    const int32_t* block_tables;
    const int32_t* prefix_lens;
    const int32_t* chunk_lens;
    int32_t* status;
    int64_t kvnew_token_stride, kvnew_head_stride;       // in elements
    int64_t page_bytes, head_bytes;
    int32_t num_requests, num_kv_heads, page_size, max_blocks, num_pages;
    int32_t few;                     // as in AppendParams
    uint32_t off_q_offsets, off_prefix;
    uint32_t off_touched;            // (8 bits) WppTouched [num_touched] of the plan
    int32_t num_touched;
    int64_t total_new_tokens;
};

struct Kv4AttnParams {
    const void* plan;
    const __nv_bfloat16* q;
    const uint8_t* k_cache;
    const uint8_t* v_cache;
    const int32_t* block_tables;
    const int32_t* prefix_lens;
    const int32_t* chunk_lens;
    __nv_bfloat16* out;
    float* lse;                      // [T][Hq] or null
    float* ws_o;                     // split partials: [slots][2][128][d]
    float* ws_lse;                   // [slots][2][128], log2 units
    int32_t* status;
    int64_t q_token_stride, q_head_stride, o_token_stride, o_head_stride;      // in elements
    int64_t page_bytes, head_bytes;
    int32_t num_q_heads, group, page_size, max_blocks, num_pages;
    uint32_t off_q_offsets, off_prefix, off_units, off_few_ctas;
    float scale_log2;
    uint32_t bf16_128;               // 128 in both halves of a word; as below
    int32_t first_tile, num_tiles;   // of the plan's units
    uint32_t* tile_counter;          // or null: every CTA has one tile
    uint32_t* few_counter;           // (few rows) or null: every CTA has the units off_few_ctas says
    int32_t num_few;                 // units of the kernel for few rows
    uint32_t f16_1024, f16_64;       // f16 1024 and 64 in both halves of a word (from here, and no constants: see codes_low)
};

struct CombineParams {
    const void* plan;
    const float* ws_o;
    const float* ws_lse;
    __nv_bfloat16* out;
    float* lse;
    int64_t o_token_stride, o_head_stride;
    int32_t num_q_heads, head_dim;
    int32_t max_rows;                // most rows of a combine record
    int32_t num_records;
    uint32_t off_q_offsets, off_combine;
};

struct RopeParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_out;            // or the K pool, as v_out is the V pool
    __nv_bfloat16* v_out;
    const uint64_t* turns;           // [rot_dim / 2], of a turn per position, in 2^-64
    const int32_t* positions;        // [T]
    const int64_t* slots;            // [T], page * page_size + slot of the page, -1: none
    int32_t* status;
    int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride, qo_token_stride, qo_head_stride,
        ko_token_stride, ko_head_stride, kv_page_stride, kv_head_stride, kv_token_stride;      // in elements
    int64_t total_tokens, num_slots;
    int32_t num_q_heads, num_k_heads, page_shift;
    int32_t rot_vecs;                // rot_dim / 16
    int32_t q_in_place, k_in_place;  // what does not turn stands already
    float magnitude;
    int32_t passes, units_per_token, few;      // (the launch's: of a warp; warps of a token; as in AppendParams)
};

constexpr int kPagesMostRequests = 16384;

struct PagesParams {
    const int32_t* prefix_lens;
    const int32_t* chunk_lens;
    const int32_t* free_pages;
    const int32_t* cursor;           // [1]: entries of free_pages that are taken
    int32_t* cursor_out;             // [2]: the same afterwards; a count of CTAs, 0 between calls
    int32_t* block_tables;
    int64_t* row_offsets;
    int32_t* positions;              // [max_tokens] or null
    int64_t* slots;                  // [max_tokens] or null
    int32_t* status;
    int32_t num_requests, max_blocks, num_pages, page_shift, num_free, max_tokens;
};

struct KdaParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const float* alpha;
    const float* beta;
    const int64_t* row_offsets;
    const int32_t* prefix_lens;
    float* state_pool;
    const int32_t* state_in;
    const int32_t* state_out;
    const int32_t* snap_slots;
    __nv_bfloat16* out;
    int32_t* status;
    int32_t num_requests, num_heads, num_slots, snap_interval, max_snaps;
};

struct LinearParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const float* log_decay;
    const int64_t* row_offsets;
    const int32_t* prefix_lens;
    float* state_pool;
    const int32_t* state_in;
    const int32_t* state_out;
    const int32_t* snap_slots;
    __nv_bfloat16* out;
    int32_t* status;
    int64_t q_token_stride, k_token_stride, v_token_stride, o_token_stride, decay_token_stride;      // in elements
    int32_t num_requests, num_heads, num_slots, snap_interval, max_snaps;
    float scale;
    int32_t few_tokens;              // chunks of at most so many are the token form's, the others the blocks' (-1: one form has all)
};

struct LinearChunkParams : LinearParams {
    int64_t seg_tokens;              // tokens of a chain's segments; its first is number row_offsets[r] / seg_tokens in the workspace
    int64_t ws_segments;             // segments that the first pass may have
    float* ws_state;                 // [2 ws_segments][H][d * d]: their own states; where a chain's first one is, the chain's state before
    float* ws_log;                   // [ws_segments][H], base 2
};

// Chunk-parallel (tensor-core) form of the recurrent layer: the inputs of KdaParams plus the workspace arrays the
// preparation kernel fills for the chain kernel.  bh = (global block index) * num_heads + head.
struct KdaGroupParams : KdaParams {
    int64_t longest;                // longest chunk this form takes; a wave with a longer one is left to the two passes behind it
    int32_t* blk_off;               // [R+1] for the two passes: their block offsets, or blk_off[0] = -1 if there is nothing left
                                    // for them; null: nothing is behind, the wave is this form's whatever its lengths
    int32_t pieces;                 // a chain is cut into so many, a CTA each
    int32_t* ticket;                // next piece to be taken: first pieces of all chains, then second ones, ...
    float4* hand;                   // [R][H] states of 64 KB between pieces, and per column warp how many blocks they have seen
    int32_t* hand_seen;             // [R][H][8], behind the ticket
};

struct KdaTcParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const float* alpha;
    const float* beta;
    const int64_t* row_offsets;
    const int32_t* prefix_lens;
    float* state_pool;
    const int32_t* state_in;
    const int32_t* state_out;
    const int32_t* snap_slots;
    __nv_bfloat16* out;
    int32_t* status;
    int32_t num_requests, num_heads, num_slots, snap_interval, max_snaps;
    int32_t seg_lo, seg_hi;         // blocks [seg_lo, seg_hi) of every request belong to this launch
    int32_t beside;                 // preparation: launched beside the chain of the segment before
    int32_t gated;                  // behind the group form: nothing to do if that did the wave (blk_off[0] < 0)
    int32_t* blk_off;               // [R+1] exclusive scan of the requests' block counts
    unsigned long long* ws_mask;    // [bh] bit t: token t of the block starts a sub-block
    float* ws_e;                    // [bh][64][128] decay product at a sub-block's last token (other rows unused)
    __nv_bfloat16 *ws_w0_h, *ws_w0_l, *ws_qt_h, *ws_qt_l, *ws_kb_h, *ws_kb_l;   // [bh][64][128] hi / lo bf16 terms
    __nv_bfloat16 *ws_m_h, *ws_m_l;                                             // [bh][64][64]
    float* ws_u0;                                                               // [bh][64][128]
};

}  // namespace wpp

extern "C" {
// maps: 0..5 the operand arrays W0, Qt, Kb (hi, lo each), 6..7 M (hi, lo), 8 U0, 9..12 q, k, v, alpha
int wpp_launch_kda_tc(const wpp::KdaTcParams* params, const CUtensorMap* maps, int max_blocks, int num_sms, int segments,
                      const int32_t* seg_begin, void* stream);
int wpp_launch_attention(int head_dim, const CUtensorMap* tq, const CUtensorMap* tk, const CUtensorMap* tv,
                         const wpp::AttnParams* p, int num_ctas, int late_rescale, void* stream);
int wpp_launch_attention_small(int head_dim, const CUtensorMap* tq, const CUtensorMap* tk, const CUtensorMap* tv,
                               const wpp::SmallAttnParams* p, int num_ctas, void* stream);
int wpp_launch_append(const wpp::AppendParams* p, int num_sms, void* stream);
int wpp_launch_kv4_append(int head_dim, const wpp::Kv4AppendParams* p, int num_sms, void* stream);
int wpp_launch_kv8_append(int head_dim, const wpp::Kv4AppendParams* p, int num_sms, void* stream);
int wpp_launch_kv8_tiles(int head_dim, const CUtensorMap* tq, const CUtensorMap* tk, const CUtensorMap* tv, const wpp::Kv4AttnParams* p,
                         int num_ctas, void* stream);
int wpp_launch_kv8_few(int head_dim, const wpp::Kv4AttnParams* p, int num_ctas, int max_rows, int log_parts, void* stream);
int wpp_launch_kv4_tiles(int head_dim, const CUtensorMap* tq, const wpp::Kv4AttnParams* p, int num_ctas, void* stream);
int wpp_launch_kv4_few(int head_dim, const wpp::Kv4AttnParams* p, int num_ctas, int max_rows, void* stream);
int wpp_launch_rope(const wpp::RopeParams* p, int head_dim, int neighbours, int write, int num_sms, void* stream);
int wpp_launch_pages(const wpp::PagesParams* p, int num_sms, void* stream);
int wpp_launch_combine(const wpp::CombineParams* p, int num_combine, void* stream);
// maps: q, k, v, alpha; form: 1, 2, 3 = CTAs of 128, 64, 32 columns of the state
int wpp_launch_kda_group(const wpp::KdaGroupParams* p, const CUtensorMap* maps, int form, void* stream);
int wpp_launch_kda(const wpp::KdaParams* p, int num_sms, int layout, void* stream);
int wpp_launch_linear_token(const wpp::LinearParams* p, int head_dim, int num_sms, void* stream);
int wpp_launch_linear_chunk(const wpp::LinearChunkParams* p, int head_dim, int64_t segments, int two_passes, void* stream);
int wpp_launch_linear_tc(const wpp::LinearChunkParams* p, const CUtensorMap* maps, int64_t segments, int two_passes, void* stream);
int wpp_launch_selftest_wait(long long limit_cycles, int32_t* status, long long* waited_cycles, void* stream);
}
