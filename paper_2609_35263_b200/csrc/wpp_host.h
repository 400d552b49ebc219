// Internal host-side declarations shared by the planner and the launch code.
#pragma once
#include <stdint.h>

#include "../../include/wpp.h"
#include "wpp_plan_format.h"

#define WPP_DEFAULT_TILE_M 256
#define WPP_MAX_TILE_M 256

#ifdef __cplusplus
extern "C" {
#endif
int wpp_resolve_desc(const wpp_batch_desc* in, wpp_batch_desc* out);
uint64_t wpp_desc_hash(const wpp_batch_desc* resolved);
int wpp_check_plan(const void* plan_host, const wpp_batch_desc* resolved, const struct WppPlanHeader** out);
/* The plan of a wave over a 4- or 8-bit cache (wpp_plan_kv4.cpp): opts resolved, lengths checked, T and pairs their sums */
size_t wpp_kv4_plan_bytes(const wpp_batch_desc* resolved, const wpp_plan_opts* opts, int64_t total_new_tokens);
int wpp_kv4_plan(const wpp_batch_desc* resolved, const wpp_plan_opts* opts, const int32_t* prefix_lens, const int32_t* chunk_lens,
                 int64_t total_new_tokens, int64_t pairs, void* plan_host, size_t plan_host_bytes, wpp_plan_info* info);
int wpp_ctx_sm_count(const wpp_ctx* ctx);
int wpp_ctx_check_device(const wpp_ctx* ctx);   /* WPP_OK iff the context's device is the current one */
#ifdef __cplusplus
}
#endif
