// C ABI of the 4-bit cache: host-side validation and planning.
#include <math.h>

#include "host.h"
#include "kv4_plan.h"
#include "launchers.h"

namespace {

using d2sd::fail;
using d2sd::hip_status;
using d2sd::ok;

constexpr int kNumCUs = 256;
constexpr long long kMaxPositions = (1ll << 30) - 64;   // of a request, so that position arithmetic stays in 32 bits
constexpr long long kMaxGroups = 1ll << 23;             // workgroups along x

// Sizes that the three cache calls share.
d2sd_status validate_cache_sizes(int batch, int num_kv_heads, int head_dim, int page_size, int dtype, int num_pages,
                                 int max_pages) {
  if (batch < 1) return fail(D2SD_ERR_INVALID_ARG, "batch must be >= 1 (got %d)", batch);
  if (num_kv_heads < 1) return fail(D2SD_ERR_INVALID_ARG, "num_kv_heads must be >= 1");
  if (head_dim != D2SD_HEAD_DIM) return fail(D2SD_ERR_UNSUPPORTED, "head_dim %d != %d", head_dim, D2SD_HEAD_DIM);
  if (page_size != D2SD_PAGE_SIZE) return fail(D2SD_ERR_UNSUPPORTED, "page_size %d != %d", page_size, D2SD_PAGE_SIZE);
  if (dtype != D2SD_F32 && dtype != D2SD_BF16) return fail(D2SD_ERR_INVALID_ARG, "dtype %d unknown", dtype);
  if (num_pages < 1 || max_pages < 1) return fail(D2SD_ERR_INVALID_ARG, "num_pages and max_pages must be >= 1");
  if (num_kv_heads > 65535) return fail(D2SD_ERR_UNSUPPORTED, "num_kv_heads %d exceeds 65535", num_kv_heads);
  if ((long long)max_pages * page_size > kMaxPositions)
    return fail(D2SD_ERR_UNSUPPORTED, "max_pages * page_size = %lld exceeds %lld", (long long)max_pages * page_size,
                kMaxPositions);
  return D2SD_OK;
}

d2sd_status validate_cache(const d2sd_kv4_cache* c) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return fail(D2SD_ERR_INVALID_ARG, "cache or one of its pointers is NULL");
  const void* const ptr[] = {c->k, c->v, c->k_scale, c->v_scale};
  const char* const names[] = {"cache->k", "cache->v", "cache->k_scale", "cache->v_scale"};
  for (int i = 0; i < 4; ++i)
    if (reinterpret_cast<uintptr_t>(ptr[i]) % (i < 2 ? 16 : 4) != 0)
      return fail(D2SD_ERR_INVALID_ARG, "%s is not %d-byte aligned", names[i], i < 2 ? 16 : 4);
  return D2SD_OK;
}

d2sd_status validate_aligned(const void* a, const char* an, const void* b, const char* bn) {
  if (reinterpret_cast<uintptr_t>(a) % 16 != 0) return fail(D2SD_ERR_INVALID_ARG, "%s is not 16-byte aligned", an);
  if (reinterpret_cast<uintptr_t>(b) % 16 != 0) return fail(D2SD_ERR_INVALID_ARG, "%s is not 16-byte aligned", bn);
  return D2SD_OK;
}

d2sd_status validate_tokens(int batch, int total, int most, int max_pages, int page_size) {
  if (total < 0 || most < 0 || most > total)
    return fail(D2SD_ERR_INVALID_ARG, "need 0 <= max_tokens <= total_tokens (got %d, %d)", most, total);
  if (total > 0 && most < 1) return fail(D2SD_ERR_INVALID_ARG, "max_tokens must be >= 1 when total_tokens > 0");
  if (most > (long long)max_pages * page_size)
    return fail(D2SD_ERR_INVALID_ARG, "max_tokens %d exceeds max_pages * page_size = %lld", most,
                (long long)max_pages * page_size);
  if (d2sd::kv4_page_groups(batch, most) > kMaxGroups)
    return fail(D2SD_ERR_UNSUPPORTED, "batch %d x max_tokens %d: too many pages for one call", batch, most);
  return D2SD_OK;
}

// ---- attention plan ----

d2sd_status validate_attn_kv4(const d2sd_attn_args* a) {
  d2sd_status s = d2sd::validate_attn(a, false);
  if (s) return s;
  if (a->k_cache || a->v_cache) return fail(D2SD_ERR_INVALID_ARG, "k_cache and v_cache must be NULL: the context is in `cache`");
  if (a->row_group != 0 || a->packed != 0) return fail(D2SD_ERR_INVALID_ARG, "row_group and packed must be 0");
  return D2SD_OK;
}

constexpr int kStepKeys = 128;
constexpr long long kMaxUnits = 1ll << 24;              // of one request's streams, which the kernels add up in 32 bits

// Two workgroups of four waves per CU are resident (bf16; one with fp32, whose
// terms take twice the registers), and that is the grid unless a share would
// fall below kMinSteps steps of keys, less than which is not worth a partial
// state (one request of one token over 4096 keys: 18.5 us with two, 21.5 with
// one, 20.0 with three).
//
// A stream's start, tree and end take as long as some steps of its keys, 10 to
// 15 us, and a share that holds many short streams would end last. They are
// charged kCharge units of cost (a step of four row tiles is 8), at most a
// share: 64 requests of one token over 500 to 16000 keys take 178 us with 3,
// 164 with 10, 146 with 20, 130 with 30 and 132 with 45.
constexpr int kMinSteps = 2;
constexpr long long kCharge = 30;

// Whether streams that are not cut, one workgroup each, end sooner. In units of
// cost, uncut they take, per round of resident workgroups, a start and the
// longest stream's steps; cut, a start and one more per stream of a share, the
// share (contexts of three quarters of the largest) and the merge, whose states
// grow with the rows. fp32 steps count for a quarter more. us cut, uncut: 64
// requests of one token over 100 to 2000 keys 46, 33 (over 500 to 16000 130,
// 150); 24 over 100 to 1000 28, 21; 16 of up to eight row tiles over 500 keys 42,
// 28, 32 over 1000 73, 53, 64 over 100 to 500 95, 75; fp32, 6 of one token and two
// KV heads over 706 keys 20.5, 28.
bool whole_pays(bool bf16, long long streams, long long resident, long long steps, long long cost, int most, int grid) {
  const double step = bf16 ? 1.0 : 1.25;
  const double uncut = fmax(1.0, (double)streams / resident) * (kCharge + step * steps * most);
  const double cut = kCharge * (1.0 + (double)streams / grid) + 0.75 * step * steps * cost / grid + 5.0 * most;
  return uncut <= cut;
}

d2sd_status make_kv4_plan(const d2sd_attn_args* a, d2sd::Kv4Plan* plan) {
  const int G = a->num_qo_heads / a->num_kv_heads;
  const bool bf16 = a->dtype == D2SD_BF16;
  const int ctx = a->stage == D2SD_STAGE_TREE ? 0 : a->max_ctx_len;
  auto tiles_of = [&](long long nodes) { return (int)((nodes * G + d2sd::kRowsPerTile - 1) / d2sd::kRowsPerTile); };
  const int tiles_most = max(1, tiles_of(a->max_nodes));
  const long long steps = (ctx + kStepKeys - 1) / kStepKeys + 1 + (a->max_nodes + 63ll) / 64;   // of a stream, at most
  if ((steps + 16) * d2sd::kv4_cost(tiles_most) * a->num_kv_heads > kMaxUnits)
    return fail(D2SD_ERR_UNSUPPORTED, "max_ctx_len %d x max_nodes %d is too much for one request", a->max_ctx_len, a->max_nodes);
  long long streams = 0, cost = 0;                      // of a step of all streams; exact with host offsets, else from the mean request
  auto count = [&](int tiles, long long times) {
    streams += times * a->num_kv_heads * (tiles / 4 + (tiles >> 1 & 1) + (tiles & 1));
    cost += times * a->num_kv_heads * d2sd::kv4_cost(tiles);
  };
  if (a->node_indptr_host) {
    for (int b = 0; b < a->batch; ++b) count(tiles_of(a->node_indptr_host[b + 1] - a->node_indptr_host[b]), 1);
  } else {
    count(max(1, tiles_of(a->total_nodes / max(1, a->batch))), a->batch);
  }
  const int most = d2sd::kv4_cost(tiles_most >= 4 ? 4 : tiles_most >= 2 ? 2 : 1);
  const long long resident = (bf16 ? 2 : 1) * kNumCUs;
  auto rounded = [](long long want) { return (int)((max(1ll, want) + 7) / 8 * 8); };
  const int cut_grid = rounded(a->kv_split > 0 ? min(streams * steps * kStepKeys / a->kv_split, 16 * resident)
                                               : min(resident, steps * cost / (kMinSteps * most)));
  plan->whole = ctx == 0 || a->total_nodes == 0 || (a->kv_split == 0 && whole_pays(bf16, streams, resident, steps, cost, most, cut_grid));
  plan->most = plan->whole ? 1 : most;
  plan->grid = plan->whole ? rounded(min(streams, 16 * resident)) : cut_grid;
  const long long charge = min(kCharge, steps * cost / plan->grid);
  for (int i = 0; i < 3; ++i) plan->charge[i] = max(1, (int)(charge / d2sd::kv4_cost(1 << i)));
  const long long pieces = plan->grid / max(1ll, streams);
  plan->span = (int)max(1ll, min(64ll, pieces));
  plan->per = pieces > 16 ? 8 : pieces > 4 ? 4 : 1;
  plan->slot_rows = min(4, tiles_most) * d2sd::kRowsPerTile;
  const size_t states = (size_t)2 * plan->grid * plan->slot_rows;
  plan->ws_bytes = plan->whole ? 0 : states * (D2SD_HEAD_DIM + 2) * sizeof(float) + (size_t)plan->grid * d2sd::kKv4CutBytes;
  plan->scale = a->sm_scale > 0.0f ? a->sm_scale : 1.0f / sqrtf((float)a->head_dim);
  return D2SD_OK;
}

}  // namespace

extern "C" {

d2sd_status d2sd_append_kv4(int batch, int num_kv_heads, int head_dim, int page_size, int dtype, int num_pages,
                            int max_pages, int max_ctx_len, const int* token_indptr, int total_tokens,
                            int max_tokens, const void* k, const void* v, const int* page_table, int* ctx_len,
                            const d2sd_kv4_cache* cache, hipStream_t stream) {
  d2sd_status s = validate_cache_sizes(batch, num_kv_heads, head_dim, page_size, dtype, num_pages, max_pages);
  if (s) return s;
  if ((s = validate_tokens(batch, total_tokens, max_tokens, max_pages, page_size))) return s;
  if (max_ctx_len < 0 || (long long)max_ctx_len > (long long)max_pages * page_size)
    return fail(D2SD_ERR_INVALID_ARG, "max_ctx_len %d outside [0, max_pages * page_size = %lld]", max_ctx_len,
                (long long)max_pages * page_size);
  if (!token_indptr || !page_table || !ctx_len || (total_tokens > 0 && (!k || !v)))
    return fail(D2SD_ERR_INVALID_ARG, "a required device pointer is NULL");
  if ((s = validate_cache(cache)) || (s = validate_aligned(k, "k", v, "v"))) return s;
  if (total_tokens == 0) return ok();
  return hip_status(d2sd::launch_append_kv4(batch, num_kv_heads, dtype, num_pages, max_pages, max_ctx_len, token_indptr,
                                            total_tokens, max_tokens, k, v, page_table, ctx_len, *cache, stream),
                    "append_kv4 launch");
}

d2sd_status d2sd_commit_accepted_kv4(int batch, int B, int num_kv_heads, int head_dim, int page_size, int dtype,
                                     int num_pages, int max_pages, int max_ctx_len, const int* node_indptr,
                                     int total_nodes, const int* path_nodes, const int* accept_len,
                                     const void* k_tree, const void* v_tree, const int* page_table, int* ctx_len,
                                     const d2sd_kv4_cache* cache, hipStream_t stream) {
  d2sd_status s = validate_cache_sizes(batch, num_kv_heads, head_dim, page_size, dtype, num_pages, max_pages);
  if (s) return s;
  if (B < 2 || B > D2SD_MAX_B) return fail(D2SD_ERR_INVALID_ARG, "B = %d outside [2, %d]", B, D2SD_MAX_B);
  if (total_nodes < 0 || max_ctx_len < 0) return fail(D2SD_ERR_INVALID_ARG, "negative size");
  if ((long long)max_ctx_len + B > (long long)max_pages * page_size)
    return fail(D2SD_ERR_INVALID_ARG, "max_ctx_len + B = %lld exceeds max_pages * page_size = %lld",
                (long long)max_ctx_len + B, (long long)max_pages * page_size);
  if (!node_indptr || !path_nodes || !accept_len || !k_tree || !v_tree || !page_table || !ctx_len)
    return fail(D2SD_ERR_INVALID_ARG, "a required device pointer is NULL");
  if ((s = validate_cache(cache)) || (s = validate_aligned(k_tree, "k_tree", v_tree, "v_tree"))) return s;
  return hip_status(d2sd::launch_commit_kv4(batch, B, num_kv_heads, dtype, num_pages, max_pages, max_ctx_len, node_indptr,
                                            total_nodes, path_nodes, accept_len, k_tree, v_tree, page_table, ctx_len,
                                            *cache, stream),
                    "commit_kv4 launch");
}

d2sd_status d2sd_read_kv4(int batch, int num_kv_heads, int head_dim, int page_size, int dtype, int num_pages,
                          int max_pages, const int* token_indptr, int total_tokens, int max_tokens,
                          const int* start, const int* page_table, const d2sd_kv4_cache* cache, void* k_out,
                          void* v_out, hipStream_t stream) {
  d2sd_status s = validate_cache_sizes(batch, num_kv_heads, head_dim, page_size, dtype, num_pages, max_pages);
  if (s) return s;
  if ((s = validate_tokens(batch, total_tokens, max_tokens, max_pages, page_size))) return s;
  if (!token_indptr || !page_table || (total_tokens > 0 && (!k_out || !v_out)))
    return fail(D2SD_ERR_INVALID_ARG, "a required device pointer is NULL");
  if ((s = validate_cache(cache)) || (s = validate_aligned(k_out, "k_out", v_out, "v_out"))) return s;
  if (total_tokens == 0) return ok();
  return hip_status(d2sd::launch_read_kv4(batch, num_kv_heads, dtype, num_pages, max_pages, token_indptr, total_tokens,
                                          max_tokens, start, page_table, *cache, k_out, v_out, stream),
                    "read_kv4 launch");
}

d2sd_status d2sd_cascade_workspace_size_kv4(const d2sd_attn_args* args, size_t* bytes) {
  d2sd_status s = validate_attn_kv4(args);
  if (s) return s;
  if (!bytes) return fail(D2SD_ERR_INVALID_ARG, "bytes is NULL");
  d2sd::Kv4Plan plan;
  if ((s = make_kv4_plan(args, &plan))) return s;
  *bytes = plan.ws_bytes;
  return ok();
}

d2sd_status d2sd_cascade_verify_attention_kv4(const d2sd_attn_args* args, const d2sd_kv4_cache* cache, void* ws,
                                              size_t ws_bytes, hipStream_t stream) {
  d2sd_status s = validate_attn_kv4(args);
  if (s) return s;
  if (!args->q || !args->page_table || !args->ctx_len || !args->k_tree || !args->v_tree || !args->node_indptr || !args->out)
    return fail(D2SD_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (args->stage != D2SD_STAGE_PREFIX && !args->anc_mask) return fail(D2SD_ERR_INVALID_ARG, "anc_mask is NULL");
  if ((s = validate_cache(cache)) || (s = validate_aligned(args->q, "q", args->out, "out")) ||
      (s = validate_aligned(args->k_tree, "k_tree", args->v_tree, "v_tree")))
    return s;
  d2sd::Kv4Plan plan;
  if ((s = make_kv4_plan(args, &plan))) return s;
  if (plan.ws_bytes > 0 && (!ws || ws_bytes < plan.ws_bytes))
    return fail(D2SD_ERR_WORKSPACE_TOO_SMALL, "workspace %zu bytes, need %zu", ws ? ws_bytes : 0, plan.ws_bytes);
  if (args->total_nodes == 0) return ok();
  if (plan.ws_bytes > 0 && reinterpret_cast<uintptr_t>(ws) % 16 != 0)
    return fail(D2SD_ERR_INVALID_ARG, "ws is not 16-byte aligned");
  hipEvent_t ev[3];
  d2sd::timing_begin(ev);
  const hipError_t e = d2sd::launch_kv4_attention(*args, *cache, plan, ws, stream, ev);
  d2sd::timing_end(ev, e == hipSuccess, !plan.whole);
  return hip_status(e, "kv4 attention launch");
}

}  // extern "C"
