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

// Row groups of one split over the batch: exact with host offsets, else from
// the mean tree.
long long row_groups(const d2sd_attn_args* a, int G, int rows_per_group) {
  long long groups = 0;
  if (a->node_indptr_host) {
    for (int b = 0; b < a->batch; ++b) {
      const long long rows = (long long)(a->node_indptr_host[b + 1] - a->node_indptr_host[b]) * G;
      groups += (rows + rows_per_group - 1) / rows_per_group;
    }
  } else {
    const double rows = (double)a->total_nodes / a->batch * G;
    groups = (long long)a->batch * max(1, (int)ceil(rows / rows_per_group));
  }
  return max(1ll, groups * a->num_kv_heads);
}

d2sd_status make_kv4_plan(const d2sd_attn_args* a, d2sd::Kv4Plan* plan) {
  const int G = a->num_qo_heads / a->num_kv_heads;
  const long long rows = (long long)a->max_nodes * G;
  const int ctx = a->stage == D2SD_STAGE_TREE ? 0 : a->max_ctx_len;
  plan->waves = rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : 8;
  const int rows_per_group = plan->waves * d2sd::kRowsPerTile;
  const long long g = row_groups(a, G, rows_per_group);
  const long long resident = (long long)kNumCUs * (plan->waves <= 2 ? 3 : plan->waves == 4 ? 2 : 1);
  const int s_lo = max(1, (ctx + d2sd::kKv4MaxSplit - 1) / d2sd::kKv4MaxSplit);
  const int s = (int)min((2 * resident + g - 1) / g, (long long)max(1, ctx / 256));
  const int splits = max(s_lo, s);
  plan->split = a->kv_split > 0 ? a->kv_split : max(64, ((ctx + splits - 1) / splits + 63) / 64 * 64);
  plan->n_ch_max = max(1, (ctx + plan->split - 1) / plan->split);
  plan->n_rg_max = (int)max(1ll, (rows + rows_per_group - 1) / rows_per_group);
  plan->items = (long long)a->batch * a->num_kv_heads * plan->n_ch_max * plan->n_rg_max;
  if (plan->items > kMaxGroups) return fail(D2SD_ERR_UNSUPPORTED, "too many work items (%lld)", plan->items);
  if ((long long)a->batch * ((long long)a->max_nodes * a->num_qo_heads / 8 + 1) > kMaxGroups)
    return fail(D2SD_ERR_UNSUPPORTED, "too many split-merge workgroups (batch %d, max_nodes %d)", a->batch, a->max_nodes);
  const size_t states = (size_t)plan->n_ch_max * a->total_nodes * a->num_qo_heads;
  plan->ws_bytes = plan->n_ch_max > 1 ? states * (D2SD_HEAD_DIM + 2) * sizeof(float) : 0;
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
  return hip_status(d2sd::launch_kv4_attention(*args, *cache, plan, ws, stream), "kv4 attention launch");
}

}  // extern "C"
