// C ABI of the logit adjustment: host-side validation.
#include "host.h"
#include "launchers.h"

using d2sd::fail;

extern "C" d2sd_status d2sd_adjust_logits(const d2sd_logits_args* a, hipStream_t stream) {
  if (!a) return fail(D2SD_ERR_INVALID_ARG, "args is NULL");
  if (a->batch < 1) return fail(D2SD_ERR_INVALID_ARG, "batch must be >= 1 (got %d)", a->batch);
  if (a->total_nodes < 0) return fail(D2SD_ERR_INVALID_ARG, "total_nodes must be >= 0");
  if (a->max_nodes < 1 || a->max_nodes > d2sd::kMaxTreeNodes)
    return fail(D2SD_ERR_INVALID_ARG, "max_nodes %d outside [1, %d]", a->max_nodes, d2sd::kMaxTreeNodes);
  if ((long long)a->mask_words * 32 < a->max_nodes)
    return fail(D2SD_ERR_INVALID_ARG, "mask_words %d too small for max_nodes %d", a->mask_words, a->max_nodes);
  if (a->vocab < 1 || a->vocab > D2SD_MAX_VOCAB)
    return fail(D2SD_ERR_INVALID_ARG, "vocab = %d outside [1, %d]", a->vocab, D2SD_MAX_VOCAB);
  if (a->dtype != D2SD_F32 && a->dtype != D2SD_BF16) return fail(D2SD_ERR_INVALID_ARG, "dtype %d unknown", a->dtype);
  if (a->max_history < 0 || a->max_bias < 0 || a->num_masks < 0)
    return fail(D2SD_ERR_INVALID_ARG, "max_history, max_bias and num_masks must be >= 0");
  if ((long long)a->batch * a->max_nodes * ((a->vocab + 2047) / 2048) >= (1ll << 24))
    return fail(D2SD_ERR_UNSUPPORTED, "batch x max_nodes x vocab / 2048 needs more than 2^24 workgroups");
  if (!a->node_indptr || !a->depth || !a->anc_mask || !a->draft_tokens || !a->logits || !a->out)
    return fail(D2SD_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (a->max_history > 0 && (!a->history || !a->history_len))
    return fail(D2SD_ERR_INVALID_ARG, "history or history_len is NULL");
  if (a->max_bias > 0 && (!a->bias_token || !a->bias_value))
    return fail(D2SD_ERR_INVALID_ARG, "bias_token or bias_value is NULL");
  if (a->num_masks > 0 && (!a->token_mask || !a->mask_row))
    return fail(D2SD_ERR_INVALID_ARG, "token_mask or mask_row is NULL");
  if (reinterpret_cast<uintptr_t>(a->logits) % 16 != 0) return fail(D2SD_ERR_INVALID_ARG, "logits is not 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(a->out) % 16 != 0) return fail(D2SD_ERR_INVALID_ARG, "out is not 16-byte aligned");
  if (a->total_nodes == 0) return d2sd::ok();
  return d2sd::hip_status(d2sd::launch_adjust_logits(*a, stream), "adjust_logits launch");
}
