// Launchers of the tree, selection, accept, commit, 4-bit cache and logit
// kernels (implemented in their .hip files); the C ABI validates arguments first. The
// attention launchers are declared in common.h next to the attention plan.
#pragma once

#include "common.h"

namespace d2sd {

hipError_t launch_tree_build(int batch, int B, int Kmax, const int* K, const int* p,
                             const int* node_indptr, int total_nodes, int mask_words, int* parent,
                             int* depth, int* path_id, uint32_t* anc_mask, int* path_leaf,
                             hipStream_t stream);

hipError_t launch_tree_from_parents(int batch, const int* node_indptr, int total_nodes, int max_nodes,
                                    int mask_words, const int* parent, int* depth, int* path_id,
                                    uint32_t* anc_mask, hipStream_t stream);

hipError_t launch_select_reanchor(int batch, int B, int Kmax, const float* conf, const int* K, int* p_out,
                                  double* r_out, hipStream_t stream);

hipError_t launch_tree_indptr(int batch, int B, int Kmax, const int* K, const int* p, int* node_indptr,
                              hipStream_t stream);

hipError_t launch_commit(int batch, int B, int hkv, int row_bytes, int num_pages, int max_pages, int max_ctx,
                         const int* node_indptr, int total_nodes, const int* path_nodes, const int* accept_len,
                         const void* k_tree, const void* v_tree, const int* page_table, int* ctx_len,
                         void* k_cache, void* v_cache, hipStream_t stream);

hipError_t launch_accept_path(int batch, int B, const int* node_indptr, int total_nodes,
                              const int* parent, const int* depth, const int* path_id,
                              const int* draft, const int* argmax, int* accept_len, int* best_path,
                              int* accept_node, int* path_nodes, int* out_tokens,
                              hipStream_t stream);

hipError_t launch_sample_targets(int batch, const int* node_indptr, int total_nodes, int max_nodes,
                                 const int* parent, const int* draft, int vocab, int dtype, const void* logits,
                                 float temperature, const float* uniform, int* context_rep, int* tokens,
                                 hipStream_t stream);

// The 4-bit cache (kv4.hip). kv4_page_groups: workgroups along x of the calls
// that go page by page.
long long kv4_page_groups(int batch, int max_tokens);

hipError_t launch_append_kv4(int batch, int hkv, int dtype, int num_pages, int max_pages, int max_ctx,
                             const int* token_indptr, int total, int max_tokens, const void* k, const void* v,
                             const int* page_table, int* ctx_len, const d2sd_kv4_cache& cache, hipStream_t stream);

hipError_t launch_commit_kv4(int batch, int B, int hkv, int dtype, int num_pages, int max_pages, int max_ctx,
                             const int* node_indptr, int total_nodes, const int* path_nodes, const int* accept_len,
                             const void* k_tree, const void* v_tree, const int* page_table, int* ctx_len,
                             const d2sd_kv4_cache& cache, hipStream_t stream);

hipError_t launch_read_kv4(int batch, int hkv, int dtype, int num_pages, int max_pages, const int* token_indptr, int total,
                           int max_tokens, const int* start, const int* page_table, const d2sd_kv4_cache& cache,
                           void* k_out, void* v_out, hipStream_t stream);

hipError_t launch_adjust_logits(const d2sd_logits_args& a, hipStream_t stream);

}  // namespace d2sd
