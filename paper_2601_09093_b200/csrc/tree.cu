// decode_attention_tree: attention of a tree of drafted tokens over the paged cache (speculative decoding: several
// continuations of a trace are drafted as a tree and verified in one pass of the model).
//
//   out[i][u][h] = sum_j softmax_j(q[i][u][h] . k[j] / sqrt(d)) v[j],   j over the S_i cached positions of row i, then over
//                  drafted token u itself and its ancestors in the tree
//
#include "attention_rows.cuh"

using namespace stepk;

extern "C" {

int decode_attention_tree_workspace_bytes(const step_pool* pool, int n, int T, size_t* bytes) {
  if (!pool || !bytes || n < 0 || T < 1 || T > kMaxTreeNodes) return STEP_ERR_INVALID_ARG;
  *bytes = tree_tc_supported(pool, n) ? tree_tc_workspace(pool, T) : attn_rows_workspace(pool, n, T);
  return STEP_OK;
}

int decode_attention_tree(step_pool* pool, int layer, const void* q, const void* k_draft, const void* v_draft,
                          const int32_t* parents, const int32_t* n_nodes, int T, const int32_t* block_table,
                          const int32_t* seq_lens, int n, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!pool || n < 0 || T < 1 || T > kMaxTreeNodes) return STEP_ERR_INVALID_ARG;
  if (layer < 0 || layer >= pool->cfg.num_layers) return STEP_ERR_INVALID_ARG;
  if (n == 0) return STEP_OK;
  if (!q || !k_draft || !v_draft || !parents || !block_table || !seq_lens || !out || n > 65535) return STEP_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)k_draft | (uintptr_t)v_draft) & 15 || (uintptr_t)out & 31) return STEP_ERR_INVALID_ARG;
  int st = on_pool_device(pool);
  if (st != STEP_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  if (tree_tc_supported(pool, n)) {
    if (!workspace || (uintptr_t)workspace & 255 || workspace_bytes < tree_tc_workspace(pool, T)) return STEP_ERR_INVALID_ARG;
    return tree_tc_launch(pool, layer, q, k_draft, v_draft, parents, n_nodes, T, block_table, seq_lens, n, out, workspace, s);
  }
  const size_t need = attn_rows_workspace(pool, n, T);
  if (need > 0 && (!workspace || (uintptr_t)workspace & 255 || workspace_bytes < need)) return STEP_ERR_INVALID_ARG;
  RowsArgs a = {};
  a.g = geo_of(pool);
  a.kv = pool->cfg.kv_storage; a.layer = layer;
  a.q = q; a.k_draft = k_draft; a.v_draft = v_draft; a.parents = parents; a.n_nodes = n_nodes; a.T = T;
  a.block_table = block_table; a.seq_lens = seq_lens; a.out = out;
  a.counters = pool->v.counters;
  if (pool->cfg.dtype == STEP_BF16) return launch_attn_rows<__nv_bfloat16, __nv_bfloat16, true, false>(pool, a, n, (float*)workspace, s);
  return launch_attn_rows<float, float, true, false>(pool, a, n, (float*)workspace, s);
}

}  // extern "C"
