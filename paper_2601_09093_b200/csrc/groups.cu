// decode_attention_groups: decode attention of traces that were forked from several prompts, each prompt read once for all of
// its traces.
//
//   out[i][h] = sum_j softmax_j(q[i][h] . K_i[j] / sqrt(d)) V_i[j],  j in [0, seq_lens[i]),
//
// where the first pages of a group's rows are the same blocks.  bf16 pools of the usual shape run on groups_tc.cu, others on
// attention_rows.cuh, which reads shared pages once for 16 / G traces.
#include "attention_rows.cuh"

using namespace stepk;

extern "C" {

int decode_attention_groups_workspace_bytes(const step_pool* pool, int n, int n_groups, size_t* bytes) {
  if (!pool || !bytes || n < 0 || n_groups < 0 || n > 65535 || n_groups > 65535) return STEP_ERR_INVALID_ARG;
  *bytes = groups_tc_supported(pool, n) ? groups_tc_workspace(pool, n, n_groups)
           : n_groups > 0               ? attn_groups_workspace(pool, n)
                                        : attn_rows_workspace(pool, n, 1);
  return STEP_OK;
}

int decode_attention_groups(step_pool* pool, int layer, const void* q, const int32_t* block_table, const int32_t* seq_lens, int n,
                            const int32_t* group_rows, const int32_t* group_pages, int n_groups, void* out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!pool || n < 0 || n_groups < 0 || layer < 0 || layer >= pool->cfg.num_layers) return STEP_ERR_INVALID_ARG;
  if (n == 0) return STEP_OK;
  if (!q || !block_table || !seq_lens || !out || n > 65535 || n_groups > 65535) return STEP_ERR_INVALID_ARG;
  if (n_groups > 0 && (!group_rows || !group_pages)) return STEP_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)out) & 15) return STEP_ERR_INVALID_ARG;
  size_t need = 0;
  int st = decode_attention_groups_workspace_bytes(pool, n, n_groups, &need);
  if (st != STEP_OK) return st;
  if (need > 0 && (!workspace || (uintptr_t)workspace & 255 || workspace_bytes < need)) return STEP_ERR_INVALID_ARG;
  st = on_pool_device(pool);
  if (st != STEP_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  if (groups_tc_supported(pool, n))
    return groups_tc_launch(pool, layer, q, block_table, seq_lens, n, group_rows, group_pages, n_groups, out, workspace, s);
  RowsArgs a = {};
  a.g = geo_of(pool);
  a.kv = pool->cfg.kv_storage; a.layer = layer;
  a.q = q; a.T = 1;
  a.block_table = block_table; a.seq_lens = seq_lens; a.out = out;
  a.counters = pool->v.counters;
  a.group_rows = group_rows; a.group_pages = group_pages; a.n_groups = n_groups;
  const bool bf16 = pool->cfg.dtype == STEP_BF16;
  float* part = (float*)workspace;
  if (n_groups > 0)
    return bf16 ? launch_attn_rows<__nv_bfloat16, __nv_bfloat16, false, false, true>(pool, a, n, part, s)
                : launch_attn_rows<float, float, false, false, true>(pool, a, n, part, s);
  return bf16 ? launch_attn_rows<__nv_bfloat16, __nv_bfloat16, false, false>(pool, a, n, part, s)
              : launch_attn_rows<float, float, false, false>(pool, a, n, part, s);
}

}  // extern "C"
