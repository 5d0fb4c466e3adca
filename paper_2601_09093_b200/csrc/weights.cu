// decode_attention_weights: decode attention that also keeps count of what the cache is used for.
//
//   p[i][h][j] = softmax_j(q[i][h] . K_i[j] / sqrt(d)),  out[i][h] = sum_j p[i][h][j] V_i[j]
//   weight_sum[i][kvh][j] += sum over the query heads h of KV head kvh of p[i][h][j]
//
// The weights are known only when a row's maximum and sum are, so the attention kernel leaves its scores (log2-scaled,
// fp32) in the workspace and a second kernel, its programmatic dependent, turns them into weights: 8 * G bytes per
// position and KV head on top of the 4 * d bytes of K and V in bf16 (a second read of K would be 2 * d).
#include "attention_rows.cuh"

using namespace stepk;

namespace {

constexpr int kAccThreads = 256;

// weight_sum[t][h][j] += sum_g exp2(scores[t][h G + g][j] - m_g) / l_g.  grid (position chunks, Hkv, n); the heads are added
// in ascending order by one thread, so the sums do not depend on the launch.
__global__ void __launch_bounds__(kAccThreads)
weights_add_kernel(Geo g, const float* __restrict__ scores, long long score_stride, const float* __restrict__ ml,
                   const int32_t* __restrict__ seq_lens, float* __restrict__ weight_sum, int weight_stride, int32_t* counters) {
  const int h = blockIdx.y, t = blockIdx.z;
  wait_for_primary();
  long long S = seq_lens[t];
  const long long cap = (long long)g.max_pages * g.P;
  if (S > cap) S = cap;
  if (S > weight_stride) { S = weight_stride; if (threadIdx.x == 0) flag_error(counters, STEP_ERR_CAPACITY); }
  const float* sc = scores + ((size_t)t * g.Hq + (size_t)h * g.G) * score_stride;
  const float* mlh = ml + ((size_t)t * g.Hq + (size_t)h * g.G) * 2;
  float* w = weight_sum + ((size_t)t * g.Hkv + h) * weight_stride;
  for (long long j = (long long)blockIdx.x * kAccThreads + threadIdx.x; j < S; j += (long long)gridDim.x * kAccThreads) {
    float sum = 0.f;
    for (int k = 0; k < g.G; ++k) sum += exp2f(sc[(size_t)k * score_stride + j] - mlh[2 * k]) / mlh[2 * k + 1];
    w[j] += sum;
  }
}

long long stride_of_scores(int weight_stride) { return ((long long)weight_stride + 15) / 16 * 16; }

}  // namespace

extern "C" {

int decode_attention_weights_workspace_bytes(const step_pool* pool, int n, int weight_stride, size_t* bytes) {
  if (!pool || !bytes || n < 0 || weight_stride < 1) return STEP_ERR_INVALID_ARG;
  const size_t rows = (size_t)n * pool->cfg.num_q_heads;
  *bytes = rows * stride_of_scores(weight_stride) * sizeof(float) + rows * 2 * sizeof(float);
  return STEP_OK;
}

int decode_attention_weights(step_pool* pool, int layer, const void* q, const int32_t* block_table, const int32_t* seq_lens,
                             int n, void* out, float* weight_sum, int weight_stride, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (!pool || n < 0 || weight_stride < 1 || layer < 0 || layer >= pool->cfg.num_layers) return STEP_ERR_INVALID_ARG;
  if (n == 0) return STEP_OK;
  if (!q || !block_table || !seq_lens || !out || !weight_sum || !workspace || n > 65535) return STEP_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)out) & 15 || (uintptr_t)workspace & 255) return STEP_ERR_INVALID_ARG;
  size_t need = 0;
  int st = decode_attention_weights_workspace_bytes(pool, n, weight_stride, &need);
  if (st != STEP_OK) return st;
  if (workspace_bytes < need) return STEP_ERR_INVALID_ARG;
  st = on_pool_device(pool);
  if (st != STEP_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  RowsArgs a = {};
  a.g = geo_of(pool);
  a.kv = pool->cfg.kv_storage; a.layer = layer;
  a.q = q; a.T = 1;
  a.block_table = block_table; a.seq_lens = seq_lens; a.out = out;
  a.scores = (float*)workspace; a.score_stride = stride_of_scores(weight_stride);
  a.ml = a.scores + (size_t)n * a.g.Hq * a.score_stride;
  a.counters = pool->v.counters;
  st = pool->cfg.dtype == STEP_BF16 ? launch_attn_rows<__nv_bfloat16, float, false, true>(a, n, s)
                                    : launch_attn_rows<float, float, false, true>(a, n, s);
  if (st != STEP_OK) return st;
  int chunks = (weight_stride + 4 * kAccThreads - 1) / (4 * kAccThreads);
  if (chunks > 64) chunks = 64;
  if (launch_dependent(weights_add_kernel, dim3(chunks, a.g.Hkv, n), dim3(kAccThreads), 0, s, a.g, a.scores, a.score_stride,
                       a.ml, seq_lens, weight_sum, weight_stride, a.counters) != cudaSuccess) return STEP_ERR_CUDA;
  return launch_ok();
}

}  // extern "C"
