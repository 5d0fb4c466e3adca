// decode_attention_weights: decode attention that also keeps count of what the cache is used for.
//
//   p[i][h][j] = softmax_j(q[i][h] . K_i[j] / sqrt(d)),  out[i][h] = sum_j p[i][h][j] V_i[j]
//   weight_sum[i][kvh][j] += sum over the query heads h of KV head kvh of p[i][h][j]
//
// The weights are known only when a row's maximum and sum are, so the attention kernel leaves its scores (log2-scaled,
// fp32) in the workspace and a second kernel, its programmatic dependent, turns them into weights: 8 * G bytes per
// position and KV head on top of the 4 * d bytes of K and V in bf16 (a second read of K would be 2 * d).
//
// 64 traces of 4.6k to 16.9k positions, 32 / 8 heads of 128 in bf16: 464 to 488 us, 2.86 GB at 5.9 to 6.2 TB/s; the streaming kernel
// is 438 of them, at the measured copy bandwidth, the rest is combining (bound by the latency of the pieces' loads) and adding
// (24 us alone: the scores come back from HBM and L2 at 5.5 TB/s).  The adding launch and the scores' workspace are sized by
// weight_stride, not by the lengths, which the host does not know: CTAs behind a trace's end return at once.
#include "attention_rows.cuh"

using namespace stepk;

namespace {

constexpr int kAccThreads = 256, kAccKeys = 4 * kAccThreads;

// x + y with subnormal numbers kept (this library's own arithmetic flushes them): a sum that a caller has let decay that far
// stays what it is where a weight is nothing.
__device__ inline float add_kept(float x, float y) {
  float z;
  asm("add.rn.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
  return z;
}

// weight_sum[t][h][j] += sum_g exp2(scores[t][h G + g][j] - m_g) / l_g.  grid (chunks of kAccKeys positions, Hkv, n), a thread
// takes four positions; the heads are added in ascending order, so the sums do not depend on the launch.
__global__ void __launch_bounds__(kAccThreads)
weights_add_kernel(Geo g, const float* __restrict__ scores, long long score_stride, const float* __restrict__ ml,
                   const int32_t* __restrict__ seq_lens, float* __restrict__ weight_sum, int weight_stride, int32_t* counters) {
  const int h = blockIdx.y, t = blockIdx.z;
  wait_for_primary();
  long long S = seq_lens[t];
  const long long cap = (long long)g.max_pages * g.P;
  if (S > cap) S = cap;
  if (S > weight_stride) { S = weight_stride; if (threadIdx.x == 0 && blockIdx.x == 0) flag_error(counters, STEP_ERR_CAPACITY); }
  const long long j = (long long)blockIdx.x * kAccKeys + threadIdx.x * 4;
  if (j >= S) return;
  const float4* sc = reinterpret_cast<const float4*>(scores + ((size_t)t * g.Hq + (size_t)h * g.G) * score_stride + j);
  const float2* mlh = reinterpret_cast<const float2*>(ml) + (size_t)t * g.Hq + (size_t)h * g.G;
  float* w = weight_sum + ((size_t)t * g.Hkv + h) * weight_stride + j;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < g.G; ++k) {
    const float4 s = __ldcs(sc + (size_t)k * (score_stride / 4));
    const float2 r = mlh[k];
    const float inv = 1.f / r.y;
    sum.x += exp2f(s.x - r.x) * inv;
    sum.y += exp2f(s.y - r.x) * inv;
    sum.z += exp2f(s.z - r.x) * inv;
    sum.w += exp2f(s.w - r.x) * inv;
  }
  if (j + 4 <= S && ((uintptr_t)w & 15) == 0) {
    float4 old = *reinterpret_cast<float4*>(w);
    old.x = add_kept(old.x, sum.x); old.y = add_kept(old.y, sum.y);
    old.z = add_kept(old.z, sum.z); old.w = add_kept(old.w, sum.w);
    *reinterpret_cast<float4*>(w) = old;
  } else {
    w[0] = add_kept(w[0], sum.x);
    if (j + 1 < S) w[1] = add_kept(w[1], sum.y);
    if (j + 2 < S) w[2] = add_kept(w[2], sum.z);
    if (j + 3 < S) w[3] = add_kept(w[3], sum.w);
  }
}

long long stride_of_scores(int weight_stride) { return ((long long)weight_stride + 15) / 16 * 16; }

}  // namespace

extern "C" {

int decode_attention_weights_workspace_bytes(const step_pool* pool, int n, int weight_stride, size_t* bytes) {
  if (!pool || !bytes || n < 0 || weight_stride < 1) return STEP_ERR_INVALID_ARG;
  const size_t rows = (size_t)n * pool->cfg.num_q_heads;
  *bytes = rows * stride_of_scores(weight_stride) * sizeof(float) + rows * 2 * sizeof(float);
  if (!attn_mma_covers(pool, n)) *bytes += 12 + attn_rows_workspace(pool, n, 1);
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
  const Geo g = geo_of(pool);
  float* scores = (float*)workspace;
  const long long score_stride = stride_of_scores(weight_stride);
  float* ml = scores + (size_t)n * g.Hq * score_stride;
  if (attn_mma_covers(pool, n)) {
    st = attn_mma_scores(pool, layer, q, block_table, seq_lens, n, out, scores, score_stride, ml, s);
  } else {
    RowsArgs a = {};
    a.g = g;
    a.kv = pool->cfg.kv_storage; a.layer = layer;
    a.q = q; a.T = 1;
    a.block_table = block_table; a.seq_lens = seq_lens; a.out = out;
    a.scores = scores; a.score_stride = score_stride; a.ml = ml;
    a.counters = pool->v.counters;
    float* part = ml + ((size_t)n * g.Hq * 2 + 3) / 4 * 4;          // 16-byte aligned
    st = pool->cfg.dtype == STEP_BF16 ? launch_attn_rows<__nv_bfloat16, float, false, true>(pool, a, n, part, s)
                                      : launch_attn_rows<float, float, false, true>(pool, a, n, part, s);
  }
  if (st != STEP_OK) return st;
  const int chunks = (int)(((long long)weight_stride + kAccKeys - 1) / kAccKeys);
  if (launch_dependent(weights_add_kernel, dim3(chunks, g.Hkv, n), dim3(kAccThreads), 0, s, g, scores, score_stride, ml,
                       seq_lens, weight_sum, weight_stride, pool->v.counters) != cudaSuccess) return STEP_ERR_CUDA;
  return launch_ok();
}

}  // extern "C"
