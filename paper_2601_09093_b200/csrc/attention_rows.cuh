// Attention of several query rows of one trace and KV head on the CUDA cores, for any element type, head size and page
// size: what decode_attention_tree and decode_attention_weights run on where their tensor-core kernels do not apply.
//
//   out[r] = sum_j softmax_j(q[r] . k[j] * scale) v[j]     over the S cached positions and, for a tree of drafted tokens,
//                                                          over the drafted tokens that row r may see
//
// One CTA takes kRows query rows of one (trace, KV head): the rows of a trace are the G heads of the group for every
// drafted token (row = token * G + head).  It walks over the keys kKeys at a time: K and V are widened to fp32 in shared
// memory, a thread makes four scores, a row's eight threads keep its running (max, sum) in fp32, and in the second product
// a thread owns up to four dims of all rows.  fp32 throughout: one rounding, of the output.
#pragma once

#include "step_internal.cuh"

#include <math.h>

namespace stepk {

constexpr int kMaxTreeNodes = 64;     // drafted tokens per trace: a node's ancestors are one 64-bit mask

__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ inline T from_f32(float x);
template <> __device__ inline float from_f32<float>(float x) { return x; }
template <> __device__ inline __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16(x); }

// Drafted tokens of trace t that exist: n_nodes[t], or all T.
__device__ inline int tree_nodes(const int32_t* n_nodes, int t, int T, int32_t* counters) {
  if (!n_nodes) return T;
  const int k = n_nodes[t];
  if (k < 0 || k > T) { if (threadIdx.x == 0) flag_error(counters, STEP_ERR_INVALID_ARG); return k < 0 ? 0 : T; }
  return k;
}

// s_mask[u] = the nodes that node u attends to: itself and its ancestors.  Called by the whole CTA (at least
// kMaxTreeNodes threads); pointer doubling, six rounds.  A parent that does not come before its node is flagged and
// read as "none".
__device__ inline void tree_masks(const int32_t* parents, int nodes, unsigned long long* s_mask, int* s_up, int32_t* counters) {
  const int u = threadIdx.x;
  if (u < nodes) {
    int p = parents[u];
    if (p >= u || p < -1) { flag_error(counters, STEP_ERR_INVALID_ARG); p = -1; }
    s_up[u] = p;
    s_mask[u] = 1ull << u;
  }
  __syncthreads();
#pragma unroll 1
  for (int reach = 1; reach < kMaxTreeNodes; reach *= 2) {
    unsigned long long m = 0;
    int up = -1;
    if (u < nodes) {
      const int p = s_up[u];
      m = s_mask[u];
      if (p >= 0) { m |= s_mask[p]; up = s_up[p]; }
    }
    __syncthreads();
    if (u < nodes) { s_mask[u] = m; s_up[u] = up; }
    __syncthreads();
  }
}

struct RowsArgs {
  Geo g;
  const void* kv; int layer;
  const void* q;                        // [n, T, Hq, d]
  const void* k_draft; const void* v_draft;   // [n, T, L, Hkv, d] (trees only)
  const int32_t* parents;               // [n, T]
  const int32_t* n_nodes;               // [n] or null
  int T;
  const int32_t* block_table; const int32_t* seq_lens;
  void* out;                            // [n, T, Hq, d]
  float* scores;                        // [n, Hq, score_stride] log2-scaled scores of the cached positions (kScores)
  long long score_stride;
  float* ml;                            // [n, Hq, 2] (max, sum) of every row, log2-scaled (kScores)
  int32_t* counters;
};

constexpr int kRows = 16, kKeys = 32, kRowsThreads = 128;

inline size_t attn_rows_smem(int d) { return ((size_t)kRows * d + (size_t)kKeys * (d + 1) + (size_t)kKeys * d) * sizeof(float); }

template <typename T, typename OutT, bool kTree, bool kScores>
__global__ void __launch_bounds__(kRowsThreads) attn_rows_kernel(RowsArgs a) {
  extern __shared__ float smf[];
  const Geo& g = a.g;
  const int d = g.d, G = g.G, h = blockIdx.y, t = blockIdx.z, r0 = blockIdx.x * kRows;
  float* s_q = smf;
  float* s_k = s_q + kRows * d;
  float* s_v = s_k + kKeys * (d + 1);
  __shared__ float s_p[kRows][kKeys + 1], s_m[kRows], s_l[kRows], s_corr[kRows];
  __shared__ unsigned long long s_mask[kMaxTreeNodes];
  __shared__ int s_up[kMaxTreeNodes];
  const int tid = threadIdx.x;
  constexpr int cpe = 16 / (int)sizeof(T);
  const int cpr = d / cpe;
  const T* kv = (const T*)a.kv;
  const int n_rows = a.T * G;

  int nodes = 1;
  if constexpr (kTree) {
    nodes = tree_nodes(a.n_nodes, t, a.T, a.counters);
    tree_masks(a.parents + (size_t)t * a.T, nodes, s_mask, s_up, a.counters);
  }
  int S = a.seq_lens[t];
  if (S < 0) S = 0;
  if ((long long)S > (long long)g.max_pages * g.P) { S = g.max_pages * g.P; if (tid == 0) flag_error(a.counters, STEP_ERR_CAPACITY); }
  const int n_keys = S + (kTree ? nodes : 0);

  for (int i = tid; i < kRows * d; i += kRowsThreads) {
    const int r = r0 + i / d;
    float x = 0.f;
    if (r < nodes * G) x = to_f32(((const T*)a.q)[(((size_t)t * a.T + r / G) * g.Hq + (size_t)h * G + r % G) * d + i % d]);
    s_q[i] = x;
  }
  const float scale = 1.4426950408889634f / sqrtf((float)d);
  const int row = tid >> 3, sub = tid & 7;               // first product: a row's eight threads take keys sub, sub + 8, ...
  const int my_r = r0 + row, my_u = my_r / G;
  const bool real = my_r < nodes * G;
  unsigned long long sees = 0;
  if constexpr (kTree) sees = real ? s_mask[my_u] : 0ull;
  float m_run = -INFINITY, l_run = 0.f;
  float acc[kRows][4];
#pragma unroll
  for (int r = 0; r < kRows; ++r) { acc[r][0] = acc[r][1] = acc[r][2] = acc[r][3] = 0.f; }

  for (int j0 = 0; j0 < n_keys; j0 += kKeys) {
    __syncthreads();
    for (int i = tid; i < 2 * kKeys * cpr; i += kRowsThreads) {
      const int which = i >= kKeys * cpr, r = which ? i - kKeys * cpr : i;
      const int key = r / cpr, c = r - key * cpr, j = j0 + key;
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (j < S) {
        const int slot = j % g.P;
        int b = a.block_table[(size_t)t * g.max_pages + j / g.P];
        if (b < 0 || b >= g.num_blocks) { flag_error(a.counters, STEP_ERR_BAD_BLOCK); b = 0; }
        raw = *reinterpret_cast<const uint4*>(kv + kv_page_base(g, a.layer, b, h, which) + kv_in_page(g, slot, c * cpe, cpe));
      } else if (kTree && j < n_keys) {
        const T* src = (const T*)(which ? a.v_draft : a.k_draft);
        raw = *reinterpret_cast<const uint4*>(src + ((((size_t)t * a.T + (j - S)) * g.L + a.layer) * g.Hkv + h) * d + c * cpe);
      }
      const T* e = reinterpret_cast<const T*>(&raw);
      float* dst = which ? s_v + key * d + c * cpe : s_k + key * (d + 1) + c * cpe;
#pragma unroll
      for (int x = 0; x < cpe; ++x) dst[x] = to_f32(e[x]);
    }
    __syncthreads();
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    const float* qr = s_q + row * d;
    for (int k = 0; k < d; ++k) {
      const float x = qr[k];
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = fmaf(x, s_k[(sub + 8 * i) * (d + 1) + k], s[i]);
    }
    float mx = m_run;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + sub + 8 * i;
      bool see = real && j < S;
      if (kTree && j >= S && j < n_keys) see = (sees >> (j - S)) & 1;
      s[i] = see ? s[i] * scale : -INFINITY;
      mx = fmaxf(mx, s[i]);
      if constexpr (kScores)
        if (see && j < a.score_stride) a.scores[((size_t)t * g.Hq + (size_t)h * G + my_r) * a.score_stride + j] = s[i];
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float base = mx == -INFINITY ? 0.f : mx;        // a row that has seen nothing yet
    const float corr = exp2f(m_run - base);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = exp2f(s[i] - base);
      s_p[row][sub + 8 * i] = p;
      sum += p;
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    l_run = l_run * corr + sum;
    m_run = mx;
    if (sub == 0) s_corr[row] = corr;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = tid + kRowsThreads * i;
      if (k >= d) break;
#pragma unroll
      for (int r = 0; r < kRows; ++r) acc[r][i] *= s_corr[r];
      for (int key = 0; key < kKeys; ++key) {
        const float v = s_v[key * d + k];
#pragma unroll
        for (int r = 0; r < kRows; ++r) acc[r][i] = fmaf(s_p[r][key], v, acc[r][i]);
      }
    }
  }
  if (sub == 0) { s_m[row] = m_run; s_l[row] = l_run; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = tid + kRowsThreads * i;
    if (k >= d) break;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int rr = r0 + r;
      if (rr >= n_rows) continue;
      const float l = s_l[r];
      ((OutT*)a.out)[(((size_t)t * a.T + rr / G) * g.Hq + (size_t)h * G + rr % G) * d + k] = from_f32<OutT>(l > 0.f ? acc[r][i] / l : 0.f);
    }
  }
  if constexpr (kScores)
    if (tid < kRows && r0 + tid < n_rows) {
      float* ml = a.ml + ((size_t)t * g.Hq + (size_t)h * G + r0 + tid) * 2;
      ml[0] = s_m[tid]; ml[1] = s_l[tid];
    }
}

template <typename T, typename OutT, bool kTree, bool kScores>
int launch_attn_rows(const RowsArgs& a, int n, cudaStream_t s) {
  const size_t smem = attn_rows_smem(a.g.d);
  auto kern = attn_rows_kernel<T, OutT, kTree, kScores>;
  if (smem > 32 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return STEP_ERR_CUDA;
  const int blocks = (a.T * a.g.G + kRows - 1) / kRows;
  kern<<<dim3(blocks, a.g.Hkv, n), kRowsThreads, smem, s>>>(a);
  return launch_ok();
}

}  // namespace stepk
