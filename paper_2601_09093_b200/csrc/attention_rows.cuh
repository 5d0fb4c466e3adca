// Attention of several query rows of one trace and KV head on the CUDA cores, for any element type, head size and page
// size: what decode_attention_tree and decode_attention_weights run on where their tensor-core kernels do not apply.
//
//   out[r] = sum_j softmax_j(q[r] . k[j] * scale) v[j]     over the S cached positions and, for a tree of drafted tokens,
//                                                          over the drafted tokens that row r may see
//
// One CTA takes kRows query rows of one (trace, KV head) - the rows of a trace are the G heads of the group for every
// drafted token (row = token * G + head) - and one of `splits` equal ranges of its keys, kKeys at a time: K and V are
// widened to fp32 in shared memory, a thread makes four scores, a row's eight threads keep its running (max, sum) in fp32,
// and in the second product a thread owns four dims of two or four rows.  fp32 throughout: one rounding, of the output.
// With more than one range the pieces are combined by rows_merge_kernel, a programmatic dependent, in ascending order.
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
  int splits;
  float* part;                          // splits > 1: [n, Hkv, rows, splits, d] values, then (max, sum) pairs
  int32_t* counters;
};

constexpr int kRows = 16, kKeys = 32, kRowsThreads = 128, kAhead = 8;

// Ranges of keys per (row block, KV head, trace): enough that about four CTAs per SM have work, each at least two tiles.
// (8 traces of up to 256 tokens, 4 heads of 64 in fp32, one new token: 229 us with one range and the products of the first
// form of this kernel.)
inline int attn_rows_splits(const step_pool* pool, int n, int T) {
  const long long units = (long long)n * pool->cfg.num_kv_heads * ((T * pool->G + kRows - 1) / kRows);
  const long long most = ((long long)pool->cfg.max_pages_per_trace * pool->cfg.page_size + T + 2 * kKeys - 1) / (2 * kKeys);
  long long s = units > 0 ? 4ll * pool->num_sms / units : 1;
  if (s > most) s = most;
  if (s > 64) s = 64;
  return s < 1 ? 1 : (int)s;
}
inline size_t attn_rows_workspace(const step_pool* pool, int n, int T) {
  const int splits = attn_rows_splits(pool, n, T);
  return splits == 1 ? 0 : (size_t)n * pool->cfg.num_kv_heads * T * pool->G * splits * (pool->cfg.head_dim + 2) * sizeof(float);
}

inline size_t attn_rows_smem(int d) { return ((size_t)kRows * (d + 4) + (size_t)kKeys * (d + 4) + (size_t)kKeys * d) * sizeof(float); }

// kRpt rows and kNi times four dims of the output per thread: kRpt 2 for d <= 64, else 4; kNi 4 for d > 128.
template <typename T, typename OutT, bool kTree, bool kScores, int kRpt, int kNi>
__global__ void __launch_bounds__(kRowsThreads) attn_rows_kernel(RowsArgs a) {
  extern __shared__ float4 smem4[];
  const Geo& g = a.g;
  const int d = g.d, G = g.G, h = blockIdx.y, t = blockIdx.z;
  const int n_rows = a.T * G, blocks = (n_rows + kRows - 1) / kRows;
  const int r0 = (int)(blockIdx.x % blocks) * kRows, split = blockIdx.x / blocks;
  const int ld = d + 4;
  float* s_q = reinterpret_cast<float*>(smem4);
  float* s_k = s_q + kRows * ld;
  float* s_v = s_k + kKeys * ld;
  __shared__ __align__(16) float s_p[kKeys][kRows + 4];
  __shared__ float s_corr[kRows], s_m[kRows], s_l[kRows];
  __shared__ unsigned long long s_mask[kMaxTreeNodes];
  __shared__ int s_up[kMaxTreeNodes];
  __shared__ const T* s_src[2][2][kKeys];                // [tile parity][K | V][key]: start of the row, null behind the last key
  const int tid = threadIdx.x;
  constexpr int cpe = 16 / (int)sizeof(T);
  const int cpr = d / cpe;
  const T* kv = (const T*)a.kv;
  dependents_may_launch();

  int nodes = 1;
  if constexpr (kTree) {
    nodes = tree_nodes(a.n_nodes, t, a.T, a.counters);
    tree_masks(a.parents + (size_t)t * a.T, nodes, s_mask, s_up, a.counters);
  }
  int S = a.seq_lens[t];
  if (S < 0) S = 0;
  if ((long long)S > (long long)g.max_pages * g.P) { S = g.max_pages * g.P; if (tid == 0) flag_error(a.counters, STEP_ERR_CAPACITY); }
  const int n_keys = S + (kTree ? nodes : 0);
  const int tiles = (n_keys + kKeys - 1) / kKeys, per = (tiles + a.splits - 1) / a.splits;
  const int it0 = min(tiles, split * per), it1 = min(tiles, it0 + per);

  // where the rows of a tile's keys are (a thread per key)
  auto locate = [&](int it) {
    if (tid < kKeys && it < it1) {
      const int j = it * kKeys + tid;
      const T *k = nullptr, *v = nullptr;
      if (j < S) {
        int b = a.block_table[(size_t)t * g.max_pages + j / g.P];
        if (b < 0 || b >= g.num_blocks) { flag_error(a.counters, STEP_ERR_BAD_BLOCK); b = 0; }
        k = kv + kv_page_base(g, a.layer, b, h, 0) + (size_t)(j % g.P) * d;
        v = k + (size_t)g.P * d;
      } else if (kTree && j < n_keys) {
        const size_t at = ((((size_t)t * a.T + (j - S)) * g.L + a.layer) * g.Hkv + h) * d;
        k = (const T*)a.k_draft + at;
        v = (const T*)a.v_draft + at;
      }
      s_src[it & 1][0][tid] = k;
      s_src[it & 1][1][tid] = v;
    }
  };
  locate(it0);
#pragma unroll 2
  for (int i = tid; i < kRows * cpr; i += kRowsThreads) {
    const int rr = i / cpr, c = i - rr * cpr, r = r0 + rr;
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (r < nodes * G)
      raw = *reinterpret_cast<const uint4*>((const T*)a.q + (((size_t)t * a.T + r / G) * g.Hq + (size_t)h * G + r % G) * d + c * cpe);
    const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int x = 0; x < cpe; ++x) s_q[rr * ld + c * cpe + x] = to_f32(e[x]);
  }
  const float scale = 1.4426950408889634f / sqrtf((float)d);
  const int row = tid >> 3, sub = tid & 7;               // first product: a row's eight threads take keys sub, sub + 8, ...
  const int my_r = r0 + row, my_u = my_r / G;
  const bool real = my_r < nodes * G;
  unsigned long long sees = 0;
  if constexpr (kTree) sees = real ? s_mask[my_u] : 0ull;
  float m_run = -INFINITY, l_run = 0.f;
  // second product: thread x of the (row group, dims) tiles owns rows kRpt * (x % groups) .. and dims 4 * (x / groups) ..
  constexpr int kGroups = kRows / kRpt;                 // (divides the threads: a thread's rows are the same in all of its tiles)
  static_assert(kRowsThreads % kGroups == 0, "rows of a thread");
  const int tiles_o = kGroups * (d / 4);
  float acc[kNi][kRpt][4];
#pragma unroll
  for (int i = 0; i < kNi; ++i)
#pragma unroll
    for (int x = 0; x < kRpt; ++x) { acc[i][x][0] = acc[i][x][1] = acc[i][x][2] = acc[i][x][3] = 0.f; }
  unsigned long long see[kRpt];                          // the drafted tokens that these rows see
#pragma unroll
  for (int y = 0; y < kRpt; ++y) {
    const int r = r0 + tid % kGroups * kRpt + y;
    see[y] = kTree && r < nodes * G ? s_mask[r / G] : 0ull;
  }
  __syncthreads();

  for (int it = it0; it < it1; ++it) {
    const int j0 = it * kKeys;
    // (kAhead loads of a thread are under way before the first of them is used)
    for (int i0 = tid; i0 < 2 * kKeys * cpr; i0 += kAhead * kRowsThreads) {
      uint4 raw[kAhead];
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        const int i = i0 + y * kRowsThreads;
        raw[y] = make_uint4(0, 0, 0, 0);
        if (i < 2 * kKeys * cpr) {
          const int which = i >= kKeys * cpr, r = which ? i - kKeys * cpr : i;
          const int key = r / cpr, c = r - key * cpr;
          const T* src = s_src[it & 1][which][key];
          if (src) {
            const int j = j0 + key;
            const int cc = g.swizzle && j < S ? ((c & ~7) | ((c ^ (j % g.P)) & 7)) : c;   // (drafts are stored as they come)
            raw[y] = *reinterpret_cast<const uint4*>(src + cc * cpe);
          }
        }
      }
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        const int i = i0 + y * kRowsThreads;
        if (i < 2 * kKeys * cpr) {
          const int which = i >= kKeys * cpr, r = which ? i - kKeys * cpr : i;
          const int key = r / cpr, c = r - key * cpr;
          const T* e = reinterpret_cast<const T*>(&raw[y]);
          float* dst = which ? s_v + key * d + c * cpe : s_k + key * ld + c * cpe;
#pragma unroll
          for (int x = 0; x < cpe; x += 4)
            *reinterpret_cast<float4*>(dst + x) = make_float4(to_f32(e[x]), to_f32(e[x + 1]), to_f32(e[x + 2]), to_f32(e[x + 3]));
        }
      }
    }
    locate(it + 1);
    __syncthreads();
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < d; k += 4) {
      const float4 x = *reinterpret_cast<const float4*>(s_q + row * ld + k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 y = *reinterpret_cast<const float4*>(s_k + (sub + 8 * i) * ld + k);
        s[i] = fmaf(x.x, y.x, s[i]); s[i] = fmaf(x.y, y.y, s[i]); s[i] = fmaf(x.z, y.z, s[i]); s[i] = fmaf(x.w, y.w, s[i]);
      }
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
      s_p[sub + 8 * i][row] = p;
      sum += p;
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    l_run = l_run * corr + sum;
    m_run = mx;
    if (sub == 0) s_corr[row] = corr;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kNi; ++i) {
      const int x = tid + i * kRowsThreads;
      if (x < tiles_o) {
        const int rg = x % kGroups * kRpt, k = x / kGroups * 4;
#pragma unroll
        for (int y = 0; y < kRpt; ++y) {
          const float c = s_corr[rg + y];
#pragma unroll
          for (int z = 0; z < 4; ++z) acc[i][y][z] *= c;
        }
        if (kTree && j0 + kKeys > S) {
          // a drafted token that a row does not see is passed over: its v may hold an infinity or a NaN, and 0 times that is NaN
#pragma unroll 4
          for (int key = 0; key < min(kKeys, n_keys - j0); ++key) {
            const float4 v = *reinterpret_cast<const float4*>(s_v + key * d + k);
            const int u = j0 + key - S;
#pragma unroll
            for (int y = 0; y < kRpt; ++y) {
              const float p = s_p[key][rg + y];
              if (u < 0 || ((see[y] >> (u & 63)) & 1)) {
                acc[i][y][0] = fmaf(p, v.x, acc[i][y][0]); acc[i][y][1] = fmaf(p, v.y, acc[i][y][1]);
                acc[i][y][2] = fmaf(p, v.z, acc[i][y][2]); acc[i][y][3] = fmaf(p, v.w, acc[i][y][3]);
              }
            }
          }
          continue;
        }
#pragma unroll 8
        for (int key = 0; key < kKeys; ++key) {
          const float4 v = *reinterpret_cast<const float4*>(s_v + key * d + k);
          float p[kRpt];
#pragma unroll
          for (int y = 0; y < kRpt; ++y) p[y] = s_p[key][rg + y];
#pragma unroll
          for (int y = 0; y < kRpt; ++y) {
            acc[i][y][0] = fmaf(p[y], v.x, acc[i][y][0]); acc[i][y][1] = fmaf(p[y], v.y, acc[i][y][1]);
            acc[i][y][2] = fmaf(p[y], v.z, acc[i][y][2]); acc[i][y][3] = fmaf(p[y], v.w, acc[i][y][3]);
          }
        }
      }
    }
    __syncthreads();
  }
  if (sub == 0) { s_m[row] = m_run; s_l[row] = l_run; }
  __syncthreads();
  const size_t head_rows = ((size_t)t * g.Hkv + h) * n_rows;          // this head's first row among all rows
  const size_t all_rows = (size_t)gridDim.z * g.Hkv * n_rows;
  float2* part_ml = reinterpret_cast<float2*>(a.part + all_rows * a.splits * d);
#pragma unroll
  for (int i = 0; i < kNi; ++i) {
    const int x = tid + i * kRowsThreads;
    if (x >= tiles_o) break;
    const int rg = x % kGroups * kRpt, k = x / kGroups * 4;
#pragma unroll
    for (int y = 0; y < kRpt; ++y) {
      const int r = r0 + rg + y;
      if (r >= n_rows) continue;
      if (a.splits > 1) {
        *reinterpret_cast<float4*>(a.part + ((head_rows + r) * a.splits + split) * d + k) =
            make_float4(acc[i][y][0], acc[i][y][1], acc[i][y][2], acc[i][y][3]);
      } else {
        const float l = s_l[rg + y], inv = l > 0.f ? 1.f / l : 0.f;
        OutT* o = (OutT*)a.out + (((size_t)t * a.T + r / G) * g.Hq + (size_t)h * G + r % G) * d + k;
#pragma unroll
        for (int z = 0; z < 4; ++z) o[z] = from_f32<OutT>(l > 0.f ? acc[i][y][z] * inv : l == 0.f ? 0.f : l);   // (a NaN stays one)
      }
    }
  }
  if (tid < kRows && r0 + tid < n_rows) {
    const float2 ml = make_float2(s_m[tid], s_l[tid]);
    if (a.splits > 1) part_ml[(head_rows + r0 + tid) * a.splits + split] = ml;
    else if (kScores) reinterpret_cast<float2*>(a.ml)[(size_t)t * g.Hq + (size_t)h * G + r0 + tid] = ml;
  }
}

// Combines the ranges of every row, in ascending order: a warp per row, lanes over the dims.
template <typename OutT, bool kScores>
__global__ void __launch_bounds__(kRowsThreads) rows_merge_kernel(RowsArgs a, int n) {
  const Geo& g = a.g;
  const int d = g.d, G = g.G, n_rows = a.T * G, lane = threadIdx.x & 31;
  const size_t all_rows = (size_t)n * g.Hkv * n_rows;
  const float2* part_ml = reinterpret_cast<const float2*>(a.part + all_rows * a.splits * d);
  dependents_may_launch();
  wait_for_primary();
  for (size_t i = (size_t)blockIdx.x * (kRowsThreads / 32) + (threadIdx.x >> 5); i < all_rows; i += (size_t)gridDim.x * (kRowsThreads / 32)) {
    const int r = (int)(i % n_rows);
    const size_t th = i / n_rows, t = th / g.Hkv, h = th % g.Hkv;
    // a lane per range (two where there are more than 32)
    float2 x0 = make_float2(-INFINITY, 0.f), x1 = x0;
    if (lane < a.splits) x0 = __ldcg(part_ml + i * a.splits + lane);
    if (lane + 32 < a.splits) x1 = __ldcg(part_ml + i * a.splits + lane + 32);
    float M = fmaxf(x0.x, x1.x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    const float off = M == -INFINITY ? 0.f : M;
    const float w0 = exp2f(x0.x - off), w1 = exp2f(x1.x - off);
    float l = w0 * x0.y + w1 * x1.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    const float inv = 1.f / l;
    OutT* out = (OutT*)a.out + ((t * a.T + r / G) * g.Hq + h * G + r % G) * d;
    for (int k0 = 0; k0 < d; k0 += 128) {
      const int k = k0 + lane * 4;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int s = 0; s < a.splits; ++s) {
        const float w = __shfl_sync(0xffffffffu, s < 32 ? w0 : w1, s & 31);
        if (k < d) {
          const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part + (i * a.splits + s) * d + k));
          sum.x = fmaf(w, v.x, sum.x); sum.y = fmaf(w, v.y, sum.y); sum.z = fmaf(w, v.z, sum.z); sum.w = fmaf(w, v.w, sum.w);
        }
      }
      if (k < d) {
        const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int z = 0; z < 4; ++z) out[k + z] = from_f32<OutT>(l > 0.f ? v[z] * inv : l == 0.f ? 0.f : l);
      }
    }
    if constexpr (kScores)
      if (lane == 0) reinterpret_cast<float2*>(a.ml)[t * g.Hq + h * G + r] = make_float2(M, l);
  }
}

// a.splits and a.part are set here; `part` has attn_rows_workspace bytes.
template <typename T, typename OutT, bool kTree, bool kScores>
int launch_attn_rows(const step_pool* pool, RowsArgs a, int n, float* part, cudaStream_t s) {
  a.splits = attn_rows_splits(pool, n, a.T);
  a.part = part;
  const int d = a.g.d;
  const size_t smem = attn_rows_smem(d);
  auto kern = d <= 64 ? attn_rows_kernel<T, OutT, kTree, kScores, 2, 1>
                      : (d <= 128 ? attn_rows_kernel<T, OutT, kTree, kScores, 4, 1> : attn_rows_kernel<T, OutT, kTree, kScores, 4, 4>);
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return STEP_ERR_CUDA;
  const int blocks = (a.T * a.g.G + kRows - 1) / kRows;
  kern<<<dim3(blocks * a.splits, a.g.Hkv, n), kRowsThreads, smem, s>>>(a);
  if (launch_ok() != STEP_OK) return STEP_ERR_CUDA;
  if (a.splits > 1) {
    const long long rows = (long long)n * a.g.Hkv * a.T * a.g.G;
    const int grid = (int)((rows + 3) / 4 < 8ll * pool->num_sms ? (rows + 3) / 4 : 8ll * pool->num_sms);
    if (launch_dependent(rows_merge_kernel<OutT, kScores>, dim3(grid), dim3(kRowsThreads), 0, s, a, n) != cudaSuccess) return STEP_ERR_CUDA;
  }
  return launch_ok();
}

}  // namespace stepk
