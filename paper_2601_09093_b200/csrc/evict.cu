// kv_pool_evict_positions: a trace whose cache is over its budget gives up the positions of least accumulated weight.
//
// Per (layer, listed trace, KV head), with S cached positions, first = S - recent and m = budget - recent:
//   C     = the m of the positions [0, first) with the largest weights (equal weights: the lower position first, NaN last)
//   slots [m, budget)  get positions [first, S) in order, the trace's most recent ones
//   slots [0, m)       a chosen position below m stays where it is; the free slots take, in ascending order, the chosen
//                      positions from m on, in ascending order
// Attention over a cache does not depend on the order of its positions, so only `recent` rows and one row per evicted
// position move; keeping all of them in order would move half the cache or more on average.  The last slots do stay in
// order, which is what makes "the most recent ones" mean the same at the next call.
//
// Three launches, each a programmatic dependent of the one before:
//   1. evict_plan_kernel    one CTA: which traces are cut; a block of its own for every kept page that is shared
//   2. evict_move_kernel    one CTA per (KV head, trace, layer): selection, then the rows and weights move
//   3. evict_finish_kernel  a cluster of CTAs: references dropped, free list, block table, lengths
#include "release.cuh"

using namespace stepk;

namespace {

struct EvictArgs {
  DevViews v;
  Geo g;
  uint4* kv;
  const int32_t* ids;
  int n;
  const float* weights; float* weights_out;   // [L, n, Hkv, stride]
  int stride, budget, recent;
  int32_t* kept;                              // [L, n, Hkv, budget]
  int32_t* old_len;                           // workspace [n]: cached positions of the entry before the call; -1: left alone
  int32_t* off;                               // workspace [n + 1]
  int32_t* new_row;                           // workspace [n, pages of a budget]
  int cpr;
};

constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads) evict_plan_kernel(EvictArgs a) {
  extern __shared__ int sm[];
  dependents_may_launch();
  int* s_need = sm;                   // blocks wanted for shared kept pages; -1: the entry is left alone
  int* s_off = sm + a.n;
  __shared__ int s_fc;
  const DevViews& v = a.v;
  const Geo& g = a.g;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nwarps = blockDim.x >> 5;
  const int nbp = (a.budget + g.P - 1) / g.P;
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    const int t = a.ids[i];
    if (t >= 0 && t < g.max_traces) v.prune_rank[t] = 0x7fffffff;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    const int t = a.ids[i];
    if (t >= 0 && t < g.max_traces) atomicMin(&v.prune_rank[t], i);
  }
  __syncthreads();
  for (int i = warp; i < a.n; i += nwarps) {
    const int t = a.ids[i];
    int need = -1;
    if (t < 0 || t >= g.max_traces || !v.live[t] || v.prune_rank[t] != i) {
      if (lane == 0) flag_error(v.counters, STEP_ERR_BAD_TRACE);
    } else {
      const int S = v.seq_lens[t];
      if (S > a.stride && S > a.budget) {
        if (lane == 0) flag_error(v.counters, STEP_ERR_CAPACITY);          // positions without a weight
      } else if (S > a.budget) {
        // the pages that stay, by block; a block out of range leaves the whole entry alone
        const int32_t* row = v.block_table + (size_t)t * g.max_pages;
        const int pages = (S + g.P - 1) / g.P;
        int shared = 0;
        bool bad = false;
        for (int p = lane; p < pages; p += 32) {
          const int b = row[p];
          if (b < 0 || b >= g.num_blocks) bad = true;
          else if (p < nbp && v.refcount[b] > 1) ++shared;
        }
        bad = __any_sync(0xffffffffu, bad);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) shared += __shfl_xor_sync(0xffffffffu, shared, o);
        if (bad) { if (lane == 0) flag_error(v.counters, STEP_ERR_BAD_BLOCK); }
        else need = shared;
      }
    }
    if (lane == 0) s_need[i] = need;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int fc = v.counters[C_FREE_COUNT];
    int remaining = fc, pages = 0;
    for (int i = 0; i < a.n; ++i) {
      a.off[i] = pages;
      const int need = s_need[i];
      if (need < 0) continue;
      if (need > remaining) { s_need[i] = -1; flag_error(v.counters, STEP_ERR_NO_BLOCKS); continue; }
      s_off[i] = fc - remaining;
      remaining -= need;
      pages += (v.seq_lens[a.ids[i]] + g.P - 1) / g.P;
    }
    a.off[a.n] = pages;
    s_fc = fc;
    v.counters[C_FREE_COUNT] = remaining;
  }
  __syncthreads();
  for (int i = warp; i < a.n; i += nwarps) {
    if (s_need[i] < 0) { if (lane == 0) a.old_len[i] = -1; continue; }
    const int t = a.ids[i];
    const int32_t* row = v.block_table + (size_t)t * g.max_pages;
    int32_t* to = a.new_row + (size_t)i * nbp;
    int taken = s_fc - 1 - s_off[i];
    for (int p0 = 0; p0 < nbp; p0 += 32) {
      const int p = p0 + lane;
      const int b = p < nbp ? row[p] : -1;
      const bool shared = b >= 0 && v.refcount[b] > 1;
      const unsigned who = __ballot_sync(0xffffffffu, shared);
      if (p < nbp) to[p] = shared ? v.free_list[taken - __popc(who & ((1u << lane) - 1))] : b;
      taken -= __popc(who);
    }
    if (lane == 0) a.old_len[i] = v.seq_lens[t];
  }
}

// ---------------------------------------------------------------- selection and moves
constexpr int kMoveThreads = 256, kMoveWarps = kMoveThreads / 32;
constexpr int kBins = 2048;                   // selection by digits of 11, 11 and 10 bits

// Larger weight -> larger key; NaN below everything; the two zeros are equal.
__device__ inline uint32_t weight_key(float w) {
  if (isnan(w)) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix sum over the CTA of kMoveThreads; *total gets the sum.
__device__ inline int move_scan(int x, int* s_warp, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kMoveWarps; ++w) {
    const int c = s_warp[w];
    if (w < warp) before += c;
    all += c;
  }
  *total = all;
  return before + incl - x;
}

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(EvictArgs a) {
  __shared__ int s_hist[kBins];
  __shared__ int s_warp[kMoveWarps];
  __shared__ int s_digit, s_left;
  const Geo& g = a.g;
  const int h = blockIdx.x, i = blockIdx.y, l = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t head = ((size_t)l * a.n + i) * g.Hkv + h;
  const float* w = a.weights + head * a.stride;
  float* w_out = a.weights_out + head * a.stride;
  int32_t* kept = a.kept + head * a.budget;
  dependents_may_launch();
  wait_for_primary();
  const int S = a.old_len[i];
  if (S < 0) {                                          // left alone: its weights go over as they are
    if (w_out != w)
      for (int j = tid; j < a.stride; j += kMoveThreads) w_out[j] = w[j];
    return;
  }
  const int first = S - a.recent, m = a.budget - a.recent;

  // ---- the m-th largest key of [0, first), and how many of the positions that have it are chosen
  uint32_t prefix = 0;
  int want = m;                                         // still to be found among the keys that share the prefix
  if (m > 0) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
      for (int b = tid; b < kBins; b += kMoveThreads) s_hist[b] = 0;
      __syncthreads();
      for (int j = tid; j < first; j += kMoveThreads) {
        const uint32_t k = weight_key(w[j]);
        if (pass == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&s_hist[(k >> shift) & ((1u << bits) - 1)], 1);
      }
      __syncthreads();
      // bins from the top: thread x owns bins [hi - 8 x - 7, hi - 8 x]
      constexpr int per = kBins / kMoveThreads;
      int c[per], sum = 0;
#pragma unroll
      for (int x = 0; x < per; ++x) { c[x] = s_hist[kBins - 1 - (tid * per + x)]; sum += c[x]; }
      int total;
      int at = move_scan(sum, s_warp, &total);
#pragma unroll
      for (int x = 0; x < per; ++x) {
        if (at < want && at + c[x] >= want) { s_digit = kBins - 1 - (tid * per + x); s_left = want - at; }
        at += c[x];
      }
      __syncthreads();
      prefix = (prefix << bits) | (uint32_t)s_digit;
      want = s_left;
      __syncthreads();
    }
  }
  // position j is chosen if its key is above the threshold, or equal to it and among the first `want` such positions

  // ---- the chosen positions from m on, ascending, into the last places of [0, m) of the list.  (Its free slots are
  // filled below in ascending order: the place a moving position waits in lies at or behind the slot that takes it.)
  int equal = 0;                                        // positions so far whose key equals the threshold
  int moving = 0;
  if (m > 0) {
    // how many come from [m, first): the chosen ones of [0, m) are counted on the way
    int stay = 0;
    for (int j0 = 0; j0 < m; j0 += kMoveThreads) {
      const int j = j0 + tid;
      const uint32_t k = j < m ? weight_key(w[j]) : 0u;
      const bool eq = j < m && k == prefix;
      int n_eq;
      const int before = move_scan(eq, s_warp, &n_eq);
      const bool c = j < m && (k > prefix || (eq && equal + before < want));
      stay += __syncthreads_count(c);
      equal += n_eq;
    }
    moving = m - stay;
    int put = m - moving;
    for (int j0 = m; j0 < first && put < m; j0 += kMoveThreads) {
      const int j = j0 + tid;
      const uint32_t k = j < first ? weight_key(w[j]) : 0u;
      const bool eq = j < first && k == prefix;
      int n_eq, n_c;
      const int before = move_scan(eq, s_warp, &n_eq);
      const bool c = j < first && (k > prefix || (eq && equal + before < want));
      const int at = move_scan(c, s_warp, &n_c);
      if (c) kept[put + at] = j;
      put += n_c;
      equal += n_eq;
    }
    __syncthreads();
    equal = 0;
    int filled = 0;
    for (int j0 = 0; j0 < m; j0 += kMoveThreads) {
      const int j = j0 + tid;
      const uint32_t k = j < m ? weight_key(w[j]) : 0u;
      const bool eq = j < m && k == prefix;
      int n_eq, n_free;
      const int before = move_scan(eq, s_warp, &n_eq);
      const bool is_free = j < m && !(k > prefix || (eq && equal + before < want));
      const int at = move_scan(is_free, s_warp, &n_free);
      int from = j;
      if (is_free) from = kept[m - moving + filled + at];
      __syncthreads();
      if (j < m) kept[j] = from;
      equal += n_eq;
      filled += n_free;
    }
  }
  for (int r = tid; r < a.recent; r += kMoveThreads) kept[m + r] = first + r;
  __syncthreads();

  // ---- rows.  A row of K (or V) is cpr chunks of 16 bytes; both rows of a position are one warp's work.
  const int nbp = (a.budget + g.P - 1) / g.P;
  const int32_t* old_row = a.v.block_table + (size_t)a.ids[i] * g.max_pages;
  const int32_t* new_row = a.new_row + (size_t)i * nbp;
  const size_t page_chunks = (size_t)g.P * a.cpr;
  uint4* base = a.kv + (size_t)l * g.num_blocks * g.Hkv * 2 * page_chunks + (size_t)h * 2 * page_chunks;
  const size_t block_chunks = (size_t)g.Hkv * 2 * page_chunks;
  const int row_chunks = 2 * a.cpr;
  auto row_at = [&](const int32_t* table, int j) { return base + (size_t)table[j / g.P] * block_chunks + (size_t)(j % g.P) * a.cpr; };
  // chunk c of the row pair (K, then V) of slot j, as stored
  auto place = [&](int j, int c) {
    const int kv = c >= a.cpr;
    const int cc = c - kv * a.cpr;
    return (size_t)kv * page_chunks + (g.swizzle ? ((cc & ~7) | ((cc ^ (j % g.P)) & 7)) : cc);
  };
  // slots [0, m): the sources are slots from m on, or the same slot of a page that was shared; nothing written here is read
  // here
  for (int j = warp; j < m; j += kMoveWarps) {
    const int from = kept[j];
    if (from == j && new_row[j / g.P] == old_row[j / g.P]) continue;
    const uint4* src = row_at(old_row, from);
    uint4* dst = row_at(new_row, j);
    for (int c = lane; c < row_chunks; c += 32) dst[place(j, c)] = src[place(from, c)];
    if (lane == 0) w_out[j] = w[from];
  }
  if (w_out != w)
    for (int j = tid; j < m; j += kMoveThreads)
      if (kept[j] == j) w_out[j] = w[j];
  __syncthreads();
  // the most recent positions, in order: a batch is read whole before it is written (a slot may be the source of an
  // earlier one, never of a later one)
  constexpr int kBatch = 4;
  for (int r0 = 0; r0 < a.recent; r0 += kMoveWarps * kBatch) {
    for (int c0 = 0; c0 < row_chunks; c0 += 32) {
      const int c = c0 + lane;
      uint4 x[kBatch];
      float ww[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int r = r0 + b * kMoveWarps + warp;
        if (r < a.recent && c < row_chunks) x[b] = row_at(old_row, first + r)[place(first + r, c)];
        if (r < a.recent && c == 0) ww[b] = w[first + r];
      }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int r = r0 + b * kMoveWarps + warp;
        if (r < a.recent && c < row_chunks) row_at(new_row, m + r)[place(m + r, c)] = x[b];
        if (r < a.recent && c == 0) w_out[m + r] = ww[b];
      }
      __syncthreads();
    }
  }
  for (int j = a.budget + tid; j < a.stride; j += kMoveThreads) w_out[j] = 0.f;
}

// ---------------------------------------------------------------- bookkeeping
// The (entry, page) pairs of all traces that were cut, in list order and page order, form one sequence; a pair whose page
// is behind the budget, or was replaced by a block of its own, drops one reference.  A block whose count reaches zero is
// pushed on the free list at the place of the last pair that names it, as a serial walk would (see release.cuh).
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kPruneThreads, 1) evict_finish_kernel(EvictArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ int s_warp[33], s_count, s_base;
  DevViews& v = a.v;
  const Geo& g = a.g;
  const int rank = (int)cluster.block_rank(), C = (int)cluster.num_blocks();
  const int nbp = (a.budget + g.P - 1) / g.P;
  wait_for_primary();
  const int E = a.off[a.n];
  const int R = ((E + C - 1) / C + blockDim.x - 1) / blockDim.x * blockDim.x;
  const int lo = min(E, rank * R), hi = min(E, lo + R);
  const int fc = v.counters[C_FREE_COUNT];
  int32_t* slot = nullptr;
  int i = 0, p = 0;
  // pair e: its place in the block table, its block if it drops a reference, else -1
  auto dropped = [&](int e) {
    i = find_list_index(a.off, a.n, e);
    p = e - a.off[i];
    slot = v.block_table + (size_t)a.ids[i] * g.max_pages + p;
    const int b = *slot;
    return p >= nbp || a.new_row[(size_t)i * nbp + p] != b ? b : -1;
  };
  for (int e = lo + threadIdx.x; e < hi; e += blockDim.x) {
    const int b = dropped(e);
    if (b < 0) continue;
    atomicSub(&v.refcount[b], 1);
    atomicMax(&v.claim[b], e);
  }
  __threadfence();
  cluster.sync();
  int pushes = 0;
  for (int e = lo + threadIdx.x; e < hi; e += blockDim.x) {
    const int b = dropped(e);
    pushes += b >= 0 && __ldcg(&v.claim[b]) == e && __ldcg(&v.refcount[b]) == 0;
  }
  int total;
  block_excl_scan(pushes, s_warp, &total);
  if (threadIdx.x == 0) s_count = total;
  cluster.sync();
  if (threadIdx.x == 0) {
    int before = 0, all = 0;
    for (int r = 0; r < C; ++r) {
      const int c = *cluster.map_shared_rank(&s_count, r);
      if (r < rank) before += c;
      all += c;
    }
    s_base = fc + before;
    if (rank == 0) v.counters[C_FREE_COUNT] = fc + all;
  }
  __syncthreads();
  int at_base = s_base;
  for (int base = lo; base < hi; base += blockDim.x) {
    const int e = base + threadIdx.x;
    int b = -1;
    bool own = false, push = false;
    if (e < hi) {
      b = dropped(e);
      if (b >= 0) {
        own = __ldcg(&v.claim[b]) == e;                  // (only its owner clears a claim)
        push = own && __ldcg(&v.refcount[b]) == 0;
        const int fresh = p < nbp ? a.new_row[(size_t)i * nbp + p] : -1;
        *slot = fresh;
        if (fresh >= 0) v.refcount[fresh] = 1;
      }
    }
    int row_total;
    const int at = at_base + block_excl_scan(push ? 1 : 0, s_warp, &row_total);
    if (push) v.free_list[at] = b;
    if (own) v.claim[b] = -1;
    at_base += row_total;
  }
  if (rank == 0)
    for (int k = threadIdx.x; k < a.n; k += blockDim.x)
      if (a.old_len[k] >= 0) v.seq_lens[a.ids[k]] = a.budget;
  cluster.sync();                        // no CTA leaves while its count may still be read
}

bool evict_sizes_ok(const step_pool* pool, int n, int budget) {
  return n >= 0 && n <= pool->cfg.max_traces && n <= kMaxTracesFast && budget >= 1 &&
         budget <= (long long)pool->cfg.max_pages_per_trace * pool->cfg.page_size;
}

}  // namespace

extern "C" {

int kv_pool_evict_workspace_bytes(const step_pool* pool, int n, int budget, size_t* bytes) {
  if (!pool || !bytes || !evict_sizes_ok(pool, n, budget)) return STEP_ERR_INVALID_ARG;
  const size_t nbp = (budget + pool->cfg.page_size - 1) / pool->cfg.page_size;
  *bytes = ((size_t)2 * n + 1 + n * nbp) * sizeof(int32_t);
  return STEP_OK;
}

int kv_pool_evict_positions(step_pool* pool, const int32_t* trace_ids, int n, const float* weights, float* weights_out,
                            int weight_stride, int budget, int recent, int32_t* kept_out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!pool || !evict_sizes_ok(pool, n, budget) || weight_stride < 1 || recent < 0 || recent > budget) return STEP_ERR_INVALID_ARG;
  if (n == 0) return STEP_OK;
  if (!trace_ids || !weights || !weights_out || !kept_out || !workspace || (uintptr_t)workspace & 255) return STEP_ERR_INVALID_ARG;
  if (weight_stride < budget || pool->cfg.num_layers > 65535 || n > 65535) return STEP_ERR_INVALID_ARG;
  size_t need = 0;
  int st = kv_pool_evict_workspace_bytes(pool, n, budget, &need);
  if (st != STEP_OK) return st;
  if (workspace_bytes < need) return STEP_ERR_INVALID_ARG;
  st = on_pool_device(pool);
  if (st != STEP_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  EvictArgs a;
  a.v = pool->v; a.g = geo_of(pool);
  a.kv = (uint4*)pool->cfg.kv_storage;
  a.ids = trace_ids; a.n = n;
  a.weights = weights; a.weights_out = weights_out; a.stride = weight_stride; a.budget = budget; a.recent = recent;
  a.kept = kept_out;
  a.old_len = (int32_t*)workspace; a.off = a.old_len + n; a.new_row = a.off + n + 1;
  a.cpr = a.g.d * pool->elem_bytes / 16;
  evict_plan_kernel<<<1, kPlanThreads, (size_t)n * 2 * sizeof(int), s>>>(a);
  if (launch_ok() != STEP_OK) return STEP_ERR_CUDA;
  if (launch_dependent(evict_move_kernel, dim3(a.g.Hkv, n, a.g.L), dim3(kMoveThreads), 0, s, a) != cudaSuccess) return STEP_ERR_CUDA;
  if (launch_dependent(evict_finish_kernel, dim3(kClusterCtas), dim3(kPruneThreads), 0, s, a) != cudaSuccess) return STEP_ERR_CUDA;
  return launch_ok();
}

}  // extern "C"
