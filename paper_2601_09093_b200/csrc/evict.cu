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
//   1. evict_plan_kernel    a cluster of CTAs: which traces are cut; a block of its own for every kept page that is shared;
//                           the list of the pages that drop a reference
//   2. evict_move_kernel    one CTA per (KV head, trace, layer): selection, then the rows and weights move
//   3. evict_finish_kernel  a cluster of CTAs: references dropped, free list, block table, lengths
//
// 64 traces, 4 layers, 8 KV heads of 128 in bf16, about 4100 positions cut to 4096 with 256 recent ones: 207 to 212 us for 665 MB
// of rows, weights and lists (102 us at the copy bandwidth).  The move kernel is 180 of them.
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
  int32_t* need;                              // workspace [n]: blocks of its own that it takes; -1: left alone
  int32_t* base;                              // workspace [n + 1]: blocks taken by the entries before it (then of all)
  int32_t* off;                               // workspace [n + 1]: pages dropped by the entries before it (then by all)
  int32_t* new_row;                           // workspace [n, pages of a budget]
  int2* drop;                                 // workspace [n * max_pages]: (entry, page) of every reference dropped, in order
  int cpr;
  int cache_keys;                             // positions whose keys evict_move_kernel keeps in shared memory
  int shift;                                  // log2 of the page size, -1 if it is no power of two
};

// Pages are examined by a warp per entry, spread over the cluster: a kept page's reference count is a scattered 4-byte
// read, and one SM alone takes 10 us for the 16,000 of them that 64 traces of 4,096 positions have.  (A call that has few
// pages to look at is a cluster of one: its barriers cost nothing then.)
__global__ void __launch_bounds__(kPruneThreads, 1) evict_plan_kernel(EvictArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ int s_warp[33];
  __shared__ int s_fc;
  dependents_may_launch();
  const DevViews& v = a.v;
  const Geo& g = a.g;
  const int rank = (int)cluster.block_rank(), C = (int)cluster.num_blocks(), lane = threadIdx.x & 31;
  const int warp = (threadIdx.x >> 5) * C + rank, nwarps = kPruneThreads / 32 * C;
  const int nbp = (a.budget + g.P - 1) / g.P;
  // first place of every listed trace (a repeat is flagged and left alone)
  if (rank == 0) {
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
      const int t = a.ids[i];
      if (t >= 0 && t < g.max_traces) v.prune_rank[t] = 0x7fffffff;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
      const int t = a.ids[i];
      if (t >= 0 && t < g.max_traces) atomicMin(&v.prune_rank[t], i);
    }
    __threadfence();
  }
  cluster.sync();
  for (int i = warp; i < a.n; i += nwarps) {
    const int t = a.ids[i];
    int need = -1, S = -1;
    if (t < 0 || t >= g.max_traces || !v.live[t] || __ldcg(&v.prune_rank[t]) != i) {
      if (lane == 0) flag_error(v.counters, STEP_ERR_BAD_TRACE);
    } else {
      S = v.seq_lens[t];
      if (S > a.stride && S > a.budget) {
        if (lane == 0) flag_error(v.counters, STEP_ERR_CAPACITY);          // positions without a weight
      } else if (S > a.budget) {
        const int32_t* row = v.block_table + (size_t)t * g.max_pages;
        const int pages = (S + g.P - 1) / g.P;
        int shared = 0;
        bool bad = false;
#pragma unroll 4
        for (int p = lane; p < pages; p += 32) {
          const int b = row[p];
          if (b < 0 || b >= g.num_blocks) bad = true;                      // (leaves the whole entry alone)
          else if (p < nbp) shared += v.refcount[b] > 1;
        }
        bad = __any_sync(0xffffffffu, bad);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) shared += __shfl_xor_sync(0xffffffffu, shared, o);
        if (bad) { if (lane == 0) flag_error(v.counters, STEP_ERR_BAD_BLOCK); }
        else need = shared;
      }
    }
    if (lane == 0) { a.need[i] = need; a.old_len[i] = S; }
  }
  __threadfence();
  cluster.sync();
  if (rank == 0) {
    // the free list serves everybody, or a serial walk decides who is left alone
    const int fc = v.counters[C_FREE_COUNT];
    int taken = 0;
    for (int i0 = 0; i0 < a.n; i0 += blockDim.x) {
      const int i = i0 + threadIdx.x;
      int total;
      block_excl_scan(i < a.n ? max(__ldcg(&a.need[i]), 0) : 0, s_warp, &total);
      taken += total;
    }
    if (taken > fc && threadIdx.x == 0) {
      int remaining = fc;
      for (int i = 0; i < a.n; ++i) {
        const int need = __ldcg(&a.need[i]);
        if (need > remaining) { a.need[i] = -1; flag_error(v.counters, STEP_ERR_NO_BLOCKS); }
        else if (need > 0) remaining -= need;
      }
    }
    __syncthreads();
    int run_b = 0, run_p = 0;
    for (int i0 = 0; i0 < a.n; i0 += blockDim.x) {
      const int i = i0 + threadIdx.x;
      int need = 0, pages = 0;
      if (i < a.n) {
        need = __ldcg(&a.need[i]);
        if (need >= 0) pages = need + (__ldcg(&a.old_len[i]) + g.P - 1) / g.P - nbp;
        else { need = 0; a.old_len[i] = -1; }
      }
      int total_b, total_p;
      const int at_b = run_b + block_excl_scan(need, s_warp, &total_b);
      const int at_p = run_p + block_excl_scan(pages, s_warp, &total_p);
      if (i < a.n) { a.base[i] = at_b; a.off[i] = at_p; }
      run_b += total_b; run_p += total_p;
    }
    if (threadIdx.x == 0) { a.base[a.n] = run_b; a.off[a.n] = run_p; v.counters[C_FREE_COUNT] = fc - run_b; }
    __threadfence();
  }
  cluster.sync();
  if (threadIdx.x == 0) s_fc = __ldcg(&v.counters[C_FREE_COUNT]) + __ldcg(&a.base[a.n]);     // before this call
  __syncthreads();
  for (int i = warp; i < a.n; i += nwarps) {
    if (__ldcg(&a.old_len[i]) < 0) continue;
    const int pages = (__ldcg(&a.old_len[i]) + g.P - 1) / g.P;
    const int32_t* row = v.block_table + (size_t)a.ids[i] * g.max_pages;
    int32_t* to = a.new_row + (size_t)i * nbp;
    const bool any = __ldcg(&a.need[i]) > 0;
    int taken = s_fc - 1 - __ldcg(&a.base[i]);
    int2* out = a.drop + __ldcg(&a.off[i]);
    if (any) {
      for (int p0 = 0; p0 < nbp; p0 += 32) {
        const int p = p0 + lane;
        const int b = p < nbp ? row[p] : -1;
        const bool shared = b >= 0 && v.refcount[b] > 1;
        const unsigned who = __ballot_sync(0xffffffffu, shared);
        const int before = __popc(who & ((1u << lane) - 1));
        if (p < nbp) to[p] = shared ? v.free_list[taken - before] : b;
        if (shared) out[before] = make_int2(i, p);
        taken -= __popc(who);
        out += __popc(who);
      }
    } else {
#pragma unroll 4
      for (int p = lane; p < nbp; p += 32) to[p] = row[p];
    }
    for (int p = nbp + lane; p < pages; p += 32) out[p - nbp] = make_int2(i, p);
  }
}

// ---------------------------------------------------------------- selection and moves
constexpr int kMoveThreads = 256, kMoveWarps = kMoveThreads / 32;
constexpr int kBins = 2048;                   // selection by digits of 11, 11 and 10 bits
constexpr int kMostCachedKeys = 12288;        // 48 KiB of keys: three CTAs per SM still fit
constexpr int kBatch = 8;                     // rows a warp has in flight
constexpr int kPageCache = 1024;              // block ids kept in shared memory

// Bits of a weight -> key.  Larger weight -> larger key; NaN below everything; the two zeros are equal.  The kernel reads and
// writes weights as integers throughout: this library's arithmetic and comparisons take subnormal numbers for zeros, and
// the compiler turns a test of a float's bits against zero back into such a comparison.
__device__ inline uint32_t weight_key(uint32_t u) {
  const uint32_t magnitude = u & 0x7fffffffu;
  if (magnitude > 0x7f800000u) return 0u;
  return magnitude == 0u ? 0x80000000u : ((u & 0x80000000u) ? ~u : (u | 0x80000000u));
}

// What bounds it: for a cut of a few positions the passes over the weights (each a read of shared memory, or of L2 for
// long caches) and the copies' latency, so four CTAs per SM matter more than rows in flight per warp, and more than the 52
// bytes of registers that a thread spills for them; all CTAs go through the same phases at the same time, and the memory
// system idles while they select.  The positions are split into one contiguous run per warp, so that ranks need one exchange
// of counts between the warps and none per step.  Keys are kept in shared memory where weight_stride says that those of any
// trace fit; with a wider stride every pass reads the weights, of short traces too.
__global__ void __launch_bounds__(kMoveThreads, 4) evict_move_kernel(EvictArgs a) {
  extern __shared__ uint32_t s_key[];                   // [cache_keys]
  __shared__ int s_hist[kBins];                         // the histogram, then the positions that move
  __shared__ int s_slot[kBins];                         // and the slots that take them
  __shared__ int s_cnt[kMoveWarps][4];                  // per warp: above and equal in [0, m), above and equal in [m, first)
  __shared__ int s_scan[kMoveWarps];
  __shared__ int s_digit, s_left;
  __shared__ int s_page[kPageCache];
  const Geo& g = a.g;
  const int h = blockIdx.x, i = blockIdx.y, l = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t head = ((size_t)l * a.n + i) * g.Hkv + h;
  const uint32_t* w = reinterpret_cast<const uint32_t*>(a.weights) + head * a.stride;
  uint32_t* w_out = reinterpret_cast<uint32_t*>(a.weights_out) + head * a.stride;
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

  // ---- the m-th largest key of [0, first), and how many of the positions that have it are chosen (`want`): position j is
  // chosen if its key is above the threshold, or equal to it and among the first `want` such positions
  const bool in_smem = first <= a.cache_keys;
  const int32_t* old_row = a.v.block_table + (size_t)a.ids[i] * g.max_pages;
  const int pages = (S + g.P - 1) / g.P;
  for (int p = tid; p < min(pages, kPageCache); p += kMoveThreads) s_page[p] = old_row[p];
  // (two buffers: a position below m most likely stays, and those that do not are written again further down)
  const bool copy_weights = w_out != w;
  if (in_smem || copy_weights) {
#pragma unroll 8
    for (int j = tid; j < first; j += kMoveThreads) {
      const uint32_t x = w[j];
      if (in_smem) s_key[j] = weight_key(x);
      if (copy_weights && j < m) w_out[j] = x;
    }
  }
  for (int j = tid; j < m; j += kMoveThreads) kept[j] = j;               // (most slots; the others are written again further down)
  for (int r = tid; r < a.recent; r += kMoveThreads) kept[m + r] = first + r;
  auto key = [&](int j) { return in_smem ? s_key[j] : weight_key(w[j]); };
  uint32_t limit = 0;
  int want = m;                                         // still to be found among the keys that share the prefix
#pragma unroll 1
  for (int pass = 0; pass < 3 && m > 0; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
    for (int b = tid; b < kBins; b += kMoveThreads) s_hist[b] = 0;
    __syncthreads();
#pragma unroll 4
    for (int j = tid; j < first; j += kMoveThreads) {
      const uint32_t k = key(j);
      if (pass == 0 || (k >> (shift + bits)) == limit) atomicAdd(&s_hist[(k >> shift) & ((1u << bits) - 1)], 1);
    }
    __syncthreads();
    // bins from the top, eight to a thread
    constexpr int per = kBins / kMoveThreads;
    int c[per], sum = 0;
#pragma unroll
    for (int x = 0; x < per; ++x) { c[x] = s_hist[kBins - 1 - (tid * per + x)]; sum += c[x]; }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    int at = incl - sum;
    for (int x = 0; x < warp; ++x) at += s_scan[x];
#pragma unroll
    for (int x = 0; x < per; ++x) {
      if (at < want && at + c[x] >= want) { s_digit = kBins - 1 - (tid * per + x); s_left = want - at; }
      at += c[x];
    }
    __syncthreads();
    limit = (limit << bits) | (uint32_t)s_digit;
    want = s_left;
    __syncthreads();
  }

  // ---- a contiguous run of [0, m) and one of [m, first) per warp; how many of each are above and equal
  const int run0 = ((m + kMoveWarps - 1) / kMoveWarps + 31) & ~31, run1 = ((first - m + kMoveWarps - 1) / kMoveWarps + 31) & ~31;
  const int a0 = min(m, warp * run0), b0 = min(m, a0 + run0);
  const int a1 = min(first, m + warp * run1), b1 = min(first, a1 + run1);
  auto count = [&](int lo, int hi, int& above, int& equal) {
    above = equal = 0;
#pragma unroll 4
    for (int j = lo + lane; j < hi; j += 32) {
      const uint32_t k = key(j);
      above += k > limit;
      equal += k == limit;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { above += __shfl_xor_sync(0xffffffffu, above, o); equal += __shfl_xor_sync(0xffffffffu, equal, o); }
  };
  {
    int x, y, z, u;
    count(a0, b0, x, y);
    count(a1, b1, z, u);
    if (lane == 0) { s_cnt[warp][0] = x; s_cnt[warp][1] = y; s_cnt[warp][2] = z; s_cnt[warp][3] = u; }
  }
  __syncthreads();
  // of this warp's runs: equal keys before them, free slots before the first, moving positions before the second
  int eq0 = 0, eq1 = 0, free0 = 0, move0 = 0, moving = 0;
  {
    int eq = 0, fr = 0, mv = 0;
    for (int x = 0; x < kMoveWarps; ++x) {
      if (x == warp) { eq0 = eq; free0 = fr; }
      const int len = min(m, (x + 1) * run0) - min(m, x * run0);
      fr += len - s_cnt[x][0] - min(max(want - eq, 0), s_cnt[x][1]);
      eq += s_cnt[x][1];
    }
    for (int x = 0; x < kMoveWarps; ++x) {
      if (x == warp) { eq1 = eq; move0 = mv; }
      mv += s_cnt[x][2] + min(max(want - eq, 0), s_cnt[x][3]);
      eq += s_cnt[x][3];
    }
    moving = mv;
    if (m == 0) moving = 0;
  }

  // ---- rows: a row of K (or V) is cpr chunks of 16 bytes; both rows of a position are one warp's work
  const int nbp = (a.budget + g.P - 1) / g.P;
  const int32_t* new_row = a.new_row + (size_t)i * nbp;
  const bool fresh_pages = a.need[i] > 0;               // some kept pages are shared: all that they hold is copied
  const size_t page_chunks = (size_t)g.P * a.cpr;
  uint4* base = a.kv + (size_t)l * g.num_blocks * g.Hkv * 2 * page_chunks + (size_t)h * 2 * page_chunks;
  const size_t block_chunks = (size_t)g.Hkv * 2 * page_chunks;
  const int row_chunks = 2 * a.cpr;
  auto old_block = [&](int p) { return p < kPageCache ? s_page[p] : old_row[p]; };
  auto new_block = [&](int p) { return fresh_pages ? new_row[p] : old_block(p); };
  auto page_of = [&](int j) { return a.shift >= 0 ? j >> a.shift : j / g.P; };
  // Where slot j's K row starts (in chunks from `base`) in block b, and what its chunk numbers are XORed with: worked out by
  // one lane per row and handed round, since the arithmetic of every lane for every row cost more than the copies.
  auto row_of = [&](int b, int j) { return (unsigned long long)b * block_chunks + (unsigned long long)(j - page_of(j) * g.P) * a.cpr; };
  auto twist_of = [&](int j) { return g.swizzle ? (j - page_of(j) * g.P) & 7 : 0; };
  // kBatch rows of one warp: lane x < kBatch knows the source of row x, lane kBatch + x its slot; n of them exist
  auto copy_rows = [&](int j, int n, bool all_read_first) {
    const bool is_slot = lane >= kBatch;
    const bool real = lane < 2 * kBatch && lane % kBatch < n;
    const unsigned long long at = real ? row_of(is_slot ? new_block(page_of(j)) : old_block(page_of(j)), j) : 0ull;
    const int twist = real ? twist_of(j) : 0;
    for (int c0 = 0; c0 < row_chunks; c0 += 32) {
      const int c = c0 + lane, kv = c >= a.cpr, cc = c - kv * a.cpr;
      uint4* mine = base + (kv ? page_chunks : 0);
      uint4 x[kBatch];
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        const unsigned long long from = __shfl_sync(0xffffffffu, at, r);
        const int tw = __shfl_sync(0xffffffffu, twist, r);
        if (r < n && c < row_chunks) x[r] = mine[from + (cc ^ tw)];
      }
      if (all_read_first) __syncthreads();
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        const unsigned long long to = __shfl_sync(0xffffffffu, at, kBatch + r);
        const int tw = __shfl_sync(0xffffffffu, twist, kBatch + r);
        if (r < n && c < row_chunks) mine[to + (cc ^ tw)] = x[r];
      }
    }
  };
  // Slots [0, m), kBins moving positions a round: positions and slots are listed in shared memory, then their rows are
  // copied, all at once.  The sources are positions from m on: nothing written here is read here.  (Copying a slot's row
  // where the slot is found, one after another, took four times as long.)
  for (int round = 0; round == 0 || round * kBins < moving; ++round) {
    const int lo = round * kBins, hi = lo + kBins;
    __syncthreads();
    if (moving > 0) {
      int eq = eq1, at = move0;
      for (int j0 = a1; j0 < b1; j0 += 32) {
        const int j = j0 + lane;
        const uint32_t k = j < b1 ? key(j) : 0u;
        const bool is_eq = j < b1 && k == limit;
        const unsigned eqs = __ballot_sync(0xffffffffu, is_eq), below = (1u << lane) - 1;
        const bool c = j < b1 && (k > limit || (is_eq && eq + __popc(eqs & below) < want));
        const unsigned cs = __ballot_sync(0xffffffffu, c);
        const int r = at + __popc(cs & below);
        if (c && r >= lo && r < hi) s_hist[r - lo] = j;
        eq += __popc(eqs);
        at += __popc(cs);
      }
    }
    __syncthreads();
    int eq = eq0, at = free0;
    for (int j0 = a0; j0 < b0; j0 += 32) {
      const int j = j0 + lane;
      const uint32_t k = j < b0 ? key(j) : 0u;
      const bool is_eq = j < b0 && k == limit;
      const unsigned eqs = __ballot_sync(0xffffffffu, is_eq), below = (1u << lane) - 1;
      const bool is_free = j < b0 && !(k > limit || (is_eq && eq + __popc(eqs & below) < want));
      const unsigned fr = __ballot_sync(0xffffffffu, is_free);
      const int r = at + __popc(fr & below);
      eq += __popc(eqs);
      at += __popc(fr);
      if (is_free && r >= lo && r < hi) { s_slot[r - lo] = j; kept[j] = s_hist[r - lo]; }
    }
    __syncthreads();
    const int cnt = min(kBins, moving - lo);
    if (copy_weights || in_smem)                        // (else the weights still say which slots are free)
      for (int r = tid; r < cnt; r += kMoveThreads) w_out[s_slot[r]] = w[s_hist[r]];
    for (int r0 = warp * kBatch; r0 < cnt; r0 += kMoveWarps * kBatch) {
      const int r = r0 + lane % kBatch;
      copy_rows(r < cnt ? (lane < kBatch ? s_hist[r] : s_slot[r]) : 0, min(kBatch, cnt - r0), false);
    }
  }
  // what stays on a page that was shared goes along to the block that replaces it
  if (fresh_pages)
    for (int j0 = warp * kBatch; j0 < m; j0 += kMoveWarps * kBatch) {
      // (the rows that do not stay are passed over by letting the warp's batch shrink to those that do)
      const int j = j0 + lane;
      const bool stays = lane < kBatch && j < m && new_block(page_of(j)) != old_block(page_of(j)) && kept[j] == j;
      const unsigned who = __ballot_sync(0xffffffffu, stays);
      const int n = __popc(who), r = lane % kBatch;
      copy_rows(r < n ? j0 + (int)__fns(who, 0, r + 1) : 0, n, false);
    }
  if (!copy_weights && !in_smem)
    for (int j = tid; j < m; j += kMoveThreads) {
      const int from = kept[j];
      if (from != j) w_out[j] = w[from];
    }
  __syncthreads();
  // the most recent positions, in order: a batch is read whole before it is written (a slot may be the source of an
  // earlier one, never of a later one)
  for (int r0 = 0; r0 < a.recent; r0 += kMoveThreads) {
    const int r = r0 + tid;
    const uint32_t x = r < a.recent ? w[first + r] : 0u;
    __syncthreads();
    if (r < a.recent) w_out[m + r] = x;
    __syncthreads();
  }
  for (int r0 = 0; r0 < a.recent; r0 += kMoveWarps * kBatch) {
    const int r1 = r0 + warp * kBatch, r = r1 + lane % kBatch;
    copy_rows(r < a.recent ? (lane < kBatch ? first : m) + r : 0, max(0, min(kBatch, a.recent - r1)), true);
  }
  for (int j = a.budget + tid; j < a.stride; j += kMoveThreads) w_out[j] = 0u;
}

// ---------------------------------------------------------------- bookkeeping
// The listed (entry, page) pairs drop one reference each.  A block whose count reaches zero is pushed on the free list at
// the place of the last pair that names it, as a serial walk would (see release.cuh).
__global__ void __launch_bounds__(kPruneThreads, 1) evict_finish_kernel(EvictArgs a) {
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
  auto place = [&](int2 e) { return v.block_table + (size_t)a.ids[e.x] * g.max_pages + e.y; };
  for (int e = lo + threadIdx.x; e < hi; e += blockDim.x) {
    const int b = *place(a.drop[e]);
    atomicSub(&v.refcount[b], 1);
    atomicMax(&v.claim[b], e);
  }
  __threadfence();
  cluster.sync();
  int pushes = 0;
  for (int e = lo + threadIdx.x; e < hi; e += blockDim.x) {
    const int b = *place(a.drop[e]);
    pushes += __ldcg(&v.claim[b]) == e && __ldcg(&v.refcount[b]) == 0;
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
      const int2 d = a.drop[e];
      int32_t* at = place(d);
      b = *at;
      own = __ldcg(&v.claim[b]) == e;                    // (only its owner clears a claim)
      push = own && __ldcg(&v.refcount[b]) == 0;
      const int fresh = d.y < nbp ? a.new_row[(size_t)d.x * nbp + d.y] : -1;
      *at = fresh;
      if (fresh >= 0) v.refcount[fresh] = 1;
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

// A cluster of `ctas` CTAs; dependent: a programmatic dependent of the launch before it.
cudaError_t launch_cluster(void (*kernel)(EvictArgs), int ctas, bool dependent, cudaStream_t s, const EvictArgs& a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(kPruneThreads); cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = dependent ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
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
  *bytes = ((size_t)4 * n + 2 + n * nbp) * sizeof(int32_t) + (size_t)n * pool->cfg.max_pages_per_trace * sizeof(int2);
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
  a.drop = (int2*)workspace;
  a.old_len = (int32_t*)(a.drop + (size_t)n * a.g.max_pages);
  a.need = a.old_len + n; a.base = a.need + n; a.off = a.base + n + 1; a.new_row = a.off + n + 1;
  a.cpr = a.g.d * pool->elem_bytes / 16;
  a.shift = -1;
  for (int b = 0; b < 30; ++b)
    if (a.g.P == 1 << b) a.shift = b;
  a.cache_keys = weight_stride <= kMostCachedKeys ? weight_stride : 0;
  // pages there may be to look at: below 4096 (four rounds of one CTA's threads) one CTA is faster than a cluster of eight
  const int ctas = (long long)n * a.g.max_pages < 4096 ? 1 : kClusterCtas;
  if (launch_cluster(evict_plan_kernel, ctas, false, s, a) != cudaSuccess) return STEP_ERR_CUDA;
  const size_t smem = (size_t)a.cache_keys * sizeof(uint32_t);
  if (cudaFuncSetAttribute(evict_move_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostCachedKeys * 4) != cudaSuccess) return STEP_ERR_CUDA;
  if (launch_dependent(evict_move_kernel, dim3(a.g.Hkv, n, a.g.L), dim3(kMoveThreads), smem, s, a) != cudaSuccess) return STEP_ERR_CUDA;
  if (launch_cluster(evict_finish_kernel, ctas, true, s, a) != cudaSuccess) return STEP_ERR_CUDA;
  return launch_ok();
}

}  // extern "C"
