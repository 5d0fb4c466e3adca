// Tensor-core form of decode_attention_groups (bf16 pools, head_dim 128, page 16).
//
// A trace's keys are the pages it shares with its group and the pages of its own.  Both kinds leave partial results
//   m = max_j s_j,  l = sum_j 2^(s_j - m),  o = sum_j 2^(s_j - m) v_j          (s in units of log 2)
// which a last kernel combines.
//
// groups_kernel works on both kinds at once, on different SMs: the shared pages are bound by the tensor cores and the
// exponentials, the own pages by HBM, and the SMs that read own pages get the more of its bandwidth the fewer they are.  Every
// CTA works out for itself who shares what (from the lengths and the groups' arrays) and how many CTAs each kind gets; the first
// leaves the outcome in the workspace for groups_merge_kernel, a programmatic dependent.
//   Own pages: the pages of all (row, KV head) sequences form one stream, cut into one equal contiguous share per warp; a warp
//   streams its share through a private ring of three pages (8 KiB, K and V rows of one head, 16 asynchronous copies of 16
//   bytes a lane: one bulk copy took the warp 450 cycles of a page's 1,750) and runs both products on 16 x 8 x 16 tiles, the G
//   heads of the group as rows: with so few rows a 128-row tensor-core tile would be nearly empty, and beginning a sequence
//   costs such a kernel four tiles' time, more than a trace's own text often has.
//   Shared pages: the query rows of a group's traces - (trace, head of the KV head's group) - are taken 256 at a time against
//   one read of the keys, as decode_attention_tree does with a trace's drafted tokens: scores by tcgen05 into tensor memory, a
//   thread per row for the softmax, probabilities as two bf16 numbers each over the scores, from where they are the second
//   product's A operand.  Two chains ("lanes") run side by side: 128 rows each of the same tile of 128 keys, or, where a row block has
//   at most 128 rows, even and odd tiles of the same rows.  The tiles of all (group, KV head, row block) sequences form one
//   stream, cut into one equal share per CTA.
//
// 64 traces of a prompt of 32,768 with own texts of up to 1,024, 32 / 8 heads: 73.5 us, 270 MB (41 us at the measured copy rate) and
// 35 GFLOP; 81 to 84 after half a second of nothing else, at the card's power limit.  (With one bf16 number for a probability 70 and 73;
// as two kernels in a row 104.)  8 prompts of 1,000 to 16,000 with 12 traces each and own texts of up to 3,000, 64 / 8 heads: 131 to
// 142 us, 0.78 to 0.84 of the measured copy.
//
// The partition is a function of lengths and groups alone and pieces are combined in stream order, so a call gives the same
// bits every time.  Every wait for a barrier is bounded (kv_pool_set_wait_limit_ns); a CTA whose wait runs out raises
// STEP_ERR_TIMEOUT and leaves when its copies and products in flight have ended.
#include "attention_tc.cuh"

#include <string.h>

using namespace stepk;

namespace {

constexpr int kSetup = 2;                         // tiles' worth of time that a sequence of shared pages takes besides its tiles
constexpr int kKSlots = 2, kVSlots = 3, kSlots = kKSlots + kVSlots;   // rings of K and of V tiles, 160 KiB: a V tile waits for its softmax
constexpr int kWarpK = 8, kWarpMma = 9, kWarpQ = 10, kWarpV = 11;
constexpr int kThreads = 384;                     // three warpgroups
constexpr int kRegsSoftmax = 208, kRegsOther = 88; // 2 x 128 x 208 + 128 x 88 = 384 x 168, what the launch has
constexpr int kTmemCols = 512;                    // S of both lanes (P over them), then O of both
constexpr float kRescale = 8.f;                   // log2 of how far a row's maximum may run ahead of its reference
constexpr unsigned long long kDrainNs = 100000000ull;

constexpr int kStreamWarps = 8, kStages = 3, kPageBytes = 2 * kP * kD * 2;

constexpr int kTableGroups = 48;                  // groups whose table fits beside the rings; a longer one lies in the workspace
// What a CTA takes, in nanoseconds (measured, 32 / 8 and 64 / 8 heads): a tile of shared pages with more than 128 rows (its products
// and exponentials) and with fewer (1.0 alone, the latency of its copies when all SMs read); a page of a warp's own; what comes
// before and behind them.  (A tile of both lanes alone takes 2.4 to 2.6 us, 2.8 at the card's power limit.  64 traces of 32,768 in turn with
// others: 76.7 us at 2150, 74.8 at 2600, 73.4 at 2800; a decode step of 2 x 32 traces of 8192, four layers: 349 at 1600, 337 at 1800, 331
// at 2000; 8 x 12 traces 133.5, 135 and 137.7.)
constexpr int kWideNs = 2800, kNarrowNs = 2000, kPageNs = 1050, kPrefixNs = 9000, kOwnNs = 5000;
constexpr int kOwnSetup = 2;                      // pages' worth of time that a sequence of own pages takes besides them

// Tiles in the prefix stream, own pages (of all KV heads; setups counted in both), CTAs that take shared pages (the others take own
// pages).
struct Header { int units, pages, n_prefix; };

// What a row's result is combined from.
struct RowPlan {                     // (positions in both streams fit 32 bits: groups_tc_supported)
  int at;                           // where the row's own pages begin in their stream, KV head 0: Hkv times this
  int begin;                        // where the tiles of the row's block of its group begin in the prefix stream, KV head 0
  int pages, tiles;                 // own pages; tiles it shares (0: none)
  int head;                         // from one KV head's tiles to the next's
  int place;                        // of its heads in the block: trace * 2 + 1 if the block has results of two lanes for a row
};

struct GroupArgs {
  const __nv_bfloat16* kv; const __nv_bfloat16* q; __nv_bfloat16* out;
  const int32_t* block_table; const int32_t* seq_lens; const int32_t* group_rows; const int32_t* group_pages;
  int32_t* counters;
  int n, n_groups, Hq, Hkv, G, layer, max_pages, num_blocks;
  int tokens;                       // traces whose heads fill a tile of query rows: 128 / G
  int box;                          // traces of one copy of query rows
  int ctas;
  float scale_log2;
  unsigned long long wait_ns;
  // workspace
  Header* header;
  RowPlan* plan;                    // [n]
  int4* cta_groups;                 // [ctas][n_groups] the groups as every CTA finds them for itself (more than kTableGroups)
  int* cta_group_at;
  float *pre_ml, *pre_o;            // [CTA][2][lane][128] (m, l) and o of the prefix pieces that are not whole sequences
  float *row_ml, *row_o;            // [lane][n][Hq] of those that are
  float *own_ml, *own_o;            // [warp][2][G] of the own pages' pieces that are not whole sequences
  float *all_ml, *all_o;            // [n][Hq] of those that are, where there are shared pages besides
};

// A probability enters the second product, whose V is bf16, as two bf16 numbers: hi = p cut off behind the bits that bf16 holds, and
// lo = p kScale - hi, rounded to nearest; sums of probabilities are multiplied by kScale in the end.  lo is at most (2^-7 + 2^-10) p, so
// that hi + lo is off by at most 2^-8 of that, 3.5e-5 of p, where the output's own rounding is up to 3.9e-3; one rounded bf16 number
// made the output's error 2.3e-3 instead of 1.7e-3 in the 2-norm.  kScale makes lo positive (where p is above 2^-116): an infinity
// in V keeps its sign in both products and their sum.  64 traces of a prompt of 32,768, SMs shared out as for one number: 68.5 us with one
// number, 74.5 with two; with hi rounded to nearest 75.6, with packed arithmetic (fma.f32x2, whose operands have to be moved together) 79.5.
constexpr float kScale = 1.f + 0x1p-10f;
__device__ inline void split2(float p0, float p1, uint32_t& hi, uint32_t& lo) {
  hi = __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
  p0 = fmaf(p0, kScale, -__uint_as_float(__float_as_uint(p0) & 0xffff0000u));
  p1 = fmaf(p1, kScale, -__uint_as_float(__float_as_uint(p1) & 0xffff0000u));
  lo = pack2(p0, p1);
}

__device__ inline int div_up(int x, int by) { return (int)(((unsigned)x + (unsigned)by - 1) / (unsigned)by); }

// One warp: how many CTAs take shared pages, so that the slower kind of CTA is as fast as can be.  (Around the ratio of the work,
// a candidate per lane: with few tiles a share is a whole number of them.)
__device__ inline int choose_prefix(const GroupArgs& a, int units, float unit_ns, int pages, int lane) {
  if (units == 0 || pages == 0) return units == 0 ? 0 : a.ctas;
  const float ratio = (float)units * unit_ns / ((float)units * unit_ns + (float)pages * (kPageNs / (float)kStreamWarps));
  const int at = (int)(ratio * a.ctas) - 12 + lane;
  float t = INFINITY;
  if (at >= 1 && at < a.ctas)
    t = fmaxf(kPrefixNs + (float)div_up(units, at) * unit_ns, kOwnNs + (float)div_up(pages, (a.ctas - at) * kStreamWarps) * kPageNs);
  float best = t;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = fminf(best, __shfl_xor_sync(0xffffffffu, best, o));
  return __shfl_sync(0xffffffffu, at, __ffs(__ballot_sync(0xffffffffu, t == best)) - 1);
}
__device__ inline int prefix_share(const Header& h, int ctas) { return div_up(h.units, ctas); }
__device__ inline int own_share(const Header& h, int ctas) { return div_up(h.pages, ctas * kStreamWarps); }

__device__ inline int length_of(const GroupArgs& a, int i, bool flag) {
  int S = a.seq_lens[i];
  if (S < 0) S = 0;
  if ((long long)S > (long long)a.max_pages * kP) { S = a.max_pages * kP; if (flag) flag_error(a.counters, STEP_ERR_CAPACITY); }
  return S;
}

// ---- the prefix stream: for every group that shares pages, for every KV head, for every block of 2 * tokens traces
struct Shape { int tiles, blocks; };
__device__ inline Shape shape_of(const GroupArgs& a, int4 g) {
  Shape x;
  x.tiles = (g.w + kTile / kP - 1) / (kTile / kP);
  x.blocks = (g.y + 2 * a.tokens - 1) / (2 * a.tokens);
  return x;
}

// ---------------------------------------------------------------- own pages
__device__ inline void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ inline void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ inline void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ inline void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ inline void mma16816(float (&c)[4], const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

constexpr size_t kRing = (size_t)kStreamWarps * kStages * kPageBytes;                      // rings of own pages
constexpr size_t kStreamSmem = 1024 + kRing + (kMaxTracesFast + 2) * 4 + 2 * kMaxTracesFast * 4;

// What every CTA works out first, in shared memory behind the rings of own pages.
struct Rows {
  int* at;                          // [n + 1] own pages of the rows before, setups counted
  int* own;                         // [n] pages that the row shares
  int* len;                         // [n] its length, at most what the table holds
};

// One warp's share of the own pages: the me-th W positions of `total`.
__device__ __forceinline__ void own_pages(const GroupArgs& a, const Rows& rw, unsigned char* sm, uint32_t base, int me, int total, int W) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int begin = (int)min((long long)total, (long long)me * W), end = min(total - begin, W) + begin;
  if (begin >= end) return;
  // the sequence that holds a position of the stream
  struct Seq { int row, h, pages, own, at; };                          // at: where it begins
  auto of_row = [&](Seq& s) { s.pages = rw.at[s.row + 1] - rw.at[s.row] - kOwnSetup; s.own = rw.own[s.row]; };
  auto row_behind = [&](int row) {                                     // that has pages
    do ++row; while (row < a.n && rw.at[row + 1] == rw.at[row]);
    return row;
  };
  auto seq_at = [&](int pos) {
    int lo = 0, hi = a.n - 1;                                          // the last row that begins at or before pos: it has pages
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (rw.at[mid] * a.Hkv <= pos) lo = mid; else hi = mid - 1;
    }
    Seq s;
    s.row = lo;
    of_row(s);
    const int off = pos - rw.at[lo] * a.Hkv, each = s.pages + kOwnSetup;
    s.h = (int)((unsigned)off / (unsigned)each);
    s.at = pos - off + s.h * each;
    return s;
  };
  auto next_seq = [&](Seq s) {
    s.at += s.pages + kOwnSetup;
    if (++s.h < a.Hkv) return s;
    s.h = 0;
    s.row = row_behind(s.row);
    if (s.row < a.n) of_row(s);
    return s;
  };
  // pages [first, last) of sequence s are in this share
  auto first_of = [&](const Seq& s) { return max(0, begin - s.at - kOwnSetup); };
  auto last_of = [&](const Seq& s) { return min(s.pages, max(0, end - s.at - kOwnSetup)); };

  // ---- the copies: up to kStages pages ahead.  Lane i holds the blocks of pages win + i of the sequence; those of the window
  // behind are asked for when a window is entered, those of the next row when a row is: a read of the table takes a page's time.
  const uint32_t ring = base + warp * kStages * kPageBytes;
  auto load_ids = [&](int row, int w) {
    if (row >= a.n) return 0;
    const int own = rw.own[row], pages = rw.at[row + 1] - rw.at[row] - kOwnSetup;
    return w + lane < pages ? a.block_table[(size_t)row * a.max_pages + own + w + lane] : 0;
  };
  // the next piece's query rows on their way to the L1
  auto prefetch_q = [&](const Seq& s) {
    if (s.row < a.n && s.at < end && lane < 2 * a.G)
      asm volatile("prefetch.global.L1 [%0];" ::"l"(a.q + ((size_t)s.row * a.Hq + (size_t)s.h * a.G) * kD + lane * 64));
  };
  Seq s = seq_at(begin), ps = s;
  int page = first_of(s), plast = last_of(s), win = page, put = 0;
  int ids = load_ids(s.row, win), ids_next = load_ids(s.row, win + 32), ids_row = win == 0 ? ids : load_ids(s.row, 0);
  int behind = row_behind(s.row), ids_behind = load_ids(behind, 0);
  bool any = page < plast;                                             // pages are left to copy
  prefetch_q(next_seq(s));
  auto issue = [&]() {
    if (!any) {
      cp_async_commit();                                               // (an empty group: the wait counts groups)
      return;
    }
    if (page - win >= 32) { win += 32; ids = ids_next; ids_next = load_ids(ps.row, win + 32); }
    int b = __shfl_sync(0xffffffffu, ids, page - win);
    if (b < 0 || b >= a.num_blocks) { if (lane == 0) flag_error(a.counters, STEP_ERR_BAD_BLOCK); b = 0; }
    const __nv_bfloat16* src = a.kv + (((size_t)a.layer * a.num_blocks + b) * a.Hkv + ps.h) * (2 * kP * kD) + lane * 8;
    const uint32_t dst = ring + put * kPageBytes + lane * 16;
#pragma unroll
    for (int x = 0; x < kPageBytes / 512; ++x) cp_async16(dst + x * 512, src + x * 256);
    cp_async_commit();
    if (++put == kStages) put = 0;
    if (++page < plast) return;
    const int row = ps.row;
    ps = next_seq(ps);
    any = ps.row < a.n && ps.at + kOwnSetup < end;
    if (!any) return;
    page = win = 0;
    plast = last_of(ps);
    if (ps.row != row) { ids_row = ids_behind; behind = row_behind(behind); ids_behind = load_ids(behind, 0); }
    ids = ids_row;
    ids_next = load_ids(ps.row, 32);
  };
  for (int x = 0; x < kStages; ++x) issue();

  const int gr = lane >> 2, tq = lane & 3;                             // rows gr, gr + 8 and columns 2 tq, 2 tq + 1 of a tile
  // where this lane's address of an ldmatrix points, for K (chunk 2 x + kc of key kk) and V (chunk 2 x + vc of key vk)
  const int kk = (lane >> 4) * 8 + (lane & 7), kc = (lane >> 3) & 1, vk = ((lane >> 3) & 1) * 8 + (lane & 7), vc = lane >> 4;
  const bool upper = a.G > 8;                                          // (rows from 8 on are heads too)
  int get = 0;
  for (; s.row < a.n && s.at + kOwnSetup < end; s = next_seq(s)) {
    const int page0 = first_of(s), cnt = last_of(s) - page0;
    const int S = rw.len[s.row] - s.own * kP;                          // own positions
    const __nv_bfloat16* q = a.q + ((size_t)s.row * a.Hq + (size_t)s.h * a.G) * kD;
    uint32_t qf[8][4];
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int r = gr + (y & 1) * 8;
        qf[x][y] = r < a.G ? __ldg(reinterpret_cast<const uint32_t*>(q + (size_t)r * kD + x * 16 + (y >> 1) * 8 + tq * 2)) : 0u;
      }
    float o[16][4] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    for (int p = page0; p < page0 + cnt; ++p) {
      cp_async_wait<kStages - 1>();                                    // this lane's part of the page has landed; everyone's:
      __syncwarp();
      const uint32_t pg = ring + get * kPageBytes;
      const int rows = S - p * kP;                                     // positions in this page and behind
      if (rows < kP) {                                                 // what a page holds behind the last position takes no part
        unsigned char* v = sm + (pg - base) + kP * kD * 2;
        for (int x = rows * 16 + lane; x < kP * 16; x += 32) *reinterpret_cast<uint4*>(v + x * 16) = make_uint4(0, 0, 0, 0);
        __syncwarp();
      }
      float sc[2][4] = {};
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        uint32_t b[4];
        const int c = 2 * x + kc;
        ldsm4(b, pg + kk * 256 + ((c & 8) | ((c ^ kk) & 7)) * 16);
        mma16816(sc[0], qf[x], b[0], b[1]);
        mma16816(sc[1], qf[x], b[2], b[3]);
      }
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          sc[y][z] *= a.scale_log2;
          if (rows < kP && y * 8 + tq * 2 + (z & 1) >= rows) sc[y][z] = -INFINITY;
          mx[z >> 1] = fmaxf(mx[z >> 1], sc[y][z]);
        }
      uint32_t pf[4], pl[4];                                           // hi and lo parts of the probabilities
      float corr[2];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        if (z == 1 && !upper) {                                        // the rows that are no heads take the others' lo parts
          corr[1] = corr[0];
          pf[1] = pl[0];
          pf[3] = pl[2];
          break;
        }
        mx[z] = fmaxf(mx[z], __shfl_xor_sync(0xffffffffu, mx[z], 1));
        mx[z] = fmaxf(mx[z], __shfl_xor_sync(0xffffffffu, mx[z], 2));
        const float mn = fmaxf(m[z], mx[z]), off = mn == -INFINITY ? 0.f : mn;
        corr[z] = exp2f(m[z] - off);
        m[z] = mn;
        const float p0 = exp2f(sc[0][2 * z] - off), p1 = exp2f(sc[0][2 * z + 1] - off);
        const float p2 = exp2f(sc[1][2 * z] - off), p3 = exp2f(sc[1][2 * z + 1] - off);
        l[z] = l[z] * corr[z] + ((p0 + p1) + (p2 + p3));
        split2(p0, p1, pf[z], pl[z]);                                  // (the sum is that of the probabilities as they are)
        split2(p2, p3, pf[2 + z], pl[2 + z]);
      }
      if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
        for (int x = 0; x < 16; ++x) { o[x][0] *= corr[0]; o[x][1] *= corr[0]; o[x][2] *= corr[1]; o[x][3] *= corr[1]; }
      }
      auto values = [&](bool twice) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          uint32_t b[4];
          const int c = 2 * x + vc;
          ldsm4_t(b, pg + kP * kD * 2 + vk * 256 + ((c & 8) | ((c ^ vk) & 7)) * 16);
          mma16816(o[2 * x], pf, b[0], b[1]);
          mma16816(o[2 * x + 1], pf, b[2], b[3]);
          if (twice) {
            mma16816(o[2 * x], pl, b[0], b[1]);
            mma16816(o[2 * x + 1], pl, b[2], b[3]);
          }
        }
      };
      if (upper) values(true); else values(false);                     // (a branch per step keeps the steps from overlapping)
      if (++get == kStages) get = 0;
      __syncwarp();                                                    // all lanes have read the page
      issue();
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      l[z] += __shfl_xor_sync(0xffffffffu, l[z], 1);
      l[z] += __shfl_xor_sync(0xffffffffu, l[z], 2);
      l[z] *= kScale;
    }
    if (!upper) {
#pragma unroll
      for (int x = 0; x < 16; ++x) { o[x][0] += o[x][2]; o[x][1] += o[x][3]; }
    }
    const bool whole = cnt == s.pages;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int r = gr + z * 8;
      if (r >= a.G) continue;
      const size_t row = (size_t)s.row * a.Hq + (size_t)s.h * a.G + r;
      if (whole && s.own == 0) {
        const float inv = 1.f / l[z];
        uint32_t* out = reinterpret_cast<uint32_t*>(a.out + row * kD) + tq;
#pragma unroll
        for (int x = 0; x < 16; ++x) out[x * 4] = pack2(o[x][2 * z] * inv, o[x][2 * z + 1] * inv);
      } else {
        const size_t slot = whole ? row : ((size_t)me * 2 + (s.at <= begin ? 0 : 1)) * a.G + r;
        float2* po = reinterpret_cast<float2*>((whole ? a.all_o : a.own_o) + slot * kD) + tq;
#pragma unroll
        for (int x = 0; x < 16; ++x) po[x * 4] = make_float2(o[x][2 * z], o[x][2 * z + 1]);
        if (tq == 0) reinterpret_cast<float2*>(whole ? a.all_ml : a.own_ml)[slot] = make_float2(m[z], l[z]);
      }
    }
    prefetch_q(next_seq(next_seq(s)));
  }
}

// ---------------------------------------------------------------- shared pages
struct Place { int g, hb, at; int4 grp; Shape x; };   // sequence hb = head * blocks + block of group g; at: how far into it, kSetup counted first
// What a share that ends at `end` holds of the sequence at place p (stream position pos).  (No tile at all only at the share's
// end, in front of a sequence's first.)
struct Part { int tile0, cnt, len; };
__device__ inline Part part_of(const Place& p, int pos, int end) {
  Part x;
  x.len = min(p.x.tiles + kSetup - p.at, end - pos);
  x.tile0 = max(0, p.at - kSetup);
  x.cnt = max(0, p.at + x.len - kSetup) - x.tile0;
  return x;
}
// The groups as this CTA keeps them: in shared memory, or, if they are many, in the workspace.
struct Table { const int4* groups; const int* at; int n; };
// One warp: the group that position pos of the stream (pos < total) lies in.
__device__ inline Place locate(const GroupArgs& a, const Table& tab, int pos, int lane) {
  int g = 0;
  for (int g0 = 0; g0 < tab.n; g0 += 32) {              // the last that begins at or before pos: it has tiles
    const unsigned m = __ballot_sync(0xffffffffu, g0 + lane < tab.n && tab.at[g0 + lane] <= pos);
    if (!m) break;
    g = g0 + 31 - __clz(m);
    if (m != 0xffffffffu) break;
  }
  Place p;
  p.g = g;
  p.grp = tab.groups[g];
  p.x = shape_of(a, p.grp);
  const int off = pos - tab.at[g], each = p.x.tiles + kSetup;
  p.hb = (int)((unsigned)off / (unsigned)each);
  p.at = off - p.hb * each;
  return p;
}
// The place behind a whole rest of a sequence.
__device__ inline void next_sequence(const GroupArgs& a, const Table& tab, Place& p) {
  p.at = 0;
  if (++p.hb < a.Hkv * p.x.blocks) return;
  p.hb = 0;
  while (++p.g < tab.n) {
    p.grp = tab.groups[p.g];
    if (p.grp.z >= 0) { p.x = shape_of(a, p.grp); return; }
  }
}
// A piece, as the query warp announces it: tiles [tile0, tile0 + cnt) of the sequence's `tiles`, for rows of traces
// [row0, row0 + rows).
struct Piece { int h, row0, rows, two, tile0, cnt, tiles, keys, slot; };

constexpr size_t kTableAt = 2 * kQBytes + kSlots * kSlotBytes;          // behind the rings and the rows' arrays
static_assert(kTableAt >= kRing + (kMaxTracesFast + 2) * 4 + 2 * kMaxTracesFast * 4, "rows and groups lie side by side");
constexpr size_t kPrefixSmem = 1024 + kTableAt + 32 * 8 + 2 * sizeof(Piece) + 64 + kTableGroups * 20;
constexpr size_t kSmem = kPrefixSmem > kStreamSmem ? kPrefixSmem : kStreamSmem;
static_assert(kSmem <= 232448 - 256, "shared memory of one CTA");

__global__ void __launch_bounds__(kThreads, 1) groups_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ GroupArgs a) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ int s_sum[kThreads / 32];
  __shared__ Header s_header;
  __shared__ float s_unit_ns;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* sm = smem_raw + (base - raw);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const bool first = blockIdx.x == 0;
  dependents_may_launch();
  if (threadIdx.x == 0) { prefetch_map(&map); prefetch_map(&map_q); }

  // ---- who shares what.  A description that is not in order is not followed at all.
  Rows rw;
  rw.at = reinterpret_cast<int*>(sm + kRing);
  rw.own = rw.at + kMaxTracesFast + 2;
  rw.len = rw.own + kMaxTracesFast;
  int4* s_grp = reinterpret_cast<int4*>(sm + kTableAt);
  int* s_grp_at = reinterpret_cast<int*>(s_grp + kTableGroups);
  bool bad = false;
  for (int g = threadIdx.x; g < a.n_groups; g += kThreads) {
    const int r0 = a.group_rows[g], r1 = a.group_rows[g + 1], pages = a.group_pages[g];
    bad |= r0 < 0 || r1 < r0 || r1 > a.n || pages < 0 || pages > a.max_pages;
  }
  for (int i = threadIdx.x; i < a.n; i += kThreads) {
    rw.own[i] = 0;
    rw.len[i] = length_of(a, i, first);
  }
  Table tab;
  tab.n = __syncthreads_or(bad) ? 0 : a.n_groups;
  if (first && threadIdx.x == 0 && tab.n != a.n_groups) flag_error(a.counters, STEP_ERR_INVALID_ARG);
  int4* grp = a.n_groups <= kTableGroups ? s_grp : a.cta_groups + (size_t)blockIdx.x * a.n_groups;
  int* grp_at = a.n_groups <= kTableGroups ? s_grp_at : a.cta_group_at + (size_t)blockIdx.x * a.n_groups;
  tab.groups = grp;
  tab.at = grp_at;
  for (int g = warp; g < tab.n; g += kThreads / 32) {
    const int r0 = a.group_rows[g], r1 = a.group_rows[g + 1], pages = a.group_pages[g];
    int members = 0, leader = -1;
    for (int i0 = r0; i0 < r1; i0 += 32) {
      const int i = i0 + lane;
      const unsigned m = __ballot_sync(0xffffffffu, i < r1 && pages > 0 && rw.len[i] >= (long long)pages * kP);
      if (m && leader < 0) leader = i0 + __ffs(m) - 1;
      members += __popc(m);
    }
    if (members < 2) leader = -1;
    if (leader >= 0)
      for (int i = r0 + lane; i < r1; i += 32)
        if (rw.len[i] >= (long long)pages * kP) {
          rw.own[i] = pages;
          if (first) a.plan[i].tiles = g + 1;                          // (for now: whose pages it shares)
        }
    if (lane == 0) grp[g] = make_int4(r0, r1 - r0, leader, pages);
  }
  __syncthreads();
  // ---- where every group's tiles begin in their stream (one warp), and every row's own pages in theirs (a thread takes `per` rows)
  if (warp == kThreads / 32 - 1) {
    int run = 0;
    float ns = 0.f;
    for (int g0 = 0; g0 < tab.n; g0 += 32) {
      const int g = g0 + lane;
      int mine = 0;
      if (g < tab.n) {
        const int4 x = grp[g];
        if (x.z >= 0) {
          const Shape sh = shape_of(a, x);
          mine = (sh.tiles + kSetup) * sh.blocks * a.Hkv;
          const int narrow = x.y - (sh.blocks - 1) * 2 * a.tokens <= a.tokens;
          ns += (float)mine * (kWideNs - (kWideNs - kNarrowNs) * narrow / (float)sh.blocks);
        }
      }
      int incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
      }
      if (g < tab.n) grp_at[g] = run + incl - mine;
      run += __shfl_sync(0xffffffffu, incl, 31);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ns += __shfl_xor_sync(0xffffffffu, ns, o);
    if (lane == 0) { s_header.units = run; s_unit_ns = ns / (float)max(1, run); }
  }
  {
    const int per = (a.n + kThreads - 1) / kThreads, i0 = threadIdx.x * per;
    auto pages_of = [&](int i) {
      const int pages = (rw.len[i] + kP - 1) / kP - rw.own[i];
      return pages > 0 ? pages + kOwnSetup : 0;
    };
    int mine = 0;
    for (int i = i0; i < min(a.n, i0 + per); ++i) mine += pages_of(i);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    int run = incl - mine + __reduce_add_sync(0xffffffffu, lane < warp ? s_sum[lane] : 0);
    for (int i = i0; i < min(a.n, i0 + per); ++i) {
      rw.at[i] = run;
      run += pages_of(i);
      if (i == a.n - 1) rw.at[a.n] = run;
    }
  }
  __syncthreads();
  Header hd;
  hd.units = s_header.units; hd.pages = rw.at[a.n] * a.Hkv;
  hd.n_prefix = choose_prefix(a, hd.units, s_unit_ns, hd.pages, lane);
  const int n_prefix = hd.n_prefix;
  if (first) {
    if (threadIdx.x == 0) *a.header = hd;
    for (int i = threadIdx.x; i < a.n; i += kThreads) {
      RowPlan p = {};
      p.at = rw.at[i];
      p.pages = max(0, rw.at[i + 1] - rw.at[i] - kOwnSetup);
      if (rw.own[i] > 0) {
        const int g = a.plan[i].tiles - 1;
        const int4 x = grp[g];
        const Shape sh = shape_of(a, x);
        const int t = i - x.x, block = t / (2 * a.tokens);
        p.tiles = sh.tiles;
        p.head = sh.blocks * (sh.tiles + kSetup);
        p.begin = grp_at[g] + block * (sh.tiles + kSetup);
        p.place = (t - block * 2 * a.tokens) * 2 + (x.y - block * 2 * a.tokens <= a.tokens);
      }
      a.plan[i] = p;
    }
  }

  if ((int)blockIdx.x >= n_prefix) {
    // ================================================ own pages
    const int n_own = a.ctas - n_prefix;
    if (warp < kStreamWarps) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
      own_pages(a, rw, sm, base, ((int)blockIdx.x - n_prefix) * kStreamWarps + warp, hd.pages, own_share(hd, n_own));
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    }
    return;
  }

  // ================================================ shared pages
  const uint32_t sm_q = base, sm_ring = base + 2 * kQBytes;
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(s_grp_at + kTableGroups);
  Piece* s_piece = reinterpret_cast<Piece*>(s_bar + 32);               // [2]
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_piece + 2);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_begun = reinterpret_cast<int*>(s_tmem + 4);                   // [3] how many fills of their buffers the K, V and query warps have begun
  const uint32_t bars = smem_u32(s_bar);
  const uint32_t bar_full = bars, bar_empty = bars + 8 * kSlots;
  const uint32_t bar_q = bars + 16 * kSlots, bar_s = bar_q + 8, bar_p = bar_s + 16, bar_o = bar_p + 32,
                 bar_qfree = bar_o + 16, bar_drain = bar_qfree + 8;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(bar_full + 8 * s, 1);               // the fetching warp's announcement of bytes
      mbar_init(bar_empty + 8 * s, 1);              // tcgen05.commit
    }
    mbar_init(bar_q, 1);                            // the query warp's announcement
    mbar_init(bar_qfree, 9);                        // tcgen05.commit: a piece's last scores; all softmax warps have begun it
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_s + 8 * s, 1);                  // tcgen05.commit: scores made (and the products before them done)
      mbar_init(bar_p + 8 * s, 4);                  // the second half of the probabilities (one arrival per warp)
      mbar_init(bar_p + 16 + 8 * s, 4);             // the first half
      mbar_init(bar_o + 8 * s, 1);                  // tcgen05.commit: a piece's last product
    }
    mbar_init(bar_drain, 1);
    *s_abort = 0;
    s_begun[0] = s_begun[1] = s_begun[2] = 0;
    mbar_init_fence();
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_async_smem();                               // (the rows' arrays, which everyone has read by now, make way for copies)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  // this CTA's share of the stream
  const int W = prefix_share(hd, n_prefix), pos0 = (int)min((long long)hd.units, (long long)blockIdx.x * W), end = min(hd.units - pos0, W) + pos0;

  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (mbar_test_wait(bar, parity)) return true;                      // (a limit of zero: this is all)
    if (*s_abort) return false;
    if (mbar_wait_bounded(bar, parity, a.wait_ns)) return true;
    flag_error(a.counters, STEP_ERR_TIMEOUT);
    *s_abort = 1;
    return false;
  };
  // the same, with one answer for the whole warp: what follows has to be executed by all of it
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  // one arrival for all of the warp's threads
  auto arrive_warp = [&](uint32_t bar) { __syncwarp(); if (lane == 0) mbar_arrive(bar); };

  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // ------------------------------------------------ softmax: lane `ln` of the CTA, row `row` of its 128
    const int ln = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t t_s = t_row + ln * 128, t_o = t_row + 256 + ln * 128;
    uint32_t ph_s = 0, ph_o = 0, ph_piece = 0;
    for (;;) {
      if (!wait_warp(bar_q, ph_piece)) break;
      const Piece pc = s_piece[ph_piece];
      if (pc.cnt == 0) break;                                          // the share is done
      arrive_warp(bar_qfree);
      float m_ref = -INFINITY, l = 0.f;
      bool started = false, ok = true;
      for (int i = pc.two ? 0 : ln; i < pc.cnt; i += pc.two ? 1 : 2) {
        if (!wait_warp(bar_s + 8 * ln, ph_s)) { ok = false; break; }
        ph_s ^= 1;
        tc_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tc_ld32_async(t_s + 32 * c, s + 32 * c);
        tc_wait_ld();
        pin<128>(s);
        const int left = pc.keys - (pc.tile0 + i) * kTile;
        if (left < kTile) {                                            // behind the last page
#pragma unroll
          for (int c = 0; c < kTile; ++c)
            if (c >= left) s[c] = 0xff800000u;
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < kTile; c += 8) {
#pragma unroll
          for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], __uint_as_float(s[c + 2 * x]), __uint_as_float(s[c + 2 * x + 1]));
        }
        const float m_new = fmaxf(m_ref, fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * a.scale_log2);
        if (!started) {
          m_ref = m_new;
          started = true;
        } else {
          const bool grow = m_new > m_ref + kRescale;
          if (__any_sync(0xffffffffu, grow)) {
            const float corr = grow ? exp2f(m_ref - m_new) : 1.f;
            if (grow) m_ref = m_new;
            l *= corr;
#pragma unroll 1
            for (int c = 0; c < kD; c += 32) {
              uint32_t o[32];
              tc_ld32_async(t_o + c, o);
              tc_wait_ld();
              pin<32>(o);
#pragma unroll
              for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * corr);
              tc_st32(t_o + c, o);
            }
          }
        }
        const float off = m_ref == -INFINITY ? 0.f : m_ref;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        // In halves: the second product of the first 64 keys runs while the others' probabilities are made.  16 keys' hi parts, then
        // their lo parts take the columns of these keys' scores.
#pragma unroll
        for (int c0 = 0; c0 < kTile; c0 += 32) {
          uint32_t p[32];
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            float p0, p1;
            fma2(p0, p1, __uint_as_float(s[c0 + c]), __uint_as_float(s[c0 + c + 1]), a.scale_log2, -off);
            p0 = exp2f(p0);
            p1 = exp2f(p1);
            add2(sum[c & 2], sum[(c & 2) + 1], p0, p1);
            split2(p0, p1, p[(c & 16) + (c & 15) / 2], p[(c & 16) + 8 + (c & 15) / 2]);
          }
          tc_st32(t_s + c0, p);
          if (c0 == 32 || c0 == 96) {
            tc_wait_st();
            tc_fence_before();
            arrive_warp(bar_p + 8 * (c0 == 32 ? 2 + ln : ln));
          }
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      if (!ok) break;
      // A piece of one tile leaves lane 1 without any: it has no products to wait for.  (Nobody waits for that lane's warps
      // either, so that a phase of the barrier which they were to see could be over, and the next one too, before they look.)
      const bool some = pc.two || ln < pc.cnt;
      if (some) {
        if (!wait_warp(bar_o + 8 * ln, ph_o)) break;
        ph_o ^= 1;
        tc_fence_after();
      }
      ph_piece ^= 1;

      // ---- the piece is done: its rows' (m, l) and o
      const int t = (pc.two ? ln * a.tokens : 0) + row / a.G;           // trace of the block
      const bool mine = row < a.tokens * a.G && t < pc.rows;
      const bool whole = pc.cnt == pc.tiles;
      const size_t at = whole ? ((size_t)(pc.two ? 0 : ln) * a.n + pc.row0 + (mine ? t : 0)) * a.Hq + (size_t)pc.h * a.G + row % a.G
                              : (((size_t)blockIdx.x * 2 + pc.slot) * 2 + ln) * kHalfRows + row;
      if (mine) reinterpret_cast<float2*>(whole ? a.row_ml : a.pre_ml)[at] = make_float2(m_ref, l * kScale);
      float* o_out = (whole ? a.row_o : a.pre_o) + at * kD;
      if (some) {
#pragma unroll
        for (int c = 0; c < kD; c += 64) {
          uint32_t o[64];
          tc_ld32_async(t_o + c, o);
          tc_ld32_async(t_o + c + 32, o + 32);
          tc_wait_ld();
          pin<64>(o);
          if (mine) {
#pragma unroll
            for (int x = 0; x < 64; x += 8) st_global32(o_out + c + x, o + x);
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == kWarpK || warp == kWarpV) {
      // ------------------------------------------------ K or V tiles into their ring
      const int kv = warp == kWarpV, ring0 = kv ? kKSlots : 0, ring_n = kv ? kVSlots : kKSlots;
      int slot = 0, begun = 0;                                         // (fills begun)
      uint32_t ph = 1;
      bool ok = true;
      // Block ids of 64 pages (eight tiles): lane i holds those of pages win + i and win + 32 + i.  The second half is asked
      // for when the first is entered, four tiles before it is needed.
      auto load_ids = [&](const Place& of, int first) {
        const int page = first + lane;
        return of.g < tab.n && page < of.grp.w ? a.block_table[(size_t)of.grp.z * a.max_pages + page] : 0;
      };
      int pos = pos0;
      if (pos < end) {
        Place pl = locate(a, tab, pos, lane);
        Part part = part_of(pl, pos, end);
        int win = (part.tile0 * (kTile / kP)) & ~31;
        int next0 = load_ids(pl, win), next1 = load_ids(pl, win + 32);
        while (pos < end && ok) {
          part = part_of(pl, pos, end);
          const int h = pl.hb / pl.x.blocks, all = pl.grp.w;
          win = (part.tile0 * (kTile / kP)) & ~31;
          int ids0 = next0, ids1 = next1;
          Place nx = pl;                                               // the sequence behind this one, its block ids too
          next_sequence(a, tab, nx);
          next0 = load_ids(nx, 0);
          next1 = load_ids(nx, 32);
          for (int i = 0; i < part.cnt; ++i) {
            const int pg0 = (part.tile0 + i) * (kTile / kP);
            if (!wait_warp(bar_empty + 8 * (ring0 + slot), ph)) { ok = false; break; }
            const uint32_t bar = bar_full + 8 * (ring0 + slot), dst = sm_ring + (ring0 + slot) * kSlotBytes;
            if (pg0 >= win + 32) { win += 32; ids0 = ids1; ids1 = load_ids(pl, win + 32); }
            const int in_win = pg0 - win, pages = min(kTile / kP, all - pg0);
            int bb = __shfl_sync(0xffffffffu, ids0, (in_win + (lane & 7)) & 31);
            if (lane < pages && (bb < 0 || bb >= a.num_blocks)) { flag_error(a.counters, STEP_ERR_BAD_BLOCK); bb = 0; }
            if (lane == 0) mbar_expect_tx(bar, pages * (kP * kD * 2));
            __syncwarp();
            if (lane < pages)                                          // a box is the K or the V of a page
              tma_load_4d(dst + lane * (kP * kD * 2), &map, 0, 0, 0, ((((a.layer * a.num_blocks) + bb) * a.Hkv + h) * 2 + kv) * (kP / 8), bar);
            __syncwarp();
            ++begun;
            if (++slot == ring_n) { slot = 0; ph ^= 1; }
          }
          pos += part.len;
          pl = nx;
        }
      }
      if (lane == 0) s_begun[kv] = begun;
    } else if (warp == kWarpQ) {
      // ------------------------------------------------ query rows of one piece after another
      uint32_t par = 0;
      int begun = 0;
      int pos = pos0;
      Place pl = {};
      if (pos < end) pl = locate(a, tab, pos, lane);
      for (;; par ^= 1) {
        Piece pc = {};
        Part part = {};
        if (pos < end) part = part_of(pl, pos, end);
        if (part.cnt > 0) {
          pc.h = pl.hb / pl.x.blocks;
          const int t0 = (pl.hb - pc.h * pl.x.blocks) * 2 * a.tokens;
          pc.row0 = pl.grp.x + t0; pc.rows = min(2 * a.tokens, pl.grp.y - t0);
          pc.two = pc.rows > a.tokens;
          pc.tile0 = part.tile0; pc.cnt = part.cnt; pc.tiles = pl.x.tiles; pc.keys = pl.grp.w * kP;
          pc.slot = pos - pl.at <= pos0 ? 0 : 1;                       // of the share: does the sequence begin inside it?
          pos += part.len;
          next_sequence(a, tab, pl);
        }
        // the scores of the piece before are made, and its announcement has been read (the very first wait passes at once)
        if (!wait_warp(bar_qfree, par ^ 1)) break;
        if (lane == 0) {
          s_piece[par] = pc;
          if (pc.cnt > 0) {
            // (rows of other groups may come along: a row of the products depends on its own query only)
            const int halves = pc.two ? 4 : 2;
            mbar_expect_tx(bar_q, halves * a.box * a.G * 128);
            for (int x = 0; x < halves; ++x)
              tma_load_3d(sm_q + (x >> 1) * kQBytes + (x & 1) * (kQBytes / 2), &map_q, (x & 1) * 64, pc.h * a.G, pc.row0 + (x >> 1) * a.tokens, bar_q);
          } else {
            mbar_arrive(bar_q);
          }
        }
        __syncwarp();
        if (lane == 0) s_begun[2] = ++begun;
        if (pc.cnt == 0) break;
      }
    } else {
      // ------------------------------------------------ products.  The tensor cores take the next few instructions only, so
      // every cycle this warp spends between them is idle time there.  Hence: the warp stays together and one thread is
      // elected for the instructions, and what is likely there long since is waited for before what is not.
      const uint32_t id_qk = umma_idesc_bf16(kTile), id_pv = umma_idesc_bf16(kD) | (1u << 16);   // B of the second is MN-major
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      int at[2] = {0, 0};
      uint32_t ph[2] = {0, 0}, ph_q = 0, ph_p[2] = {0, 0};
      bool ok = true;
      // waits for the next tile of K (0) or V (1); its slot
      auto next = [&](int kv) -> int {
        const int s = (kv ? kKSlots : 0) + at[kv];
        ok = ok && wait_warp(bar_full + 8 * s, ph[kv]);
        if (++at[kv] == (kv ? kVSlots : kKSlots)) { at[kv] = 0; ph[kv] ^= 1; }
        return s;
      };
      auto probabilities = [&](int ln, bool first_half) {
        ok = ok && wait_warp(bar_p + 8 * (first_half ? 2 + ln : ln), ph_p[ln]);
        if (!first_half) ph_p[ln] ^= 1;
        tc_fence_after();
      };
      // (the elected thread's part of it)
      auto scores = [&](int ln, int q, int s) {
        const uint32_t qa = sm_q + q * kQBytes, kb = sm_ring + s * kSlotBytes;
#pragma unroll
        for (int x = 0; x < 8; ++x)
          tc_mma_bf16(tm + ln * 128, umma_desc_sw128(qa + (x >> 2) * (kQBytes / 2) + (x & 3) * 32),
                      umma_desc_k(kb + (x >> 2) * 1024 + (x & 3) * 32), id_qk, x != 0);
        tc_commit(bar_s + 8 * ln);
      };
      // steps of 16 keys; those of a tile behind the last page are left out, so nothing that lies there matters
      auto values = [&](int ln, int s, bool first, int from, int steps) {
        const uint32_t vb = sm_ring + s * kSlotBytes;
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (x >= from && x < steps) {
            tc_mma_bf16_ta(tm + 256 + ln * 128, tm + ln * 128 + x * 16, umma_desc_v(vb + x * 4096), id_pv, !(first && x == 0));
            tc_mma_bf16_ta(tm + 256 + ln * 128, tm + ln * 128 + x * 16 + 8, umma_desc_v(vb + x * 4096), id_pv, 1);
          }
      };
      while (ok) {
        ok = wait_warp(bar_q, ph_q);
        const Piece pc = s_piece[ph_q];
        const int cnt = pc.cnt, keys = pc.keys - pc.tile0 * kTile;
        auto steps = [&](int i) { return min(8, (keys - i * kTile) / 16); };
        ph_q ^= 1;
        if (!ok || cnt == 0) break;
        tc_fence_after();
        if (pc.two) {
          int k = next(0);
          if (ok && elect_one()) {
            scores(0, 0, k);
            scores(1, 1, k);
            tc_commit(bar_empty + 8 * k);
            if (cnt == 1) tc_commit(bar_qfree);
          }
          __syncwarp();
          for (int i = 0; i < cnt && ok; ++i) {
            const int v = next(1);
            const bool more = i + 1 < cnt;
            if (more) k = next(0);
            probabilities(0, true);
            if (ok && elect_one()) values(0, v, i == 0, 0, min(4, steps(i)));
            __syncwarp();
            probabilities(0, false);
            if (ok && elect_one()) {
              values(0, v, i == 0, 4, steps(i));
              if (more) scores(0, 0, k); else tc_commit(bar_o);
            }
            __syncwarp();
            probabilities(1, true);
            if (ok && elect_one()) values(1, v, i == 0, 0, min(4, steps(i)));
            __syncwarp();
            probabilities(1, false);
            if (ok && elect_one()) {
              values(1, v, i == 0, 4, steps(i));
              tc_commit(bar_empty + 8 * v);
              if (more) { scores(1, 1, k); tc_commit(bar_empty + 8 * k); } else tc_commit(bar_o + 8);
              if (i + 2 == cnt) tc_commit(bar_qfree);
            }
            __syncwarp();
          }
        } else {
          for (int i = 0; i < min(cnt, 2); ++i) {
            const int k = next(0);
            if (ok && elect_one()) {
              scores(i, 0, k);
              tc_commit(bar_empty + 8 * k);
              if (i + 1 == cnt) tc_commit(bar_qfree);
            }
            __syncwarp();
          }
          for (int i = 0; i < cnt && ok; ++i) {
            const int ln = i & 1, v = next(1);
            probabilities(ln, true);
            if (ok && elect_one()) values(ln, v, i < 2, 0, min(4, steps(i)));
            __syncwarp();
            probabilities(ln, false);
            if (ok && elect_one()) {
              values(ln, v, i < 2, 4, steps(i));
              tc_commit(bar_empty + 8 * v);
              if (i + 2 >= cnt) tc_commit(bar_o + 8 * ln);
            }
            __syncwarp();
            if (i + 2 < cnt) {
              const int k = next(0);
              if (ok && elect_one()) {
                scores(ln, 0, k);
                tc_commit(bar_empty + 8 * k);
                if (i + 3 == cnt) tc_commit(bar_qfree);
              }
              __syncwarp();
            }
          }
        }
      }
      __syncwarp();
      if (elect_one()) {
        tc_commit(bar_drain);                                          // no product is in flight when the tensor memory goes back
        mbar_wait_bounded(bar_drain, 0);
      }
      __syncwarp();
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  // A wait has run out: copies in flight still write this CTA's shared memory.  (Decided here, where no warp can begin one any
  // more and *s_abort is final.)
  if (*s_abort) {
    // fills 0, 1, 2, .. of a barrier complete its phases in that order: the last one's parity
    auto landed = [&](uint32_t bar, int fills) { if (fills > 0) mbar_wait_bounded(bar, (fills - 1) & 1, kDrainNs); };
    const int begun = warp == kWarpK ? s_begun[0] : (warp == kWarpV ? s_begun[1] : s_begun[2]);
    if (lane == 0 && warp == kWarpK)
      for (int s = 0; s < kKSlots; ++s) landed(bar_full + 8 * s, (begun - s + kKSlots - 1) / kKSlots);
    if (lane == 0 && warp == kWarpV)
      for (int s = 0; s < kVSlots; ++s) landed(bar_full + 8 * (kKSlots + s), (begun - s + kVSlots - 1) / kVSlots);
    if (lane == 0 && warp == kWarpQ) landed(bar_q, begun);
    __syncthreads();
  }
  if (warp == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}
// ---------------------------------------------------------------- one result per row
constexpr int kMergeWarps = 4, kMergeAhead = 8;

// A warp per query row (kTeam: a CTA, whose warps take a run of the pieces each), lanes over the 128 dims: the shared pages' pieces,
// then the row's own, in stream order with a running (max, sum, values); the loads of kMergeAhead pieces are under way at once.
// With few rows there are many pieces of each: 16 traces of one prompt of 16,000, 34 pieces a row, took a warp 10 us.
template <bool kTeam>
__global__ void __launch_bounds__(kMergeWarps * 32) groups_merge_kernel(const __grid_constant__ GroupArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ float2 s_ml[kTeam ? kMergeWarps : 1];
  __shared__ float4 s_o[kTeam ? kMergeWarps : 1][32];
  wait_for_primary();
  const Header hd = *a.header;
  const int W = max(1, own_share(hd, max(1, a.ctas - hd.n_prefix))), Wp = max(1, prefix_share(hd, max(1, hd.n_prefix)));
  for (int r = kTeam ? blockIdx.x : blockIdx.x * kMergeWarps + warp; r < a.n * a.Hq; r += gridDim.x * (kTeam ? 1 : kMergeWarps)) {
    const int i = r / a.Hq, hq = r - i * a.Hq, h = hq / a.G, sub = hq - h * a.G;
    const RowPlan pl = a.plan[i];
    const int at = pl.at * a.Hkv + h * (pl.pages + kOwnSetup);
    const int w0 = pl.pages > 0 ? (at + kOwnSetup) / W : 0, w1 = pl.pages > 0 ? (at + kOwnSetup + pl.pages - 1) / W : -1;
    if (pl.tiles == 0 && w0 == w1) continue;                           // written already
    // the pieces of the shared pages: shares p0 .. p1, each with one result or (narrow) one per lane
    const int begin = pl.begin + h * pl.head;
    const int narrow = pl.place & 1, trace = pl.place >> 1, ln = trace / a.tokens, row = ln * kHalfRows + (trace - ln * a.tokens) * a.G + sub;
    const int p0 = pl.tiles > 0 ? (begin + kSetup) / Wp : 0;
    const int pieces = pl.tiles > 0 ? ((begin + kSetup + pl.tiles - 1) / Wp - p0 + 1) << narrow : 0;
    const bool whole = pieces == 1 << narrow;                          // one share has all tiles
    const int all = pieces + (w1 - w0 + 1);
    float M = -INFINITY, den = 0.f;
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
    const int from = kTeam ? all * warp / kMergeWarps : 0, to = kTeam ? all * (warp + 1) / kMergeWarps : all;
    for (int k0 = from; k0 < to; k0 += kMergeAhead) {
      float2 ml[kMergeAhead];
      float4 o[kMergeAhead];
#pragma unroll
      for (int y = 0; y < kMergeAhead; ++y) {
        const int k = k0 + y;
        ml[y] = make_float2(-INFINITY, 0.f);
        if (k >= to) continue;
        const float *mls, *os;
        size_t slot;
        if (k < pieces) {
          const int s = p0 + (k >> narrow), by = k & narrow;
          mls = whole ? a.row_ml : a.pre_ml;
          os = whole ? a.row_o : a.pre_o;
          slot = whole ? (size_t)by * a.n * a.Hq + r : ((size_t)s * 2 + (begin <= s * Wp ? 0 : 1)) * 2 * kHalfRows + by * kHalfRows + row;
        } else {
          const int s = w0 + k - pieces;
          mls = w0 == w1 ? a.all_ml : a.own_ml;
          os = w0 == w1 ? a.all_o : a.own_o;
          slot = w0 == w1 ? r : ((size_t)s * 2 + (at <= s * W ? 0 : 1)) * a.G + sub;
        }
        ml[y] = __ldcg(reinterpret_cast<const float2*>(mls) + slot);
        o[y] = __ldcg(reinterpret_cast<const float4*>(os + slot * kD) + lane);
      }
      float Mb = M;
#pragma unroll
      for (int y = 0; y < kMergeAhead; ++y)
        if (ml[y].y != 0.f) Mb = fmaxf(Mb, ml[y].x);
      const float off = Mb == -INFINITY ? 0.f : Mb, keep = exp2f(M - off);
      den *= keep; num.x *= keep; num.y *= keep; num.z *= keep; num.w *= keep;
#pragma unroll
      for (int y = 0; y < kMergeAhead; ++y) {
        if (ml[y].y == 0.f) continue;                                  // none, or a lane that had no tile: nothing stands there
        const float wgt = exp2f(ml[y].x - off);
        den += wgt * ml[y].y;
        num.x += wgt * o[y].x; num.y += wgt * o[y].y; num.z += wgt * o[y].z; num.w += wgt * o[y].w;
      }
      M = Mb;
    }
    if constexpr (kTeam) {
      if (lane == 0) s_ml[warp] = make_float2(M, den);
      s_o[warp][lane] = num;
      __syncthreads();
      float Mb = -INFINITY;
#pragma unroll
      for (int w = 0; w < kMergeWarps; ++w) Mb = fmaxf(Mb, s_ml[w].x);
      const float off = Mb == -INFINITY ? 0.f : Mb;
      den = 0.f;
      num = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kMergeWarps; ++w) {
        const float wgt = exp2f(s_ml[w].x - off);
        const float4 o = s_o[w][lane];
        den += wgt * s_ml[w].y;
        num.x += wgt * o.x; num.y += wgt * o.y; num.z += wgt * o.z; num.w += wgt * o.w;
      }
      __syncthreads();                                                 // (the next row's results go to the same place)
      if (warp != 0) continue;
    }
    const float inv = all == 0 ? 0.f : 1.f / den;                      // a row without any key: zeros
    reinterpret_cast<uint2*>(a.out + (size_t)r * kD)[lane] = make_uint2(pack2(num.x * inv, num.y * inv), pack2(num.z * inv, num.w * inv));
  }
}

// Lays the workspace out (from `ws` on; null: only its size).
size_t lay_out(const step_pool* pool, int n, int n_groups, char* ws, GroupArgs* a) {
  const Geo g = geo_of(pool);
  const size_t ctas = pool->num_sms, warps = ctas * kStreamWarps, rows = (size_t)n * g.Hq;
  size_t off = 0;
  auto take = [&](size_t bytes) { char* p = ws + off; off += (bytes + 255) / 256 * 256; return p; };
  GroupArgs x = {};
  x.header = (Header*)take(sizeof(Header));
  x.plan = (RowPlan*)take((size_t)n * sizeof(RowPlan));
  if (n_groups > kTableGroups) {
    x.cta_groups = (int4*)take(ctas * n_groups * sizeof(int4));
    x.cta_group_at = (int*)take(ctas * n_groups * 4);
  }
  x.own_ml = (float*)take(warps * 2 * g.G * 8);
  x.own_o = (float*)take(warps * 2 * g.G * kD * 4);
  if (n_groups > 0) {
    x.pre_ml = (float*)take(ctas * 4 * kHalfRows * 8);
    x.pre_o = (float*)take(ctas * 4 * kHalfRows * kD * 4);
    x.row_ml = (float*)take(2 * rows * 8);
    x.row_o = (float*)take(2 * rows * kD * 4);
    x.all_ml = (float*)take(rows * 8);
    x.all_o = (float*)take(rows * kD * 4);
  }
  if (a) *a = x;
  return off;
}

}  // namespace

namespace stepk {

// (positions in the streams of own and of shared pages are 32-bit numbers)
bool groups_tc_supported(const step_pool* pool, int n) {
  return attention_tc_covers(pool, n) && pool->num_sms >= 2 && (long long)n * pool->cfg.num_kv_heads * ((long long)pool->cfg.max_pages_per_trace + 3) < (1ll << 31);
}

void make_pool_map(step_pool* pool) {
  CUtensorMap map;
  static_assert(sizeof(map) <= sizeof(pool->tmap_kv_bytes), "tensor map");
  if (!attention_tc_fits(pool) || !encode_pool_map(pool, &map)) return;
  memcpy(pool->tmap_kv_bytes, &map, sizeof(map));
  pool->tmap_kv_set = true;
}

size_t groups_tc_workspace(const step_pool* pool, int n, int n_groups) { return lay_out(pool, n, n_groups, nullptr, nullptr); }

int groups_tc_launch(step_pool* pool, int layer, const void* q, const int32_t* block_table, const int32_t* seq_lens, int n,
                     const int32_t* group_rows, const int32_t* group_pages, int n_groups, void* out, void* workspace, cudaStream_t s) {
  const Geo g = geo_of(pool);
  if (!pool->tmap_kv_set) return STEP_ERR_CUDA;
  if (!pool->groups_ready) {                                           // (threads that come here at once do the same)
    // (warps that ask for more registers than the launch has would wait for good)
    cudaFuncAttributes fa;
    if (cudaFuncSetAttribute(groups_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) != cudaSuccess ||
        cudaFuncGetAttributes(&fa, groups_kernel) != cudaSuccess || fa.numRegs * kThreads < 256 * kRegsSoftmax + 128 * kRegsOther) return STEP_ERR_CUDA;
    pool->groups_ready = true;
  }
  GroupArgs a;
  lay_out(pool, n, n_groups, (char*)workspace, &a);
  a.kv = (const __nv_bfloat16*)pool->cfg.kv_storage; a.q = (const __nv_bfloat16*)q; a.out = (__nv_bfloat16*)out;
  a.block_table = block_table; a.seq_lens = seq_lens; a.group_rows = group_rows; a.group_pages = group_pages;
  a.counters = pool->v.counters;
  a.n = n; a.n_groups = n_groups; a.Hq = g.Hq; a.Hkv = g.Hkv; a.G = g.G; a.layer = layer; a.max_pages = g.max_pages; a.num_blocks = g.num_blocks;
  a.tokens = kHalfRows / g.G;
  a.box = a.tokens < n ? a.tokens : n;
  a.ctas = pool->num_sms;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)kD);
  a.wait_ns = pool->wait_limit_ns;
  CUtensorMap map, map_q;
  memcpy(&map, pool->tmap_kv_bytes, sizeof(map));
  // queries: a box is one half of the dims of the G heads of a group, for as many traces as make a tile of rows
  const cuuint64_t q_dims[3] = {kD, (cuuint64_t)g.Hq, (cuuint64_t)n};
  const cuuint64_t q_strides[2] = {kD * 2, (cuuint64_t)g.Hq * kD * 2};
  const cuuint32_t q_box[3] = {64, (cuuint32_t)g.G, (cuuint32_t)a.box}, estr[3] = {1, 1, 1};
  if (!encode_tiled(&map_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), q_dims, q_strides, q_box, estr,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE))
    return STEP_ERR_CUDA;
  groups_kernel<<<a.ctas, kThreads, kSmem, s>>>(map, map_q, a);
  if (launch_ok() != STEP_OK) return STEP_ERR_CUDA;
  const long long rows = (long long)n * g.Hq, most = 16ll * a.ctas;
  const bool team = rows <= 8ll * a.ctas;
  const long long ctas = team ? rows : (rows + kMergeWarps - 1) / kMergeWarps;
  if (launch_dependent(team ? groups_merge_kernel<true> : groups_merge_kernel<false>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kMergeWarps * 32), 0, s, a) !=
      cudaSuccess) return STEP_ERR_CUDA;
  return launch_ok();
}

}  // namespace stepk
