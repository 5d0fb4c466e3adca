// Tensor-core form of decode_attention_tree (bf16 pools, head_dim 128, page 16).
//
// The query rows of one trace and KV head are the G heads of its group for every drafted token (row = token * G + head,
// up to 64 * 16 of them).  Against one read of the cache they do 4 * 128 operations per row and position, against 512
// bytes: 64 rows are a small fraction of what the tensor cores do in the time of that read, 256 rows are about as much.
// So every K and V byte is brought to an SM once per 256 rows, and the products run on tcgen05 with M = 128:
//   * keys are taken 128 at a time: the cached positions, then the drafted tokens, as one sequence.  Whole pages are
//     fetched by TMA, K and V of a page as one box each: the pool stores a row's 16-byte chunks swizzled by the slot, so a
//     box that takes a page as [8-row group][half of the dims][8 rows][64 dims] lands in shared memory in the arrangement
//     the tensor cores read (rows of 128 bytes, 128-byte swizzle), K as a K-major operand of the first product, V as an
//     MN-major operand of the second.  What lies behind the last whole page - the end of the cache, drafted tokens - is
//     copied row by row (cp.async), with zeros up to a multiple of 16 keys, where the second product stops: what a page
//     holds behind a trace's end never reaches it.  A row's probability of a drafted token that it does not see is 0, and 0
//     times an infinity or a NaN is NaN: the query warp looks at v of a piece's drafted tokens ahead of time, such elements
//     become zeros in the tile, and the rows that do see the token get them added behind the piece's output;
//   * scores S (128 x 128, fp32) are made in tensor memory; 128 threads, a row each, read them, keep the running maximum
//     and sum in fp32, and write the probabilities back as bf16 (one rounding, half a step of 2^-8 at most; the sum takes
//     them unrounded) over the same columns, from where they are the A operand of the second product, which adds to O
//     (128 x 128, fp32) in tensor memory.  bf16 because both operands of a product have one type and V's is bf16; the output
//     is rounded to it anyway, and the two roundings together are 2.3e-3 off in the 2-norm where the second alone makes
//     1.7e-3 (a second term of the probabilities would be half as many products again, in a kernel that above 128 rows waits
//     for them).  O is rescaled only when a row's maximum has grown by more than 2^8 (the probabilities are relative to an older
//     maximum until then; a published method), so the accumulators are almost never touched;
//   * two such chains ("lanes") run side by side in a CTA, so that the tensor cores work on one while the other is at
//     its softmax.  Up to 128 rows: the lanes take even and odd tiles of the same rows and are combined at the end.
//     More: the lanes take 128 rows each of the same tile, and 256 rows are one row group;
//   * the tiles of all (trace, KV head, row group) sequences form one stream - a sequence counts kSetup tiles more than it
//     has, which is about what beginning and ending one costs - that is cut into one equal contiguous share per CTA;
//     what a share holds of a sequence is a piece.  A piece that is not a whole sequence leaves its
//     (m, l, O) in the share's first or last slot, and tree_merge_kernel - a programmatic dependent - combines the pieces of
//     every sequence in stream order.  Row groups without a drafted token of theirs (a short tree) are not in the stream;
//   * query rows come by TMA too (a box: the group's heads of as many tokens as fit 128 rows), the next piece's
//     as soon as the last scores of the current one are made, so that the next piece's first scores overlap this one's last
//     softmax and its output.
// Warps: 4 + 4 softmax (lane 0, lane 1), one that fetches K, one for V (a TMA instruction takes its thread some 70 cycles:
// with both in one warp that warp set the pace), one that issues the products, one for the query rows.
// 64 traces x 16 nodes over 4.6k to 16.9k positions, 32 / 8 heads: 457 to 522 us from device to device, 2.83 GB at 5.4 to 6.2 TB/s
// (0.83 to 0.95 of the measured copy).  32 traces x 64 nodes over 2k to 25.6k positions, 64 / 8 heads: 854 to 1080 us (the
// power cap), 0.70 PFLOP at 0.65 to 0.82 PFLOP/s.  There a lane has one buffer for scores and probabilities, so that its softmax
// waits for the second product of this tile and the first of the next, and the other lane does not fill the gap: the tensor
// pipe is busy half of the time.  Also, in a trace's last row group whose drafted tokens fit the first 128 rows, the second
// lane works on rows that are not there (the number of lanes is one per launch): an eighth of all that case's work.
// A trace without drafted tokens has its tiles read all the same, for nothing.
// Every wait is bounded (kv_pool_set_wait_limit_ns); one that runs out raises STEP_ERR_TIMEOUT and the CTA winds down: no warp
// begins anything more, the products in flight are waited for, and when all warps are through and nothing new can start, so
// is every copy that was begun (each with a limit of its own).  Only then is the shared memory given up.
#include "attention_rows.cuh"
#include "async_copy.cuh"
#include "tensor_core.cuh"

#include <string.h>

using namespace stepk;

namespace {

constexpr int kP = 16, kD = 128;
constexpr int kTile = 128;                        // keys per tile
constexpr int kSetup = 4;                         // tiles' worth of time that a sequence takes besides its tiles (see above)
constexpr int kSlotBytes = kTile * kD * 2;        // K or V of one tile
constexpr int kQBytes = kHalfRows * kD * 2;       // 128 query rows, same arrangement
constexpr int kKSlots = 2, kVSlots = 3, kSlots = kKSlots + kVSlots;   // rings of K and of V tiles, 160 KiB: a V tile waits for its softmax
constexpr int kXCols = 16;                        // columns per round in which the lanes exchange their sums (below 128 rows)
constexpr int kXBytes = 2 * kXCols * kHalfRows * 4;
constexpr int kWarpK = 8, kWarpMma = 9, kWarpQ = 10, kWarpV = 11;
constexpr int kThreads = 384;                      // three warpgroups
constexpr int kRegsSoftmax = 208, kRegsOther = 88; // 2 x 128 x 208 + 128 x 88 = 384 x 168, what the launch has
constexpr int kTmemCols = 512;                    // S of both lanes (P over them), then O of both
constexpr float kRescale = 8.f;                   // log2 of how far a row's maximum may run ahead of its reference
constexpr unsigned long long kDrainNs = 100000000ull;

struct TreeArgs {
  const __nv_bfloat16* kv;
  const __nv_bfloat16* q; const __nv_bfloat16* k_draft; const __nv_bfloat16* v_draft;
  const int32_t* parents; const int32_t* n_nodes;
  const int32_t* block_table; const int32_t* seq_lens;
  __nv_bfloat16* out;
  float* ws_ml;                     // [share][2][group rows][2]
  float* ws_o;                      // [share][2][group rows][kD]
  int32_t* counters;
  int n, T, Hq, Hkv, G, L, layer, max_pages, num_blocks;
  int tokens;                       // drafted tokens whose heads fill a tile of query rows: 128 / G
  int lanes;                        // tiles of query rows in a group: 1 or 2
  int group_rows;                   // 128 or 256
  int shares;                       // CTAs of the attention launch
  float scale_log2;
  unsigned long long wait_ns;       // limit of every wait for a barrier
};

// ---- the stream of tiles
__device__ inline int cached(const TreeArgs& a, int t, bool flag) {
  int S = a.seq_lens[t];
  if (S < 0) S = 0;
  if ((long long)S > (long long)a.max_pages * kP) { S = a.max_pages * kP; if (flag) flag_error(a.counters, STEP_ERR_CAPACITY); }
  return S;
}
__device__ inline int nodes_of(const TreeArgs& a, int t, bool flag) {
  if (!a.n_nodes) return a.T;
  const int k = a.n_nodes[t];
  if (flag && (k < 0 || k > a.T)) flag_error(a.counters, STEP_ERR_INVALID_ARG);
  return min(max(k, 0), a.T);
}
// Trace t in the stream: tiles of a sequence, row groups that hold one of its drafted tokens (one at least: a trace without
// any key has one tile, of which nothing is written).
struct Shape { int S, nodes, tiles, groups; };
__device__ inline Shape shape_of(const TreeArgs& a, int t, bool flag) {
  Shape x;
  x.S = cached(a, t, flag);
  x.nodes = nodes_of(a, t, flag);
  const long long keys = (long long)x.S + x.nodes;
  x.tiles = keys > 0 ? (int)((keys + kTile - 1) / kTile) : 1;
  x.groups = max(1, (x.nodes + a.tokens * a.lanes - 1) / (a.tokens * a.lanes));
  return x;
}
// The stream: for every trace, for every KV head, for every row group, the sequence's tiles.  A warp's place in it:
struct Place { int t, hr, at; Shape x; };   // at: how far into the sequence, its kSetup counted first
// (64-bit divisions take hundreds of cycles and stand in front of a small call's first copies)
__device__ inline long long div_up(long long x, int by) {
  return x + by <= 0x7fffffffll ? (long long)((unsigned)(x + by - 1) / (unsigned)by) : (x + by - 1) / by;
}
// One warp: `total` tiles in all, W tiles per share; the place of position pos_of(W) if that lies inside the stream (else
// t = -1).  The first 32 traces' shapes are read once.
template <typename PosOf>
__device__ inline Place locate(const TreeArgs& a, int lane, bool flag, PosOf pos_of, long long& total, long long& W) {
  Shape x0 = {};
  long long sum = 0;
  for (int t = lane; t < a.n; t += 32) {
    const Shape x = shape_of(a, t, flag);
    if (t < 32) x0 = x;
    sum += (long long)(x.tiles + kSetup) * x.groups;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  total = sum * a.Hkv;
  W = div_up(total, a.shares);
  const long long pos = pos_of(W);
  Place p = {};
  p.t = -1;
  if (pos >= total) return p;
  long long run = 0;
  for (int base = 0; base < a.n; base += 32) {
    const int t = base + lane;
    Shape x = x0;
    if (base > 0) x = t < a.n ? shape_of(a, t, false) : Shape{};
    const long long mine = t < a.n ? (long long)(x.tiles + kSetup) * x.groups * a.Hkv : 0;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    const unsigned past = __ballot_sync(0xffffffffu, run + incl > pos);      // (lanes behind the last trace count nothing)
    if (past) {
      const int who = __ffs(past) - 1;
      const long long r = pos - (run + __shfl_sync(0xffffffffu, incl - mine, who));
      p.t = base + who;
      p.x.S = __shfl_sync(0xffffffffu, x.S, who);
      p.x.nodes = __shfl_sync(0xffffffffu, x.nodes, who);
      p.x.tiles = __shfl_sync(0xffffffffu, x.tiles, who);
      p.x.groups = __shfl_sync(0xffffffffu, x.groups, who);
      p.hr = r <= 0x7fffffffll ? (int)((unsigned)r / (unsigned)(p.x.tiles + kSetup)) : (int)(r / (p.x.tiles + kSetup));
      p.at = (int)(r - (long long)p.hr * (p.x.tiles + kSetup));
      return p;
    }
    run += __shfl_sync(0xffffffffu, incl, 31);
  }
  return p;
}
// What a share that ends at `end` holds of the sequence at place p (stream position pos): tiles [tile0, tile0 + cnt) of it,
// `len` of the stream.  (No tile at all only at the share's end, in front of a sequence's first.)
struct Part { int tile0, cnt; long long len; };
__device__ inline Part part_of(const Place& p, long long pos, long long end) {
  Part x;
  x.len = min((long long)(p.x.tiles + kSetup - p.at), end - pos);
  x.tile0 = max(0, p.at - kSetup);
  x.cnt = max(0, (int)(p.at + x.len) - kSetup) - x.tile0;
  return x;
}
// The place behind a whole rest of a sequence.
__device__ inline void next_sequence(const TreeArgs& a, Place& p) {
  p.at = 0;
  if (++p.hr < a.Hkv * p.x.groups) return;
  p.hr = 0;
  if (++p.t < a.n) p.x = shape_of(a, p.t, false);
}
// A piece, as the query warps announce it: tiles [tile0, tile0 + cnt) of the sequence's `tiles`.
struct Piece {
  int t, h, u0, tile0, cnt, tiles, S, nodes;
  unsigned long long odd;         // its drafted tokens whose v holds an infinity or a NaN
};

// ---- instructions
// One thread of a warp that is together (the same one every time).
__device__ inline bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ inline void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ inline void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ inline void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ inline void mbar_arrive_n(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// 16 bytes, or 16 zero bytes (src is then not read)
__device__ inline void cp_async16_or_zero(uint32_t dst, const void* src, bool real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
// 32 columns of this thread's TMEM lane, without waiting for them
__device__ inline void tc_ld32_async(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ inline void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// The values of an asynchronous load may be used only behind the wait: ties them to this place.
template <int N> __device__ inline void pin(uint32_t* r) {
#pragma unroll
  for (int i = 0; i < N; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
__device__ inline void tc_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
         "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
         "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
         "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
         "r"(taddr) : "memory");
}
__device__ inline void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] * B[smem]
__device__ inline void tc_mma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// A K or V tile in a ring slot: groups of 8 rows (tokens), a group as two halves of 8 rows x 128 bytes with the 128-byte
// swizzle.  Byte offset of 16-byte chunk `at` (0 .. 15, as stored) of row rr:
__device__ inline uint32_t tile_chunk(int rr, int at) { return (rr >> 3) * 2048 + (at >> 3) * 1024 + (rr & 7) * 128 + (at & 7) * 16; }
// K as a K-major operand: the next 8 keys (N) are 2048 bytes further; dims from 64 on start 1024 bytes further.
__device__ inline uint64_t umma_desc_k(uint32_t smem_addr) {
  const uint32_t lo = ((smem_addr >> 4) & 0x3FFFu) | (1u << 16);
  const uint32_t hi = (2048u >> 4) | (1u << 14) | (2u << 29);
  return ((uint64_t)hi << 32) | lo;
}
// V as an MN-major operand: 64 of the N index (dims) are 128 contiguous bytes, the next 64 lie 1024 bytes further (leading
// byte offset), the next 8 of the K index (tokens) 2048 bytes (stride byte offset).
__device__ inline uint64_t umma_desc_v(uint32_t smem_addr) {
  const uint32_t lo = ((smem_addr >> 4) & 0x3FFFu) | ((1024u >> 4) << 16);
  const uint32_t hi = (2048u >> 4) | (1u << 14) | (2u << 29);
  return ((uint64_t)hi << 32) | lo;
}
// 32 bytes (a whole sector) per thread
__device__ inline void st_global32(void* dst, const uint32_t* r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(dst), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// Two fp32 operations in one instruction.
__device__ inline void fma2(float& x, float& y, float ax, float ay, float b, float c) {
  asm("{\n\t.reg .b64 a, b, c, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%5, %5};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(x), "=f"(y) : "f"(ax), "f"(ay), "f"(b), "f"(c));
}
__device__ inline void add2(float& x, float& y, float ax, float ay) {
  asm("{\n\t.reg .b64 a, b, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%0, %1};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "+f"(x), "+f"(y) : "f"(ax), "f"(ay));
}
__device__ inline float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ inline uint32_t pack2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Whether one of a pair of bf16 values is an infinity or a NaN; the pair with zeros for those.
__device__ inline bool not_finite(uint32_t pair) { return ((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ inline uint32_t only_finite(uint32_t pair) {
  return pair & ((pair & 0x7f80u) == 0x7f80u ? 0xffff0000u : ~0u) & ((pair & 0x7f800000u) == 0x7f800000u ? 0xffffu : ~0u);
}
// One warp: those of drafted tokens [u0, u1) of trace t whose v holds an infinity or a NaN.
__device__ inline unsigned long long odd_tokens(const TreeArgs& a, int t, int h, int u0, int u1, int lane) {
  const __nv_bfloat16* v = a.v_draft + (((size_t)t * a.T * a.L + a.layer) * a.Hkv + h) * kD + (lane & 15) * 8;
  uint32_t lo = 0u, hi = 0u;
  for (int u = u0 + (lane >> 4); u < u1; u += 16) {
    uint4 x[8];
#pragma unroll
    for (int y = 0; y < 8; ++y)
      x[y] = u + 2 * y < u1 ? *reinterpret_cast<const uint4*>(v + (size_t)(u + 2 * y) * a.L * a.Hkv * kD) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int y = 0; y < 8; ++y)
      if (not_finite(x[y].x) || not_finite(x[y].y) || not_finite(x[y].z) || not_finite(x[y].w)) {
        const uint32_t bit = 1u << ((u + 2 * y) & 31);
        if (u + 2 * y < 32) lo |= bit; else hi |= bit;
      }
  }
  return (unsigned long long)__reduce_or_sync(0xffffffffu, hi) << 32 | __reduce_or_sync(0xffffffffu, lo);
}
// One warp, when the rows of piece pc have been written (slot: of this share, if the piece is not a whole sequence): what is
// not finite in v of its odd tokens is added to the rows that see them.
__device__ inline void add_odd(const TreeArgs& a, const Piece& pc, int slot, int lane) {
#pragma unroll 1
  for (int r = 0; r < a.group_rows; ++r) {
    const int row = r % kHalfRows, u = pc.u0 + r / kHalfRows * a.tokens + row / a.G;
    if (row >= a.tokens * a.G || u >= pc.nodes) continue;
    __nv_bfloat16* out = a.out + (((size_t)pc.t * a.T + u) * a.Hq + (size_t)pc.h * a.G + row % a.G) * kD;
    float* o_out = a.ws_o + (((size_t)blockIdx.x * 2 + slot) * a.group_rows + r) * kD;
#pragma unroll 1
    for (int w = u; w >= 0;) {
      const __nv_bfloat16* v = a.v_draft + ((((size_t)pc.t * a.T + w) * a.L + a.layer) * a.Hkv + pc.h) * kD;
      if ((pc.odd >> w) & 1)
#pragma unroll 1
        for (int c = lane; c < kD; c += 32) {
          const float x = __bfloat162float(v[c]);
          if ((__float_as_uint(x) & 0x7f800000u) != 0x7f800000u) continue;
          if (pc.cnt == pc.tiles) out[c] = __float2bfloat16(__bfloat162float(out[c]) + x);
          else o_out[c] += x;
        }
      const int up = a.parents[(size_t)pc.t * a.T + w];
      w = up < w ? up : -1;
    }
  }
}

template <bool kTwoRows>   // the lanes take 128 rows each of a 256-row group; else even and odd tiles of the same 128 rows
__global__ void __launch_bounds__(kThreads, 1) tree_tc_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ TreeArgs a) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* sm = smem_raw + (base - raw);
  constexpr int kQAll = (kTwoRows ? 2 : 1) * kQBytes, kX = kTwoRows ? 0 : kXBytes;
  const uint32_t sm_q = base, sm_ring = base + kQAll + kX;
  float* s_x = reinterpret_cast<float*>(sm + kQAll);                   // [2][kXCols][128]: columns lane 0 gives, lane 1 gives
  unsigned char* tail = sm + kQAll + kX + kSlots * kSlotBytes;
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(tail);
  unsigned long long* s_mask = reinterpret_cast<unsigned long long*>(s_bar + 32);   // [2][64] by piece parity
  Piece* s_piece = reinterpret_cast<Piece*>(s_mask + 128);             // [2]
  int* s_up = reinterpret_cast<int*>(s_piece + 2);                     // [64]
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_up + 64);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_begun = reinterpret_cast<int*>(s_tmem + 4);                   // [3] how many fills of their buffers the K, V and query warps have begun
  float* s_ml = reinterpret_cast<float*>(s_tmem + 8);                  // [2][128][2] (below 128 rows)
  const uint32_t bars = smem_u32(s_bar);
  const uint32_t bar_full = bars, bar_empty = bars + 8 * kSlots;
  const uint32_t bar_q = bars + 16 * kSlots, bar_s = bar_q + 8, bar_p = bar_s + 16, bar_o = bar_p + 32,
                 bar_both = bar_o + 16, bar_qfree = bar_both + 8, bar_drain = bar_qfree + 8;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    prefetch_map(&map);
    prefetch_map(&map_q);
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(bar_full + 8 * s, 33);              // a fetching warp's threads, and its announcement of bytes
      mbar_init(bar_empty + 8 * s, 1);              // tcgen05.commit
    }
    mbar_init(bar_q, 1);                            // the query warp's announcement
    mbar_init(bar_qfree, 9);                        // tcgen05.commit: a piece's last scores; all softmax warps have begun it
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_s + 8 * s, 1);                  // tcgen05.commit: scores made (and the products before them done)
      mbar_init(bar_p + 8 * s, 4);                  // (one arrival per warp: arrivals at one barrier queue up)
      mbar_init(bar_p + 16 + 8 * s, 4);             // the first half of the probabilities (above 128 rows)
      mbar_init(bar_o + 8 * s, 1);                  // tcgen05.commit: a piece's last product
    }
    mbar_init(bar_both, 8);
    mbar_init(bar_drain, 1);
    *s_abort = 0;
    mbar_init_fence();
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  dependents_may_launch();
  const uint32_t tmem = *s_tmem;
  // this CTA's share of the stream and the place it begins at: every warp that walks it asks
  auto my_share = [&](bool flag, long long& pos0, long long& end) {
    long long total, W;
    const Place p = locate(a, lane, flag, [](long long w) { return (long long)blockIdx.x * w; }, total, W);
    pos0 = min(total, (long long)blockIdx.x * W);
    end = min(total, pos0 + W);
    return p;
  };

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

  int last_piece = -1, last_slot = 0;                                  // (query warp) whose rows are written when all is done
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // ------------------------------------------------ softmax: lane `ln` of the CTA, row `row` of its 128
    const int ln = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t t_s = t_row + ln * 128, t_o = t_row + 256 + ln * 128;
    uint32_t ph_s = 0, ph_piece = 0, ph_both = 0;
    bool ok = true, first = true;
    for (;;) {
      if (!wait_warp(bar_q, ph_piece)) { ok = false; break; }
      const Piece pc = s_piece[ph_piece];
      if (pc.cnt == 0) break;                                          // the share is done
      const int S = pc.S, u = pc.u0 + (kTwoRows ? ln * a.tokens : 0) + row / a.G;
      const bool mine = row < a.tokens * a.G && u < pc.nodes;
      const unsigned long long sees = mine ? s_mask[ph_piece * 64 + u] : 0ull;
      arrive_warp(bar_qfree);

      float m_ref = -INFINITY, l = 0.f;
      bool started = false;
      for (int i = kTwoRows ? 0 : ln; i < pc.cnt; i += kTwoRows ? 1 : 2) {
        if (!wait_warp(bar_s + 8 * ln, ph_s)) { ok = false; break; }
        ph_s ^= 1;
        tc_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tc_ld32_async(t_s + 32 * c, s + 32 * c);
        tc_wait_ld();
        pin<128>(s);
        const int j0 = (pc.tile0 + i) * kTile;
        if (j0 + kTile > S) {                                          // the end of the cache, drafted tokens
#pragma unroll
          for (int c = 0; c < kTile; ++c) {
            const int j = j0 + c - S;                                  // < 0: cached; else drafted token j
            const bool see = j < 0 || (j < 64 && ((sees >> (j & 63)) & 1));
            if (!see) s[c] = 0xff800000u;
          }
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
        // (in halves where the tensor cores wait for it: the second product of the first 64 keys runs while the others'
        // probabilities are made)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int c = half * 64; c < half * 64 + 64; c += 2) {
            float p0, p1;
            fma2(p0, p1, __uint_as_float(s[c]), __uint_as_float(s[c + 1]), a.scale_log2, -off);
            p0 = exp2f(p0);
            p1 = exp2f(p1);
            add2(sum[c & 2], sum[(c & 2) + 1], p0, p1);
            s[c / 2] = pack2(p0, p1);
          }
          tc_st32(t_s + half * 32, s + half * 32);
          if (kTwoRows || half == 1) {
            tc_wait_st();
            tc_fence_before();
            arrive_warp(bar_p + 8 * (half == 0 ? 2 + ln : ln));
          }
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      if (!ok || !wait_warp(bar_o + 8 * ln, ph_piece)) { ok = false; break; }
      tc_fence_after();
      ph_piece ^= 1;

      // ---- the piece is done
      const bool whole = pc.cnt == pc.tiles;
      const size_t slot = (size_t)blockIdx.x * 2 + (first ? 0 : 1);
      first = false;
      float2* ml_out = reinterpret_cast<float2*>(a.ws_ml) + slot * a.group_rows + (kTwoRows ? ln * 128 : 0) + row;
      float* o_out = a.ws_o + (slot * a.group_rows + (kTwoRows ? ln * 128 : 0) + row) * kD;
      __nv_bfloat16* out = a.out + (((size_t)pc.t * a.T + (mine ? u : 0)) * a.Hq + (size_t)pc.h * a.G + (mine ? row % a.G : 0)) * kD;
      // N columns, from c on, of this thread's row
      auto put = [&](int c, uint32_t* o, int N, float inv) {
        if (!mine) return;
        if (whole) {
#pragma unroll
          for (int x = 0; x < N / 2; ++x) o[x] = pack2(__uint_as_float(o[2 * x]) * inv, __uint_as_float(o[2 * x + 1]) * inv);
#pragma unroll
          for (int x = 0; x < N / 2; x += 8) st_global32(out + c + 2 * x, o + x);
        } else {
#pragma unroll
          for (int x = 0; x < N; x += 8) st_global32(o_out + c + x, o + x);
        }
      };
      if constexpr (kTwoRows) {
        if (!whole && mine) *ml_out = make_float2(m_ref, l);
        const float inv = 1.f / l;
#pragma unroll
        for (int c = 0; c < kD; c += 64) {
          uint32_t o[64];
          tc_ld32_async(t_o + c, o);
          tc_ld32_async(t_o + c + 32, o + 32);
          tc_wait_ld();
          pin<64>(o);
          put(c, o, 32, inv);
          put(c + 32, o + 32, 32, inv);
        }
      } else {
        // the two lanes hold the even and the odd tiles of the same rows: each takes 64 columns of the sum, the other
        // lane's part of them through shared memory
        s_ml[(ln * 128 + row) * 2] = m_ref;
        s_ml[(ln * 128 + row) * 2 + 1] = l;
        const bool some = ln < pc.cnt;                                 // a piece of one tile leaves lane 1 without any
        uint32_t o[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tc_ld32_async(t_o + 32 * c, o + 32 * c);
        tc_wait_ld();
        pin<128>(o);
        if (!some) {
#pragma unroll
          for (int c = 0; c < 128; ++c) o[c] = 0u;
        }
        if (ln) {                                                      // so that o[0 .. 63] are kept, o[64 .. 127] given
#pragma unroll
          for (int c = 0; c < 64; ++c) { const uint32_t x = o[c]; o[c] = o[64 + c]; o[64 + c] = x; }
        }
        float w_own = 0.f, w_other = 0.f, inv = 0.f;
#pragma unroll
        for (int c = 0; c < 64; c += kXCols) {
#pragma unroll
          for (int x = 0; x < kXCols; ++x) s_x[(ln * kXCols + x) * 128 + row] = __uint_as_float(o[64 + c + x]);
          arrive_warp(bar_both);
          if (!wait_warp(bar_both, ph_both)) { ok = false; break; }
          ph_both ^= 1;
          if (c == 0) {
            const float m0 = s_ml[row * 2], m1 = s_ml[(128 + row) * 2], l0 = s_ml[row * 2 + 1], l1 = s_ml[(128 + row) * 2 + 1];
            const float M = fmaxf(m0, m1), off = M == -INFINITY ? 0.f : M;
            const float w0 = exp2f(m0 - off), w1 = exp2f(m1 - off);
            const float lsum = l0 * w0 + l1 * w1;
            inv = 1.f / lsum;
            w_own = ln == 0 ? w0 : w1;
            w_other = ln == 0 ? w1 : w0;
            if (!whole && mine && ln == 0) *ml_out = make_float2(M, lsum);
          }
#pragma unroll
          for (int x = 0; x < kXCols; ++x)
            o[c + x] = __float_as_uint(__uint_as_float(o[c + x]) * w_own + s_x[((1 - ln) * kXCols + x) * 128 + row] * w_other);
          put((ln == 0 ? 0 : 64) + c, o + c, kXCols, inv);
          arrive_warp(bar_both);                                       // the exchange area may be written again
          if (!wait_warp(bar_both, ph_both)) { ok = false; break; }
          ph_both ^= 1;
        }
        if (!ok) break;
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
   if (warp == kWarpK || warp == kWarpV) {
    // ------------------------------------------------ K or V tiles into their ring
    const int kv = warp == kWarpV, ring0 = kv ? kKSlots : 0, ring_n = kv ? kVSlots : kKSlots;
    int slot = 0, begun = 0;                                           // (fills begun)
    uint32_t ph = 1;
    bool ok = true;
    Place pl = {};
    int h = 0;
    // Block ids of 64 pages (eight tiles): lane i holds those of pages win + i and win + 32 + i.  The second half is asked
    // for when the first is entered, four tiles before it is needed: with a read of the table in front of every tile, the read's
    // latency set the pace of the whole kernel (1,800 cycles a tile and operand).
    int win = 0, ids0 = 0, ids1 = 0;
    Part part = {};
    auto load_ids = [&](const Place& of, int first) {
      const int page = first + lane;
      return of.t >= 0 && of.t < a.n && (long long)page * kP < of.x.S ? a.block_table[(size_t)of.t * a.max_pages + page] : 0;
    };
    // tile i of the piece into the next slot
    auto fetch = [&](int i) {
      if (!ok) return;
      if (!wait_warp(bar_empty + 8 * (ring0 + slot), ph)) { ok = false; return; }
      const uint32_t bar = bar_full + 8 * (ring0 + slot), dst = sm_ring + (ring0 + slot) * kSlotBytes;
      const int j0 = (part.tile0 + i) * kTile;
      const int S = pl.x.S, nodes = pl.x.nodes;
      if (j0 / kP >= win + 32) { win += 32; ids0 = ids1; ids1 = load_ids(pl, win + 32); }
      const int in_win = j0 / kP - win;
      // block of page pg (0 .. 7) of this tile; one out of range is flagged and read as block 0
      auto block_of = [&](int pg) {
        int bb = __shfl_sync(0xffffffffu, in_win < 32 ? ids0 : ids1, (in_win + pg) & 31);
        if (bb < 0 || bb >= a.num_blocks) { flag_error(a.counters, STEP_ERR_BAD_BLOCK); bb = 0; }
        return bb;
      };
      // whole pages by TMA; behind the last of them (the end of the cache, drafted tokens) row by row, zeros up to a
      // multiple of 16 keys, which is as far as the second product goes
      const int pages = min(kTile / kP, max(0, (S - j0) / kP));
      if (lane == 0 && pages > 0) mbar_expect_tx(bar, pages * (kP * kD * 2));
      __syncwarp();
      const int own = block_of(lane & 7);
      if (lane < pages)                                                // a box is the K or the V of a page
        tma_load_4d(dst + lane * (kP * kD * 2), &map, 0, 0, 0, ((((a.layer * a.num_blocks) + own) * a.Hkv + h) * 2 + kv) * (kP / 8), bar);
      if (pages == kTile / kP) {
        if (lane == 0) mbar_arrive_n(bar, 32);
      } else {
        // two rows of 16 chunks at a time; a cached row is copied as it is stored, which is the arrangement wanted here
        const int c = lane & 15, rows = min(kTile, (S + nodes - j0 + 15) & ~15);
        const int bb = block_of(pages);                                // the page that the cache ends in
        const __nv_bfloat16* tail = a.kv + ((((size_t)a.layer * a.num_blocks + bb) * a.Hkv + h) * 2 + kv) * (kP * kD) + c * 8;
        const __nv_bfloat16* draft = (kv ? a.v_draft : a.k_draft) + (((size_t)pl.t * a.T * a.L + a.layer) * a.Hkv + h) * kD + c * 8;
        const size_t draft_row = (size_t)a.L * a.Hkv * kD;
#pragma unroll 4
        for (int rr = pages * kP + (lane >> 4); rr < rows; rr += 2) {
          const int j = j0 + rr;
          const bool real = j < S + nodes;
          const __nv_bfloat16* src = j < S ? tail + (rr % kP) * kD : (real ? draft + (size_t)(j - S) * draft_row : a.kv);
          cp_async16_or_zero(dst + tile_chunk(rr, j < S ? c : (c & 8) | ((c ^ rr) & 7)), src, real);
        }
        cp_async_arrive_when_done(bar);
        if (lane == 0 && pages == 0) mbar_arrive(bar);                 // (the announcement of bytes is the other form of this arrival)
      }
      __syncwarp();
      ++begun;
      if (++slot == ring_n) { slot = 0; ph ^= 1; }
    };
    long long pos, end;
    pl = my_share(kv == 0 && blockIdx.x == 0, pos, end);
    part = part_of(pl, pos, end);
    const int win0 = (part.tile0 * (kTile / kP)) & ~31;
    int next0 = load_ids(pl, win0), next1 = load_ids(pl, win0 + 32);
    while (pos < end && ok) {
      part = part_of(pl, pos, end);
      h = pl.hr / pl.x.groups;
      win = (part.tile0 * (kTile / kP)) & ~31;
      ids0 = next0;
      ids1 = next1;
      Place nx = pl;                                                   // the sequence behind this one, its block ids too
      next_sequence(a, nx);
      next0 = load_ids(nx, 0);
      next1 = load_ids(nx, 32);
      for (int i = 0; i < part.cnt; ++i) fetch(i);
      pos += part.len;
      pl = nx;
    }
    cp_async_wait_all();
    if (lane == 0) s_begun[kv] = begun;
  } else if (warp == kWarpQ) {
    // ------------------------------------------------ query rows and ancestor masks of one piece after another
    uint32_t par = 0;
    int made = 0, begun = 0;                                           // pieces announced; those and the end of the share
    if (lane == 0) s_begun[2] = 0;
    long long pos, end;
    Place pl = my_share(false, pos, end);
    for (;; par ^= 1) {
      Piece pc = {};
      Part part = {};
      if (pos < end) part = part_of(pl, pos, end);
      if (part.cnt > 0) {
        pc.t = pl.t; pc.h = pl.hr / pl.x.groups; pc.u0 = (pl.hr - pc.h * pl.x.groups) * a.tokens * a.lanes;
        pc.tile0 = part.tile0; pc.cnt = part.cnt; pc.tiles = pl.x.tiles; pc.S = pl.x.S; pc.nodes = pl.x.nodes;
        int up[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) up[x] = lane + 32 * x < pc.nodes ? a.parents[(size_t)pc.t * a.T + lane + 32 * x] : -1;
        pc.odd = odd_tokens(a, pc.t, pc.h, max(0, pc.tile0 * kTile - pc.S), min(pc.nodes, (pc.tile0 + pc.cnt) * kTile - pc.S), lane);
#pragma unroll
        for (int x = 0; x < 2; ++x) {                                  // (the other piece's masks are the ones in use)
          const int u = lane + 32 * x;
          int p = up[x];
          if (u >= pc.nodes) break;
          if (p >= u || p < -1) { flag_error(a.counters, STEP_ERR_INVALID_ARG); p = -1; }
          s_up[u] = p;
        }
        __syncwarp();
        for (int u = lane; u < pc.nodes; u += 32) {
          unsigned long long m = 0;
          for (int w = u; w >= 0; w = s_up[w]) m |= 1ull << w;
          s_mask[par * 64 + u] = m;
        }
        __syncwarp();
        pos += part.len;
        next_sequence(a, pl);
      }
      // the scores of the piece before are made, and its announcement has been read (the very first wait passes at once)
      if (!wait_warp(bar_qfree, par ^ 1)) break;
      // all softmax warps have begun that piece, so the one before it is written
      if (made >= 2 && s_piece[par].odd) add_odd(a, s_piece[par], made == 2 ? 0 : 1, lane);
      __syncwarp();
      if (pc.cnt > 0) ++made;
      if (lane == 0) {
        s_piece[par] = pc;
        if (pc.cnt > 0) {
          // (rows of tokens that the trace does not have may come along: a row of the products depends on its own query only)
          const int tiles = kTwoRows && pc.u0 + a.tokens < pc.nodes ? 2 : 1, box = min(a.tokens, a.T) * a.G * 128;
          mbar_expect_tx(bar_q, 2 * tiles * box);
          for (int x = 0; x < 2 * tiles; ++x)
            tma_load_3d(sm_q + (x >> 1) * kQBytes + (x & 1) * (kQBytes / 2), &map_q, (x & 1) * 64, pc.h * a.G, pc.t * a.T + pc.u0 + (x >> 1) * a.tokens, bar_q);
        } else {
          mbar_arrive(bar_q);
        }
      }
      __syncwarp();
      if (lane == 0) s_begun[2] = ++begun;
      if (pc.cnt == 0) break;
    }
    last_piece = made > 0 ? (int)(par ^ 1) : -1;
    last_slot = made > 1;
    // out rows behind a trace's last drafted token
    for (int t = blockIdx.x; t < a.n; t += gridDim.x) {
      const int nodes = nodes_of(a, t, false);
      uint4* dst = reinterpret_cast<uint4*>(a.out + ((size_t)t * a.T + nodes) * a.Hq * kD);
      const int chunks = (a.T - nodes) * a.Hq * (kD / 8);
      for (int x = lane; x < chunks; x += 32) dst[x] = make_uint4(0, 0, 0, 0);
    }
  } else {
    // ------------------------------------------------ products.  The tensor cores take the next few instructions only, so
    // every cycle this warp spends between them is idle time there once they are what limits the kernel (more than 128
    // rows).  Hence: the warp stays together and one thread is elected for the instructions (a wait in a single thread's
    // branch costs twice the cycles), and what is likely there long since is waited for before what is not.
    const uint32_t id_qk = umma_idesc_bf16(kTile), id_pv = umma_idesc_bf16(kD) | (1u << 16);   // B of the second is MN-major
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    int at[2] = {0, 0};
    uint32_t ph[2] = {0, 0}, ph_q = 0, ph_p[2] = {0, 0};
    bool ok = true;
    // waits for the next tile of K (0) or V (1); its slot.  Rows copied by cp.async came through the generic proxy.
    auto next = [&](int kv, bool copied) -> int {
      const int s = (kv ? kKSlots : 0) + at[kv];
      ok = ok && wait_warp(bar_full + 8 * s, ph[kv]);
      if (copied) fence_async_smem();
      if (++at[kv] == (kv ? kVSlots : kKSlots)) { at[kv] = 0; ph[kv] ^= 1; }
      return s;
    };
    auto probabilities = [&](int ln, bool first_half) {
      ok = ok && wait_warp(bar_p + 8 * (first_half ? 2 + ln : ln), ph_p[ln]);
      if (!first_half) ph_p[ln] ^= 1;
      tc_fence_after();
    };
    // (the elected thread's part of it)
    auto scores = [&](int ln, int s) {
      const uint32_t qa = sm_q + (kTwoRows ? ln * kQBytes : 0), kb = sm_ring + s * kSlotBytes;
#pragma unroll
      for (int x = 0; x < 8; ++x)
        tc_mma_bf16(tm + ln * 128, umma_desc_sw128(qa + (x >> 2) * (kQBytes / 2) + (x & 3) * 32),
                    umma_desc_k(kb + (x >> 2) * 1024 + (x & 3) * 32), id_qk, x != 0);
      tc_commit(bar_s + 8 * ln);
    };
    // steps of 16 keys; those of a tile behind the last key are left out, so nothing that lies there matters
    auto values = [&](int ln, int s, bool first, int from, int steps) {
      const uint32_t vb = sm_ring + s * kSlotBytes;
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (x >= from && x < steps) tc_mma_bf16_ta(tm + 256 + ln * 128, tm + ln * 128 + x * 8, umma_desc_v(vb + x * 4096), id_pv, !(first && x == 0));
    };
    while (ok) {
      ok = wait_warp(bar_q, ph_q);
      const int cnt = s_piece[ph_q].cnt, S = s_piece[ph_q].S - s_piece[ph_q].tile0 * kTile, keys = S + s_piece[ph_q].nodes;
      const unsigned long long odd = s_piece[ph_q].odd;
      auto copied = [&](int i) { return (i + 1) * kTile > S; };
      // zeros for what is not finite in v of drafted tokens (tile i of the piece, in slot s)
      auto tame = [&](int i, int s) {
        if (odd == 0 || !copied(i)) return;
        for (int rr = lane >> 4; rr < kTile; rr += 2) {
          const int u = i * kTile + rr - S, c = lane & 15;
          if (u < 0 || u >= keys - S || !((odd >> u) & 1)) continue;
          uint4* x = reinterpret_cast<uint4*>(sm + (sm_ring - base) + s * kSlotBytes + tile_chunk(rr, c));
          *x = make_uint4(only_finite(x->x), only_finite(x->y), only_finite(x->z), only_finite(x->w));
        }
        fence_async_smem();
        __syncwarp();
      };
      auto steps = [&](int i) { return min(8, (keys - i * kTile + 15) / 16); };
      ph_q ^= 1;
      if (!ok || cnt == 0) break;
      tc_fence_after();
      if constexpr (kTwoRows) {
        int k = next(0, copied(0));
        if (ok && elect_one()) {
          scores(0, k);
          scores(1, k);
          tc_commit(bar_empty + 8 * k);
          if (cnt == 1) tc_commit(bar_qfree);
        }
        for (int i = 0; i < cnt && ok; ++i) {
          const int v = next(1, copied(i));
          if (ok) tame(i, v);
          const bool more = i + 1 < cnt;
          if (more) k = next(0, copied(i + 1));
          probabilities(0, true);
          if (ok && elect_one()) values(0, v, i == 0, 0, min(4, steps(i)));
          __syncwarp();
          probabilities(0, false);
          if (ok && elect_one()) {
            values(0, v, i == 0, 4, steps(i));
            if (more) scores(0, k); else tc_commit(bar_o);
          }
          __syncwarp();
          probabilities(1, true);
          if (ok && elect_one()) values(1, v, i == 0, 0, min(4, steps(i)));
          __syncwarp();
          probabilities(1, false);
          if (ok && elect_one()) {
            values(1, v, i == 0, 4, steps(i));
            tc_commit(bar_empty + 8 * v);
            if (more) { scores(1, k); tc_commit(bar_empty + 8 * k); } else tc_commit(bar_o + 8);
            if (i + 2 == cnt) tc_commit(bar_qfree);
          }
          __syncwarp();
        }
      } else {
        // (bound by the stream of tiles: the second product does not wait for a tile of K)
        for (int i = 0; i < min(cnt, 2); ++i) {
          const int k = next(0, copied(i));
          if (ok && elect_one()) {
            scores(i, k);
            tc_commit(bar_empty + 8 * k);
            if (i + 1 == cnt) tc_commit(bar_qfree);
          }
          __syncwarp();
        }
        for (int i = 0; i < cnt && ok; ++i) {
          const int v = next(1, copied(i));
          if (ok) tame(i, v);
          probabilities(i & 1, false);
          if (ok && elect_one()) {
            values(i & 1, v, i < 2, 0, steps(i));
            tc_commit(bar_empty + 8 * v);
            if (i + 2 >= cnt) tc_commit(bar_o + 8 * (i & 1));
            if (cnt == 1) tc_commit(bar_o + 8);                        // lane 1 has nothing to do
          }
          __syncwarp();
          if (i + 2 < cnt) {
            const int k = next(0, copied(i + 2));
            if (ok && elect_one()) {
              scores(i & 1, k);
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
      tc_commit(bar_drain);                                            // no product is in flight when the tensor memory goes back
      mbar_wait_bounded(bar_drain, 0);
    }
    __syncwarp();
  }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  // A wait has run out: copies in flight still write this CTA's shared memory.  (Decided here, where no warp can begin one any
  // more and *s_abort is final: a fetching warp may be through with its share before another warp's wait runs out.)
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
  if (warp == kWarpQ && last_piece >= 0 && !*s_abort && s_piece[last_piece].odd) add_odd(a, s_piece[last_piece], last_slot, lane);
  if (warp == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Combines the pieces of every sequence that more than one share holds.  A CTA takes one border between two shares (and 32
// of the rows): if the sequence it cuts has no border before it, the CTA combines all of that sequence's pieces, a warp per
// query row, lanes over the 128 dims, in stream order with a running (max, sum, weighted values).  The same bits whatever
// ran when.  The search stands in front of the wait for the attention kernel: it runs early on SMs that have no CTA of that
// kernel left (beside one there are no registers for it).
constexpr int kMergeWarps = 8, kMergeRows = 32;

__global__ void __launch_bounds__(kMergeWarps * 32) tree_merge_kernel(TreeArgs a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __shared__ Place s_place;
  __shared__ long long s_W;
  const int w0 = blockIdx.x;                                           // the share in front of the border
  if (warp == 0) {
    long long total, W;
    const Place p = locate(a, lane, false, [&](long long w) { return (w0 + 1) * w; }, total, W);
    if (lane == 0) { s_place = p; s_W = W; }
  }
  __syncthreads();
  wait_for_primary();
  const Place p = s_place;
  const long long W = s_W, start = (w0 + 1) * W - p.at;                // where the sequence begins
  // no border, no cut, or not the sequence's first cut
  if (p.t < 0 || p.at <= kSetup || start + kSetup < w0 * W) return;
  const int h = p.hr / p.x.groups, u0 = (p.hr - h * p.x.groups) * a.tokens * a.lanes;
  const int w1 = (int)((start + kSetup + p.x.tiles - 1) / W);
  for (int rr = blockIdx.y * kMergeRows + warp; rr < (int)(blockIdx.y + 1) * kMergeRows; rr += kMergeWarps) {
    const int row = rr % kHalfRows, u = u0 + rr / kHalfRows * a.tokens + row / a.G;
    if (row >= a.tokens * a.G || u >= p.x.nodes) continue;
    float M = -INFINITY, den = 0.f;
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int w = w0; w <= w1; ++w) {
      const size_t slot = (size_t)w * 2 + (start <= (long long)w * W ? 0 : 1);
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(a.ws_ml + (slot * a.group_rows + rr) * 2));
      const float4 o = __ldcg(reinterpret_cast<const float4*>(a.ws_o + (slot * a.group_rows + rr) * kD) + lane);
      const float Mb = fmaxf(M, ml.x), off = Mb == -INFINITY ? 0.f : Mb;   // a row may see nothing of a piece
      const float keep = exp2f(M - off), wgt = exp2f(ml.x - off);
      den = den * keep + wgt * ml.y;
      num.x = num.x * keep + wgt * o.x; num.y = num.y * keep + wgt * o.y;
      num.z = num.z * keep + wgt * o.z; num.w = num.w * keep + wgt * o.w;
      M = Mb;
    }
    const float inv = 1.f / den;
    reinterpret_cast<uint2*>(a.out + (((size_t)p.t * a.T + u) * a.Hq + (size_t)h * a.G + row % a.G) * kD)[lane] =
        make_uint2(pack2(num.x * inv, num.y * inv), pack2(num.z * inv, num.w * inv));
  }
}

size_t smem_bytes(bool two_rows) {
  return 1024 + (two_rows ? 2 * kQBytes : kQBytes + kXBytes + 512 * 4) + kSlots * kSlotBytes + 32 * 8 + 128 * 8 + 2 * sizeof(Piece) + 64 * 4 + 32;
}
static_assert(1024 + 2 * kQBytes + kSlots * kSlotBytes + 32 * 8 + 128 * 8 + 2 * sizeof(Piece) + 64 * 4 + 32 <= 232448, "shared memory of one CTA");

}  // namespace

namespace stepk {

bool tree_tc_supported(const step_pool* pool, int n) {
  const kv_pool_config& c = pool->cfg;
  return c.dtype == STEP_BF16 && c.head_dim == kD && c.page_size == kP && pool->swizzle && n <= kMaxTracesFast && pool->fast_path > 0 &&
         (long long)c.num_layers * c.num_blocks * c.num_kv_heads * 2 * kP < (1ll << 31) && encode_tiled_fn() != nullptr;
}

size_t tree_tc_workspace(const step_pool* pool, int T) {
  const size_t rows = T > kHalfRows / pool->G ? 2 * kHalfRows : kHalfRows;
  return (size_t)pool->num_sms * 2 * rows * (kD + 2) * sizeof(float);
}

int tree_tc_launch(step_pool* pool, int layer, const void* q, const void* k_draft, const void* v_draft, const int32_t* parents,
                   const int32_t* n_nodes, int T, const int32_t* block_table, const int32_t* seq_lens, int n, void* out,
                   void* workspace, cudaStream_t s) {
  const Geo g = geo_of(pool);
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return STEP_ERR_CUDA;
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  if (!pool->tree_ready) {
    // the pool as groups of 8 rows of 128 dims, seen as [group][half of the dims][row][64 dims]; a box is the two groups of a
    // page's K or V
    CUtensorMap fresh;
    static_assert(sizeof(fresh) <= sizeof(pool->tmap_kv_bytes), "tensor map");
    const cuuint64_t dims[4] = {64, 8, 2, (cuuint64_t)g.L * g.num_blocks * g.Hkv * 2 * (kP / 8)};
    const cuuint64_t strides[3] = {256, 128, 2048};
    const cuuint32_t box[4] = {64, 8, 2, kP / 8};
    if (enc(&fresh, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, pool->cfg.kv_storage, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return STEP_ERR_CUDA;
    memcpy(pool->tmap_kv_bytes, &fresh, sizeof(fresh));
    if (cudaFuncSetAttribute(tree_tc_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(true)) != cudaSuccess ||
        cudaFuncSetAttribute(tree_tc_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(false)) != cudaSuccess)
      return STEP_ERR_CUDA;
    pool->tree_ready = true;
  }
  CUtensorMap map;
  memcpy(&map, pool->tmap_kv_bytes, sizeof(map));
  TreeArgs a;
  a.kv = (const __nv_bfloat16*)pool->cfg.kv_storage;
  a.q = (const __nv_bfloat16*)q; a.k_draft = (const __nv_bfloat16*)k_draft; a.v_draft = (const __nv_bfloat16*)v_draft;
  a.parents = parents; a.n_nodes = n_nodes; a.block_table = block_table; a.seq_lens = seq_lens;
  a.out = (__nv_bfloat16*)out;
  a.counters = pool->v.counters;
  a.n = n; a.T = T; a.Hq = g.Hq; a.Hkv = g.Hkv; a.G = g.G; a.L = g.L; a.layer = layer; a.max_pages = g.max_pages; a.num_blocks = g.num_blocks;
  a.tokens = kHalfRows / g.G;
  a.lanes = T > a.tokens ? 2 : 1;
  a.group_rows = a.lanes * kHalfRows;
  a.shares = pool->num_sms;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)kD);
  a.wait_ns = pool->wait_limit_ns;
  a.ws_o = (float*)workspace;
  a.ws_ml = a.ws_o + (size_t)a.shares * 2 * a.group_rows * kD;
  const size_t smem = smem_bytes(a.lanes == 2);
  auto kern = a.lanes == 2 ? tree_tc_kernel<true> : tree_tc_kernel<false>;
  // queries: a box is one half of the dims of the G heads of a group, for as many tokens as make a tile of rows
  CUtensorMap map_q;
  const cuuint64_t q_dims[3] = {kD, (cuuint64_t)g.Hq, (cuuint64_t)n * T};
  const cuuint64_t q_strides[2] = {kD * 2, (cuuint64_t)g.Hq * kD * 2};
  const cuuint32_t q_box[3] = {64, (cuuint32_t)g.G, (cuuint32_t)(a.tokens < T ? a.tokens : T)};
  if (enc(&map_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), q_dims, q_strides, q_box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return STEP_ERR_CUDA;
  kern<<<a.shares, kThreads, smem, s>>>(map, map_q, a);
  if (launch_ok() != STEP_OK) return STEP_ERR_CUDA;
  if (a.shares > 1 &&
      launch_dependent(tree_merge_kernel, dim3(a.shares - 1, a.group_rows / kMergeRows), dim3(kMergeWarps * 32), 0, s, a) != cudaSuccess) return STEP_ERR_CUDA;
  return launch_ok();
}

}  // namespace stepk
