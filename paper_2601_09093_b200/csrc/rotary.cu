// Rotary positions: rotate_positions turns queries or keys by their positions, store_kv_rotated turns keys on their way into
// the paged cache (and the queries of the same tokens along with them).
//
//   pair i of a head's first D = rotary_dim dims (i and i + D/2, or 2i and 2i + 1), at position p:
//   (y1, y2) = scale * ( x1 cos a - x2 sin a,  x2 cos a + x1 sin a ),  a = p * f_i;      transposed: a = -p * f_i
//
// Angles.  f_i enters as turns per position in units of 2^-64 (a 64-bit integer, made once on the host): p times that, modulo
// 2^64, IS the angle modulo a turn, with an error of p * 2^-65 turns from the table's rounding - 1.7e-13 radians at a position of
// a million, where a 32-bit product p * f would be off by 0.03.  The two top bits are the quadrant (rounded to nearest), what is
// left - at most an eighth of a turn - becomes a float, which rounds it by at most 2^-28 of a turn, and goes through sincospif.
// One 64-bit multiplication per pair and position, shared by all heads of the token.
//
// Both kernels are bound by memory: every element is read once and written once.  A thread owns kU = 16 bytes worth of
// pairs ("unit"): two 16-byte chunks of a head - one in each half, or two neighbours - so that it reads and writes whole
// chunks and both members of its pairs, in place as well.  Values are turned in fp32 and rounded once; subnormal ones are kept (this
// file is compiled without fast arithmetic, to the same registers and times).
#include "step_internal.cuh"

#include <math.h>

#include <atomic>

using namespace stepk;

namespace {

// Cosine and sine (times scale) of p * step turns, step in units of 2^-64.
__device__ inline void angle_of(long long p, unsigned long long step, float scale, float& c, float& s) {
  const unsigned long long phase = (unsigned long long)p * step;
  const unsigned quadrant = (unsigned)((phase + (1ull << 61)) >> 62);
  const long long rest = (long long)(phase - ((unsigned long long)quadrant << 62));    // in [-2^61, 2^61)
  float sn, cs;
  sincospif((float)rest * 0x1p-63f, &sn, &cs);
  c = (quadrant & 1) ? sn : cs;
  s = (quadrant & 1) ? cs : sn;
  if (quadrant == 1 || quadrant == 2) c = -c;
  if (quadrant & 2) s = -s;
  c *= scale;
  s *= scale;
}

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ inline T from_float(float x);
template <> __device__ inline float from_float<float>(float x) { return x; }
template <> __device__ inline __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16(x); }

// The two chunks of a unit, turned.
template <typename T, bool kPairs>
__device__ inline void turn_unit(uint4& a, uint4& b, const float* c, const float* s) {
  constexpr int kU = 16 / (int)sizeof(T);
  alignas(16) T x[2 * kU];
  *reinterpret_cast<uint4*>(x) = a;
  *reinterpret_cast<uint4*>(x + kU) = b;
#pragma unroll
  for (int i = 0; i < kU; ++i) {
    const int i1 = kPairs ? 2 * i : i, i2 = kPairs ? 2 * i + 1 : i + kU;
    const float x1 = to_float(x[i1]), x2 = to_float(x[i2]);
    x[i1] = from_float<T>(x1 * c[i] - x2 * s[i]);
    x[i2] = from_float<T>(x2 * c[i] + x1 * s[i]);
  }
  a = *reinterpret_cast<uint4*>(x);
  b = *reinterpret_cast<uint4*>(x + kU);
}
// Chunks of unit u in a head of D rotated dims.
template <typename T, bool kPairs>
__device__ inline void chunks_of(int u, int D, int& a, int& b) {
  constexpr int kU = 16 / (int)sizeof(T);
  a = kPairs ? 2 * u : u;
  b = kPairs ? 2 * u + 1 : u + D / (2 * kU);
}

// ---------------------------------------------------------------- rotate_positions
// x / by for 0 <= x < 2^31 and a divisor that the host knows: two instructions instead of twenty.
struct Quotient {
  unsigned by, mul, shift;
};
inline Quotient quotient(int by) {
  Quotient q;
  q.by = (unsigned)by;
  int log = 0;
  while ((1ll << log) < by) ++log;
  q.shift = by == 1 ? 0 : log - 1;
  q.mul = (unsigned)(((1ull << (31 + log)) + by - 1) / by);            // (not used for 1)
  return q;
}
__device__ inline int over(int x, const Quotient& q) { return q.by == 1 ? x : (int)(__umulhi((unsigned)x, q.mul) >> q.shift); }

struct RotateDev {
  const void* x; void* out;
  const int32_t* positions; long long position_batch;
  const unsigned long long* table;
  long long x_batch, x_row, x_head, out_batch, out_row, out_head;      // elements
  int batch, rows, heads, d, D;
  float scale, sign;
  int copy_tail;                    // dims behind D are copied (not in place)
  int heads_per_task, tasks_per_row;                                   // rotate_rows_kernel
  int rows_per_cta;                                                    // rotate_flat_kernel
  Quotient by_rows, by_half, by_units, by_heads, by_tail;
};

constexpr int kRotateThreads = 256, kRotateAhead = 2, kRotateAngles = 2048;   // (ahead 4: 104 registers, 35 us for 8191 rows of 40 heads instead of 31)
constexpr int kRotateWarps = kRotateThreads / 32;

// Rows of many heads: a warp takes one row and a range of its heads.  It makes the cosines and sines of the row's pairs once (in
// shared memory); a lane keeps those of its unit and goes through the heads with nothing but adds, as many heads at once as there
// is room for.  64 x 1024 rows of 64 heads of 128 in bf16: 328 us, 6.5 TB/s (the measured copy); numbering the units
// of all heads and rows, as rotate_flat_kernel does, took 662 us: 60 instructions of indexing per unit.
template <typename T, bool kPairs>
__global__ void __launch_bounds__(kRotateThreads) rotate_rows_kernel(const __grid_constant__ RotateDev a) {
  constexpr int kU = 16 / (int)sizeof(T);
  __shared__ __align__(16) float2 s_angle[kRotateAngles];               // (read two at a time)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long task = (long long)blockIdx.x * kRotateWarps + warp;
  const long long row = task / a.tasks_per_row;
  if (row >= (long long)a.batch * a.rows) return;
  const int h0 = (int)(task - row * a.tasks_per_row) * a.heads_per_task, h1 = min(a.heads, h0 + a.heads_per_task);
  const int bi = (int)(row / a.rows), ri = (int)(row - (long long)bi * a.rows);
  const T* x = (const T*)a.x + bi * a.x_batch + ri * a.x_row;
  T* out = (T*)a.out + bi * a.out_batch + ri * a.out_row;
  const int half = a.D / 2, units = a.D / (2 * kU), across = min(units, 32), together = 32 / across;
  float2* angle = s_angle + warp * (kRotateAngles / kRotateWarps);
  const int p = a.positions ? a.positions[bi * a.position_batch + ri] : ri;
  for (int i = lane; i < half; i += 32) {
    float c, s;
    angle_of(p, a.table[i], a.scale, c, s);
    angle[i] = make_float2(c, s * a.sign);
  }
  __syncwarp();
  const int sub = lane / across;
  for (int u0 = 0; u0 < units; u0 += across) {
    const int u = u0 + lane - sub * across;
    if (sub >= together || u >= units) continue;
    float c[kU], s[kU];
#pragma unroll
    for (int i = 0; i < kU; i += 2) {
      const float4 v = reinterpret_cast<const float4*>(angle + u * kU)[i / 2];
      c[i] = v.x; s[i] = v.y; c[i + 1] = v.z; s[i + 1] = v.w;
    }
    int ca, cb;
    chunks_of<T, kPairs>(u, a.D, ca, cb);
    for (int h = h0 + sub; h < h1; h += kRotateAhead * together) {
      uint4 va[kRotateAhead], vb[kRotateAhead];
#pragma unroll
      for (int y = 0; y < kRotateAhead; ++y) {
        const int hy = h + y * together;
        if (hy < h1) {
          const uint4* src = reinterpret_cast<const uint4*>(x + hy * a.x_head);
          va[y] = src[ca];
          vb[y] = src[cb];
        }
      }
#pragma unroll
      for (int y = 0; y < kRotateAhead; ++y) {
        const int hy = h + y * together;
        if (hy < h1) {
          turn_unit<T, kPairs>(va[y], vb[y], c, s);
          uint4* dst = reinterpret_cast<uint4*>(out + hy * a.out_head);
          dst[ca] = va[y];
          dst[cb] = vb[y];
        }
      }
    }
  }
  if (a.copy_tail) {
    const int first = a.D / kU, tail = a.d / kU - first;
    for (int i = lane; i < (h1 - h0) * tail; i += 32) {
      const int hy = over(i, a.by_tail), ch = first + i - hy * tail;
      reinterpret_cast<uint4*>(out + (h0 + hy) * a.out_head)[ch] = reinterpret_cast<const uint4*>(x + (h0 + hy) * a.x_head)[ch];
    }
  }
}

// Rows of few heads: a CTA takes up to rows_per_cta rows.  Cosines and sines of all pairs of its rows once,
// into shared memory; then its threads go through the units of all heads of all rows, kRotateAhead of them under way at once.
// 33 x 1021 rows of 5 heads of 64, fp32, half of each turned, 86 MB: 16.5 us on the same inputs again (they stay in the L2), where a warp
// per row took 37 (most of its lanes idle); 20.5 on inputs in turn (floor 13.2).  What bounds it is rounds of memory latency in a row - the
// angles, the first units, a second round of few units, then the copied dims - at 35 % of the issue slots.
template <typename T, bool kPairs>
__global__ void __launch_bounds__(kRotateThreads) rotate_flat_kernel(const __grid_constant__ RotateDev a) {
  constexpr int kU = 16 / (int)sizeof(T);
  __shared__ __align__(16) float2 s_angle[kRotateAngles];               // (read two at a time)
  const int row0 = blockIdx.x * a.rows_per_cta, n_rows = min(a.rows_per_cta, a.batch * a.rows - row0);
  const int heads = a.heads, half = a.D / 2, units = a.D / (2 * kU);
  for (int x = threadIdx.x; x < n_rows * half; x += kRotateThreads) {
    const int r = over(x, a.by_half), pair = x - r * half, bi = over(row0 + r, a.by_rows), ri = row0 + r - bi * a.rows;
    float c, s;
    angle_of(a.positions ? a.positions[bi * a.position_batch + ri] : ri, a.table[pair], a.scale, c, s);
    s_angle[x] = make_float2(c, s * a.sign);
  }
  __syncthreads();
  // (row, head) number x of this CTA: where it lies
  auto place = [&](int x, int& r, long long& in, long long& out) {
    r = over(x, a.by_heads);
    const int h = x - r * heads, bi = over(row0 + r, a.by_rows), ri = row0 + r - bi * a.rows;
    in = bi * a.x_batch + ri * a.x_row + h * a.x_head;
    out = bi * a.out_batch + ri * a.out_row + h * a.out_head;
  };
  const int items = n_rows * heads * units;
  for (int i0 = threadIdx.x; i0 < items; i0 += kRotateAhead * kRotateThreads) {
    uint4 va[kRotateAhead], vb[kRotateAhead];
    uint4 *da[kRotateAhead], *db[kRotateAhead];
    const float4* cs[kRotateAhead];
#pragma unroll
    for (int y = 0; y < kRotateAhead; ++y) {
      const int i = i0 + y * kRotateThreads;
      if (i >= items) continue;
      const int x = over(i, a.by_units), u = i - x * units;
      int r, ca, cb;
      long long in, out;
      place(x, r, in, out);
      chunks_of<T, kPairs>(u, a.D, ca, cb);
      const uint4* src = reinterpret_cast<const uint4*>((const T*)a.x + in);
      va[y] = src[ca];
      vb[y] = src[cb];
      da[y] = reinterpret_cast<uint4*>((T*)a.out + out) + ca;
      db[y] = reinterpret_cast<uint4*>((T*)a.out + out) + cb;
      cs[y] = reinterpret_cast<const float4*>(s_angle + r * half + u * kU);
    }
#pragma unroll
    for (int y = 0; y < kRotateAhead; ++y) {
      if (i0 + y * kRotateThreads >= items) continue;
      float c[kU], s[kU];
#pragma unroll
      for (int x = 0; x < kU; x += 2) {
        const float4 v = cs[y][x / 2];
        c[x] = v.x; s[x] = v.y; c[x + 1] = v.z; s[x + 1] = v.w;
      }
      turn_unit<T, kPairs>(va[y], vb[y], c, s);
      *da[y] = va[y];
      *db[y] = vb[y];
    }
  }
  if (a.copy_tail) {
    const int first = a.D / kU, tail = a.d / kU - first, chunks = n_rows * heads * tail;
    for (int i0 = threadIdx.x; i0 < chunks; i0 += kRotateAhead * kRotateThreads) {
      uint4 v[kRotateAhead], *dst[kRotateAhead];
#pragma unroll
      for (int y = 0; y < kRotateAhead; ++y) {
        const int i = i0 + y * kRotateThreads;
        if (i >= chunks) continue;
        const int x = over(i, a.by_tail), c = first + i - x * tail;
        int r;
        long long in, out;
        place(x, r, in, out);
        v[y] = reinterpret_cast<const uint4*>((const T*)a.x + in)[c];
        dst[y] = reinterpret_cast<uint4*>((T*)a.out + out) + c;
      }
#pragma unroll
      for (int y = 0; y < kRotateAhead; ++y)
        if (i0 + y * kRotateThreads < chunks) *dst[y] = v[y];
    }
  }
}

// Any alignment, any even D: a thread takes one pair, or one dim behind D, at a time, with a handful of divisions to know which.  8191 rows of
// 40 heads of 96 in bf16, 24 dims turned: 180 us, where 32 dims turned in whole chunks take 33 and the bytes 19.
template <typename T, bool kPairs>
__global__ void __launch_bounds__(256) rotate_any_kernel(const __grid_constant__ RotateDev a) {
  const int half = a.D / 2, items = half + (a.copy_tail ? a.d - a.D : 0);
  const long long all = (long long)a.batch * a.rows * a.heads * items;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
    const int e = (int)(i % items);
    long long r = i / items;
    const int h = (int)(r % a.heads);
    r /= a.heads;
    const int bi = (int)(r / a.rows), ri = (int)(r - (long long)bi * a.rows);
    const T* x = (const T*)a.x + bi * a.x_batch + ri * a.x_row + h * a.x_head;
    T* out = (T*)a.out + bi * a.out_batch + ri * a.out_row + h * a.out_head;
    if (e >= half) { out[e + half] = x[e + half]; continue; }
    const int p = a.positions ? a.positions[bi * a.position_batch + ri] : ri;
    float c, s;
    angle_of(p, a.table[e], a.scale, c, s);
    s *= a.sign;
    const int i1 = kPairs ? 2 * e : e, i2 = kPairs ? 2 * e + 1 : e + half;
    const float x1 = to_float(x[i1]), x2 = to_float(x[i2]);
    out[i1] = from_float<T>(x1 * c - x2 * s);
    out[i2] = from_float<T>(x2 * c + x1 * s);
  }
}

// ---------------------------------------------------------------- store_kv_rotated
struct StoreDev {
  Geo g;
  const int32_t* block_table; const int32_t* seq_lens; const uint8_t* live; int32_t* counters;
  void* kv;
  const int32_t* ids; const int32_t* start; const int32_t* positions;
  const void* k; const void* v; const void* q; void* q_out;
  long long k_row, v_row, q_row, q_layer, q_out_row, q_out_layer;       // elements
  const unsigned long long* table;
  int D; float scale;
  int layer0, n_layers, n_tokens;
  int layers_per_cta;
};

constexpr int kMaxPairs = 256;                                           // head_dim <= 512

// A CTA takes one (entry, token) row and a range of layers: cosines and sines of its position once, into shared memory;
// where the row goes (block and slot, the same for every layer and head) once; then its warps share the heads.
// kChunks: whole units (D a multiple of two chunks); else pair by pair.  32 tokens for 64 traces, 36 layers of 32 / 8 heads of 128 in
// bf16, with their queries: 290 us, 1.81 GB at 6.3 TB/s; one token, one layer: the latency of three dependent reads (the store and
// attention to the row together 12.4 us, 13.1 with the page looked up after the trace's length, a fourth).  Pair by pair (D no multiple of two
// chunks) a lane moves 2 or 4 bytes at a time: 32 tokens for 64 traces, 8 layers of 32 / 8 heads of 96 in bf16, 24 dims turned: 199 us, where
// 32 dims turned take 66 and the bytes 46.
template <typename T, bool kPairs, bool kChunks>
__global__ void __launch_bounds__(256) store_kernel(const StoreDev a) {
  constexpr int kU = 16 / (int)sizeof(T);
  __shared__ float s_c[kMaxPairs], s_s[kMaxPairs];
  const Geo& g = a.g;
  const int i = blockIdx.x / a.n_tokens, tok = blockIdx.x - i * a.n_tokens;
  const int st = a.start[i], t = a.ids[i];
  if (st < 0) return;                                                    // no room was made for this entry
  const bool reporter = threadIdx.x == 0 && tok == 0 && blockIdx.y == 0;
  if (t < 0 || t >= g.max_traces) { if (reporter) flag_error(a.counters, STEP_ERR_BAD_TRACE); return; }
  const long long p = (long long)(a.positions ? a.positions[i] : st) + tok;
  const int half = a.D / 2;
  for (int x = threadIdx.x; x < half; x += 256) angle_of(p, a.table[x], a.scale, s_c[x], s_s[x]);
  const bool live = a.live[t];
  const int S = a.seq_lens[t];
  // (the page is looked up along with the trace's length, before that has been compared: one round of reads less.
  // slot stays signed: unsigned took 51 registers instead of 48, four CTAs per SM instead of five: 325 us instead of 308 for the 64
  // traces above and attention to one layer)
  const unsigned page = ((unsigned)st + tok) / (unsigned)g.P;
  const int slot = (int)((unsigned)st + tok - page * g.P);
  const int b = a.block_table[(size_t)t * g.max_pages + min(page, (unsigned)g.max_pages - 1u)];
  if (!live) { if (reporter) flag_error(a.counters, STEP_ERR_BAD_TRACE); return; }
  if ((long long)st + a.n_tokens > S || (long long)S > (long long)g.max_pages * g.P) {
    if (reporter) flag_error(a.counters, STEP_ERR_INVALID_ARG);
    return;
  }
  if (b < 0 || b >= g.num_blocks) { if (threadIdx.x == 0 && blockIdx.y == 0) flag_error(a.counters, STEP_ERR_BAD_BLOCK); return; }
  __syncthreads();
  const int l0 = blockIdx.y * a.layers_per_cta, l1 = min(a.n_layers, l0 + a.layers_per_cta);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = 256 / 32;
  const int cpr = g.d / kU;                                              // chunks of a head's row
  const size_t head_stride = (size_t)2 * g.P * g.d, layer_stride = (size_t)g.num_blocks * g.Hkv * head_stride;
  // K row of (layer l of this call, head 0); V's is P * d further
  T* const kv0 = (T*)a.kv + (size_t)a.layer0 * layer_stride + (size_t)b * g.Hkv * head_stride + (size_t)slot * g.d;
  const T* const k0 = (const T*)a.k + (long long)blockIdx.x * a.k_row;
  const T* const v0 = (const T*)a.v + (long long)blockIdx.x * a.v_row;
  const T* const q0 = (const T*)a.q + (long long)blockIdx.x * a.q_row;
  T* const qo0 = (T*)a.q_out + (long long)blockIdx.x * a.q_out_row;
  auto stored = [&](int c) { return g.swizzle ? ((c & ~7) | ((c ^ slot) & 7)) : c; };   // where a row's chunk c stands

  // ---- values: as they are
  const int kv_heads = (l1 - l0) * g.Hkv;
  for (int x = threadIdx.x; x < kv_heads * cpr; x += 256) {
    const int hh = x / cpr, c = x - hh * cpr, l = l0 + hh / g.Hkv, h = hh % g.Hkv;
    reinterpret_cast<uint4*>(kv0 + (size_t)l * layer_stride + h * head_stride + (size_t)g.P * g.d)[stored(c)] =
        reinterpret_cast<const uint4*>(v0 + ((size_t)l * g.Hkv + h) * g.d)[c];
  }
  // ---- keys and queries: heads hh of [0, total) are turned; from(hh) and to(hh) say where a head's row is
  const int units = kChunks ? a.D / (2 * kU) : 1, across = min(units, 32), together = 32 / across;
  const int sub = lane / across;
  auto turn_heads = [&](int total, auto from, auto to, auto at) {
    if constexpr (kChunks) {
      for (int u0 = 0; u0 < units; u0 += across) {
        const int u = u0 + lane - sub * across;
        if (sub >= together || u >= units) continue;
        float c[kU], s[kU];
#pragma unroll
        for (int x = 0; x < kU; ++x) { c[x] = s_c[u * kU + x]; s[x] = s_s[u * kU + x]; }
        int ca, cb;
        chunks_of<T, kPairs>(u, a.D, ca, cb);
        // (a head at a time: with two under way the 32 more registers cost a CTA per SM, and 339 us instead of 308)
        for (int hh = warp * together + sub; hh < total; hh += warps * together) {
          const uint4* src = reinterpret_cast<const uint4*>(from(hh));
          uint4* dst = reinterpret_cast<uint4*>(to(hh));
          uint4 va = src[ca], vb = src[cb];
          turn_unit<T, kPairs>(va, vb, c, s);
          dst[at(ca)] = va;
          dst[at(cb)] = vb;
        }
      }
    } else {
      for (int x = threadIdx.x; x < total * half; x += 256) {
        const int hh = x / half, e = x - hh * half;
        const T* src = from(hh);
        T* dst = to(hh);
        const int i1 = kPairs ? 2 * e : e, i2 = kPairs ? 2 * e + 1 : e + half;
        const float x1 = to_float(src[i1]), x2 = to_float(src[i2]);
        dst[at(i1 / kU) * kU + i1 % kU] = from_float<T>(x1 * s_c[e] - x2 * s_s[e]);
        dst[at(i2 / kU) * kU + i2 % kU] = from_float<T>(x2 * s_c[e] + x1 * s_s[e]);
      }
    }
    const int tail = g.d - a.D;                                          // dims that are not turned
    if (kChunks) {
      for (int x = threadIdx.x; x < total * (tail / kU); x += 256) {
        const int hh = x / (tail / kU), c = a.D / kU + x % (tail / kU);
        reinterpret_cast<uint4*>(to(hh))[at(c)] = reinterpret_cast<const uint4*>(from(hh))[c];
      }
    } else {
      for (int x = threadIdx.x; x < total * tail; x += 256) {
        const int hh = x / tail, e = a.D + x % tail;
        to(hh)[at(e / kU) * kU + e % kU] = from(hh)[e];
      }
    }
  };
  turn_heads(kv_heads, [&](int hh) { return k0 + ((size_t)l0 * g.Hkv + hh) * g.d; },
             [&](int hh) { return kv0 + (size_t)(l0 + hh / g.Hkv) * layer_stride + (hh % g.Hkv) * head_stride; }, stored);
  if (a.q)
    turn_heads((l1 - l0) * g.Hq, [&](int hh) { return q0 + (long long)(l0 + hh / g.Hq) * a.q_layer + (hh % g.Hq) * g.d; },
               [&](int hh) { return qo0 + (long long)(l0 + hh / g.Hq) * a.q_out_layer + (hh % g.Hq) * g.d; }, [](int c) { return c; });
}

bool rotary_valid(const step_rotary* r, int head_dim) {
  return r && r->table && r->rotary_dim >= 2 && r->rotary_dim % 2 == 0 && r->rotary_dim <= head_dim &&
         (r->interleaved == 0 || r->interleaved == 1) && isfinite(r->scale) && !((uintptr_t)r->table & 7);
}

typedef void (*StoreForm)(const StoreDev);
template <typename T>
StoreForm store_form(bool pairs, bool chunks) {
  if (chunks) return pairs ? store_kernel<T, true, true> : store_kernel<T, false, true>;
  return pairs ? store_kernel<T, true, false> : store_kernel<T, false, false>;
}

// Multiprocessors of the current device, asked for once per device; 0: not to be told.
int sms_here() {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev < kDevices && (n = known[dev]) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  if (dev < kDevices) known[dev] = n;
  return n;
}

template <typename T>
int launch_rotate(const RotateDev& a0, int pairs, cudaStream_t s) {
  constexpr int kU = 16 / (int)sizeof(T);
  RotateDev a = a0;
  const int sms = sms_here();
  if (sms == 0) return STEP_ERR_CUDA;
  const long long strides = a.x_batch | a.x_row | a.x_head | a.out_batch | a.out_row | a.out_head;
  const int tail = a.copy_tail ? (a.d - a.D) / kU : 0;
  // whole 16-byte chunks wherever the shape allows it, and what a CTA or a warp of those kernels counts in 32 bits fits: a head's copied
  // dims are at most 2^16 chunks (times 512 rows of fewer than 64 heads), a row's heads at most 2^30
  const bool chunks = a.D % (2 * kU) == 0 && a.D / 2 <= kRotateAngles / kRotateWarps && (!a.copy_tail || a.d % kU == 0) && strides % kU == 0 &&
                      !(((uintptr_t)a.x | (uintptr_t)a.out) & 15) && tail <= 1 << 16 && a.heads <= 1 << 30;
  const long long rows = (long long)a.batch * a.rows;
  const int half = a.D / 2, units = a.D / (2 * kU);
  a.by_tail = quotient(tail && chunks ? tail : 1);
  // (the flat form numbers its rows, and what one CTA goes through, in 31 bits)
  if (chunks && (long long)a.heads * units < 32 * kRotateAhead && rows <= 0x3fffffffll) {
    // kRotateAhead units a thread, unless that leaves SMs without work
    const int most = kRotateAngles / half, row_units = a.heads * units;
    long long per = (kRotateAhead * kRotateThreads + row_units - 1) / row_units;
    if (per > most) per = most;
    if (per > rows / (2 * sms)) per = rows / (2 * sms);
    a.rows_per_cta = per < 1 ? 1 : (int)per;
    a.by_rows = quotient(a.rows); a.by_half = quotient(half); a.by_units = quotient(units); a.by_heads = quotient(a.heads);
    const unsigned ctas = (unsigned)((rows + a.rows_per_cta - 1) / a.rows_per_cta);
    if (pairs) rotate_flat_kernel<T, true><<<ctas, kRotateThreads, 0, s>>>(a);
    else rotate_flat_kernel<T, false><<<ctas, kRotateThreads, 0, s>>>(a);
  } else if (chunks) {
    // a warp takes all heads of a row; where that leaves SMs without work, or is more than 32 bits count, fewer
    const int together = units < 32 ? 32 / units : 1;
    int per = a.heads;
    while (per > together && (rows * ((a.heads + per - 1) / per) < 16ll * sms || (long long)per * tail > 1 << 30)) per = (per + 1) / 2;
    per = (per + together - 1) / together * together;
    a.heads_per_task = per;
    a.tasks_per_row = (a.heads + per - 1) / per;
    const long long ctas = (rows * a.tasks_per_row + kRotateWarps - 1) / kRotateWarps;
    if (ctas > 0x7fffffffll) return STEP_ERR_INVALID_ARG;
    if (pairs) rotate_rows_kernel<T, true><<<(unsigned)ctas, kRotateThreads, 0, s>>>(a);
    else rotate_rows_kernel<T, false><<<(unsigned)ctas, kRotateThreads, 0, s>>>(a);
  } else {
    const long long items = rows * a.heads * (a.D / 2 + (a.copy_tail ? a.d - a.D : 0));
    const long long ctas = (items + 255) / 256 < 16 * sms ? (items + 255) / 256 : 16 * sms;
    if (pairs) rotate_any_kernel<T, true><<<(unsigned)ctas, 256, 0, s>>>(a);
    else rotate_any_kernel<T, false><<<(unsigned)ctas, 256, 0, s>>>(a);
  }
  return launch_ok();
}

}  // namespace

extern "C" {

int step_rotary_table(const step_rotary_config* cfg, uint64_t* table_out, step_rotary* rotary_out) {
  if (!cfg || !table_out || !rotary_out) return STEP_ERR_INVALID_ARG;
  const int D = cfg->rotary_dim;
  if (D < 2 || D % 2 != 0 || (cfg->interleaved != 0 && cfg->interleaved != 1)) return STEP_ERR_INVALID_ARG;
  if (!(isfinite(cfg->base) && cfg->base > 1.0) || !(isfinite(cfg->output_scale) && cfg->output_scale >= 0.0)) return STEP_ERR_INVALID_ARG;
  const int kind = cfg->scaling;
  if (kind < STEP_ROTARY_PLAIN || kind > STEP_ROTARY_BANDS) return STEP_ERR_INVALID_ARG;
  const long double s = cfg->factor;
  if (kind != STEP_ROTARY_PLAIN && !(isfinite(cfg->factor) && cfg->factor > 0.0)) return STEP_ERR_INVALID_ARG;
  if (kind == STEP_ROTARY_BASE && D == 2) return STEP_ERR_INVALID_ARG;
  const bool ramp = kind == STEP_ROTARY_YARN || kind == STEP_ROTARY_BANDS;
  if (ramp && (!(isfinite(cfg->original_positions) && cfg->original_positions > 0.0) ||
               !(isfinite(cfg->fast) && cfg->slow > 0.0 && cfg->fast > cfg->slow))) return STEP_ERR_INVALID_ARG;
  if (cfg->divisors)
    for (int i = 0; i < D / 2; ++i)
      if (!(isfinite(cfg->divisors[i]) && cfg->divisors[i] > 0.0)) return STEP_ERR_INVALID_ARG;
  const long double turn = 6.283185307179586476925286766559005768L;
  long double log_base = logl((long double)cfg->base);
  if (kind == STEP_ROTARY_BASE) log_base += logl(s) * D / (D - 2);
  long double first = 0.0L, last = 0.0L;                 // YARN: the pairs between which the stretching sets in
  if (kind == STEP_ROTARY_YARN) {
    const long double L = cfg->original_positions;
    first = floorl(D * logl(L / (cfg->fast * turn)) / (2 * log_base));
    last = ceill(D * logl(L / (cfg->slow * turn)) / (2 * log_base));
    if (first < 0) first = 0;
    if (last > D - 1) last = D - 1;
  }
  for (int i = 0; i < D / 2; ++i) {
    long double f = expl(-2.0L * i / D * log_base), stretched = 0.0L;
    if (kind == STEP_ROTARY_LINEAR) stretched = 1.0L;
    if (kind == STEP_ROTARY_YARN) stretched = (i - first) / (last - first > 0.001L ? last - first : 0.001L);
    if (kind == STEP_ROTARY_BANDS) stretched = (cfg->fast - cfg->original_positions * f / turn) / ((long double)cfg->fast - cfg->slow);
    if (stretched < 0) stretched = 0;
    if (stretched > 1) stretched = 1;
    if (stretched > 0) f = f * (1.0L - stretched) + f / s * stretched;
    if (cfg->divisors) f /= cfg->divisors[i];
    // turns per position; whole turns do not matter at whole positions
    long double x = f / turn;
    if (!(x < 0x1p16L)) return STEP_ERR_INVALID_ARG;     // (x is good to 2^-60 of itself: nothing would be left at far positions)
    x = (x - floorl(x)) * 0x1p64L;
    uint64_t u = x < 0x1p64L ? (uint64_t)x : 0;
    if (x < 0x1p64L && x - (long double)u >= 0.5L) ++u;
    table_out[i] = u;
  }
  double scale = cfg->output_scale;
  if (scale == 0.0) scale = kind == STEP_ROTARY_YARN && cfg->factor > 1.0 ? 0.1 * log(cfg->factor) + 1.0 : 1.0;
  if (!isfinite((float)scale)) return STEP_ERR_INVALID_ARG;
  rotary_out->table = nullptr;
  rotary_out->rotary_dim = D;
  rotary_out->interleaved = cfg->interleaved;
  rotary_out->scale = (float)scale;
  return STEP_OK;
}

int rotate_positions(const rotate_args* a, const step_rotary* rotary, void* stream) {
  if (!a || a->batch < 0 || a->rows < 0 || a->heads < 0 || a->head_dim < 1) return STEP_ERR_INVALID_ARG;
  if (a->dtype != STEP_BF16 && a->dtype != STEP_FP32) return STEP_ERR_INVALID_ARG;
  if ((a->transpose != 0 && a->transpose != 1) || !rotary_valid(rotary, a->head_dim)) return STEP_ERR_INVALID_ARG;
  if (a->batch == 0 || a->rows == 0 || a->heads == 0) return STEP_OK;
  if (!a->x || !a->out) return STEP_ERR_INVALID_ARG;
  const uintptr_t unit = a->dtype == STEP_BF16 ? 1 : 3;
  if (((uintptr_t)a->x | (uintptr_t)a->out) & unit || (uintptr_t)a->positions & 3) return STEP_ERR_INVALID_ARG;
  RotateDev r = {};
  r.x = a->x; r.out = a->out;
  r.positions = a->positions; r.position_batch = a->position_batch;
  r.table = (const unsigned long long*)rotary->table;
  r.x_batch = a->x_batch; r.x_row = a->x_row; r.x_head = a->x_head;
  r.out_batch = a->out_batch; r.out_row = a->out_row; r.out_head = a->out_head;
  r.batch = a->batch; r.rows = a->rows; r.heads = a->heads; r.d = a->head_dim; r.D = rotary->rotary_dim;
  if (r.batch == 1) r.x_batch = r.out_batch = 0;         // (a stride that is not used may be anything)
  if (r.rows == 1) r.x_row = r.out_row = 0;
  if (r.heads == 1) r.x_head = r.out_head = 0;
  // results that would share a place, or lie over x in another order, depend on which thread comes first
  if ((r.batch > 1 && r.out_batch == 0) || (r.rows > 1 && r.out_row == 0) || (r.heads > 1 && r.out_head == 0)) return STEP_ERR_INVALID_ARG;
  if (r.x == r.out && (r.x_batch != r.out_batch || r.x_row != r.out_row || r.x_head != r.out_head)) return STEP_ERR_INVALID_ARG;
  r.scale = rotary->scale; r.sign = a->transpose ? -1.f : 1.f;
  r.copy_tail = a->x != a->out && r.D < r.d;
  return a->dtype == STEP_BF16 ? launch_rotate<__nv_bfloat16>(r, rotary->interleaved, (cudaStream_t)stream)
                               : launch_rotate<float>(r, rotary->interleaved, (cudaStream_t)stream);
}

int store_kv_rotated(step_pool* pool, const kv_store_args* a, const step_rotary* rotary, void* stream) {
  if (!pool || !a || a->n < 0 || a->n_tokens < 0) return STEP_ERR_INVALID_ARG;
  const kv_pool_config& cfg = pool->cfg;
  if (a->layer0 < 0 || a->n_layers < 1 || a->layer0 > cfg.num_layers - a->n_layers) return STEP_ERR_INVALID_ARG;
  if (!rotary_valid(rotary, cfg.head_dim)) return STEP_ERR_INVALID_ARG;
  if (a->n == 0 || a->n_tokens == 0) return STEP_OK;
  if (!a->trace_ids || !a->start || !a->k || !a->v || !a->q != !a->q_out) return STEP_ERR_INVALID_ARG;
  const long long rows = (long long)a->n * a->n_tokens;
  if (rows > 0x7fffffffll) return STEP_ERR_INVALID_ARG;
  const int cpe = 16 / pool->elem_bytes;
  const long long k_row = rows > 1 ? a->k_row : 0, v_row = rows > 1 ? a->v_row : 0;      // (a stride that is not used may be anything)
  const long long q_row = rows > 1 ? a->q_row : 0, q_out_row = rows > 1 ? a->q_out_row : 0;
  const long long q_layer = a->n_layers > 1 ? a->q_layer : 0, q_out_layer = a->n_layers > 1 ? a->q_out_layer : 0;
  if (((uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)a->q | (uintptr_t)a->q_out) & 15) return STEP_ERR_INVALID_ARG;
  if (a->q && ((rows > 1 && q_out_row == 0) || (a->n_layers > 1 && q_out_layer == 0))) return STEP_ERR_INVALID_ARG;   // (as above)
  if (a->q && a->q == a->q_out && (q_row != q_out_row || q_layer != q_out_layer)) return STEP_ERR_INVALID_ARG;
  if ((k_row | v_row) % cpe != 0 || (a->q && (q_row | q_layer | q_out_row | q_out_layer) % cpe != 0)) return STEP_ERR_INVALID_ARG;
  const int st = on_pool_device(pool);
  if (st != STEP_OK) return st;
  StoreDev d = {};
  d.g = geo_of(pool);
  d.block_table = pool->v.block_table; d.seq_lens = pool->v.seq_lens; d.live = pool->v.live; d.counters = pool->v.counters;
  d.kv = cfg.kv_storage;
  d.ids = a->trace_ids; d.start = a->start; d.positions = a->positions;
  d.k = a->k; d.v = a->v; d.q = a->q; d.q_out = a->q_out;
  d.k_row = k_row; d.v_row = v_row; d.q_row = q_row; d.q_layer = q_layer; d.q_out_row = q_out_row; d.q_out_layer = q_out_layer;
  d.table = (const unsigned long long*)rotary->table;
  d.D = rotary->rotary_dim; d.scale = rotary->scale;
  d.layer0 = a->layer0; d.n_layers = a->n_layers; d.n_tokens = a->n_tokens;
  // a CTA takes all layers of a row; where that leaves SMs without work, fewer
  int splits = (int)((2ll * pool->num_sms + rows - 1) / rows);
  if (splits > a->n_layers) splits = a->n_layers;
  d.layers_per_cta = (a->n_layers + splits - 1) / splits;
  const dim3 grid((unsigned)rows, (unsigned)((a->n_layers + d.layers_per_cta - 1) / d.layers_per_cta));
  cudaStream_t s = (cudaStream_t)stream;
  const bool chunks = d.D % (2 * cpe) == 0;
  auto kernel = cfg.dtype == STEP_BF16 ? store_form<__nv_bfloat16>(rotary->interleaved, chunks) : store_form<float>(rotary->interleaved, chunks);
  kernel<<<grid, 256, 0, s>>>(d);
  return launch_ok();
}

}  // extern "C"
