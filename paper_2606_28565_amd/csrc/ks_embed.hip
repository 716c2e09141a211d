// Dropout, the lookup of a table's rows by id, and the table's gradient (ks.h).
//
//   k_embed        dst_i = drop(factor src_i), src_i the table's row of id i (the
//                  lookup) or row i itself (dropout)
//   k_embed_back   rows of the table's gradient, of parts of the order
//   k_embed_join   the sums of ids that have rows in more than one part
//
// A lane's work is a block of eight columns of one row: 16 bytes of bfloat16, 32 of
// fp32, and exactly one Philox block's draws.  Each element is read and written once, and
// bytes bound all three: the draws (20 multiplications to 64 bits a block) are made
// while loads are on their way, and a dropout takes as long as a copy by the same kernel.
// Reads fetch lines of 128 bytes, needed or not, and stores off the 64-byte grid cost
// more than their bytes: 2,000,003 rows of 32 fp32 columns pass in 91 us, 16 of the 32
// in 86, 15 in 127 (260 MB fetched, 128 written).
//
// 16,381 rows of 4096 bf16 columns looked up: 45 us (123 MB fetched, 134 written: 5.7
// TB/s).  2,000,003 rows of 16 fp32 columns in rows of 32, with dropout: 34 us (136 MB).  Dropout
// of 134M bf16 elements: 86 us (537 MB, 6.2 TB/s; a copy of 4 GiB reaches 4.7).
#include <hip/hip_runtime.h>

#include "ks_columns.h"

namespace ks {

namespace {

constexpr int kThreads = 256;

// rows of any alignment of the type's
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 any_u32x4 __attribute__((aligned(2)));
typedef u32x2 any_u32x2 __attribute__((aligned(2)));
typedef uint32_t any_u32 __attribute__((aligned(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));   // (an array would get an address, and memory)
typedef f32x2 any_f32x2 __attribute__((aligned(4)));
typedef f32x4 any_f32x4 __attribute__((aligned(4)));

template <bool B16>
struct Eight {
  u32x4 w[B16 ? 1 : 2];
  __device__ __forceinline__ float operator[](int j) const {
    // (the element as a value: a cast of the element itself takes the vector's first)
    const uint32_t v = B16 ? w[0][j / 2] : w[B16 ? 0 : j / 4][j % 4];
    if constexpr (B16) return __builtin_bit_cast(float, j & 1 ? v & 0xFFFF0000u : v << 16);
    else return __builtin_bit_cast(float, v);
  }
};

// Where a row's last block is not whole (kPart), it is loaded with the row's last eight
// columns, which `align8` moves down: one load for all lanes, where loads of four, two and
// one element wait for each other.  Rows of fewer than eight columns (kFew) have no such
// place.
enum Kind { kWhole, kPart, kFew };

struct Place {
  int64_t at;        // element in the row
  bool part;         // not whole
};
template <int KIND>
__device__ __forceinline__ Place place_of(const Cols &c, uint32_t b) {
  if constexpr (KIND == kWhole) return {8 * (int64_t)b, false};
  if constexpr (KIND == kFew) return {0, true};
  const bool part = b + 1 == c.blocks;
  return {8 * (int64_t)b - (part ? 8 - c.rem : 0), part};
}

template <bool B16, int KIND>
__device__ __forceinline__ Eight<B16> load8(const void *base, int64_t at, const Cols &c) {
  Eight<B16> o;
  if constexpr (KIND == kFew) {
    o.w[0] = u32x4{0, 0, 0, 0};
    if constexpr (!B16) o.w[1] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (uint32_t j = 0; j < 7; ++j) {
      if (j >= c.rem) break;
      if constexpr (B16) o.w[0][j / 2] |= (uint32_t)((const uint16_t *)base)[at + j] << (16 * (j & 1));
      else o.w[j / 4][j % 4] = ((const uint32_t *)base)[at + j];
    }
  } else {
    const char *p = (const char *)base + (B16 ? 2 : 4) * at;
    o.w[0] = *(const any_u32x4 *)p;
    if constexpr (!B16) o.w[1] = *(const any_u32x4 *)(p + 16);
  }
  return o;
}

// b where the mask is set, else a (one instruction; a choice between elements of a vector
// would become a choice of the index)
__device__ __forceinline__ uint32_t choose(uint32_t mask, uint32_t b, uint32_t a) { return (mask & b) | (~mask & a); }

// the last rem of eight elements down to the first places (with `part`; behind them stays
// anything)
template <bool B16, int KIND>
__device__ __forceinline__ void align8(Eight<B16> &x, const Cols &c, bool part) {
  if constexpr (KIND != kPart) return;
  const uint32_t by = 8 - c.rem, mask = part ? 0xFFFFFFFFu : 0u;
  constexpr int N = B16 ? 4 : 8;
  uint32_t w[N];
#pragma unroll
  for (int j = 0; j < N; ++j) w[j] = x.w[j / 4][j % 4];
  if (B16 && (by & 1)) {
#pragma unroll
    for (int j = 0; j < N; ++j) w[j] = choose(mask, __builtin_amdgcn_alignbit(j + 1 < N ? w[j + 1 < N ? j + 1 : 0] : 0u, w[j], 16), w[j]);
  }
#pragma unroll
  for (int s = 1; s < N; s *= 2)
    if (by & (B16 ? 2 * s : s)) {
#pragma unroll
      for (int j = 0; j + s < N; ++j) w[j] = choose(mask, w[j + s], w[j]);
    }
#pragma unroll
  for (int j = 0; j < N; ++j) x.w[j / 4][j % 4] = w[j];
}

__device__ __forceinline__ uint32_t pair(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

template <bool B16, int KIND>
__device__ __forceinline__ void store8(void *base, int64_t at, f32x8 v, bool part, uint32_t rem) {
  const bool whole = KIND == kWhole || (KIND == kPart && !part);
  if constexpr (B16) {
    char *p = (char *)base + 2 * at;
    const u32x4 w = {pair(v[0], v[1]), pair(v[2], v[3]), pair(v[4], v[5]), pair(v[6], v[7])};
    if (whole) {
      *(any_u32x4 *)p = w;
      return;
    }
    if (rem & 4) *(any_u32x2 *)p = u32x2{w[0], w[1]};
    if (rem & 2) *(any_u32 *)(p + 2 * (rem & 4)) = rem & 4 ? w[2] : w[0];
    if (rem & 1) *(uint16_t *)(p + 2 * (rem & 6)) = (uint16_t)(rem & 4 ? (rem & 2 ? w[3] : w[2]) : (rem & 2 ? w[1] : w[0]));
  } else {
    float *p = (float *)base + at;
    if (whole) {
      *(any_f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
      *(any_f32x4 *)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
      return;
    }
    const bool up = rem & 4;
    if (up) *(any_f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
    if (rem & 2) *(any_f32x2 *)(p + (rem & 4)) = up ? f32x2{v[4], v[5]} : f32x2{v[0], v[1]};
    if (rem & 1) p[rem & 6] = up ? (rem & 2 ? v[6] : v[4]) : (rem & 2 ? v[2] : v[0]);
  }
}

// ------------------------------------------------------------ draws
struct Draws {
  uint32_t w[4];
  __device__ __forceinline__ uint32_t operator[](int j) const { return j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu; }
};
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);   // (one instruction; the compiler makes two)
}
__device__ __forceinline__ Draws philox(const Drop &d, uint64_t block, uint32_t step) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = step, c3 = d.site;
  uint32_t k0 = d.key0, k1 = d.key1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = xor3((uint32_t)(b >> 32), c1, k0);
    c1 = (uint32_t)b;
    c2 = xor3((uint32_t)(a >> 32), c3, k1);
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}
__device__ __forceinline__ uint32_t step_of(const Drop &d) { return d.step_dev ? *d.step_dev : d.step; }

// l / blocks and, in b, the rest; l < 2^32.  (ceil(2^32 / blocks) is at most blocks - 1 too
// large: one too many, where l is large)
__device__ __forceinline__ uint32_t row_in(const Cols &c, uint32_t l, uint32_t &b) {
  uint32_t q = c.magic ? __umulhi(l, c.magic) : l;
  if (c.magic && (uint64_t)q * c.blocks > l) --q;
  b = l - q * c.blocks;
  return q;
}

// ------------------------------------------------------------ lookup and dropout
// U blocks a lane: their ids, then their rows on the way together, the draws made
// meanwhile (2,000,003 rows of 16 fp32 columns in rows of 32: 34 us; with the draws
// before the rows' loads 56).  Two where bfloat16 is looked up or written, else one:
// lookups of 2^25 bf16 elements in rows of 256 to 4096 columns take 22 to 26 us with two,
// 24 to 27 with one, 22 to 27 with four; of fp32 ones 47 to 51, 45 to 49, 48 to 54; dropout
// of as many bf16 elements 27, 24 and 29.
template <bool LOOKUP, bool S16, bool D16>
constexpr int kAhead = LOOKUP && (S16 || D16) ? 2 : 1;

template <bool LOOKUP, bool S16, bool D16, bool DROP, int KIND>
__global__ __launch_bounds__(kThreads) void k_embed(EmbedParams a) {
  constexpr int U = kAhead<LOOKUP, S16, D16>;
  const uint32_t l = blockIdx.x * (kThreads * U) + threadIdx.x;
  int64_t row[U];
  uint32_t b[U], id[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    row[u] = a.row0 + row_in(a.cols, a.block0 + l + u * kThreads, b[u]);
    if constexpr (LOOKUP) id[u] = a.ids[min(row[u], a.n_rows - 1)];
  }
  // an id beyond the table reads its last row, to no use; a table without rows none
  Eight<S16> x[U];
  bool known[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    known[u] = !LOOKUP || id[u] < a.n_ids;
    const int64_t at = LOOKUP ? (int64_t)min(id[u], a.n_ids - 1) : min(row[u], a.n_rows - 1);
    x[u] = {};
    if (a.n_ids) x[u] = load8<S16, KIND>(a.src, at * a.src_ld + place_of<KIND>(a.cols, b[u]).at, a.cols);
  }
  Draws d[U];
  if constexpr (DROP) {
    const uint32_t step = step_of(a.drop);
#pragma unroll
    for (int u = 0; u < U; ++u) d[u] = philox(a.drop, a.first + l + u * kThreads, step);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (row[u] >= a.n_rows) break;
    const bool part = place_of<KIND>(a.cols, b[u]).part;
    align8<S16, KIND>(x[u], a.cols, part);
    const uint32_t least = known[u] ? a.drop.least : 1u << 16;   // (no draw is as large)
    f32x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (DROP ? d[u][j] >= least : known[u]) ? x[u][j] * a.factor : 0.0f;
    store8<D16, KIND>(a.dst, row[u] * a.dst_ld + 8 * (int64_t)b[u], v, part, a.cols.rem);
  }
}

// ------------------------------------------------------------ the table's gradient
// The order's places are split evenly, whatever ids they have: a group of `wide` lanes
// (the blocks of a row) walks `each` places in a row and adds up rows until the id
// changes; `groups` of them, one behind the other, are a workgroup.  An id that begins and
// ends in a group's places is written there.  Of the others a group keeps what ends in
// it (head) and what goes on behind it (out), which a scan over the workgroup's groups
// joins; what goes on beyond the workgroup k_embed_join joins.  The order of all sums
// goes by sizes alone.
//
// A thread's sum: 64 additions in a row, then one for each such run.
//
// 2,000,003 rows of 16 fp32 columns in rows of 32, 67 ids: 52 us (291 MB fetched, 5.6 TB/s)
// and the join 6.  16,381 rows of 2048 bf16 columns, 32,000 ids: 60 us (334 MB, most of
// them zeros for ids without rows, 5.6 TB/s) and the join 6.  By ids instead of places (a
// group for an id of up to 128 rows, workgroups for longer ones) they were 152 and 147 us
// with the join.
template <bool B16, bool DROP, int KIND>
__global__ __launch_bounds__(kBackThreads) void k_embed_back(EmbedBackParams a) {
  const int64_t wg = a.wg0 + blockIdx.x;
  const uint32_t n = min(a.off[a.n_ids], (uint32_t)a.n_rows);   // (behind: rows without an id)
  if (wg >= (int64_t)a.runs * a.tiles) {
    // ids without rows
    const uint32_t l = (uint32_t)(wg - a.fill_wg0) * (kBackThreads * kBackFill) + threadIdx.x;
#pragma unroll
    for (int u = 0; u < kBackFill; ++u) {
      uint32_t q;
      const int64_t v = a.fill_row0 + row_in(a.quads, a.fill_quad0 + l + u * kBackThreads, q);
      if (v >= a.n_ids || a.off[v] < a.off[v + 1]) continue;
      float *o = a.grad + v * a.grad_ld + 4 * (int64_t)q;
      if (a.quads.rem == 0 || q + 1 < a.quads.blocks) {
        if (a.past) __builtin_nontemporal_store(f32x4{}, (f32x4 *)o);
        else *(any_f32x4 *)o = f32x4{};
      } else {
        for (uint32_t j = 0; j < a.quads.rem; ++j) o[j] = 0.0f;
      }
    }
    return;
  }
  constexpr uint32_t kBatch = B16 ? 8 : 4;
  __shared__ float val[kBackThreads][8];
  __shared__ uint32_t stop[kBackThreads];
  const uint32_t step = DROP ? step_of(a.drop) : 0;
  const uint32_t part = (uint32_t)(wg / a.tiles), tile = (uint32_t)(wg % a.tiles), lo = part * a.run;
  if (lo >= n) return;
  const uint32_t wide = a.wide, groups = kBackThreads / wide;
  const uint32_t g = threadIdx.x / wide, b = tile * wide + threadIdx.x % wide;
  const bool in = g < groups && b < a.cols.blocks;
  const Place at = place_of<KIND>(a.cols, min(b, a.cols.blocks - 1));
  const uint32_t p0 = min(lo + g * a.each, n), p1 = g < groups ? min(p0 + a.each, n) : p0;
  auto write = [&](uint32_t v, f32x8 s) {
    if (!in || v >= a.n_ids) return;
    s *= a.factor;
    store8<false, KIND>(a.grad, (int64_t)v * a.grad_ld + 8 * (int64_t)b, s, at.part, a.cols.rem);
  };

  f32x8 head = {}, out = {};
  bool has_head = false, has_out = false, through = false;   // through: what goes on came from before
  uint32_t head_id = 0;
  if (p0 < p1) {
    uint32_t cur = a.id[p0];
    bool from_before = p0 > 0 && a.id[p0 - 1] == cur;
    f32x8 acc = {}, sum = {};
    uint32_t since = 0;
    for (uint32_t p = p0; p < p1; p += kBatch) {
      uint32_t id[kBatch], row[kBatch];
      Eight<B16> x[kBatch];
#pragma unroll
      for (uint32_t u = 0; u < kBatch; ++u) {
        const uint32_t q = min(p + u, p1 - 1);
        id[u] = a.id[q];
        row[u] = a.row[q];
      }
#pragma unroll
      for (uint32_t u = 0; u < kBatch; ++u)
        x[u] = load8<B16, KIND>(a.dy, (int64_t)min(row[u], (uint32_t)a.n_rows - 1) * a.ld + at.at, a.cols);
#pragma unroll
      for (uint32_t u = 0; u < kBatch; ++u) {
        if (p + u >= p1) break;
        if (id[u] != cur) {
          acc += sum;
          if (from_before) {
            head = acc;
            head_id = cur;
            has_head = true;
          } else {
            write(cur, acc);
          }
          acc = sum = f32x8{};
          since = 0;
          cur = id[u];
          from_before = false;
        }
        align8<B16, KIND>(x[u], a.cols, at.part);
        if (row[u] < a.n_rows) {
          if constexpr (DROP) {
            const Draws d = philox(a.drop, (uint64_t)row[u] * a.cols.blocks + b, step);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += d[j] >= a.drop.least ? x[u][j] : 0.0f;
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += x[u][j];
          }
        }
        if (++since == 64) {
          acc += sum;
          sum = f32x8{};
          since = 0;
        }
      }
    }
    acc += sum;
    const bool goes_on = p1 < n && a.id[p1] == cur;
    if (goes_on) {
      out = acc;
      has_out = true;
      through = from_before;
    } else if (from_before) {
      head = acc;
      head_id = cur;
      has_head = true;
    } else {
      write(cur, acc);
    }
  }
  // out of the groups before that goes on through them: to each group, what enters it
  f32x8 carry = out;
  bool begun = !(has_out && through);   // the id that goes on has begun in this workgroup
  for (uint32_t d = 1; d < groups; d *= 2) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) val[threadIdx.x][j] = carry[j];
    stop[threadIdx.x] = begun;
    __syncthreads();
    if (g >= d && g < groups && !begun) {
#pragma unroll
      for (int j = 0; j < 8; ++j) carry[j] += val[threadIdx.x - d * wide][j];
      begun = stop[threadIdx.x - d * wide];
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) val[threadIdx.x][j] = carry[j];
  stop[threadIdx.x] = begun;
  __syncthreads();
  if (!in) return;
  float *slot = a.part + ((int64_t)(2 * part) * a.cols.blocks + b) * 8;
  auto keep = [&](const f32x8 &s, int which) {
#pragma unroll
    for (int j = 0; j < 8; ++j) slot[(int64_t)which * a.cols.blocks * 8 + j] = s[j];
  };
  if (has_head) {
    bool here = false;
    if (g > 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) head[j] = val[threadIdx.x - wide][j] + head[j];
      here = stop[threadIdx.x - wide];
    }
    if (here) write(head_id, head);
    else keep(head, 0);
  }
  if (has_out && g == groups - 1) keep(carry, begun ? 1 : 0);   // what goes on beyond the workgroup
}

// An id that begins in this part and goes on: its sum here, then those of the parts
// that it goes on in.  A thread has four columns; `lanes` threads share them, each with
// every lanes-th part, joined in 64 bits.
constexpr int kJoinCols = 4;
__global__ __launch_bounds__(kBackThreads) void k_embed_join(EmbedBackParams a, uint32_t tiles) {
  __shared__ double room[kBackThreads][kJoinCols];
  const int64_t at = a.wg0 + blockIdx.x;
  const uint32_t part = (uint32_t)(at / tiles), tile = (uint32_t)(at % tiles);
  const uint32_t next = (part + 1) * a.run;   // (not the last part: in the order)
  const uint32_t n = min(a.off[a.n_ids], (uint32_t)a.n_rows), v = a.id[next - 1], after = a.id[next];
  if (next >= n || v != after || v >= a.n_ids) return;
  const uint32_t begin = a.off[v], end = a.off[v + 1];
  if (begin < part * a.run || begin >= next) return;
  const uint32_t last = min((max(end, next + 1) - 1) / a.run, a.runs - 1);
  const uint32_t quads = a.cols.blocks * 8 / kJoinCols, wide = min(quads, (uint32_t)kBackThreads), lanes = kBackThreads / wide;
  const uint32_t l = threadIdx.x / wide, q = tile * wide + threadIdx.x % wide;
  double sum[kJoinCols] = {};
  if (l < lanes && q < quads) {
    const float *base = a.part + (int64_t)q * kJoinCols;
    auto at = [&](int64_t slot) { return *(const f32x4 *)(base + slot * quads * kJoinCols); };
    if (l == 0) {
      const f32x4 p = at(2 * (int64_t)part + 1);
#pragma unroll
      for (int j = 0; j < kJoinCols; ++j) sum[j] = (double)p[j];
    }
    // sixteen on their way at a time, the last time too
    constexpr uint32_t kAhead = 16;
    for (uint32_t k = part + 1 + l; k <= last; k += kAhead * lanes) {
      f32x4 p[kAhead];
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) p[u] = at(2 * (int64_t)min(k + u * lanes, last));
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u)
#pragma unroll
        for (int j = 0; j < kJoinCols; ++j) sum[j] += k + u * lanes <= last ? (double)p[u][j] : 0.0;
    }
  }
  for (uint32_t half = kBackThreads / 2; half > 0; half /= 2) {
    if (half >= lanes) continue;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kJoinCols; ++j) room[threadIdx.x][j] = sum[j];
    __syncthreads();
    if (l < half && l + half < lanes) {
#pragma unroll
      for (int j = 0; j < kJoinCols; ++j) sum[j] += room[threadIdx.x + half * wide][j];
    }
  }
  if (l > 0) return;
  const uint32_t width = a.cols.rem ? a.cols.blocks * 8 - 8 + a.cols.rem : a.cols.blocks * 8;
#pragma unroll
  for (int j = 0; j < kJoinCols; ++j)
    if (kJoinCols * q + j < width) a.grad[(int64_t)v * a.grad_ld + kJoinCols * q + j] = (float)(sum[j] * a.factor);
}

// launch(first workgroup, workgroups): as many at a time as blocks and quads of a launch
// take 32 bits for
template <class F>
hipError_t in_launches(int64_t wgs, F &&launch) {
  constexpr int64_t kMost = int64_t(1) << 20;
  for (int64_t at = 0; at < wgs; at += kMost) {
    launch(at, (uint32_t)(wgs - at < kMost ? wgs - at : kMost));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

int kind_of(const Cols &c) { return c.rem == 0 ? kWhole : c.blocks > 1 ? kPart : kFew; }

template <bool LOOKUP, bool S16, bool D16, bool DROP, int KIND>
hipError_t embed(EmbedParams p, hipStream_t s) {
  constexpr int kBlocks = kThreads * kAhead<LOOKUP, S16, D16>;
  return in_launches((p.n_rows * (int64_t)p.cols.blocks + kBlocks - 1) / kBlocks, [&](int64_t at, uint32_t wgs) {
    p.first = (uint64_t)at * kBlocks;
    p.row0 = (int64_t)(p.first / p.cols.blocks);
    p.block0 = (uint32_t)(p.first % p.cols.blocks);
    hipLaunchKernelGGL((k_embed<LOOKUP, S16, D16, DROP, KIND>), dim3(wgs), dim3(kThreads), 0, s, p);
  });
}

template <bool LOOKUP, bool S16, bool D16, bool DROP>
hipError_t embed_kind(const EmbedParams &p, hipStream_t s) {
  const int kind = kind_of(p.cols);
  return kind == kWhole ? embed<LOOKUP, S16, D16, DROP, kWhole>(p, s)
                        : kind == kPart ? embed<LOOKUP, S16, D16, DROP, kPart>(p, s) : embed<LOOKUP, S16, D16, DROP, kFew>(p, s);
}

template <bool S16, bool D16>
hipError_t lookup(const EmbedParams &p, hipStream_t s) {
  return p.drop.least ? embed_kind<true, S16, D16, true>(p, s) : embed_kind<true, S16, D16, false>(p, s);
}

template <bool B16>
hipError_t dropout(const EmbedParams &p, hipStream_t s) {
  return p.drop.least ? embed_kind<false, B16, B16, true>(p, s) : embed_kind<false, B16, B16, false>(p, s);
}

template <bool B16, bool DROP>
hipError_t embed_back_parts(EmbedBackParams p, hipStream_t s) {
  const int kind = kind_of(p.cols);
  const int64_t parts = (int64_t)p.runs * p.tiles;
  return in_launches(parts + p.fill_wgs, [&](int64_t at, uint32_t wgs) {
    p.wg0 = at;
    p.fill_wg0 = at > parts ? at : parts;   // the launch's first one for ids without rows
    const int64_t quads = (p.fill_wg0 - parts) * (kBackThreads * kBackFill);
    p.fill_row0 = quads / p.quads.blocks;
    p.fill_quad0 = (uint32_t)(quads % p.quads.blocks);
    if (kind == kWhole) hipLaunchKernelGGL((k_embed_back<B16, DROP, kWhole>), dim3(wgs), dim3(kBackThreads), 0, s, p);
    else if (kind == kPart) hipLaunchKernelGGL((k_embed_back<B16, DROP, kPart>), dim3(wgs), dim3(kBackThreads), 0, s, p);
    else hipLaunchKernelGGL((k_embed_back<B16, DROP, kFew>), dim3(wgs), dim3(kBackThreads), 0, s, p);
  });
}

template <bool B16>
hipError_t embed_back(EmbedBackParams p, hipStream_t s) {
  hipError_t e = p.drop.least ? embed_back_parts<B16, true>(p, s) : embed_back_parts<B16, false>(p, s);
  if (e == hipSuccess && p.runs > 1) {
    const uint32_t quads = p.cols.blocks * 8 / kJoinCols, tiles = (quads + kBackThreads - 1) / kBackThreads;
    e = in_launches((int64_t)(p.runs - 1) * tiles, [&](int64_t at, uint32_t wgs) {
      p.wg0 = at;
      hipLaunchKernelGGL(k_embed_join, dim3(wgs), dim3(kBackThreads), 0, s, p, tiles);
    });
  }
  return e;
}

}  // namespace

hipError_t launch_embed(const EmbedParams &p, bool src16, bool dst16, hipStream_t s) {
  if (!p.ids) return src16 ? dropout<true>(p, s) : dropout<false>(p, s);
  if (src16) return dst16 ? lookup<true, true>(p, s) : lookup<true, false>(p, s);
  return dst16 ? lookup<false, true>(p, s) : lookup<false, false>(p, s);
}

hipError_t launch_embed_back(const EmbedBackParams &p, bool dy16, hipStream_t s) {
  return dy16 ? embed_back<true>(p, s) : embed_back<false>(p, s);
}

}  // namespace ks
