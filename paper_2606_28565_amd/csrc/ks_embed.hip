// Dropout, the lookup of a table's rows by id, and the table's gradient (ks.h).
//
//   k_embed        dst_i = drop(factor src_i), src_i the table's row of id i (the
//                  lookup) or row i itself (dropout)
//   k_embed_back   rows of the table's gradient: of ids with few rows, and the sums
//                  over parts of the order of the others
//   k_embed_join   the sums of ids that have rows in more than one part
//
// A lane's work is a block of eight columns of one row: 16 bytes of bfloat16, 32 of
// fp32, and exactly one Philox block's draws.  Each element is read and written once, so
// bytes bound all three.
#include <hip/hip_runtime.h>

#include "ks_internal.h"

namespace ks {

namespace {

constexpr int kThreads = 256;

// eight elements, by default as zeros; rows of any alignment of the type's
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

// the first `rem` of a row's last block (1 .. 7; the same in all lanes), or eight
template <bool B16>
__device__ __forceinline__ Eight<B16> load8(const void *base, int64_t at, bool whole, uint32_t rem) {
  Eight<B16> o;
  if constexpr (B16) {
    const char *p = (const char *)base + 2 * at;
    if (whole) {
      o.w[0] = *(const any_u32x4 *)p;
      return o;
    }
    o.w[0] = u32x4{0, 0, 0, 0};
    if (rem & 4) {
      const u32x2 v = *(const any_u32x2 *)p;
      o.w[0][0] = v[0];
      o.w[0][1] = v[1];
    }
    if (rem & 2) {
      const uint32_t v = *(const any_u32 *)(p + 2 * (rem & 4));
      if (rem & 4) o.w[0][2] = v;
      else o.w[0][0] = v;
    }
    if (rem & 1) {
      const uint32_t v = *(const uint16_t *)(p + 2 * (rem & 6));
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) o.w[0][j] = rem / 2 == j ? v : o.w[0][j];
    }
  } else {
    const uint32_t *p = (const uint32_t *)base + at;
    if (whole) {
      o.w[0] = *(const any_u32x4 *)p;
      o.w[1] = *(const any_u32x4 *)(p + 4);
      return o;
    }
    o.w[0] = o.w[1] = u32x4{0, 0, 0, 0};
    u32x4 v = {0, 0, 0, 0};
    if (rem & 4) o.w[0] = *(const any_u32x4 *)p;
    if (rem & 2) {
      const u32x2 h = *(const any_u32x2 *)(p + (rem & 4));
      v[0] = h[0];
      v[1] = h[1];
    }
    if (rem & 1) {
      const uint32_t h = p[rem & 6];
      v[0] = rem & 2 ? v[0] : h;
      v[2] = rem & 2 ? h : 0;
    }
    if (rem & 4) o.w[1] = v;
    else o.w[0] = v;
  }
  return o;
}

__device__ __forceinline__ uint32_t pair(float lo, float hi) {
  return __builtin_bit_cast(uint16_t, (__bf16)lo) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16;
}

template <bool B16>
__device__ __forceinline__ void store8(void *base, int64_t at, f32x8 v, bool whole, uint32_t rem) {
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
__device__ __forceinline__ Draws philox(const Drop &d, uint64_t block, uint32_t step) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = step, c3 = d.site;
  uint32_t k0 = d.key0, k1 = d.key1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}
__device__ __forceinline__ uint32_t step_of(const Drop &d) { return d.step_dev ? *d.step_dev : d.step; }

// row and block of the l-th block from row 0 on; l < 2^31
__device__ __forceinline__ uint32_t row_in(const Cols &c, uint32_t l, uint32_t &b) {
  uint32_t q = c.magic ? __umulhi(l, c.magic) : l;
  // (ceil(2^32 / blocks) is at most blocks - 1 over: one too many, where l is large)
  if (c.magic && q * c.blocks > l) --q;
  b = l - q * c.blocks;
  return q;
}
// ... of the workgroup's lane l: the workgroup starts at block `first` of all
__device__ __forceinline__ int64_t row_of(const Cols &c, int64_t first, uint32_t l, uint32_t &b) {
  const int64_t row = (uint64_t)first < (uint64_t(1) << 32) ? (int64_t)((uint32_t)first / c.blocks) : first / c.blocks;
  return row + row_in(c, (uint32_t)(first - row * c.blocks) + l, b);
}
__device__ __forceinline__ bool whole(const Cols &c, uint32_t b) { return c.rem == 0 || b + 1 < c.blocks; }

// ------------------------------------------------------------ lookup and dropout
template <bool S16, bool D16, bool DROP>
__global__ __launch_bounds__(kThreads) void k_embed(EmbedParams a) {
  uint32_t b;
  const int64_t first = (a.wg0 + blockIdx.x) * kThreads;
  const int64_t i = row_of(a.cols, first, threadIdx.x, b);
  if (i >= a.n_rows) return;
  const bool all = whole(a.cols, b);
  const int64_t id = a.ids ? (int64_t)a.ids[i] : i;
  f32x8 v = {};
  if (!a.ids || id < a.n_ids) {
    const Eight<S16> x = load8<S16>(a.src, id * a.src_ld + 8 * (int64_t)b, all, a.cols.rem);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = x[j] * a.factor;
  }
  if constexpr (DROP) {
    const Draws d = philox(a.drop, (uint64_t)(first + threadIdx.x), step_of(a.drop));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = d[j] >= a.drop.least ? v[j] : 0.0f;
  }
  store8<D16>(a.dst, i * a.dst_ld + 8 * (int64_t)b, v, all, a.cols.rem);
}

// ------------------------------------------------------------ the table's gradient
// acc += drop(dy of the row at place p of the order), columns of block b
template <bool B16, bool DROP>
__device__ __forceinline__ void add_row(f32x8 &acc, const EmbedBackParams &a, uint32_t p, uint32_t b, bool all, uint32_t step) {
  const uint32_t i = a.row[p];
  if (i >= a.n_rows) return;
  const Eight<B16> x = load8<B16>(a.dy, (int64_t)i * a.ld + 8 * (int64_t)b, all, a.cols.rem);
  if constexpr (DROP) {
    const Draws d = philox(a.drop, (uint64_t)i * a.cols.blocks + b, step);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += d[j] >= a.drop.least ? x[j] : 0.0f;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += x[j];
  }
}

// the places of id v
__device__ __forceinline__ void places(const EmbedBackParams &a, uint32_t v, uint32_t &begin, uint32_t &end) {
  const uint32_t n = (uint32_t)a.n_rows;
  begin = min(a.off[v], n);
  end = min(a.off[v + 1], n);
}

template <bool B16, bool DROP>
__global__ __launch_bounds__(kBackThreads) void k_embed_back(EmbedBackParams a) {
  const uint32_t step = DROP ? step_of(a.drop) : 0;
  const int64_t at = a.wg0 + blockIdx.x;
  if (at < a.short_wgs) {
    uint32_t b;
    const int64_t v = row_of(a.cols, at * kBackThreads, threadIdx.x, b);
    if (v >= a.n_ids) return;
    uint32_t p, end;
    places(a, (uint32_t)v, p, end);
    if (end > p && end - p > kBackShort) return;
    const bool all = whole(a.cols, b);
    f32x8 acc = {};
    for (; p < end; ++p) add_row<B16, DROP>(acc, a, p, b, all, step);
    acc *= a.factor;
    store8<false>(a.grad, v * a.grad_ld + 8 * (int64_t)b, acc, all, a.cols.rem);
    return;
  }
  // the ids with many rows that have some among this workgroup's places
  __shared__ uint32_t begins[kBackMost], n_begins;
  __shared__ float red[kBackThreads][8];
  const uint32_t wg = (uint32_t)(at - a.short_wgs), part = wg / a.tiles, tile = wg % a.tiles;
  const uint32_t n = (uint32_t)a.n_rows, lo = part * a.run, hi = n - lo < a.run ? n : lo + a.run;
  if (threadIdx.x == 0) n_begins = 0;
  __syncthreads();
  for (uint32_t p = lo + threadIdx.x; p < hi; p += kBackThreads) {
    const uint32_t v = a.id[p];
    if (v >= a.n_ids || (p > lo && a.id[p - 1] == v)) continue;
    uint32_t s, e;
    places(a, v, s, e);
    if (e > s && e - s > kBackShort) {
      const uint32_t k = atomicAdd(&n_begins, 1u);   // (in any order: their sums do not meet)
      if (k < kBackMost) begins[k] = p;
    }
  }
  __syncthreads();
  const uint32_t many = min(n_begins, (uint32_t)kBackMost);
  const uint32_t wide = min(a.cols.blocks, (uint32_t)kBackThreads), groups = kBackThreads / wide;
  const uint32_t g = threadIdx.x / wide, b = tile * wide + threadIdx.x % wide;
  const bool in = g < groups && b < a.cols.blocks;
  const bool all = whole(a.cols, b);
  for (uint32_t k = 0; k < many; ++k) {
    const uint32_t v = a.id[begins[k]];
    uint32_t s, e;
    places(a, v, s, e);
    const uint32_t from = max(s, lo), to = min(e, hi);
    f32x8 acc = {};
    if (in) {
      // by runs of 64 rows a thread: 64 additions in a row, then one for each run
      for (uint32_t p = from + g; p < to;) {
        f32x8 sum = {};
        for (int i = 0; i < 64 && p < to; ++i, p += groups) add_row<B16, DROP>(sum, a, p, b, all, step);
        acc += sum;
      }
    }
    for (uint32_t half = 128; half > 0; half /= 2) {
      if (half >= groups) continue;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) red[threadIdx.x][j] = acc[j];
      __syncthreads();
      if (in && g < half && g + half < groups) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += red[threadIdx.x + half * wide][j];
      }
    }
    if (!in || g > 0) continue;
    if (s >= lo && e <= hi) {
      acc *= a.factor;
      store8<false>(a.grad, (int64_t)v * a.grad_ld + 8 * (int64_t)b, acc, all, a.cols.rem);
    } else {
      float *o = a.part + ((int64_t)(2 * part + (s >= lo)) * a.cols.blocks + b) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = acc[j];
    }
  }
}

// An id that begins in this part and goes on: its sum here, then those of the parts
// that it goes on in, in order
__global__ __launch_bounds__(kBackThreads) void k_embed_join(EmbedBackParams a, uint32_t tiles) {
  const int64_t at = a.wg0 + blockIdx.x;
  const uint32_t part = (uint32_t)(at / tiles), tile = (uint32_t)(at % tiles);
  const uint32_t next = (part + 1) * a.run;   // (not the last part: in the order)
  const uint32_t v = a.id[next - 1];
  if (v >= a.n_ids) return;
  uint32_t s, e;
  places(a, v, s, e);
  if (s < part * a.run || s >= next || e <= next || e - s <= kBackShort) return;
  const uint32_t last = min((e - 1) / a.run, a.runs - 1);
  const uint32_t cols = a.cols.blocks * 8, c = tile * kBackThreads + threadIdx.x;
  if (c >= (a.cols.rem ? cols - 8 + a.cols.rem : cols)) return;
  double sum = a.part[(int64_t)(2 * part + 1) * cols + c];
  for (uint32_t k = part + 1; k <= last; ++k) sum += a.part[(int64_t)(2 * k) * cols + c];
  a.grad[(int64_t)v * a.grad_ld + c] = (float)(sum * a.factor);
}

// launch(first workgroup, workgroups): as many as a launch takes at a time
template <class F>
hipError_t in_launches(int64_t wgs, F &&launch) {
  constexpr int64_t kMost = int64_t(1) << 23;
  for (int64_t at = 0; at < wgs; at += kMost) {
    launch(at, (uint32_t)(wgs - at < kMost ? wgs - at : kMost));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <bool S16, bool D16>
hipError_t embed(EmbedParams p, hipStream_t s) {
  return in_launches((p.n_rows * (int64_t)p.cols.blocks + kThreads - 1) / kThreads, [&](int64_t at, uint32_t wgs) {
    p.wg0 = at;
    if (p.drop.least) hipLaunchKernelGGL((k_embed<S16, D16, true>), dim3(wgs), dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((k_embed<S16, D16, false>), dim3(wgs), dim3(kThreads), 0, s, p);
  });
}

template <bool B16>
hipError_t embed_back(EmbedBackParams p, hipStream_t s) {
  hipError_t e = in_launches(p.short_wgs + (int64_t)p.runs * p.tiles, [&](int64_t at, uint32_t wgs) {
    p.wg0 = at;
    if (p.drop.least) hipLaunchKernelGGL((k_embed_back<B16, true>), dim3(wgs), dim3(kBackThreads), 0, s, p);
    else hipLaunchKernelGGL((k_embed_back<B16, false>), dim3(wgs), dim3(kBackThreads), 0, s, p);
  });
  if (e == hipSuccess && p.runs > 1) {
    const uint32_t tiles = (p.cols.blocks * 8 + kBackThreads - 1) / kBackThreads;
    e = in_launches((int64_t)(p.runs - 1) * tiles, [&](int64_t at, uint32_t wgs) {
      p.wg0 = at;
      hipLaunchKernelGGL(k_embed_join, dim3(wgs), dim3(kBackThreads), 0, s, p, tiles);
    });
  }
  return e;
}

}  // namespace

hipError_t launch_embed(const EmbedParams &p, bool src16, bool dst16, hipStream_t s) {
  if (src16) return dst16 ? embed<true, true>(p, s) : embed<true, false>(p, s);
  return dst16 ? embed<false, true>(p, s) : embed<false, false>(p, s);
}

hipError_t launch_embed_back(const EmbedBackParams &p, bool dy16, hipStream_t s) {
  return dy16 ? embed_back<true>(p, s) : embed_back<false>(p, s);
}

}  // namespace ks
