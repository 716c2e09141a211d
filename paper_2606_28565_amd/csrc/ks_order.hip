// The rows by id (ks.h, ks_embed_sort): a stable counting sort by digits of at most
// 10 bits, the low ones first.  An id at or beyond n_ids sorts as n_ids.
//
//   k_order_count   how often each digit occurs in each chunk of the keys
//   k_order_sum     for a digit, how often it occurs in the chunks before each, and in all
//   k_order_place   each key to its place: its digit's first one, the chunk's before it,
//                   and its rank among the chunk's equal ones
//   k_order_off     off[] from the sorted ids, where more than one pass made them
//   k_order_small   all passes for up to 16,384 keys, which one workgroup holds
//
// The rank comes from one ballot per bit: the lanes with the same digit are a mask, and
// what the wave had before stands in its own counters in LDS.  No atomic's order enters.
#include <hip/hip_runtime.h>

#include "ks_internal.h"

namespace ks {

namespace {

constexpr int kThreads = kOrderThreads, kWaves = kThreads / 64, kRounds = kOrderKeys / kThreads;
constexpr int kBins = 1 << kOrderBits;

__device__ __forceinline__ uint32_t key_of(uint32_t id, uint32_t n_ids) { return id < n_ids ? id : n_ids; }

// the lanes that hold the same digit, among those with `in`
__device__ __forceinline__ uint64_t same_lanes(uint32_t digit, bool in, int bits) {
  uint64_t m = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const bool set = digit >> b & 1;
    const uint64_t s = __ballot(set);
    m &= set ? s : ~s;
  }
  return m;
}

// exclusive prefix sums over the workgroup's threads
__device__ __forceinline__ uint32_t before(uint32_t v, uint32_t (&room)[kWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(sum, d);
    if (lane >= d) sum += o;
  }
  __syncthreads();
  if (lane == 63) room[wave] = sum;
  __syncthreads();
  uint32_t base = 0;
  for (int w = 0; w < wave; ++w) base += room[w];
  return base + sum - v;
}

// A wave's rank of `digit` among its keys so far, and the count that it leaves for the next
template <class T>
__device__ __forceinline__ uint32_t rank_of(T *count, uint32_t digit, bool in, int bits) {
  const uint64_t m = same_lanes(digit, in, bits);
  const int lane = threadIdx.x & 63;
  uint32_t rank = 0;
  if (in) {
    const uint32_t had = count[digit];
    rank = had + (uint32_t)__popcll(m & ((uint64_t(1) << lane) - 1));
    if (m >> lane == 1) count[digit] = (T)(had + (uint32_t)__popcll(m));   // the last of them
  }
  // (a lane reads next what another one has written)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return rank;
}

// K keys a thread; keys and rows pass through LDS between two digits.  (Places and counts
// of 16,384 keys fit 16 bits.)
constexpr uint32_t kOffHere = 4096;   // ids up to which the offsets are found here
template <int K>
__global__ __launch_bounds__(kThreads) void k_order_small(OrderParams a) {
  __shared__ uint32_t keys[kThreads * K], room[kWaves];
  __shared__ uint16_t rows[kThreads * K], count[kWaves][kBins];
  const uint32_t bins = 1u << a.bits, n = a.n_rows;
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, from = wave * (64 * K) + lane;
  uint32_t k[K], row[K], rank[K];
#pragma unroll
  for (int r = 0; r < K; ++r) {
    const uint32_t p = from + 64 * r;
    row[r] = p;
    k[r] = p < n ? key_of(a.ids[p], a.n_ids) : 0;
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    for (uint32_t i = threadIdx.x; i < kWaves * bins; i += kThreads) count[i >> a.bits][i & (bins - 1)] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < K; ++r)
      if (wave * (64 * K) + 64 * r < n) rank[r] = rank_of(count[wave], k[r] >> shift & (bins - 1), from + 64 * r < n, a.bits);
    __syncthreads();
    {
      const uint32_t d = threadIdx.x;
      uint32_t total = 0;
      if (d < bins)
        for (int w = 0; w < kWaves; ++w) {
          const uint32_t c = count[w][d];
          count[w][d] = (uint16_t)total;
          total += c;
        }
      const uint32_t first = before(total, room);
      if (d < bins)
        for (int w = 0; w < kWaves; ++w) count[w][d] = (uint16_t)(count[w][d] + first);
      if (a.passes == 1 && d < bins && d <= a.n_ids) a.off[d] = first;
    }
    __syncthreads();
    const bool last = pass + 1 == a.passes;
#pragma unroll
    for (int r = 0; r < K; ++r) {
      if (from + 64 * r >= n) continue;
      const uint32_t at = count[wave][k[r] >> shift & (bins - 1)] + rank[r];
      keys[at] = k[r];
      if (last) {
        a.id[at] = k[r];
        a.row[at] = row[r];
      } else {
        rows[at] = (uint16_t)row[r];
      }
    }
    __syncthreads();
    if (last) break;
#pragma unroll
    for (int r = 0; r < K; ++r) {
      if (from + 64 * r >= n) continue;
      k[r] = keys[from + 64 * r];
      row[r] = rows[from + 64 * r];
    }
  }
  if (a.passes == 1 || a.n_ids > kOffHere) return;
  for (uint32_t v = threadIdx.x; v <= a.n_ids; v += kThreads) {
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if (keys[mid] < v) lo = mid + 1;
      else hi = mid;
    }
    a.off[v] = lo;
  }
}

__global__ __launch_bounds__(kThreads) void k_order_count(OrderParams a, const uint32_t *key, int shift) {
  __shared__ uint32_t count[kBins];
  const uint32_t bins = 1u << a.bits;
  for (uint32_t d = threadIdx.x; d < bins; d += kThreads) count[d] = 0;
  __syncthreads();
  const uint32_t lo = blockIdx.x * a.chunk, hi = a.n_rows - lo < a.chunk ? a.n_rows : lo + a.chunk;
  for (uint32_t p = lo + threadIdx.x; p < hi; p += kThreads) atomicAdd(&count[key_of(key[p], a.n_ids) >> shift & (bins - 1)], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < bins; d += kThreads) a.hist[(size_t)d * a.chunks + blockIdx.x] = count[d];
}

__global__ __launch_bounds__(kThreads) void k_order_sum(OrderParams a) {
  __shared__ uint32_t room[kWaves];
  uint32_t *h = a.hist + (size_t)blockIdx.x * a.chunks, sum = 0;
  for (uint32_t c0 = 0; c0 < a.chunks; c0 += kThreads) {
    const uint32_t c = c0 + threadIdx.x, v = c < a.chunks ? h[c] : 0;
    const uint32_t at = before(v, room);
    if (c < a.chunks) h[c] = sum + at;
    for (int w = 0; w < kWaves; ++w) sum += room[w];
  }
  if (threadIdx.x == 0) a.total[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void k_order_place(OrderParams a, const uint32_t *key, const uint32_t *row, uint32_t *to_key,
                                                          uint32_t *to_row, int shift, bool only) {
  __shared__ uint32_t count[kWaves][kBins], base[kBins], room[kWaves];
  const uint32_t bins = 1u << a.bits;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  {
    const uint32_t d = threadIdx.x, first = before(d < bins ? a.total[d] : 0, room);
    if (d < bins) base[d] = first + a.hist[(size_t)d * a.chunks + blockIdx.x];
    if (only && blockIdx.x == 0 && d <= a.n_ids && d < bins) a.off[d] = first;
  }
  const uint32_t lo = blockIdx.x * a.chunk, hi = a.n_rows - lo < a.chunk ? a.n_rows : lo + a.chunk;
  for (uint32_t from = lo; from < hi; from += kOrderKeys) {
    for (uint32_t d = threadIdx.x; d < kWaves * bins; d += kThreads) count[d >> a.bits][d & (bins - 1)] = 0;
    __syncthreads();
    uint32_t k[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const uint32_t p = from + wave * (64 * kRounds) + 64 * r + lane;
      k[r] = p < hi ? key_of(key[p], a.n_ids) : 0;
      rank[r] = rank_of(count[wave], k[r] >> shift & (bins - 1), p < hi, a.bits);
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < bins; d += kThreads) {
      uint32_t at = base[d];
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = count[w][d];
        count[w][d] = at;
        at += c;
      }
      base[d] = at;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const uint32_t p = from + wave * (64 * kRounds) + 64 * r + lane;
      if (p >= hi) continue;
      const uint32_t at = count[wave][k[r] >> shift & (bins - 1)] + rank[r];
      to_key[at] = k[r];
      to_row[at] = row ? row[p] : p;
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void k_order_off(OrderParams a) {
  const uint32_t v = blockIdx.x * 256 + threadIdx.x;
  if (v > a.n_ids) return;
  uint32_t lo = 0, hi = a.n_rows;   // the first place of an id at least v
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.id[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  a.off[v] = lo;
}

}  // namespace

hipError_t launch_order(const OrderParams &p, hipStream_t s) {
  const uint32_t *key = p.ids, *row = nullptr;
  const dim3 wg(kThreads);
  const bool small = p.n_rows > 0 && p.n_rows <= kThreads * 16;
  if (small) {
    if (p.n_rows <= kThreads * 4) hipLaunchKernelGGL(k_order_small<4>, dim3(1), wg, 0, s, p);
    else if (p.n_rows <= kThreads * 8) hipLaunchKernelGGL(k_order_small<8>, dim3(1), wg, 0, s, p);
    else hipLaunchKernelGGL(k_order_small<16>, dim3(1), wg, 0, s, p);
  }
  for (int i = 0; i < p.passes && p.n_rows > 0 && !small; ++i) {
    const bool last = (p.passes - 1 - i) % 2 == 0;
    uint32_t *to_key = last ? p.id : p.tmp_id, *to_row = last ? p.row : p.tmp_row;
    hipLaunchKernelGGL(k_order_count, dim3(p.chunks), wg, 0, s, p, key, i * p.bits);
    hipLaunchKernelGGL(k_order_sum, dim3(1u << p.bits), wg, 0, s, p);
    hipLaunchKernelGGL(k_order_place, dim3(p.chunks), wg, 0, s, p, key, row, to_key, to_row, i * p.bits, p.passes == 1);
    key = to_key;
    row = to_row;
  }
  if (p.n_rows == 0 || (p.passes > 1 && !(small && p.n_ids <= kOffHere)))
    hipLaunchKernelGGL(k_order_off, dim3(p.n_ids / 256 + 1), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace ks
