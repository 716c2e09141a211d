// The rows by id (ks.h, ks_embed_sort): a stable counting sort by digits of 8 to
// 10 bits, the low ones first.  An id at or beyond n_ids sorts as n_ids.
//
//   k_order_count   how often each digit occurs in each chunk of the keys
//   k_order_sum     for a digit, how often it occurs in the chunks before each, and in all
//                   (of many chunks)
//   k_order_place   each key to its place: its digit's first one, the chunk's before it,
//                   and its rank among the chunk's equal ones
//   k_order_off     off[] from the sorted ids, where more than one pass made them
//   k_order_within  for few keys of two digits, placed by the high one: a workgroup for each
//                   high digit places its keys by the low one, and knows its ids' offsets
//   k_order_small   all passes for up to 8192 keys, which one workgroup holds
//
// The rank comes from one ballot per bit: the lanes with the same digit are a mask, and
// what the wave had before stands in its own counters in LDS.  No atomic's order enters.
//
// Launches bound small calls: 4099 rows of 67 ids take 7 us, of 32,000 15, 16,381 rows 8 and
// 18.  300,007 rows of 1009 ids take 15 us, 2,000,003 of 67 26, of 131,072 75 (24 MB a pass
// at least, 5 us: what is left is scattered stores and the counting's way through LDS).
#include <hip/hip_runtime.h>

#include "ks_columns.h"

namespace ks {

namespace {

constexpr int kRounds = kOrderKeys / kOrderThreads;
constexpr int kSmallThreads = 1024;

__device__ __forceinline__ uint32_t key_of(uint32_t id, uint32_t n_ids) { return id < n_ids ? id : n_ids; }

// Keys behind the last one have all bits set: they come last in each pass, behind the keys
// of their digit, so that all lanes always hold a key.
constexpr uint32_t kBehind = 0xFFFFFFFFu;

// the lanes that hold the same digit: for each of its bits those that have it set or not as
// this one has
template <int BITS>
__device__ __forceinline__ uint64_t same_lanes(uint32_t digit) {
  uint32_t lo = 0xFFFFFFFFu, hi = 0xFFFFFFFFu;
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const uint32_t set = (uint32_t)((int32_t)(digit << (31 - b)) >> 31);
    const uint64_t s = __ballot(set != 0);
    lo &= ~((uint32_t)s ^ set);
    hi &= ~((uint32_t)(s >> 32) ^ set);
  }
  return (uint64_t)hi << 32 | lo;
}

// inclusive prefix sums over a wave
__device__ __forceinline__ uint32_t prefix(uint32_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// exclusive prefix sums over a workgroup's W waves
template <int W>
__device__ __forceinline__ uint32_t before(uint32_t v, uint32_t (&room)[W]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t sum = prefix(v);
  if (lane == 63) room[wave] = sum;
  __syncthreads();
  uint32_t base = 0;
  for (int w = 0; w < wave; ++w) base += room[w];
  return base + sum - v;
}

// The ranks of K keys a lane, 64 consecutive ones at a time, among the wave's keys of the same
// digit; count: the wave's counters, which keep how many of each digit it has
template <int BITS, int K, class T>
__device__ __forceinline__ void ranks(uint32_t (&rank)[K], const uint32_t (&key)[K], T *count, int shift) {
#pragma unroll
  for (int r = 0; r < K; ++r) {
    const uint32_t digit = key[r] >> shift & ((1u << BITS) - 1);
    const uint64_t m = same_lanes<BITS>(digit);
    const uint32_t lo = (uint32_t)m, hi = (uint32_t)(m >> 32), all = __popc(lo) + __popc(hi);
    const uint32_t had = count[digit], below = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
    rank[r] = had + below;
    if (below + 1 == all) count[digit] = (T)(had + all);   // the last of them
    // (a lane reads next what another one has written)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// K keys a thread; keys and rows pass through LDS between two digits.  (Places and counts
// of so few keys fit 16 bits.)  4000 keys in two digits take 13 us so, and the offsets; in five
// launches of the kernels below 20.
constexpr uint32_t kOffHere = 4096;   // ids up to which the offsets are found here
template <int BITS, int K>
__global__ __launch_bounds__(kSmallThreads) void k_order_small(OrderParams a) {
  constexpr uint32_t kBins = 1u << BITS, bins = kBins;
  __shared__ uint32_t keys[kSmallThreads * K], room[kSmallThreads / 64];
  __shared__ uint16_t rows[kSmallThreads * K], count[kSmallThreads / 64][kBins];
  const uint32_t n = a.n_rows;
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, from = wave * (64 * K) + lane;
  uint32_t k[K], row[K], rank[K];
#pragma unroll
  for (int r = 0; r < K; ++r) {
    const uint32_t p = from + 64 * r;
    row[r] = p;
    k[r] = p < n ? key_of(a.ids[p], a.n_ids) : kBehind;
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * BITS;
    for (uint32_t i = threadIdx.x; i < kSmallThreads / 64 * bins; i += kSmallThreads) count[i >> BITS][i & (bins - 1)] = 0;
    __syncthreads();
    ranks<BITS>(rank, k, count[wave], shift);
    __syncthreads();
    {
      const uint32_t d = threadIdx.x;
      uint32_t total = 0;
      if (d < bins)
        for (int w = 0; w < kSmallThreads / 64; ++w) {
          const uint32_t c = count[w][d];
          count[w][d] = (uint16_t)total;
          total += c;
        }
      const uint32_t first = before(total, room);
      if (d < bins)
        for (int w = 0; w < kSmallThreads / 64; ++w) count[w][d] = (uint16_t)(count[w][d] + first);
      if (a.passes == 1 && d < bins && d <= a.n_ids) a.off[d] = first;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < K; ++r) {
      const uint32_t at = count[wave][k[r] >> shift & (bins - 1)] + rank[r];
      keys[at] = k[r];
      rows[at] = (uint16_t)row[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < K; ++r) {
      k[r] = keys[from + 64 * r];
      row[r] = rows[from + 64 * r];
    }
  }
#pragma unroll
  for (int r = 0; r < K; ++r) {
    if (from + 64 * r >= n) continue;
    a.id[from + 64 * r] = k[r];
    a.row[from + 64 * r] = row[r];
  }
  if (a.passes == 1 || a.n_ids > kOffHere) return;
  for (uint32_t v = threadIdx.x; v <= a.n_ids; v += kSmallThreads) {
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if (keys[mid] < v) lo = mid + 1;
      else hi = mid;
    }
    a.off[v] = lo;
  }
}

template <int BITS>
__global__ __launch_bounds__(kOrderThreads) void k_order_count(OrderParams a, const uint32_t *key, int shift) {
  constexpr uint32_t kBins = 1u << BITS, bins = kBins;
  __shared__ uint32_t count[kBins];
  for (uint32_t d = threadIdx.x; d < bins; d += kOrderThreads) count[d] = 0;
  __syncthreads();
  const uint32_t lo = blockIdx.x * a.chunk, hi = a.n_rows - lo < a.chunk ? a.n_rows : lo + a.chunk;
  for (uint32_t p = lo + threadIdx.x; p < hi; p += kOrderThreads)
    atomicAdd(&count[key_of(key[p], a.n_ids) >> shift & (bins - 1)], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < bins; d += kOrderThreads) a.hist[(size_t)blockIdx.x * bins + d] = count[d];
}

// Sixteen digits a workgroup, their chunks in 64 slices.  With few chunks k_order_place adds
// up their counts itself (65,536 keys of 32,000 ids: 27 us in five launches, 29 in
// seven).
constexpr uint32_t kFewChunks = 32;
constexpr uint32_t kSumDigits = 16, kSumSlices = 64;
template <int BITS>
__global__ __launch_bounds__(kSumDigits * kSumSlices) void k_order_sum(OrderParams a) {
  constexpr uint32_t bins = 1u << BITS;
  __shared__ uint32_t room[kSumSlices][kSumDigits];
  const uint32_t i = threadIdx.x % kSumDigits, slice = threadIdx.x / kSumDigits, d = blockIdx.x * kSumDigits + i;
  const uint32_t per = (a.chunks + kSumSlices - 1) / kSumSlices, lo = min(slice * per, a.chunks), hi = min(lo + per, a.chunks);
  uint32_t *h = a.hist + d;
  uint32_t sum = 0;
#pragma unroll 8
  for (uint32_t c = lo; c < hi; ++c) sum += h[(size_t)c * bins];
  room[slice][i] = sum;
  __syncthreads();
  uint32_t at = 0;
#pragma unroll 8
  for (uint32_t s = 0; s < slice; ++s) at += room[s][i];
  if (slice == kSumSlices - 1) a.total[d] = at + sum;
#pragma unroll 8
  for (uint32_t c = lo; c < hi; ++c) {
    const uint32_t v = h[(size_t)c * bins];
    h[(size_t)c * bins] = at;
    at += v;
  }
}

// Keys [lo, hi) to their places: base[d] is where the next key with digit d goes (shared;
// a barrier before the call), count room for the waves' counters
template <int BITS, int W>
__device__ __forceinline__ void place_keys(uint32_t n_ids, const uint32_t *key, const uint32_t *row, uint32_t *to_key, uint32_t *to_row,
                                           uint32_t lo, uint32_t hi, int shift, uint32_t (&base)[1 << BITS],
                                           uint32_t (&count)[W][1 << BITS]) {
  constexpr uint32_t kBins = 1u << BITS;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (uint32_t from = lo; from < hi; from += 64 * W * kRounds) {
    for (uint32_t d = threadIdx.x; d < W * kBins; d += 64 * W) count[d >> BITS][d & (kBins - 1)] = 0;
    uint32_t k[kRounds], rank[kRounds];
    const uint32_t p0 = from + wave * (64 * kRounds) + lane;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) k[r] = p0 + 64 * r < hi ? key_of(key[p0 + 64 * r], n_ids) : kBehind;
    __syncthreads();
    ranks<BITS>(rank, k, count[wave], shift);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < kBins; d += 64 * W) {
      uint32_t at = base[d];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const uint32_t c = count[w][d];
        count[w][d] = at;
        at += c;
      }
      base[d] = at;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const uint32_t p = p0 + 64 * r;
      if (p >= hi) continue;
      const uint32_t at = count[wave][k[r] >> shift & (kBins - 1)] + rank[r];
      to_key[at] = k[r];
      to_row[at] = row ? row[p] : p;
    }
    __syncthreads();
  }
}

template <int BITS>
__global__ __launch_bounds__(kOrderThreads) void k_order_place(OrderParams a, const uint32_t *key, const uint32_t *row, uint32_t *to_key,
                                                               uint32_t *to_row, int shift, bool only) {
  constexpr uint32_t kBins = 1u << BITS, bins = kBins;
  constexpr int W = kOrderThreads / 64;
  __shared__ uint32_t count[W][kBins], base[kBins], room[W];
  // workgroups go to the eight dies in turn: consecutive chunks, whose keys of one digit go
  // to consecutive places, to the same one, so that few lines are written by two
  const uint32_t per = (a.chunks + 7) / 8, chunk = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (chunk >= a.chunks) return;
  {
    // consecutive digits a thread
    constexpr int D = kBins < kOrderThreads ? 1 : kBins / kOrderThreads;
    uint32_t total[D], chunks_before[D], sum = 0;
#pragma unroll
    for (int i = 0; i < D; ++i) {
      const uint32_t d = threadIdx.x * D + i;
      total[i] = chunks_before[i] = 0;
      if (d < bins) {
        const uint32_t *h = a.hist + d;
        if (a.chunks > kFewChunks) {
          total[i] = a.total[d];
          chunks_before[i] = h[(size_t)chunk * bins];
        } else {
#pragma unroll 8
          for (uint32_t c = 0; c < a.chunks; ++c) {
            const uint32_t v = h[(size_t)c * bins];
            total[i] += v;
            chunks_before[i] += c < chunk ? v : 0;
          }
        }
      }
      sum += total[i];
    }
    uint32_t first = before(sum, room);
#pragma unroll
    for (int i = 0; i < D; ++i) {
      const uint32_t d = threadIdx.x * D + i;
      if (d < bins) base[d] = first + chunks_before[i];
      if (only && chunk == 0 && d <= a.n_ids && d < bins) a.off[d] = first;
      first += total[i];
    }
  }
  const uint32_t lo = chunk * a.chunk, hi = a.n_rows - lo < a.chunk ? a.n_rows : lo + a.chunk;
  place_keys<BITS>(a.n_ids, key, row, to_key, to_row, lo, hi, shift, base, count);
}

// From 4097 keys to kWithin: 16,381 of 32,000 ids, a fifth of them under one high digit, take 18 us
// so, 23 by the low digit first in five launches; all under one, in one workgroup, 42.
// 3000 take 14, 13 in k_order_small.
constexpr uint32_t kWithin = 16384;
template <int BITS>
__global__ __launch_bounds__(kSmallThreads) void k_order_within(OrderParams a) {
  constexpr uint32_t kBins = 1u << BITS;
  constexpr int W = kSmallThreads / 64, D = kBins < kSmallThreads ? 1 : kBins / kSmallThreads;
  __shared__ uint32_t count[W][kBins], base[kBins], room[W], ends[2];
  // where this high digit's keys are: how many lower ones there are, and how many of its own
  const uint32_t high = blockIdx.x;
  uint32_t lower = 0, own = 0;
  for (uint32_t i = threadIdx.x; i < a.chunks << BITS; i += kSmallThreads) {
    const uint32_t v = a.hist[i], d = i & (kBins - 1);
    lower += d < high ? v : 0;
    own += d == high ? v : 0;
  }
  for (uint32_t d = threadIdx.x; d < kBins; d += kSmallThreads) base[d] = 0;
  if (threadIdx.x < 2) ends[threadIdx.x] = 0;
#pragma unroll
  for (int d = 32; d > 0; d /= 2) {
    lower += __shfl_xor(lower, d);
    own += __shfl_xor(own, d);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    atomicAdd(&ends[0], lower);
    atomicAdd(&ends[1], own);
  }
  __syncthreads();
  const uint32_t lo = ends[0], hi = min(lo + ends[1], a.n_rows);
  for (uint32_t p = lo + threadIdx.x; p < hi; p += kSmallThreads) atomicAdd(&base[a.tmp_id[p] & (kBins - 1)], 1u);
  __syncthreads();
  uint32_t total[D], sum = 0;
#pragma unroll
  for (int i = 0; i < D; ++i) {
    const uint32_t d = threadIdx.x * D + i;
    total[i] = d < kBins ? base[d] : 0;
    sum += total[i];
  }
  uint32_t first = lo + before(sum, room);   // (a barrier between the reads and the writes)
#pragma unroll
  for (int i = 0; i < D; ++i) {
    const uint32_t d = threadIdx.x * D + i;
    if (d < kBins) {
      base[d] = first;
      if ((high << BITS) + d <= a.n_ids) a.off[(high << BITS) + d] = first;
    }
    first += total[i];
  }
  __syncthreads();
  place_keys<BITS>(a.n_ids, a.tmp_id, a.tmp_row, a.id, a.row, lo, hi, 0, base, count);
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

template <int BITS>
hipError_t order(const OrderParams &p, hipStream_t s) {
  const uint32_t *key = p.ids, *row = nullptr;
  const dim3 wg(kOrderThreads), small_wg(kSmallThreads);
  const bool within = p.passes == 2 && p.n_ids > kOffHere && p.n_rows > kSmallThreads * 4 && p.n_rows <= kWithin;
  const bool small = !within && p.n_rows > 0 && p.n_rows <= kSmallThreads * 8;
  if (within) {
    hipLaunchKernelGGL((k_order_count<BITS>), dim3(p.chunks), wg, 0, s, p, key, BITS);
    hipLaunchKernelGGL((k_order_place<BITS>), dim3((p.chunks + 7) / 8 * 8), wg, 0, s, p, key, row, p.tmp_id, p.tmp_row, BITS, false);
    hipLaunchKernelGGL((k_order_within<BITS>), dim3((p.n_ids >> BITS) + 1), small_wg, 0, s, p);
    return hipGetLastError();
  }
  if (small) {
    if (p.n_rows <= kSmallThreads * 4) hipLaunchKernelGGL((k_order_small<BITS, 4>), dim3(1), small_wg, 0, s, p);
    else hipLaunchKernelGGL((k_order_small<BITS, 8>), dim3(1), small_wg, 0, s, p);
  }
  for (int i = 0; i < p.passes && p.n_rows > 0 && !small; ++i) {
    const bool last = (p.passes - 1 - i) % 2 == 0;
    uint32_t *to_key = last ? p.id : p.tmp_id, *to_row = last ? p.row : p.tmp_row;
    hipLaunchKernelGGL((k_order_count<BITS>), dim3(p.chunks), wg, 0, s, p, key, i * BITS);
    if (p.chunks > kFewChunks) hipLaunchKernelGGL((k_order_sum<BITS>), dim3((1u << BITS) / kSumDigits), dim3(kSumDigits * kSumSlices), 0, s, p);
    hipLaunchKernelGGL((k_order_place<BITS>), dim3((p.chunks + 7) / 8 * 8), wg, 0, s, p, key, row, to_key, to_row, i * BITS, p.passes == 1);
    key = to_key;
    row = to_row;
  }
  if (p.n_rows == 0 || (p.passes > 1 && !(small && p.n_ids <= kOffHere)))
    hipLaunchKernelGGL(k_order_off, dim3(p.n_ids / 256 + 1), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_order(const OrderParams &p, hipStream_t s) {
  static_assert(kOrderBits == kOrderFew + 2, "one of these");
  return p.bits == kOrderFew ? order<kOrderFew>(p, s) : p.bits == kOrderBits ? order<kOrderBits>(p, s) : order<kOrderFew + 1>(p, s);
}

}  // namespace ks
