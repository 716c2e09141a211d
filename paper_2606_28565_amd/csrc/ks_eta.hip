// The loss on log eta at given z and its gradient (ks.h, ks_eta_loss).
//
//   k_eta_sum     dz before the division by sum w, and a workgroup's sum w rho, sum w
//   k_eta_scale   those sums of a family, in order, in 64 bits; dz over sum w
//   k_eta_one     both for families of few rows: a workgroup for each
//
// A workgroup works on rows of one family.  z, eta and the weight are read once and dz is
// written twice and read once, from the caches where it fits them: an exponential, two
// logarithms and a reciprocal a row are dear enough to keep what they give.
//
// 2,000,003 rows with weights: 16 us (32 MB: 7 at the rate of a copy; two launches are 8
// with few rows).  4099 rows in one launch: 5 us, as long as the call takes on the host;
// in two 8.  32,000 rows in one launch 11, in two 8: one up to 8192 rows of a family.
#include <hip/hip_runtime.h>

#include "ks_columns.h"
#include "ks_gated.h"

namespace ks {

namespace {

using gated::EtaTerm;
using gated::eta_term;

constexpr int kThreads = 256;
constexpr int kRows = 4;   // of a thread, on their way together

__device__ __forceinline__ int family_of(const EtaParams &p, int wg) {
  int f = 0;   // (all offsets read at once: no chain of scalar loads)
#pragma unroll
  for (int i = 1; i < KS_NFAM; ++i) f += wg >= p.wg[i];
  return f;
}

// sums of a pair over the workgroup's T threads, in every thread
template <int T>
__device__ __forceinline__ void sums(double &a, double &b) {
  __shared__ double room[T / 64][2];
#pragma unroll
  for (int d = 32; d > 0; d /= 2) {
    a += __shfl_xor(a, d);
    b += __shfl_xor(b, d);
  }
  if ((threadIdx.x & 63) == 0) {
    room[threadIdx.x >> 6][0] = a;
    room[threadIdx.x >> 6][1] = b;
  }
  __syncthreads();
  a = b = 0.0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) {
    a += room[w][0];
    b += room[w][1];
  }
}

// dz before the division and the sums of rows [begin, end); thread t takes rows t, t + T, ..
template <int T>
__device__ __forceinline__ void rows(const EtaParams &p, int64_t begin, int64_t end, double &sum, double &total) {
  for (int64_t i0 = begin + threadIdx.x; i0 < end; i0 += kRows * T) {
    float eta[kRows], w[kRows], z[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t i = i0 + u * T < end ? i0 + u * T : end - 1;
      eta[u] = p.eta[i];
      w[u] = p.weight ? p.weight[i] : 1.0f;
      z[u] = p.z[i];
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      if (i0 + u * T >= end) break;
      const bool counts = eta[u] > 0.0f && eta[u] < __builtin_inff() && w[u] > 0.0f && w[u] < __builtin_inff();
      const EtaTerm t = eta_term<true>(z[u], eta[u], w[u], p.huber);
      if (counts) {
        sum += (double)t.loss;
        total += (double)w[u];
      }
      p.dz[i0 + u * T] = counts ? t.dz : 0.0f;
    }
  }
}

__global__ __launch_bounds__(kThreads) void k_eta_sum(EtaParams p) {
  const int wg = blockIdx.x, f = family_of(p, wg);
  const int64_t begin = p.fam_off[f] + (wg - p.wg[f]) * p.rows;
  const int64_t end = begin + p.rows < p.fam_off[f + 1] ? begin + p.rows : p.fam_off[f + 1];
  double sum = 0.0, total = 0.0;
  rows<kThreads>(p, begin, end, sum, total);
  sums<kThreads>(sum, total);
  if (threadIdx.x == 0) {
    p.part[2 * wg] = sum;
    p.part[2 * wg + 1] = total;
  }
}

// (the last KS_NFAM workgroups: the losses)
__global__ __launch_bounds__(kThreads) void k_eta_scale(EtaParams p) {
  const int wg = blockIdx.x, last = p.wg[KS_NFAM], f = wg < last ? family_of(p, wg) : wg - last;
  const int64_t begin = p.fam_off[f] + (wg - p.wg[f]) * p.rows;
  const int64_t end = wg >= last ? begin : begin + p.rows < p.fam_off[f + 1] ? begin + p.rows : p.fam_off[f + 1];
  // (on their way before the sums)
  float dz[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const int64_t i = begin + threadIdx.x + u * kThreads;
    dz[u] = i < end ? p.dz[i] : 0.0f;
  }
  double sum = 0.0, total = 0.0;
  for (int i = p.wg[f] + (int)threadIdx.x; i < p.wg[f + 1]; i += kThreads) {
    sum += p.part[2 * i];
    total += p.part[2 * i + 1];
  }
  sums<kThreads>(sum, total);
  const double scale = total > 0.0 ? 1.0 / total : 0.0;
  if (wg >= last) {
    if (threadIdx.x == 0) p.loss[f] = (float)(sum * scale);
    return;
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const int64_t i = begin + threadIdx.x + u * kThreads;
    if (i < end) p.dz[i] = (float)(dz[u] * scale);
  }
  for (int64_t i = begin + threadIdx.x + kRows * kThreads; i < end; i += kThreads) p.dz[i] = (float)(p.dz[i] * scale);
}

__global__ __launch_bounds__(kEtaWide) void k_eta_one(EtaParams p) {
  const int f = blockIdx.x;
  const int64_t begin = p.fam_off[f], end = p.fam_off[f + 1];
  double sum = 0.0, total = 0.0;
  rows<kEtaWide>(p, begin, end, sum, total);
  sums<kEtaWide>(sum, total);
  const double scale = total > 0.0 ? 1.0 / total : 0.0;
  if (threadIdx.x == 0) p.loss[f] = (float)(sum * scale);
  // (each thread reads what it has written)
  for (int64_t i = begin + threadIdx.x; i < end; i += kEtaWide) p.dz[i] = (float)(p.dz[i] * scale);
}

}  // namespace

hipError_t launch_eta_loss(const EtaParams &p, hipStream_t s) {
  const uint32_t wgs = (uint32_t)p.wg[KS_NFAM];
  if (wgs == 0) {
    hipLaunchKernelGGL(k_eta_one, dim3(KS_NFAM), dim3(kEtaWide), 0, s, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(k_eta_sum, dim3(wgs), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL(k_eta_scale, dim3(wgs + KS_NFAM), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace ks
