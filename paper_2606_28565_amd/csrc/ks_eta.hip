// The loss on log eta at given z and its gradient (ks.h, ks_eta_loss).
//
//   k_eta_sum     dz before the division by sum w, and a workgroup's sum w rho, sum w
//   k_eta_scale   those sums of a family, in order, in 64 bits; dz over sum w
//
// A workgroup works on rows of one family.
#include <hip/hip_runtime.h>

#include "ks_gated.h"
#include "ks_internal.h"

namespace ks {

namespace {

using gated::EtaTerm;
using gated::eta_term;

constexpr int kThreads = 256;

__device__ __forceinline__ int family_of(const EtaParams &p, int wg) {
  int f = 0;   // (all offsets read at once: no chain of scalar loads)
#pragma unroll
  for (int i = 1; i < KS_NFAM; ++i) f += wg >= p.wg[i];
  return f;
}

// sums of a pair over the workgroup, in every thread
__device__ __forceinline__ void sums(double &a, double &b) {
  __shared__ double room[kThreads][2];
  room[threadIdx.x][0] = a;
  room[threadIdx.x][1] = b;
  __syncthreads();
  for (int d = kThreads / 2; d > 0; d /= 2) {
    if ((int)threadIdx.x < d) {
      room[threadIdx.x][0] += room[threadIdx.x + d][0];
      room[threadIdx.x][1] += room[threadIdx.x + d][1];
    }
    __syncthreads();
  }
  a = room[0][0];
  b = room[0][1];
}

__global__ __launch_bounds__(kThreads) void k_eta_sum(EtaParams p) {
  const int wg = blockIdx.x, f = family_of(p, wg);
  const int64_t begin = p.fam_off[f] + (wg - p.wg[f]) * p.rows;
  const int64_t end = begin + p.rows < p.fam_off[f + 1] ? begin + p.rows : p.fam_off[f + 1];
  double sum = 0.0, total = 0.0;
  for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) {
    const float eta = p.eta[i], w = p.weight ? p.weight[i] : 1.0f;
    float dz = 0.0f;
    if (eta > 0.0f && eta < __builtin_inff() && w > 0.0f && w < __builtin_inff()) {
      const EtaTerm t = eta_term(p.z[i], eta, w, p.huber);
      dz = t.dz;
      sum += (double)t.loss;
      total += (double)w;
    }
    p.dz[i] = dz;
  }
  sums(sum, total);
  if (threadIdx.x == 0) {
    p.part[2 * wg] = sum;
    p.part[2 * wg + 1] = total;
  }
}

// (the last KS_NFAM workgroups: the losses)
__global__ __launch_bounds__(kThreads) void k_eta_scale(EtaParams p) {
  const int wg = blockIdx.x, last = p.wg[KS_NFAM], f = wg < last ? family_of(p, wg) : wg - last;
  double sum = 0.0, total = 0.0;
  for (int i = p.wg[f] + (int)threadIdx.x; i < p.wg[f + 1]; i += kThreads) {
    sum += p.part[2 * i];
    total += p.part[2 * i + 1];
  }
  sums(sum, total);
  const double scale = total > 0.0 ? 1.0 / total : 0.0;
  if (wg >= last) {
    if (threadIdx.x == 0) p.loss[f] = (float)(sum * scale);
    return;
  }
  const int64_t begin = p.fam_off[f] + (wg - p.wg[f]) * p.rows;
  const int64_t end = begin + p.rows < p.fam_off[f + 1] ? begin + p.rows : p.fam_off[f + 1];
  for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) p.dz[i] = (float)(p.dz[i] * scale);
}

}  // namespace

hipError_t launch_eta_loss(const EtaParams &p, hipStream_t s) {
  const uint32_t wgs = (uint32_t)p.wg[KS_NFAM];
  if (wgs) hipLaunchKernelGGL(k_eta_sum, dim3(wgs), dim3(kThreads), 0, s, p);
  hipLaunchKernelGGL(k_eta_scale, dim3(wgs + KS_NFAM), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace ks
