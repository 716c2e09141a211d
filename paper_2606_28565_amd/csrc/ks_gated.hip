// Gated heads over feature rows: the block, its gradients and the loss on
// log eta (ks.h).  Rows are grouped by family; a workgroup works on rows of one.
//
//   k_gated_forward   z, and for a fit the loss sums and dz of each row
//   k_gated_backward  weight gradients of a workgroup's rows, held in registers
//   k_gated_rows      gradients of the rows
//   k_gated_reduce    sums of the workgroups' gradients in a fixed order
//
// The derivative at a row, with s = sigma(g), a = g s:
//   du = dz w3 a,  dg = dz w3 u (s + a (1 - s)),  dw3 += dz a u.
// w3 is one factor of a unit over all rows, so the backward kernel leaves it out
// and k_gated_reduce multiplies the finished sums by it.
#include <hip/hip_runtime.h>

#include "ks_gated.h"
#include "ks_internal.h"

namespace ks {

using gated::Block;
using gated::gbf16x8;
using gated::gf32x4;
using gated::gu32x4;
using gated::sigmoid;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float bf16_value(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }

// round to nearest even
__device__ __forceinline__ uint16_t bf16_of(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

template <bool BF16>
__device__ __forceinline__ float element(const void *p, int64_t i) {
  if constexpr (BF16) return bf16_value(((const uint16_t *)p)[i]);
  else return ((const float *)p)[i];
}

__device__ __forceinline__ int family_of(const int32_t (&off)[KS_NFAM + 1], int wg) {
  int f = 0;
  while (wg >= off[f + 1]) ++f;
  return f;
}

// eight consecutive elements of a row as packed bf16 (one) or fp32 (two) quads
template <bool BF16>
__device__ __forceinline__ void load8(gu32x4 (&v)[BF16 ? 1 : 2], const void *x, int64_t i, bool vec) {
  if constexpr (BF16) {
    const uint16_t *p = (const uint16_t *)x + i;
    if (vec) {
      v[0] = *(const gu32x4 *)p;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[0][j] = p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
    }
  } else {
    const uint32_t *p = (const uint32_t *)x + i;
    if (vec) {
      v[0] = *(const gu32x4 *)p;
      v[1] = *(const gu32x4 *)(p + 4);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j >> 2][j & 3] = p[j];
    }
  }
}

// ------------------------------------------------------------ forward
template <bool BF16, int IN, bool LOSS>
__global__ __launch_bounds__(kThreads, 2) void k_gated_forward(GatedParams p) {
  using G = Block<BF16, IN>;
  __shared__ __align__(16) uint32_t lds[G::kLds];
  constexpr int E = BF16 ? 2 : 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wg = blockIdx.x, f = family_of(p.fwd_wg, wg);
  const size_t w = (size_t)f * p.hidden * IN * E;
  G::stage(lds, (const char *)p.w1 + w, (const char *)p.w2 + w, (const char *)p.w3 + (size_t)f * p.hidden * E,
           (const char *)p.b3 + f * E, p.hidden, (int)threadIdx.x, kThreads);
  __syncthreads();
  const int64_t begin = p.fam_off[f] + (int64_t)(wg - p.fwd_wg[f]) * p.fwd_tiles * 64;
  const int64_t fam_end = p.fam_off[f + 1];
  const int64_t end = begin + (int64_t)p.fwd_tiles * 64 < fam_end ? begin + (int64_t)p.fwd_tiles * 64 : fam_end;
  double sum = 0.0, total = 0.0;
  for (int64_t row0 = begin + 64 * wave; row0 < end; row0 += 64 * (kThreads / 64)) {
    typename G::Rows x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = row0 + 32 * i + (lane & 31);
      const int64_t at = (r < end ? r : end - 1) * p.ldx + (lane >> 5) * 8;
#pragma unroll
      for (int kc = 0; kc < G::KC; ++kc) load8<BF16>(x.v[i][kc], p.x, at + 16 * kc, p.vec);
    }
    const float z = G::z_of(x, lds);
    const int64_t row = row0 + lane;
    if (row < end) {
      if (p.z) p.z[row] = z;
      if constexpr (LOSS) {
        const float eta = p.eta[row], wt = p.weight ? p.weight[row] : 1.0f;
        const bool counts = eta > 0.0f && eta < __builtin_inff() && wt > 0.0f && wt < __builtin_inff();
        float dz = 0.0f;
        if (counts) {
          // log(1 + e^-z), without overflow
          const float res = fmaxf(-z, 0.0f) + log1pf(expf(-fabsf(z))) - logf(eta);
          const float big = fabsf(res);
          const float rho = big <= p.huber ? 0.5f * res * res : p.huber * (big - 0.5f * p.huber);
          const float slope = big <= p.huber ? res : copysignf(p.huber, res);
          // d/dz log(1 + e^-z) = -sigma(-z)
          dz = -wt * (__builtin_isnan(res) ? res : slope) * sigmoid(-z);
          sum += (double)(wt * (__builtin_isnan(res) ? res : rho));
          total += (double)wt;
        }
        if (p.dz_out) p.dz_out[row] = dz;
      }
    }
  }
  if constexpr (LOSS) {
    __shared__ double part[kThreads / 64][2];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      sum += __shfl_xor(sum, d);
      total += __shfl_xor(total, d);
    }
    if (lane == 0) {
      part[wave][0] = sum;
      part[wave][1] = total;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
      double v = 0.0;
      for (int i = 0; i < kThreads / 64; ++i) v += part[i][threadIdx.x];
      p.loss_part[2 * wg + threadIdx.x] = v;
    }
  }
}

// ------------------------------------------------------------ backward
// A wave takes 64 units (their weights and gradients in its registers) and 16
// rows at a time on the 16x16 instructions: the rows as the row operand, so a
// lane holds the gates and ups of one unit for four rows, and what it makes of
// them is the row operand of the next product, dW (units x features) += dg^T x,
// without any exchange between lanes.  That product is fp32 for either precision
// (x is exact in it), so gradients are sums of unrounded terms.  The workgroup's
// four waves are the unit groups times row groups; row groups are joined in LDS.
template <bool BF16, int IN>
struct Back {
  static constexpr int KC = IN / 16, NB = kGatedGroup / 16;
  // a lane's share of a 16-row (or 16-unit) operand: features 4 q .. 4 q + 3 of
  // each 16 (fp32, bf16 with 16 inputs), 8 q .. 8 q + 7 (bf16, 32 inputs)
  struct Op {
    uint32_t v[BF16 ? IN / 8 : IN / 4];
  };
  __device__ static __forceinline__ Op load(const void *x, int64_t i, int q, bool vec) {
    Op o;
    if constexpr (BF16) {
      constexpr int N = IN / 4;
      const uint16_t *p = (const uint16_t *)x + i + N * q;
      if (vec) {
        if constexpr (IN == 16) {
          const u32x2 t = *(const u32x2 *)p;
          o.v[0] = t[0], o.v[1] = t[1];
        } else {
          const gu32x4 t = *(const gu32x4 *)p;
#pragma unroll
          for (int j = 0; j < 4; ++j) o.v[j] = t[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) o.v[j] = p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
      }
    } else {
      const uint32_t *p = (const uint32_t *)x + i + 4 * q;
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        if (vec) {
          const gu32x4 t = *(const gu32x4 *)(p + 16 * k);
#pragma unroll
          for (int j = 0; j < 4; ++j) o.v[4 * k + j] = t[j];
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) o.v[4 * k + j] = p[16 * k + j];
        }
      }
    }
    return o;
  }
  __device__ static __forceinline__ void keep(Op &o, bool k) {
#pragma unroll
    for (auto &v : o.v) v = k ? v : 0u;
  }
  __device__ static __forceinline__ gf32x4 product(const Op &a, const Op &b) {
    gf32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (BF16 && IN == 16) {
      c = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, u32x2{a.v[0], a.v[1]}),
                                                    __builtin_bit_cast(s16x4, u32x2{b.v[0], b.v[1]}), c, 0, 0, 0);
    } else if constexpr (BF16) {
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(gbf16x8, gu32x4{a.v[0], a.v[1], a.v[2], a.v[3]}),
                                                  __builtin_bit_cast(gbf16x8, gu32x4{b.v[0], b.v[1], b.v[2], b.v[3]}), c, 0,
                                                  0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < IN / 4; ++j)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, a.v[j]), __builtin_bit_cast(float, b.v[j]), c, 0, 0,
                                                 0);
    }
    return c;
  }
};

template <bool BF16, int IN>
__global__ __launch_bounds__(kThreads, 2) void k_gated_backward(GatedParams p) {
  using K = Back<BF16, IN>;
  using Op = typename K::Op;
  constexpr int KC = K::KC, NB = K::NB;
  const int lane = threadIdx.x & 63, q = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int HG = gated_groups(p.hidden), RG = 4 / HG;
  const int hg = wave % HG, rg = wave / HG;
  const int wg = blockIdx.x, f = family_of(p.bwd_wg, wg);
  const bool works = rg < RG;
  gf32x4 dw[2][NB][KC] = {};
  float d3[NB] = {}, d0 = 0.0f;
  if (works) {
    Op wgt[2][NB];
    const size_t at = (size_t)f * p.hidden * IN;
    const bool vec = ((reinterpret_cast<uintptr_t>(p.w1) | reinterpret_cast<uintptr_t>(p.w2)) & 15) == 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int unit = hg * kGatedGroup + 16 * b + c;
      const int64_t i = at + (size_t)(unit < p.hidden ? unit : p.hidden - 1) * IN;
      wgt[0][b] = K::load(p.w1, i, q, vec);
      wgt[1][b] = K::load(p.w2, i, q, vec);
      K::keep(wgt[0][b], unit < p.hidden);
      K::keep(wgt[1][b], unit < p.hidden);
    }
    const int64_t begin = p.fam_off[f] + (int64_t)(wg - p.bwd_wg[f]) * p.bwd_rows;
    const int64_t fam_end = p.fam_off[f + 1];
    const int64_t end = begin + p.bwd_rows < fam_end ? begin + p.bwd_rows : fam_end;
    for (int64_t row0 = begin + 16 * rg; row0 < end; row0 += 16 * RG) {
      auto clamp = [&](int64_t r) { return r < end ? r : end - 1; };
      float dza = p.dz[clamp(row0 + c)], dz[4];
      Op xa = K::load(p.x, clamp(row0 + c) * p.ldx, q, p.vec);
      float xb[4][KC];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t row = clamp(row0 + 4 * q + r);
        dz[r] = p.dz[row];
#pragma unroll
        for (int k = 0; k < KC; ++k) xb[r][k] = element<BF16>(p.x, row * p.ldx + 16 * k + c);
      }
      // a row without weight adds nothing, whatever it holds
      if (row0 + c >= end) dza = 0.0f;
      K::keep(xa, dza != 0.0f);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (row0 + 4 * q + r >= end) dz[r] = 0.0f;
#pragma unroll
        for (int k = 0; k < KC; ++k) xb[r][k] = dz[r] != 0.0f ? xb[r][k] : 0.0f;
      }
      d0 += dza;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const gf32x4 g = K::product(xa, wgt[0][b]), u = K::product(xa, wgt[1][b]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float s = sigmoid(g[r]), a = g[r] * s;
          const float du = dz[r] * a;
          const float dg = dz[r] * u[r] * (fmaf(-a, s, a) + s);
          d3[b] = fmaf(du, u[r], d3[b]);
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            dw[0][b][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(dg, xb[r][k], dw[0][b][k], 0, 0, 0);
            dw[1][b][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(du, xb[r][k], dw[1][b][k], 0, 0, 0);
          }
        }
      }
    }
    // rows 4 q .. of a unit, and the 16 lanes of a row group's rows
#pragma unroll
    for (int d = 16; d < 64; d *= 2)
#pragma unroll
      for (int b = 0; b < NB; ++b) d3[b] += __shfl_xor(d3[b], d);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) d0 += __shfl_xor(d0, d);
  }
  // the row groups' sums onto the first's, in order
  constexpr int kWords = 2 * NB * KC * 4 + NB + 1;
  __shared__ float join[3][kWords][64];
  if (works && rg > 0) {
    float(*o)[64] = join[(rg - 1) * HG + hg];
    int n = 0;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n++][lane] = dw[m][b][k][i];
#pragma unroll
    for (int b = 0; b < NB; ++b) o[n++][lane] = d3[b];
    o[n][lane] = d0;
  }
  __syncthreads();
  if (!works || rg > 0) return;
  for (int g = 1; g < RG; ++g) {
    const float(*o)[64] = join[(g - 1) * HG + hg];
    int n = 0;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) dw[m][b][k][i] += o[n++][lane];
#pragma unroll
    for (int b = 0; b < NB; ++b) d3[b] += o[n++][lane];
    d0 += o[n][lane];
  }
  float *out = p.part + (size_t)wg * gated_part_size(p.hidden, IN);
  float *mine = out + hg * kGatedGroup * (2 * IN + 1);
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < KC; ++k)
          mine[(m * kGatedGroup + 16 * b + 4 * q + i) * IN + 16 * k + c] = dw[m][b][k][i];
  if (q == 0) {
#pragma unroll
    for (int b = 0; b < NB; ++b) mine[kGatedGroup * 2 * IN + 16 * b + c] = d3[b];
  }
  if (hg == 0 && lane == 0) out[gated_part_size(p.hidden, IN) - 1] = d0;
}

// ------------------------------------------------------------ rows' gradients
// dx = W1^T dg + W2^T du: units are summed over, so here the units are the row
// operand of the projections (a lane holds four units of one row) and what it
// makes of them is the column operand of the next product.  fp32 throughout,
// from fp32 copies of the weights in LDS; rows of IN + 4 floats keep both the
// 16-byte reads along a row and the reads across rows off each other's banks.
template <bool BF16, int IN>
__global__ __launch_bounds__(kThreads, 2) void k_gated_rows(GatedParams p) {
  constexpr int KC = IN / 16, LD = IN + 4, RT = 2, H = gated::kMaxHidden;
  __shared__ __align__(16) float lw[2][H][LD];
  __shared__ __align__(16) float l3[H];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4, c = lane & 15;
  const int wg = blockIdx.x, f = family_of(p.fwd_wg, wg);
  const int nb = (p.hidden + 15) / 16;
  for (int i = threadIdx.x; i < nb * 16 * IN; i += kThreads) {
    const int h = i / IN, d = i % IN;
    const int64_t at = ((int64_t)f * p.hidden + h) * IN + d;
    lw[0][h][d] = h < p.hidden ? element<BF16>(p.w1, at) : 0.0f;
    lw[1][h][d] = h < p.hidden ? element<BF16>(p.w2, at) : 0.0f;
  }
  for (int h = threadIdx.x; h < nb * 16; h += kThreads)
    l3[h] = h < p.hidden ? element<BF16>(p.w3, (int64_t)f * p.hidden + h) : 0.0f;
  __syncthreads();
  const int64_t begin = p.fam_off[f] + (int64_t)(wg - p.fwd_wg[f]) * p.fwd_tiles * 64;
  const int64_t fam_end = p.fam_off[f + 1];
  const int64_t end = begin + (int64_t)p.fwd_tiles * 64 < fam_end ? begin + (int64_t)p.fwd_tiles * 64 : fam_end;
  for (int64_t row0 = begin + 16 * RT * wave; row0 < end; row0 += 16 * RT * (kThreads / 64)) {
    float x[RT][KC][4], dz[RT];
    gf32x4 acc[RT][KC] = {};
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t r = row0 + 16 * t + c, at = r < end ? r : end - 1;
      dz[t] = r < end ? p.dz[at] : 0.0f;
#pragma unroll
      for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = element<BF16>(p.x, at * p.ldx + 16 * k + 4 * q + j);
          x[t][k][j] = dz[t] != 0.0f ? v : 0.0f;
        }
    }
#pragma unroll 1
    for (int b = 0; b < nb; ++b) {
      gf32x4 g[RT] = {}, u[RT] = {};
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const gf32x4 wa = *(const gf32x4 *)&lw[0][16 * b + c][16 * k + 4 * q];
        const gf32x4 wb = *(const gf32x4 *)&lw[1][16 * b + c][16 * k + 4 * q];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            g[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(wa[j], x[t][k][j], g[t], 0, 0, 0);
            u[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(wb[j], x[t][k][j], u[t], 0, 0, 0);
          }
      }
      const gf32x4 w3 = *(const gf32x4 *)&l3[16 * b + 4 * q];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float wa[KC], wb[KC];
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          wa[k] = lw[0][16 * b + 4 * q + r][16 * k + c];
          wb[k] = lw[1][16 * b + 4 * q + r][16 * k + c];
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const float dy = dz[t] * w3[r];
          const float s = sigmoid(g[t][r]), a = g[t][r] * s;
          const float du = dy * a, dg = dy * u[t][r] * (fmaf(-a, s, a) + s);
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            acc[t][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(wa[k], dg, acc[t][k], 0, 0, 0);
            acc[t][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(wb[k], du, acc[t][k], 0, 0, 0);
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t r = row0 + 16 * t + c;
      if (r >= end) continue;
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        // (a row without weight gets zeros even where a weight is not finite)
        gf32x4 v = acc[t][k];
        if (dz[t] == 0.0f) v = gf32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t at = r * p.g_ldx + 16 * k + 4 * q;
        if constexpr (BF16) {
          uint16_t *o = (uint16_t *)p.g_x + at;
          if (p.g_vec) {
            *(u32x2 *)o = u32x2{bf16_of(v[0]) | (uint32_t)bf16_of(v[1]) << 16, bf16_of(v[2]) | (uint32_t)bf16_of(v[3]) << 16};
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = bf16_of(v[i]);
          }
        } else {
          float *o = (float *)p.g_x + at;
          if (p.g_vec) {
            *(gf32x4 *)o = v;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = v[i];
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------ reduce
// The workgroups' sums of a family, in order: 32 elements per workgroup, eight
// threads each over an eighth of the family's workgroups, joined in LDS; in
// 64 bits.  dW1 and dW2 get their unit's w3 here, and a loss's gradients the
// family's 1 / sum w.
constexpr int kRedEl = 32, kRedParts = kThreads / kRedEl;

template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_gated_reduce(GatedParams p, int chunks) {
  const int f = blockIdx.x / chunks, ch = blockIdx.x % chunks;
  const int IN = p.in_dim, H = p.hidden, HI = H * IN;
  double scale = 1.0;
  if (p.eta) {
    __shared__ double ls[kThreads][2];
    double a = 0.0, b = 0.0;
    for (int w = p.fwd_wg[f] + (int)threadIdx.x; w < p.fwd_wg[f + 1]; w += kThreads) {
      a += p.loss_part[2 * w];
      b += p.loss_part[2 * w + 1];
    }
    ls[threadIdx.x][0] = a;
    ls[threadIdx.x][1] = b;
    __syncthreads();
    for (int d = kThreads / 2; d > 0; d /= 2) {
      if ((int)threadIdx.x < d) {
        ls[threadIdx.x][0] += ls[threadIdx.x + d][0];
        ls[threadIdx.x][1] += ls[threadIdx.x + d][1];
      }
      __syncthreads();
    }
    const double total = ls[0][1];
    scale = total > 0.0 ? 1.0 / total : 0.0;
    if (ch == 0 && threadIdx.x == 0) p.loss[f] = total > 0.0 ? (float)(ls[0][0] * scale) : 0.0f;
  }
  if (!p.g_w1) return;
  __shared__ double part[kRedParts][kRedEl];
  const int el = threadIdx.x % kRedEl, sl = threadIdx.x / kRedEl;
  const int e = ch * kRedEl + el;
  const int size = gated_part_size(H, IN);
  // where the element stands in a workgroup's sums
  int at = -1, unit = -1;
  if (e < 2 * HI) {
    const int m = e >= HI, i = m ? e - HI : e;
    unit = i / IN;
    at = (unit / kGatedGroup) * kGatedGroup * (2 * IN + 1) + (m * kGatedGroup + unit % kGatedGroup) * IN + i % IN;
  } else if (e < 2 * HI + H) {
    const int h = e - 2 * HI;
    at = (h / kGatedGroup) * kGatedGroup * (2 * IN + 1) + kGatedGroup * 2 * IN + h % kGatedGroup;
  } else if (e == 2 * HI + H) {
    at = size - 1;
  }
  const int first = p.bwd_wg[f], n = p.bwd_wg[f + 1] - first;
  const int per = (n + kRedParts - 1) / kRedParts;
  double v = 0.0;
  if (at >= 0) {
    const int lo = sl * per, hi = min(lo + per, n);
    const float *src = p.part + (size_t)first * size + at;
#pragma unroll 8
    for (int i = lo; i < hi; ++i) v += (double)src[(size_t)i * size];
  }
  part[sl][el] = v;
  __syncthreads();
  if (sl > 0 || at < 0) return;
  for (int i = 1; i < kRedParts; ++i) v += part[i][el];
  v *= scale;
  if (unit >= 0 && n > 0) v *= (double)element<BF16>(p.w3, (int64_t)f * H + unit);
  if (n == 0) v = 0.0;
  if (e < HI) p.g_w1[(size_t)f * HI + e] = (float)v;
  else if (e < 2 * HI) p.g_w2[(size_t)f * HI + e - HI] = (float)v;
  else if (e < 2 * HI + H) p.g_w3[(size_t)f * H + e - 2 * HI] = (float)v;
  else p.g_b3[f] = (float)v;
}

}  // namespace

// ------------------------------------------------------------ launchers
template <bool LOSS>
static void forward_of(const GatedParams &p, hipStream_t s) {
  const dim3 grid(p.fwd_wg[KS_NFAM]), block(kThreads);
  if (p.bf16) {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_forward<true, 16, LOSS>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_forward<true, 32, LOSS>), grid, block, 0, s, p);
  } else {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_forward<false, 16, LOSS>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_forward<false, 32, LOSS>), grid, block, 0, s, p);
  }
}

hipError_t launch_gated_forward(const GatedParams &p, hipStream_t s) {
  if (p.fwd_wg[KS_NFAM] == 0) return hipSuccess;
  if (p.eta) forward_of<true>(p, s);
  else forward_of<false>(p, s);
  return hipGetLastError();
}

hipError_t launch_gated_backward(const GatedParams &p, hipStream_t s) {
  const dim3 grid(p.bwd_wg[KS_NFAM]), block(kThreads);
  if (grid.x == 0) return hipSuccess;
  if (p.bf16) {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_backward<true, 16>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_backward<true, 32>), grid, block, 0, s, p);
  } else {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_backward<false, 16>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_backward<false, 32>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

hipError_t launch_gated_rows(const GatedParams &p, hipStream_t s) {
  const dim3 grid(p.fwd_wg[KS_NFAM]), block(kThreads);
  if (grid.x == 0) return hipSuccess;
  if (p.bf16) {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_rows<true, 16>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_rows<true, 32>), grid, block, 0, s, p);
  } else {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_rows<false, 16>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_rows<false, 32>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

hipError_t launch_gated_reduce(const GatedParams &p, hipStream_t s) {
  const int elements = p.g_w1 ? 2 * p.hidden * p.in_dim + p.hidden + 1 : 1;
  const int chunks = (elements + kRedEl - 1) / kRedEl;
  const dim3 grid(KS_NFAM * chunks), block(kThreads);
  if (p.bf16) hipLaunchKernelGGL((k_gated_reduce<true>), grid, block, 0, s, p, chunks);
  else hipLaunchKernelGGL((k_gated_reduce<false>), grid, block, 0, s, p, chunks);
  return hipGetLastError();
}

}  // namespace ks
