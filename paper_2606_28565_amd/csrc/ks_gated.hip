// Gated heads over feature rows: the block, its gradients and the loss on
// log eta (ks.h).  Rows are grouped by family; a workgroup works on rows of one.
//
//   k_gated_forward   z, or the loss alone
//   k_gated_fit       weight gradients of a workgroup's rows, held in registers: of
//                     a given dz, or of the loss, whose dz it forms on the way
//   k_gated_rows      gradients of the rows
//   k_gated_reduce    sums of the workgroups' gradients in a fixed order
//
// The derivative at a row, with s = sigma(g), a = g s:
//   du = dz w3 a,  dg = dz w3 u silu'(g),  silu'(g) = s + s (g - a),  dw3 += dz a u.
// w3 is one factor of a unit over all rows, so k_gated_fit leaves it out and
// k_gated_reduce multiplies the finished sums by it.  dz is one factor of a row
// over all units, so it goes to the rows' side of the product, dW = (..)^T (dz x).
// And u = W2 x, so sum dz a u = W2 . (sum dz a x): dw3 follows from the finished
// sum of dW2.
#include <hip/hip_runtime.h>

#include "ks_gated.h"
#include "ks_internal.h"

namespace ks {

using gated::Block;
using gated::gbf16x8;
using gated::gf32x4;
using gated::gu32x4;
using gated::sigmoid;
using gated::split2;

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

// One row's part of the loss on log eta: w rho(r), and w drho/dz.  log(1 + e^-z) is
// max(-z, 0) + log(1 + e), e = exp(-|z|) <= 1.  On the hardware's exponential and
// logarithm (within 2^-23 relative, the logarithm near 1 too): the exponent's
// rounding is put back to first order, and the logarithm of the rounded 1 + e
// corrected for that rounding, which keeps it exact relative to a small e.
struct EtaTerm {
  float loss, dz;
};
__device__ __forceinline__ EtaTerm eta_term(float z, float eta, float weight, float huber) {
  constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
  const float t = fabsf(z) * -kLog2e, lo = fmaf(fabsf(z), -kLog2e, -t) - fabsf(z) * 1.92596299e-8f;
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e * kLn2, lo, e);
  if (!(fabsf(z) < 126.0f)) e = z == z ? 0.0f : z;   // (below the normal range; t - t is no number at infinity)
  const float w = 1.0f + e;
  const float log1 = fmaf(__builtin_amdgcn_logf(w), kLn2, (e - (w - 1.0f)) * __builtin_amdgcn_rcpf(w));
  const float at = eta < 0x1p-126f ? eta * 0x1p32f : eta;   // (the logarithm takes normal numbers)
  const float res = fmaxf(-z, 0.0f) + log1 - (__builtin_amdgcn_logf(at) - (eta < 0x1p-126f ? 32.0f : 0.0f)) * kLn2;
  const float size = fabsf(res);
  const bool far = size > huber;   // (a NaN stays one)
  const float rho = far ? huber * (size - 0.5f * huber) : 0.5f * res * res;
  const float slope = far ? copysignf(huber, res) : res;
  return {weight * rho, -weight * slope * sigmoid(-z)};   // d log(1 + e^-z) / dz = -sigma(-z)
}

// ------------------------------------------------------------ forward
// N waves share the weights in LDS: four, or, where 256 units of 32 fp32 inputs
// leave room for one workgroup per CU only, eight (two per SIMD).
template <bool BF16, int IN, int HID, bool LOSS, int N>
__global__ __launch_bounds__(64 * N, 2) void k_gated_forward(GatedParams p) {
  using G = Block<BF16, IN, HID>;
  __shared__ __align__(16) uint32_t lds[G::kLds];
  constexpr int E = BF16 ? 2 : 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wg = blockIdx.x, f = family_of(p.fwd_wg, wg);
  const size_t w = (size_t)f * p.hidden * IN * E;
  G::stage(lds, (const char *)p.w1 + w, (const char *)p.w2 + w, (const char *)p.w3 + (size_t)f * p.hidden * E,
           (const char *)p.b3 + f * E, p.hidden, (int)threadIdx.x, 64 * N);
  __syncthreads();
  const int64_t begin = p.fam_off[f] + (int64_t)(wg - p.fwd_wg[f]) * p.fwd_tiles * 64;
  const int64_t fam_end = p.fam_off[f + 1];
  const int64_t end = begin + (int64_t)p.fwd_tiles * 64 < fam_end ? begin + (int64_t)p.fwd_tiles * 64 : fam_end;
  double sum = 0.0, total = 0.0;
  for (int64_t row0 = begin + 64 * wave; row0 < end; row0 += 64 * N) {
    typename G::Rows x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = row0 + 32 * i + (lane & 31);
      const int64_t at = (r < end ? r : end - 1) * p.ldx + (lane >> 5) * 8;
#pragma unroll
      for (int kc = 0; kc < G::KC; ++kc) {
        gu32x4 raw[BF16 ? 1 : 2];
        load8<BF16>(raw, p.x, at + 16 * kc, p.vec);
        if constexpr (BF16) x.v[i][kc][0] = raw[0];
        else G::split8(__builtin_bit_cast(gf32x4, raw[0]), __builtin_bit_cast(gf32x4, raw[1]), x.v[i][kc]);
      }
    }
    const float z = G::z_of(x, lds);
    const int64_t row = row0 + lane;
    if (row < end) {
      if (p.z) p.z[row] = z;
      if constexpr (LOSS) {
        const float eta = p.eta[row], wt = p.weight ? p.weight[row] : 1.0f;
        const bool counts = eta > 0.0f && eta < __builtin_inff() && wt > 0.0f && wt < __builtin_inff();
        if (counts) {
          sum += (double)eta_term(z, eta, wt, p.huber).loss;
          total += (double)wt;
        }
      }
    }
  }
  if constexpr (LOSS) {
    __shared__ double part[N][2];
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
      for (int i = 0; i < N; ++i) v += part[i][threadIdx.x];
      p.loss_part[2 * wg + threadIdx.x] = v;
    }
  }
}

// ------------------------------------------------------------ gradients
// A wave takes 16 NB units (their weights and gradients in its registers) and 16 T
// rows at a time on the 16x16x32 instruction: the rows as the row operand, so a
// lane holds the gates and ups of one unit for four rows of a tile, and what it makes
// of them is the row operand of the next product, dW (units x features), without
// any exchange between lanes.  The workgroup's W waves are the unit groups times row
// groups; for the loss, the unit groups exchange their parts of each row's z through
// LDS (one barrier per 16 T rows, two buffers); row groups are joined in LDS at the
// end.
//
// Which eight of the instruction's 32 inner indices a lane holds is free, as long as
// both operands agree: of a tile's 16 rows (or 16 fp32 features) a lane has four, so
// one instruction takes two of the six products of pieces.  dz x is split for either
// precision: gradients are sums of unrounded terms, to 2^-25 of each.
template <bool BF16, int IN>
struct Back {
  static constexpr int KC = IN / 16;
  static constexpr bool kWide = !BF16 && IN == 32;   // most registers per unit: fewer units, one tile
  static constexpr int NB = kWide ? 2 : 4, W = kWide ? 8 : 4, T = kWide ? 1 : 2;
  static constexpr int kGroup = 16 * NB;
  // a lane's part of a row (or of a unit's weights): features 4 q .. 4 q + 3 for 16
  // inputs, 8 q .. 8 q + 7 for 32, as read
  static constexpr int kRaw = BF16 ? IN / 8 : IN / 4;
  struct Raw {
    uint32_t v[kRaw];
  };
  __device__ static __forceinline__ Raw load(const char *x, int q, bool vec) {
    constexpr int kBytes = 4 * kRaw;
    Raw o;
    const char *p = x + q * kBytes;
    if (vec) {
      if constexpr (kBytes == 8) {
        const u32x2 t = *(const u32x2 *)p;
        o.v[0] = t[0], o.v[1] = t[1];
      } else {
#pragma unroll
        for (int i = 0; i < kRaw / 4; ++i) {
          const gu32x4 t = *(const gu32x4 *)(p + 16 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) o.v[4 * i + j] = t[j];
        }
      }
    } else if constexpr (BF16) {
      const uint16_t *h = (const uint16_t *)p;
#pragma unroll
      for (int j = 0; j < kRaw; ++j) o.v[j] = h[2 * j] | (uint32_t)h[2 * j + 1] << 16;
    } else {
#pragma unroll
      for (int j = 0; j < kRaw; ++j) o.v[j] = ((const uint32_t *)p)[j];
    }
    return o;
  }
  __device__ static __forceinline__ void keep(Raw &o, bool k) {
#pragma unroll
    for (auto &v : o.v) v = k ? v : 0u;
  }
  // the operands of the projections.  fp32: with 16 inputs two pieces at a time (X0 X2,
  // X1 X1, X0 X0 against W2 W0, W0 W1, W0 W1), with 32 one piece (0, 1, 2)
  static constexpr int kX = BF16 ? 1 : 3, kW = BF16 ? 1 : IN == 16 ? 2 : 3;
  struct Rows {
    gu32x4 v[kX];
  };
  struct Units {
    gu32x4 v[kW];
  };
  __device__ static __forceinline__ void pieces(const Raw &o, uint32_t (&p)[3][kRaw / 2 > 0 ? kRaw / 2 : 1]) {
#pragma unroll
    for (int j = 0; j < kRaw / 2; ++j)
      split2(__builtin_bit_cast(float, o.v[2 * j]), __builtin_bit_cast(float, o.v[2 * j + 1]), p[0][j], p[1][j], p[2][j]);
  }
  __device__ static __forceinline__ Rows rows(const Raw &o) {
    Rows r;
    if constexpr (BF16) {
      r.v[0] = gu32x4{o.v[0], o.v[1], IN == 16 ? 0u : o.v[kRaw - 2], IN == 16 ? 0u : o.v[kRaw - 1]};
    } else {
      uint32_t p[3][kRaw / 2];
      pieces(o, p);
      if constexpr (IN == 16) {
        r.v[0] = gu32x4{p[0][0], p[0][1], p[2][0], p[2][1]};
        r.v[1] = gu32x4{p[1][0], p[1][1], p[1][0], p[1][1]};
        r.v[2] = gu32x4{p[0][0], p[0][1], p[0][0], p[0][1]};
      } else {
#pragma unroll
        for (int i = 0; i < 3; ++i) r.v[i] = gu32x4{p[i][0], p[i][1], p[i][kRaw / 2 - 2], p[i][kRaw / 2 - 1]};
      }
    }
    return r;
  }
  __device__ static __forceinline__ Units units(const Raw &o) {
    Units r;
    if constexpr (BF16) {
      r.v[0] = rows(o).v[0];
    } else {
      uint32_t p[3][kRaw / 2];
      pieces(o, p);
      if constexpr (IN == 16) {
        r.v[0] = gu32x4{p[2][0], p[2][1], p[0][0], p[0][1]};
        r.v[1] = gu32x4{p[0][0], p[0][1], p[1][0], p[1][1]};
      } else {
#pragma unroll
        for (int i = 0; i < 3; ++i) r.v[i] = gu32x4{p[i][0], p[i][1], p[i][kRaw / 2 - 2], p[i][kRaw / 2 - 1]};
      }
    }
    return r;
  }
  __device__ static __forceinline__ gf32x4 mfma(const gu32x4 &a, const gu32x4 &b, const gf32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(gbf16x8, a), __builtin_bit_cast(gbf16x8, b), c, 0, 0, 0);
  }
  // rows x units (a lane: rows 4 q .. 4 q + 3 of unit c)
  __device__ static __forceinline__ gf32x4 product(const Rows &x, const Units &w) {
    gf32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (BF16 && IN == 16) {
      c = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, u32x2{x.v[0][0], x.v[0][1]}),
                                                    __builtin_bit_cast(s16x4, u32x2{w.v[0][0], w.v[0][1]}), c, 0, 0, 0);
    } else if constexpr (BF16) {
      c = mfma(x.v[0], w.v[0], c);
    } else if constexpr (IN == 16) {
      c = mfma(x.v[0], w.v[0], c);
      c = mfma(x.v[1], w.v[1], c);
      c = mfma(x.v[2], w.v[1], c);
    } else {
      c = mfma(x.v[2], w.v[0], c);
      c = mfma(x.v[1], w.v[1], c);
      c = mfma(x.v[0], w.v[2], c);
      c = mfma(x.v[1], w.v[0], c);
      c = mfma(x.v[0], w.v[1], c);
      c = mfma(x.v[0], w.v[0], c);
    }
    return c;
  }
};

// the sum of a row of 16 lanes, in each of them
template <int CTRL>
__device__ __forceinline__ float row_add(float v) {
  const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true);
  return v + __builtin_bit_cast(float, o);
}
__device__ __forceinline__ float row_sum(float v) {
  v = row_add<0x128>(v);   // row_ror:8, 4, 2, 1
  v = row_add<0x124>(v);
  v = row_add<0x122>(v);
  return row_add<0x121>(v);
}

template <bool BF16, int IN, bool LOSS>
__global__ __launch_bounds__((64 * Back<BF16, IN>::W), 2) void k_gated_fit(GatedParams p) {
  using K = Back<BF16, IN>;
  using Raw = typename K::Raw;
  constexpr int KC = K::KC, NB = K::NB, T = K::T, W = K::W, R = 16 * T;
  constexpr int kWords = 2 * NB * KC * 4 + 1;
  __shared__ float join[W - 1][kWords][64];
  __shared__ __align__(16) float zbuf[2][W][R];   // a wave's part of z of the rows in hand
  __shared__ __align__(16) float dzbuf[W][R];
  const int lane = threadIdx.x & 63, q = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int HG = gated_groups(p.hidden, K::kGroup), RG = W / HG;
  const int hg = wave % HG, rg = wave / HG;
  const int wg = blockIdx.x, f = family_of(p.bwd_wg, wg);
  const bool works = rg < RG;
  const int64_t begin = p.fam_off[f] + (int64_t)(wg - p.bwd_wg[f]) * p.bwd_rows;
  const int64_t fam_end = p.fam_off[f + 1];
  const int64_t end = begin + p.bwd_rows < fam_end ? begin + p.bwd_rows : fam_end;
  const int steps = (int)((end - begin + R * RG - 1) / (R * RG));   // the same for every wave
  gf32x4 dw[2][NB][KC] = {};
  float d0 = 0.0f;
  double sum = 0.0, total = 0.0;
  typename K::Units wgt[2][NB];
  float w3[NB] = {};
  {
    constexpr int E = BF16 ? 2 : 4;
    const bool vec = ((reinterpret_cast<uintptr_t>(p.w1) | reinterpret_cast<uintptr_t>(p.w2)) & 15) == 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int unit = hg * K::kGroup + 16 * b + c;
      const bool there = works && unit < p.hidden;
      const size_t at = ((size_t)f * p.hidden + (there ? unit : 0)) * IN * E;
      Raw a1 = K::load((const char *)p.w1 + at, q, vec), a2 = K::load((const char *)p.w2 + at, q, vec);
      K::keep(a1, there);
      K::keep(a2, there);
      wgt[0][b] = K::units(a1);
      wgt[1][b] = K::units(a2);
      if (LOSS && there) w3[b] = element<BF16>(p.w3, (int64_t)f * p.hidden + unit);
    }
  }
  const float b3 = LOSS ? element<BF16>(p.b3, f) : 0.0f;
  // Rows row0 .. row0 + R - 1 of a step; past the last row a lane reads the last.
  const uint32_t ld = (uint32_t)p.ldx * (BF16 ? 2 : 4);
  const int i_row = lane & (R - 1);   // the row whose loss (or dz) the lane forms
  const uint32_t off_a = __umul24(c, ld), off_b = __umul24(4 * q, ld) + c * (BF16 ? 2 : 4);
  Raw xa[T];
  float in0 = 0.0f, in1 = 1.0f, dza[T];
  auto fetch = [&](int64_t row0) {
    const int64_t base = row0 < end ? row0 : end - 1;
    const int left = end - base < R ? (int)(end - base) : R;   // rows there
    const char *x = (const char *)p.x + base * ld;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const uint32_t r = min(16 * t + c, left - 1);
      xa[t] = K::load(left == R ? x + (size_t)(16 * t) * ld + off_a : x + __umul24(r, ld), q, p.vec);
      if (!LOSS) dza[t] = p.dz[base + r];
    }
    const int64_t mine = base + min(i_row, left - 1);
    if (LOSS) {
      in0 = p.eta[mine];
      if (p.weight) in1 = p.weight[mine];
    } else {
      in0 = p.dz[mine];
    }
  };
  int64_t row0 = begin + R * rg;
  if (works) fetch(row0);
#pragma unroll 1
  for (int step = 0; step < steps; ++step, row0 += R * RG) {
    float av[T][NB][4], gv[T][NB][4], zp[T][4] = {};
    float xb[T][4][KC];
    const float cur0 = in0, cur1 = in1;
    if (works) {
      typename K::Rows xc[T];
#pragma unroll
      for (int t = 0; t < T; ++t) {
        // (a row whose dz is 0 adds nothing, whatever it holds)
        if (!LOSS) K::keep(xa[t], dza[t] != 0.0f && row0 + 16 * t + c < end);
        xc[t] = K::rows(xa[t]);
      }
      if (row0 + R <= end) {
        const char *x = (const char *)p.x + row0 * ld;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int k = 0; k < KC; ++k)
              xb[t][r][k] = element<BF16>(x + (size_t)(16 * t + r) * ld + off_b, 16 * k);
      } else {
        const int64_t base = row0 < end ? row0 : end - 1;
        const int last = (int)(end - base) - 1;
        const char *x = (const char *)p.x + base * ld;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int k = 0; k < KC; ++k)
              xb[t][r][k] = element<BF16>(x + __umul24(min(16 * t + 4 * q + r, last), ld), 16 * k + c);
      }
      fetch(row0 + R * RG);
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const gf32x4 g = K::product(xc[t], wgt[0][b]), u = K::product(xc[t], wgt[1][b]);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float s = sigmoid(g[r]), a = g[r] * s;
            av[t][b][r] = a;
            gv[t][b][r] = u[r] * fmaf(s, g[r] - a, s);   // u silu'(g)
            if (LOSS) zp[t][r] = fmaf(w3[b], a * u[r], zp[t][r]);
          }
        }
    }
    float dz = 0.0f;
    if constexpr (LOSS) {
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) zp[t][r] = row_sum(zp[t][r]);
      float(*zb)[R] = zbuf[step & 1];
      if (works && c == 0) {
#pragma unroll
        for (int t = 0; t < T; ++t) *(gf32x4 *)&zb[wave][16 * t + 4 * q] = gf32x4{zp[t][0], zp[t][1], zp[t][2], zp[t][3]};
      }
      if (HG > 1) __syncthreads();
      else __builtin_amdgcn_wave_barrier();
      if (works) {
        float z = b3;
        for (int h = 0; h < HG; ++h) z += zb[rg * HG + h][i_row];
        const int64_t row = row0 + i_row;
        const bool there = row < end;
        const bool counts = there && cur0 > 0.0f && cur0 < __builtin_inff() && cur1 > 0.0f && cur1 < __builtin_inff();
        const EtaTerm e = eta_term(z, cur0, cur1, p.huber);
        if (counts) dz = e.dz;
        if (hg == 0 && lane < R && there) {
          if (p.z) p.z[row] = z;
          if (counts) {
            sum += (double)e.loss;
            total += (double)cur1;
          }
        }
      }
    } else {
      if (row0 + i_row < end) dz = cur0;
    }
    if (works) {
      if (hg == 0 && lane < R) d0 += dz;
      dzbuf[wave][i_row] = dz;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const gf32x4 d = *(const gf32x4 *)&dzbuf[wave][16 * t + 4 * q];
        if constexpr (LOSS) {
          // A row that does not count may hold anything: where its z is not finite,
          // neither need be what is made of it (z is, only if all of it is).
          bool odd = false;
#pragma unroll
          for (int r = 0; r < 4; ++r) odd = odd || (d[r] == 0.0f && !(fabsf(zp[t][r]) < __builtin_inff()));
          if (__ballot(odd)) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int b = 0; b < NB; ++b) {
                if (d[r] == 0.0f) av[t][b][r] = gv[t][b][r] = 0.0f;
              }
          }
        }
        // the features' operand: Q0 Q2, Q1 Q1, Q0 Q0 of dz x against P2 P0, P1 P0, P1 P0
        gu32x4 xq[KC][3];
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          float v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = d[r] != 0.0f ? d[r] * xb[t][r][k] : 0.0f;
          uint32_t a[3], b[3];
          split2(v[0], v[1], a[0], a[1], a[2]);
          split2(v[2], v[3], b[0], b[1], b[2]);
          xq[k][0] = gu32x4{a[0], b[0], a[2], b[2]};
          xq[k][1] = gu32x4{a[1], b[1], a[1], b[1]};
          xq[k][2] = gu32x4{a[0], b[0], a[0], b[0]};
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const float(&v)[4] = m ? av[t][b] : gv[t][b];
            uint32_t a0[3], a1[3];
            split2(v[0], v[1], a0[0], a0[1], a0[2]);
            split2(v[2], v[3], a1[0], a1[1], a1[2]);
            const gu32x4 lo = {a0[2], a1[2], a0[0], a1[0]}, hi = {a0[1], a1[1], a0[0], a1[0]};
#pragma unroll
            for (int k = 0; k < KC; ++k) dw[m][b][k] = K::mfma(lo, xq[k][0], dw[m][b][k]);
#pragma unroll
            for (int k = 0; k < KC; ++k) dw[m][b][k] = K::mfma(hi, xq[k][1], dw[m][b][k]);
#pragma unroll
            for (int k = 0; k < KC; ++k) dw[m][b][k] = K::mfma(hi, xq[k][2], dw[m][b][k]);
          }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
#pragma unroll
  for (int d = 1; d < R; d *= 2) d0 += __shfl_xor(d0, d);
  if constexpr (LOSS) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      sum += __shfl_xor(sum, d);
      total += __shfl_xor(total, d);
    }
    __shared__ double part[W][2];
    if (lane == 0) {
      part[wave][0] = sum;
      part[wave][1] = total;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
      double v = 0.0;
      for (int i = 0; i < W; ++i) v += part[i][threadIdx.x];
      p.loss_part[2 * wg + threadIdx.x] = v;
    }
  }
  // the row groups' sums onto the first's, in order
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
    d0 += o[n][lane];
  }
  float *out = p.part + (size_t)wg * gated_part_size(p.hidden, IN);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int unit0 = hg * K::kGroup + 16 * b;
    float *mine = out + (unit0 / kGatedGroup) * kGatedGroup * 2 * IN;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < KC; ++k)
          mine[(m * kGatedGroup + unit0 % kGatedGroup + 4 * q + i) * IN + 16 * k + c] = dw[m][b][k][i];
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
    const int32_t *wgs = p.g_w1 ? p.bwd_wg : p.fwd_wg;   // of the kernel that summed the loss
    for (int w = wgs[f] + (int)threadIdx.x; w < wgs[f + 1]; w += kThreads) {
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
    at = (unit / kGatedGroup) * kGatedGroup * 2 * IN + (m * kGatedGroup + unit % kGatedGroup) * IN + i % IN;
  } else if (e == 2 * HI) {
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
  if (sl > 0) return;   // (the first half of the first wave is left)
  for (int i = 1; i < kRedParts; ++i) v += part[i][el];
  v = n > 0 ? v * scale : 0.0;
  if (e >= HI && e < 2 * HI) {
    // dw3 of the unit: its 16 or 32 elements are this many lanes of the half
    const int d = e % IN;
    double w = n > 0 ? v * (double)element<BF16>(p.w2, (int64_t)f * HI + e - HI) : 0.0;
    for (int o = IN / 2; o > 0; o /= 2) w += __shfl_xor(w, o);
    if (d == 0) p.g_w3[(size_t)f * H + unit] = (float)w;
  }
  if (at < 0) return;
  if (unit >= 0 && n > 0) v *= (double)element<BF16>(p.w3, (int64_t)f * H + unit);
  if (e < HI) p.g_w1[(size_t)f * HI + e] = (float)v;
  else if (e < 2 * HI) p.g_w2[(size_t)f * HI + e - HI] = (float)v;
  else p.g_b3[f] = (float)v;
}

}  // namespace

// ------------------------------------------------------------ launchers
template <bool LOSS>
static void forward_of(const GatedParams &p, hipStream_t s) {
  const dim3 grid(p.fwd_wg[KS_NFAM]);
  if (p.bf16) {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_forward<true, 16, 256, LOSS, 4>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_gated_forward<true, 32, 256, LOSS, 4>), grid, dim3(256), 0, s, p);
  } else {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_forward<false, 16, 256, LOSS, 4>), grid, dim3(256), 0, s, p);
    else if (p.hidden <= 128) hipLaunchKernelGGL((k_gated_forward<false, 32, 128, LOSS, 4>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((k_gated_forward<false, 32, 256, LOSS, 8>), grid, dim3(512), 0, s, p);
  }
}

hipError_t launch_gated_forward(const GatedParams &p, hipStream_t s) {
  if (p.fwd_wg[KS_NFAM] == 0) return hipSuccess;
  if (p.eta) forward_of<true>(p, s);
  else forward_of<false>(p, s);
  return hipGetLastError();
}

template <bool BF16, int IN, bool LOSS>
static void fit_kind(const GatedParams &p, hipStream_t s) {
  hipLaunchKernelGGL((k_gated_fit<BF16, IN, LOSS>), dim3(p.bwd_wg[KS_NFAM]), dim3(64 * Back<BF16, IN>::W), 0, s, p);
}
template <bool LOSS>
static void fit_of(const GatedParams &p, hipStream_t s) {
  if (p.bf16) p.in_dim == 16 ? fit_kind<true, 16, LOSS>(p, s) : fit_kind<true, 32, LOSS>(p, s);
  else p.in_dim == 16 ? fit_kind<false, 16, LOSS>(p, s) : fit_kind<false, 32, LOSS>(p, s);
}

hipError_t launch_gated_fit(const GatedParams &p, hipStream_t s) {
  if (p.bwd_wg[KS_NFAM] == 0) return hipSuccess;
  if (p.eta) fit_of<true>(p, s);
  else fit_of<false>(p, s);
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
  const int elements = p.g_w1 ? 2 * p.hidden * p.in_dim + 1 : 1;
  const int chunks = (elements + kRedEl - 1) / kRedEl;
  const dim3 grid(KS_NFAM * chunks), block(kThreads);
  if (p.bf16) hipLaunchKernelGGL((k_gated_reduce<true>), grid, block, 0, s, p, chunks);
  else hipLaunchKernelGGL((k_gated_reduce<false>), grid, block, 0, s, p, chunks);
  return hipGetLastError();
}

}  // namespace ks
