// Gated heads over feature rows: the block, its gradients and the loss on
// log eta (ks.h).  Rows are grouped by family; a workgroup works on rows of one.
//
//   k_gated_forward   z, and for a fit the loss sums and dz of each row
//   k_gated_sums      weight gradients of a workgroup's rows, held in registers
//                     (for few rows with the loss's forward pass)
//   k_gated_rows      gradients of the rows
//   k_gated_reduce    sums of the workgroups' gradients in a fixed order
//
// The derivative at a row, with s = sigma(g), a = g s:
//   du = dz w3 a,  dg = dz w3 u silu'(g),  silu'(g) = s + s (g - a),  dw3 += dz a u.
// w3 is one factor of a unit over all rows, so k_gated_sums leaves it out and
// k_gated_reduce multiplies the finished sums by it.  dz is one factor of a row
// over all units: fp32 heads have it on the rows' side of the product, dW =
// (..)^T (dz x); bf16 heads, whose rows are one exact piece, on the units' side.
// And u = W2 x, so sum dz a u = W2 . (sum dz a x): dw3 follows from the finished
// sum of dW2.
#include <hip/hip_runtime.h>

#include "ks_gated.h"
#include "ks_internal.h"

namespace ks {

using gated::Block;
using gated::EtaTerm;
using gated::eta_term;
using gated::gbf16x8;
using gated::gf32x16;
using gated::gf32x4;
using gated::gu32x4;
using gated::sigmoid;
using gated::split2;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t any16 __attribute__((may_alias));

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
  int f = 0;   // (all offsets read at once: no chain of scalar loads)
#pragma unroll
  for (int i = 1; i < KS_NFAM; ++i) f += wg >= off[i];
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
// N waves share the weights in LDS: four, or, where 256 units of 32 fp32 inputs
// leave room for one workgroup per CU only, eight (two per SIMD).
template <bool BF16, int IN, int HID, bool LOSS, int N>
__global__ __launch_bounds__(64 * N, 2) void k_gated_forward(GatedParams p) {
  using G = Block<BF16, IN, HID>;
  __shared__ __align__(16) uint32_t lds[G::kLds];
  constexpr int E = BF16 ? 2 : 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wg = blockIdx.x, f = family_of(p.fwd_wg, wg);
  const int64_t begin = p.fam_off[f] + (int64_t)(wg - p.fwd_wg[f]) * p.fwd_tiles * 64;
  const int64_t fam_end = p.fam_off[f + 1];
  const int64_t end = begin + (int64_t)p.fwd_tiles * 64 < fam_end ? begin + (int64_t)p.fwd_tiles * 64 : fam_end;
  gu32x4 raw[2][G::KC][BF16 ? 1 : 2];
  auto fetch = [&](int64_t row0) {   // past the last row a lane reads the last
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = row0 + 32 * i + (lane & 31);
      const int64_t at = (r < end ? r : end - 1) * p.ldx + (lane >> 5) * 8;
#pragma unroll
      for (int kc = 0; kc < G::KC; ++kc) load8<BF16>(raw[i][kc], p.x, at + 16 * kc, p.vec);
    }
  };
  fetch(begin + 64 * wave);   // (with the weights on their way too)
  const size_t w = (size_t)f * p.hidden * IN * E;
  G::stage(lds, (const char *)p.w1 + w, (const char *)p.w2 + w, (const char *)p.w3 + (size_t)f * p.hidden * E,
           (const char *)p.b3 + f * E, p.hidden, (int)threadIdx.x, 64 * N);
  __syncthreads();
  double sum = 0.0, total = 0.0;
  for (int64_t row0 = begin + 64 * wave; row0 < end; row0 += 64 * N) {
    typename G::Rows x;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int kc = 0; kc < G::KC; ++kc) {
        if constexpr (BF16) x.v[i][kc][0] = raw[i][kc][0];
        else G::split8(__builtin_bit_cast(gf32x4, raw[i][kc][0]), __builtin_bit_cast(gf32x4, raw[i][kc][1]), x.v[i][kc]);
      }
    const float z = G::z_of(x, lds);
    const int64_t row = row0 + lane;
    if (row < end) {
      if (p.z) p.z[row] = z;
      if constexpr (LOSS) {
        const float eta = p.eta[row], wt = p.weight ? p.weight[row] : 1.0f;
        const bool counts = eta > 0.0f && eta < __builtin_inff() && wt > 0.0f && wt < __builtin_inff();
        const EtaTerm e = eta_term(z, eta, wt, p.huber);
        if (counts) {
          sum += (double)e.loss;
          total += (double)wt;
        }
        if (p.dz_out) p.dz_out[row] = counts ? e.dz : 0.0f;
      }
    }
    fetch(row0 + 64 * N);
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
// dW1 = sum (u silu'(g)) (dz x)^T, dW2 = sum a (dz x)^T over a workgroup's rows.  A
// wave takes 32 units (their weights and gradients in its registers) and 32 rows at a
// time on the 32x32x16 instruction: the rows as the row operand of the projections,
// so a lane holds the gates and ups of one unit for 16 of the rows, and what it makes
// of them is the row operand of the next product, units x features, without any
// exchange between lanes.  The eight waves are the unit groups (HG) times row groups
// (RG).  What depends on the rows alone is made once for all of them: each wave
// brings 16 rows a step, as the projections' operand and as the column operand of dW,
// and leaves both in LDS.  What a unit makes of a row is three bf16 pieces, exactly.
// The column operand is dz x in three pieces and six products for fp32 heads; for
// bf16 heads it is the rows as they are and three products, dz a multiplication of
// each of a unit's two terms.  (With dz x there too, six products, and two pieces of
// the terms, within 2^-18 of each, 2M rows of 32-256 took 421 us and weight
// gradients came out with 3e-6 where fp32 sums have 2e-6; with three pieces 530 us.
// So 402 to 424 us, and 3e-7.)
//
// Which rows a lane's eight inner indices of dW stand for is free, as long as both
// operands agree: those it has, 8 (i / 4) + 4 (its half) + i mod 4 of each 16.  With 16
// inputs the instruction's 32 columns are the features twice: for fp32 heads against
// the first and the second piece of dz x (then the third and nothing), a unit's gradient
// the sum of the two halves; bf16 heads have no use for the second.
//
// Vector work bounds it: 6 instructions, an exponential and a reciprocal for each gate
// (bf16: 8) and 11 to make what it makes into pieces, for each 48 (bf16: 16) cycles of
// the matrix unit: 2M rows of bf16 32-256, the vector units 93% and the matrix units 30%
// busy.  A wave alone issues a vector instruction every 7.5 cycles, four per SIMD one
// every 2.7 (FMA) to 5 (conversions; so only the first piece is one): hence 128
// registers and 32 units per wave; and the 32x32x16 instruction runs beside them where
// 16x16x32 does not (two waves of each kind per SIMD, multiplications: 888 cycles, alone
// 659 and 369; 16x16x32 671, alone 326 and 369).  (64 units per wave, z exchanged between
// the unit groups and dz formed on the way, one pass in all: 776 us, where this and
// k_gated_forward take 570.)
template <bool BF16, int IN>
struct Back {
  static constexpr int KC = IN / 16, W = 8;
  static constexpr int NP = BF16 ? 1 : 3;      // pieces of the projections' operands
  static constexpr int NQ = BF16 ? 1 : IN == 16 ? 2 : 3;   // column operands of dW
  // eight consecutive values as pieces
  __device__ static __forceinline__ void pieces(const gu32x4 (&raw)[BF16 ? 1 : 2], gu32x4 (&x)[NP]) {
    if constexpr (BF16) x[0] = raw[0];
    else Block<false, IN, 32>::split8(__builtin_bit_cast(gf32x4, raw[0]), __builtin_bit_cast(gf32x4, raw[1]), x);
  }
  __device__ static __forceinline__ gf32x16 mfma(const gu32x4 &a, const gu32x4 &b, const gf32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(gbf16x8, a), __builtin_bit_cast(gbf16x8, b), c, 0, 0, 0);
  }
};

// LOSS: the loss's forward pass in the same launch, for few rows (one step each) and
// for fp32 heads of 32 inputs.  A wave's weights are the row operand there: a lane
// then holds 16 of its units for one row, adds up their part of z, and the unit groups'
// parts meet in LDS.
//
// A launch takes kGatedRun rows of each workgroup.  MORE: a later launch, which goes on
// from there and adds to what the workgroup stored (one whose rows have ended, zeros).
template <bool BF16, int IN, bool LOSS, bool MORE>
__global__ __launch_bounds__(512, (!LOSS && (BF16 || IN == 16) ? 4 : 2)) void k_gated_sums(GatedParams p) {
  using K = Back<BF16, IN>;
  constexpr int KC = K::KC, W = K::W, NP = K::NP, NQ = K::NQ, R = 16 * W;   // rows of a step
  constexpr int kTiles = R / 32;
  constexpr int kX = kTiles * KC * NP * 64 * 4, kQ = kTiles * 2 * NQ * 64 * 4, kJoin = (W - 1) * 16 * 64;
  __shared__ __align__(16) uint32_t lds[kX + kQ > kJoin ? kX + kQ : kJoin];
  __shared__ __align__(16) float dzs[W][16];
  __shared__ float w3s[LOSS ? 256 : 1], zs[LOSS ? W : 1][LOSS ? R : 1];   // [unit group]: its part of z
  double sum = 0.0, total = 0.0;
  gu32x4(*lx)[KC][NP][64] = reinterpret_cast<gu32x4(*)[KC][NP][64]>(lds);          // [tile]: rows
  gu32x4(*lq)[2][NQ][64] = reinterpret_cast<gu32x4(*)[2][NQ][64]>(lds + kX);       // [tile][16 rows]: dz x
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int HG = (p.hidden + kGatedGroup - 1) / kGatedGroup, RG = HG > 4 ? 1 : HG > 2 ? 2 : 4;   // (four tiles)
  const int hg = wave % HG, rg = wave / HG;
  const bool works = rg < RG;
  const int wg = blockIdx.x, f = family_of(p.bwd_wg, wg);
  const int64_t first = p.fam_off[f] + (int64_t)(wg - p.bwd_wg[f]) * p.bwd_rows, begin = MORE ? first + p.run : first;
  const int64_t end = min(min(first + p.bwd_rows, p.fam_off[f + 1]), begin + kGatedRun);
  gf32x16 dw[2] = {gf32x16{}, gf32x16{}};
  float d0 = 0.0f;
  gu32x4 wgt[2][KC][NP];
  {
    const bool vec = ((reinterpret_cast<uintptr_t>(p.w1) | reinterpret_cast<uintptr_t>(p.w2)) & 15) == 0;
    const int unit = hg * kGatedGroup + n;
    const bool there = works && unit < p.hidden;
    const int64_t at = ((int64_t)f * p.hidden + (there ? unit : 0)) * IN + 8 * h;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        gu32x4 raw[BF16 ? 1 : 2];
        load8<BF16>(raw, m ? p.w2 : p.w1, at + 16 * k, vec);
#pragma unroll
        for (auto &v : raw) v = there ? v : gu32x4{0, 0, 0, 0};
        K::pieces(raw, wgt[m][k]);
      }
  }
  // the wave's 16 rows of a step: 16 of tile wave / 2
  const int tile = wave >> 1, half = wave & 1;
  const uint32_t ld = (uint32_t)p.ldx;
  const int oct = lane >> 4;                       // the eight features a lane brings of row c
  const bool brings = IN == 32 || oct < 2;
  const int col = IN == 32 ? n : c;                // ... and the feature of its rows
  constexpr int E = BF16 ? 2 : 4;
  const uint32_t off_row = __umul24(c, ld * E) + (brings ? 8 * E * oct : 0), off_col = __umul24(4 * h, ld * E) + col * E;
  gu32x4 raw[BF16 ? 1 : 2];
  float v[8], dzc;
  auto fetch = [&](int64_t mine) {
    if (mine + 16 <= end) {
      const char *x = (const char *)p.x + mine * ld * E;
      load8<BF16>(raw, x + off_row, 0, p.vec);
      dzc = LOSS ? 0.0f : p.dz[mine + c];
      if constexpr (!BF16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = element<BF16>(x + (size_t)(8 * (i >> 2) + (i & 3)) * ld * E + off_col, 0);
      }
    } else {   // past the last row a lane reads the last
      const int64_t base = mine < end ? mine : end - 1;
      const int last = (int)(end - base) - 1;
      load8<BF16>(raw, p.x, (base + min(c, last)) * ld + (brings ? 8 * oct : 0), p.vec);
      dzc = LOSS ? 0.0f : p.dz[base + min(c, last)];
      if constexpr (!BF16) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          v[i] = element<BF16>(p.x, (base + min(8 * (i >> 2) + 4 * h + (i & 3), last)) * ld + col);
      }
      if (mine + c >= end) dzc = 0.0f;
    }
  };
  // (a step's rows are on their way while the step before is worked on; fp32 with 16
  // inputs has no registers left for them, it spills two of its 130 as it is, and a LOSS
  // has one step otherwise)
  constexpr bool kAhead = BF16 ? !LOSS : IN == 32;
  if (kAhead) fetch(begin + 16 * wave);
  if (LOSS && threadIdx.x < 256)
    w3s[threadIdx.x] = (int)threadIdx.x < p.hidden ? element<BF16>(p.w3, (int64_t)f * p.hidden + threadIdx.x) : 0.0f;
#pragma unroll 1
  for (int64_t row0 = begin; row0 < end; row0 += R) {
    if (!kAhead) fetch(row0 + 16 * wave);
    __syncthreads();   // (the step before is done with the room)
    auto put = [&]() {
      gu32x4 x[NP];
      K::pieces(raw, x);
#pragma unroll
      for (int i = 0; i < NP; ++i) lx[tile][oct >> 1][i][16 * half + c + 32 * (oct & 1)] = x[i];
    };
    if constexpr (LOSS) {
      const int64_t row = row0 + 16 * wave + c;
      const bool in = row < end;
      const float eta = p.eta[in ? row : end - 1], wt = p.weight ? p.weight[in ? row : end - 1] : 1.0f;
      if (brings) put();
      __syncthreads();
      if (works) {
#pragma unroll 1
        for (int t = rg; t < kTiles; t += RG) {
          if (row0 + 32 * t >= end) break;
          gf32x16 g = {}, u = {};
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            auto both = [&](int i, int j) {
              g = K::mfma(wgt[0][k][j], lx[t][k][i][lane], g);
              u = K::mfma(wgt[1][k][j], lx[t][k][i][lane], u);
            };
            if constexpr (!BF16) {
              both(2, 0);
              both(1, 1);
              both(0, 2);
              both(1, 0);
              both(0, 1);
            }
            both(0, 0);
          }
          float z = 0.0f;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            z = fmaf(g[r] * sigmoid(g[r]) * u[r], w3s[hg * kGatedGroup + 8 * (r >> 2) + 4 * h + (r & 3)], z);
          z += __shfl_xor(z, 32);
          if (h == 0) zs[hg][32 * t + n] = z;
        }
      }
      __syncthreads();
      float z = element<BF16>(p.b3, f);
      for (int i = 0; i < HG; ++i) z += zs[i][16 * wave + c];
      const bool counts = in && eta > 0.0f && eta < __builtin_inff() && wt > 0.0f && wt < __builtin_inff();
      const EtaTerm e = eta_term(z, eta, wt, p.huber);
      dzc = counts ? e.dz : 0.0f;
      if (oct == 0) {
        if (in && p.z) p.z[row] = z;
        if (counts) {
          sum += (double)e.loss;
          total += (double)wt;
        }
      }
    }
    {
      // (a row whose dz is 0 adds nothing, whatever it holds)
      const bool on = dzc != 0.0f;
      if (oct == 0) {
        d0 += dzc;
        dzs[wave][c] = dzc;
      }
      if (brings && !(LOSS && on)) {
#pragma unroll
        for (auto &r : raw) r = on ? r : gu32x4{0, 0, 0, 0};
        put();
      }
      __builtin_amdgcn_wave_barrier();
      if constexpr (BF16) {
        // (the rows as they lie in LDS now: those without dz are zeros)
        const any16 *own = (const any16 *)&lx[tile][col >> 4][0][16 * half + 4 * h + 32 * ((col >> 3) & 1)] + (col & 7);
        gu32x4 q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const any16 *at = own + 8 * (8 * (i >> 1) + 2 * (i & 1));
          q[i] = at[0] | (uint32_t)at[8] << 16;
        }
        lq[tile][half][0][lane] = q;
      } else {
        gu32x4 qp[3];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const gf32x4 dz = *(const gf32x4 *)&dzs[wave][8 * j + 4 * h];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t p0, p1, p2;
            const float a = dz[2 * i] != 0.0f ? dz[2 * i] * v[4 * j + 2 * i] : 0.0f;
            const float b = dz[2 * i + 1] != 0.0f ? dz[2 * i + 1] * v[4 * j + 2 * i + 1] : 0.0f;
            split2(a, b, p0, p1, p2);
            qp[0][2 * j + i] = p0, qp[1][2 * j + i] = p1, qp[2][2 * j + i] = p2;
          }
        }
        if constexpr (IN == 32) {
#pragma unroll
          for (int i = 0; i < 3; ++i) lq[tile][half][i][lane] = qp[i];
        } else {
          lq[tile][half][0][lane] = n < 16 ? qp[0] : qp[1];
          lq[tile][half][1][lane] = n < 16 ? qp[2] : gu32x4{0, 0, 0, 0};
        }
      }
    }
    __syncthreads();
    if (kAhead) fetch(row0 + R + 16 * wave);
    if (works) {
#pragma unroll 1
      for (int t = rg; t < kTiles; t += RG) {
        if (row0 + 32 * t >= end) break;
        gf32x16 g = {}, u = {};
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          gu32x4 x[NP];
#pragma unroll
          for (int i = 0; i < NP; ++i) x[i] = lx[t][k][i][lane];
          auto both = [&](int i, int j) {
            g = K::mfma(x[i], wgt[0][k][j], g);
            u = K::mfma(x[i], wgt[1][k][j], u);
          };
          if constexpr (!BF16) {
            both(2, 0);
            both(1, 1);
            both(0, 2);
            both(1, 0);
            both(0, 1);
          }
          both(0, 0);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          gu32x4 w[2][3];   // pieces of what the unit makes of 8 rows: for dW1, dW2
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float a[2], e[2];
#pragma unroll
            for (int o = 0; o < 2; ++o) {
              const int r = 2 * i + o;
              const float gr = g[8 * j + r], s = sigmoid(gr), si = gr * s;
              e[o] = u[8 * j + r] * fmaf(s, gr - si, s);   // u silu'(g)
              a[o] = si;
              if constexpr (BF16) {
                const float dz = dzs[2 * t + j][8 * (r >> 2) + 4 * h + (r & 3)];
                e[o] *= dz;
                a[o] *= dz;
              }
            }
            uint32_t p0, p1, p2;
            split2(e[0], e[1], p0, p1, p2);
            w[0][0][i] = p0, w[0][1][i] = p1, w[0][2][i] = p2;
            split2(a[0], a[1], p0, p1, p2);
            w[1][0][i] = p0, w[1][1][i] = p1, w[1][2][i] = p2;
          }
          gu32x4 x[NQ];
#pragma unroll
          for (int i = 0; i < NQ; ++i) x[i] = lq[t][j][i][lane];
          auto add = [&](int i, int k) {
            dw[0] = K::mfma(w[0][i], x[k], dw[0]);
            dw[1] = K::mfma(w[1][i], x[k], dw[1]);
          };
          if constexpr (BF16) {
            add(2, 0);
            add(1, 0);
          } else if constexpr (IN == 32) {
            add(2, 0);
            add(1, 1);
            add(0, 2);
            add(1, 0);
            add(0, 1);
          } else {
            add(0, 1);
            add(2, 0);
            add(1, 0);
          }
          add(0, 0);
        }
      }
    }
  }
  // db3, the loss, and the row groups' sums onto the first's in order (in the same room)
  __shared__ float d0s[W];
  __shared__ double loss[LOSS ? W : 1][2];
  if constexpr (LOSS) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      sum += __shfl_xor(sum, d);
      total += __shfl_xor(total, d);
    }
    if (lane == 0) {
      loss[wave][0] = sum;
      loss[wave][1] = total;
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) d0 += __shfl_xor(d0, d);
  if (lane == 0) d0s[wave] = d0;
  float(*join)[16][64] = reinterpret_cast<float(*)[16][64]>(lds);
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    __syncthreads();
    if (works && rg > 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) join[(rg - 1) * HG + hg][i][lane] = dw[m][i];
    }
    __syncthreads();
    if (works && rg == 0) {
      for (int g = 1; g < RG; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) dw[m][i] += join[(g - 1) * HG + hg][i][lane];
    }
  }
  if (!works || rg > 0) return;
  float *out = p.part + (size_t)wg * gated_part_size(p.hidden, IN);
  float *own = out + hg * kGatedGroup * 2 * IN;
  auto at = [&](int m, int i) { return own + (m * kGatedGroup + 8 * (i >> 2) + 4 * h + (i & 3)) * IN + n; };
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if constexpr (IN == 16 && !BF16) dw[m][i] += __shfl_xor(dw[m][i], 16);   // the features' second half of the columns
  if (n < IN) {
    if constexpr (MORE) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) dw[m][i] += *at(m, i);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) *at(m, i) = dw[m][i];
  }
  if (hg == 0 && lane == 0) {
    float v = 0.0f;
    for (int i = 0; i < W; ++i) v += d0s[i];
    float *last = out + gated_part_size(p.hidden, IN) - 1;
    *last = MORE ? *last + v : v;
    if constexpr (LOSS) {
      for (int i = 1; i < W; ++i) {
        sum += loss[i][0];
        total += loss[i][1];
      }
      p.loss_part[2 * wg] = MORE ? p.loss_part[2 * wg] + sum : sum;
      p.loss_part[2 * wg + 1] = MORE ? p.loss_part[2 * wg + 1] + total : total;
    }
  }
}

// ------------------------------------------------------------ rows' gradients
// dx = W1^T dg + W2^T du: units are summed over, so here the units are the row
// operand of the projections, as in k_gated_forward (a lane holds 16 units of one row),
// and what it makes of them is the column operand of the next product, features x rows,
// whose row operand is the weights transposed: eight units of a feature per lane, in
// the order in which a lane has them.  Both forms of 128 units' weights are in LDS;
// wider heads take them in two parts for 512 rows at a time.  With 16 inputs the
// instruction's 32 rows are the features twice, against the first and the second piece
// of an fp32 weight (then the third and nothing).
//
// (100,003 rows of fp32 32-67 on the fp32 instruction: 32 us; so 24 us.)
template <bool BF16, int IN>
__global__ __launch_bounds__(512, 2) void k_gated_rows(GatedParams p) {
  constexpr int HID = 128, E = BF16 ? 2 : 4, W = 8, T = 2;
  using G = Block<BF16, IN, HID>;
  constexpr int KC = G::KC, NP = G::NP, NT = IN == 32 ? NP : BF16 ? 1 : 2;   // operands of the weights transposed
  __shared__ __align__(16) uint32_t lds[G::kLds];
  __shared__ __align__(16) gu32x4 lt[HID / 32][2][2][NT][64];   // [32 units][W1, W2][16 units]
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wg = blockIdx.x, f = family_of(p.row_wg, wg);
  const int64_t begin = p.fam_off[f] + (int64_t)(wg - p.row_wg[f]) * p.row_rows;
  const int64_t fam_end = p.fam_off[f + 1];
  const int64_t end = begin + p.row_rows < fam_end ? begin + p.row_rows : fam_end;
  const int parts = (p.hidden + HID - 1) / HID;
  for (int64_t row0 = begin; row0 < end; row0 += 32 * T * W) {
    gf32x16 acc[T] = {};
    for (int part = 0; part < parts; ++part) {
      const int hid = min(p.hidden - part * HID, HID), nb = (hid + 31) / 32;
      if (parts > 1 || row0 == begin) {
        if (part > 0 || row0 > begin) __syncthreads();
        const int64_t unit0 = (int64_t)f * p.hidden + part * HID;
        const char *w1 = (const char *)p.w1 + unit0 * IN * E, *w2 = (const char *)p.w2 + unit0 * IN * E;
        G::stage(lds, w1, w2, (const char *)p.w3 + unit0 * E, (const char *)p.b3 + f * E, hid, (int)threadIdx.x, 64 * W);
        for (int i = threadIdx.x; i < nb * 4 * 64; i += 64 * W) {
          const int l = i & 63, j = (i >> 6) & 1, m = (i >> 7) & 1, blk = i >> 8;
          const int feature = l & (IN - 1);
          float v[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int unit = 32 * blk + 16 * j + 8 * (u >> 2) + 4 * (l >> 5) + (u & 3);
            v[u] = element<BF16>(m ? w2 : w1, (int64_t)(unit < hid ? unit : 0) * IN + feature);
            if (unit >= hid) v[u] = 0.0f;
          }
          gu32x4 q[3];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            uint32_t p0, p1, p2;
            split2<true>(v[2 * u], v[2 * u + 1], p0, p1, p2);
            q[0][u] = p0, q[1][u] = p1, q[2][u] = p2;
          }
          const gu32x4 none = {0, 0, 0, 0};
          const bool second = IN == 16 && (l & 16);
          if constexpr (IN == 32) {
#pragma unroll
            for (int u = 0; u < NT; ++u) lt[blk][m][j][u][l] = q[u];
          } else {
            lt[blk][m][j][0][l] = !second ? q[0] : BF16 ? none : q[1];
            if constexpr (NT == 2) lt[blk][m][j][1][l] = !second ? q[2] : none;
          }
        }
        __syncthreads();
      }
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const int64_t r0 = row0 + 32 * (W * t + wave);
        if (r0 >= end) break;
        const int64_t row = r0 + n, at = row < end ? row : end - 1;
        const float dz = row < end ? p.dz[at] : 0.0f;
        gu32x4 x[KC][NP];
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          gu32x4 raw[BF16 ? 1 : 2];
          load8<BF16>(raw, p.x, at * p.ldx + 16 * k + 8 * h, p.vec);
          // (a row whose dz is 0 gets zeros, whatever it holds)
#pragma unroll
          for (auto &r : raw) r = dz != 0.0f ? r : gu32x4{0, 0, 0, 0};
          Back<BF16, IN>::pieces(raw, x[k]);
        }
#pragma unroll 1
        for (int blk = 0; blk < nb; ++blk) {
          const uint32_t *w = lds + blk * G::kBlk;
          gf32x16 g = {}, u = {};
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            auto both = [&](int i, int j) {
              g = Back<BF16, IN>::mfma(*(const gu32x4 *)(w + k * G::kFrag + 256 * i + 4 * lane), x[k][j], g);
              u = Back<BF16, IN>::mfma(*(const gu32x4 *)(w + (KC + k) * G::kFrag + 256 * i + 4 * lane), x[k][j], u);
            };
            if constexpr (!BF16) {
              both(2, 0);
              both(1, 1);
              both(0, 2);
              both(1, 0);
              both(0, 1);
            }
            both(0, 0);
          }
          const float *w3 = (const float *)w + 2 * KC * G::kFrag + 16 * h;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            gu32x4 d[2][3];   // dg and du of 16 units in pieces
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float a[2], e[2];
#pragma unroll
              for (int o = 0; o < 2; ++o) {
                const int r = 8 * j + 2 * i + o;
                const float dy = dz * w3[r], gr = g[r], s = sigmoid(gr), si = gr * s;
                a[o] = dy * si;
                e[o] = dy * u[r] * fmaf(s, gr - si, s);
              }
              uint32_t p0, p1, p2;
              split2(e[0], e[1], p0, p1, p2);
              d[0][0][i] = p0, d[0][1][i] = p1, d[0][2][i] = p2;
              split2(a[0], a[1], p0, p1, p2);
              d[1][0][i] = p0, d[1][1][i] = p1, d[1][2][i] = p2;
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              auto add = [&](int i, int k) { acc[t] = Back<BF16, IN>::mfma(lt[blk][m][j][i][lane], d[m][k], acc[t]); };
              if constexpr (BF16) {
                add(0, 2);
                add(0, 1);
              } else if constexpr (IN == 32) {
                add(2, 0);
                add(1, 1);
                add(0, 2);
                add(1, 0);
                add(0, 1);
              } else {
                add(1, 0);
                add(0, 2);
                add(0, 1);
              }
              add(0, 0);
            }
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int64_t row = row0 + 32 * (W * t + wave) + n;
      if (row >= end) continue;
      const bool on = p.dz[row] != 0.0f;   // (zeros even where a weight is not finite)
#pragma unroll
      for (int i = 0; i < IN / 8; ++i) {
        gf32x4 v;
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          const float s = IN == 16 && !BF16 ? acc[t][4 * i + o] + acc[t][8 + 4 * i + o] : acc[t][4 * i + o];
          v[o] = on ? s : 0.0f;
        }
        const int64_t at = row * p.g_ldx + 8 * i + 4 * h;
        if constexpr (BF16) {
          uint16_t *o = (uint16_t *)p.g_x + at;
          if (p.g_vec) {
            *(u32x2 *)o = u32x2{bf16_of(v[0]) | (uint32_t)bf16_of(v[1]) << 16, bf16_of(v[2]) | (uint32_t)bf16_of(v[3]) << 16};
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = bf16_of(v[k]);
          }
        } else {
          float *o = (float *)p.g_x + at;
          if (p.g_vec) {
            *(gf32x4 *)o = v;
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = v[k];
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
  if (p.g_w1 && at >= 0) {
    const int lo = sl * per, hi = min(lo + per, n);
    const float *src = p.part + (size_t)first * size + at;
#pragma unroll 8
    for (int i = lo; i < hi; ++i) v += (double)src[(size_t)i * size];
  }
  // (the loss's sums after the loads above are on their way)
  double scale = 1.0;
  if (p.eta) {
    __shared__ double ls[kThreads][2];
    double a = 0.0, b = 0.0;
    for (int w = p.loss_wg[f] + (int)threadIdx.x; w < p.loss_wg[f + 1]; w += kThreads) {
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

template <bool LOSS, bool MORE>
static hipError_t sums_of(const GatedParams &p, hipStream_t s) {
  const dim3 grid(p.bwd_wg[KS_NFAM]), block(512);
  if constexpr (LOSS && MORE) {   // (the others take a loss of so many rows in two launches)
    if (p.bf16 || p.in_dim == 16) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_gated_sums<false, 32, true, true>), grid, block, 0, s, p);
  } else if (p.bf16) {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_sums<true, 16, LOSS, MORE>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_sums<true, 32, LOSS, MORE>), grid, block, 0, s, p);
  } else {
    if (p.in_dim == 16) hipLaunchKernelGGL((k_gated_sums<false, 16, LOSS, MORE>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((k_gated_sums<false, 32, LOSS, MORE>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

hipError_t launch_gated_sums(const GatedParams &p, bool loss, hipStream_t s) {
  if (p.bwd_wg[KS_NFAM] == 0) return hipSuccess;
  hipError_t e = loss ? sums_of<true, false>(p, s) : sums_of<false, false>(p, s);
  GatedParams q = p;
  for (q.run = kGatedRun; e == hipSuccess && q.run < p.bwd_rows; q.run += kGatedRun)
    e = loss ? sums_of<true, true>(q, s) : sums_of<false, true>(q, s);
  return e;
}

hipError_t launch_gated_rows(const GatedParams &p, hipStream_t s) {
  const dim3 grid(p.row_wg[KS_NFAM]), block(512);
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
