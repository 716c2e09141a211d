// The gated efficiency head's device code: the block that the evaluation
// (ks_kernels.hip) and the row operators (ks_gated.hip) share.
//
//   z = w3 . (silu(W1 x) * (W2 x)) + b3,   silu(g) = g / (1 + exp(-g))
//
// A wave takes 64 rows: two column blocks of 32 on the 32x32x16 matrix
// instruction, the weights its row operand from LDS.  One lane then holds 16
// of a 32-unit block's gates and ups of one row, so the activation, the product
// and the dot product with w3 stay in the lane's registers; one exchange of the
// wave's halves at the end completes the sums over the units.
//
// fp32 operands are split into three bf16 pieces that sum to them exactly (from
// 2^-102 up; below, what is lost is under 2^-126) and the six products of the
// largest pieces are taken: the three left out are at most 2^-24 of the product (the
// second piece is at most 2^-9 of the number and the third 2^-16), its own rounding in
// fp32.
// The bf16 instruction runs beside other waves' vector work, most of the way; the fp32
// one does not (two waves of each per SIMD: 32x32x16 bf16 and multiplications take 888
// cycles, alone 659 and 369; 16x16x4 fp32 940, alone 578 and 367), and the vector work
// is what bounds this block: an exponential, a reciprocal and five more per gate.
//
// 2M rows of bf16 32-256: 165 us, the vector units 91% busy.  1M rows of fp32 32-256:
// 158 us (six products at the rate of a large bf16 product: 159; on the fp32
// instruction it took 305).
#pragma once

#include <stdint.h>

namespace ks {
namespace gated {

typedef __bf16 gbf16x8 __attribute__((ext_vector_type(8)));
typedef float gf32x16 __attribute__((ext_vector_type(16)));
typedef float gf32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t gu32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxHidden = 256;

// 1 / (1 + exp(-g)).  exp(-g) overflows to infinity below -88: 0, as it should.
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504088896340736f));
}

// two floats -> packed bfloat16 pair, round to nearest even
typedef __bf16 gbf16x2 __attribute__((ext_vector_type(2)));
typedef float gf32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((gf32x2{lo, hi}), gbf16x2));
}
// a pair of values as three packed pairs of pieces.  (A piece could be taken off in one
// instruction, the dot product with (-1, 0) or (0, -1), but that one waits for the
// matrix instructions of every wave, as the shift or mask and the subtraction do not.)
//
// The first piece is rounded, so what is left is at most 2^-9; the second is cut
// off, so that what it leaves, at most 2^-16, fits the third exactly.  (Were the first
// cut off too, all three would have the value's sign: the instruction drops what lies
// far below its running sum, and a sum of one sign over 2M rows then came out 2.7e-6
// low where it is 3e-7 off.)
__device__ __forceinline__ uint32_t upper(float v) { return __builtin_bit_cast(uint32_t, v) & 0xFFFF0000u; }
__device__ __forceinline__ uint32_t pack_upper(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302);
}
// ANY: numbers up to fp32's largest, whose nearest bfloat16 is infinity from 3.396e38 up:
// they leave the largest finite one as the first piece.
template <bool ANY = false>
__device__ __forceinline__ void split2(float a, float b, uint32_t &p0, uint32_t &p1, uint32_t &p2) {
  constexpr float kTop = 0x1.fep127f;
  p0 = ANY ? pack2(__builtin_amdgcn_fmed3f(a, -kTop, kTop), __builtin_amdgcn_fmed3f(b, -kTop, kTop)) : pack2(a, b);
  a -= __builtin_bit_cast(float, p0 << 16);
  b -= __builtin_bit_cast(float, p0 & 0xFFFF0000u);
  p1 = pack_upper(a, b);
  a -= __builtin_bit_cast(float, upper(a));
  b -= __builtin_bit_cast(float, upper(b));
  p2 = pack_upper(a, b);
}

// 1 + e^-z: the exponent's rounding, 2^-24 of |z| log2 e, is put back to first order
__device__ __forceinline__ float eta_of(float z) {
  constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
  const float t = z * -kLog2e, lo = fmaf(z, -kLog2e, -t) - z * 1.92596299e-8f, e = __builtin_amdgcn_exp2f(t);
  return 1.0f + (fabsf(z) < 80.0f ? fmaf(e * kLn2, lo, e) : e);
}

// HID: the widest block that fits the LDS room (any narrower one too)
template <bool BF16, int IN, int HID>
struct Block {
  static constexpr int KC = IN / 16;                  // 16-feature chunks
  static constexpr int NP = BF16 ? 1 : 3;             // pieces of an operand
  static constexpr int kFrag = NP * 256;              // dwords of 32 units x 16 features
  static constexpr int kBlk = 2 * KC * kFrag + 32;    // of 32 units: gates, ups, w3 by register and half
  static constexpr int kLds = HID / 32 * kBlk + 4;
  static constexpr int OFF_B3 = kLds - 4, OFF_NB = kLds - 3;

  // unit of register r in lane half h of a block's products
  __device__ static __forceinline__ int unit_of(int h, int r) { return 8 * (r >> 2) + 4 * h + (r & 3); }

  // eight values as packed pieces
  __device__ static __forceinline__ void split8(const gf32x4 &a, const gf32x4 &b, gu32x4 (&p)[NP]) {
    if constexpr (!BF16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t p0, p1, p2;
        split2<true>(j < 2 ? a[2 * j] : b[2 * j - 4], j < 2 ? a[2 * j + 1] : b[2 * j - 3], p0, p1, p2);
        p[0][j] = p0;
        p[1][j] = p1;
        p[2][j] = p2;
      }
    }
  }

  // a family's weights into LDS; units past hidden are zero (and add nothing)
  __device__ static void stage(uint32_t *lds, const void *w1, const void *w2, const void *w3, const void *b3, int hidden,
                               int tid, int n_threads) {
    const int nb = (hidden + 31) / 32;
    constexpr int E = BF16 ? 2 : 4;
    const bool vec = ((reinterpret_cast<uintptr_t>(w1) | reinterpret_cast<uintptr_t>(w2)) & 15) == 0;
    // one lane's 8 features of a fragment: 16 bytes of bf16, 32 of fp32
    for (int i = tid; i < nb * 2 * KC * 64; i += n_threads) {
      const int lane = i & 63, fr = i >> 6;
      const int kc = fr % KC, m = (fr / KC) & 1, mb = fr / (2 * KC);
      const int unit = mb * 32 + (lane & 31);
      const char *src = (const char *)(m ? w2 : w1) + ((size_t)unit * IN + kc * 16 + (lane >> 5) * 8) * E;
      uint32_t *dst = lds + mb * kBlk + (m * KC + kc) * kFrag + lane * 4;
      gu32x4 v0 = {0, 0, 0, 0}, v1 = {0, 0, 0, 0};
      if (unit < hidden) {
        if (vec) {
          v0 = *(const gu32x4 *)src;
          if constexpr (!BF16) v1 = *(const gu32x4 *)(src + 16);
        } else if constexpr (BF16) {
          const uint16_t *h = (const uint16_t *)src;
#pragma unroll
          for (int j = 0; j < 4; ++j) v0[j] = h[2 * j] | (uint32_t)h[2 * j + 1] << 16;
        } else {
          const uint32_t *f = (const uint32_t *)src;
#pragma unroll
          for (int j = 0; j < 4; ++j) v0[j] = f[j], v1[j] = f[4 + j];
        }
      }
      if constexpr (BF16) {
        *(gu32x4 *)dst = v0;
      } else {
        gu32x4 p[NP];
        split8(__builtin_bit_cast(gf32x4, v0), __builtin_bit_cast(gf32x4, v1), p);
#pragma unroll
        for (int j = 0; j < NP; ++j) *(gu32x4 *)(dst + 256 * j) = p[j];
      }
    }
    for (int i = tid; i < nb * 32; i += n_threads) {
      const int mb = i >> 5, unit = mb * 32 + unit_of((i >> 4) & 1, i & 15);
      float w = 0.0f;
      if (unit < hidden)
        w = BF16 ? __builtin_bit_cast(float, (uint32_t)((const uint16_t *)w3)[unit] << 16) : ((const float *)w3)[unit];
      ((float *)lds)[mb * kBlk + 2 * KC * kFrag + (i & 31)] = w;
    }
    if (tid == 0) {
      ((float *)lds)[OFF_B3] = BF16 ? __builtin_bit_cast(float, (uint32_t)*(const uint16_t *)b3 << 16) : *(const float *)b3;
      lds[OFF_NB] = (uint32_t)nb;
    }
  }

  // the column operand of 64 rows: a lane holds, of row (lane mod 32) of each
  // column block, the eight features of its half
  struct Rows {
    gu32x4 v[2][KC][NP];
  };

  // c += W x for the two column blocks in turn (neither instruction waits for the
  // one before it), small pieces first
  __device__ static __forceinline__ void products(const uint32_t *frag, int lane, const Rows &x, int kc, gf32x16 (&c)[2]) {
    gbf16x8 a[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) a[j] = __builtin_bit_cast(gbf16x8, *(const gu32x4 *)(frag + 256 * j + lane * 4));
    auto both = [&](int i, int j) {
      c[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], __builtin_bit_cast(gbf16x8, x.v[0][kc][j]), c[0], 0, 0, 0);
      c[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], __builtin_bit_cast(gbf16x8, x.v[1][kc][j]), c[1], 0, 0, 0);
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

  // z of row (lane) of the 64
  __device__ static __forceinline__ float z_of(const Rows &x, const uint32_t *lds) {
    const int lane = threadIdx.x & 63;
    const int nb = __builtin_amdgcn_readfirstlane(lds[OFF_NB]);
    float z[2] = {0.0f, 0.0f};
#pragma unroll 1
    for (int mb = 0; mb < nb; ++mb) {
      const uint32_t *blk = lds + mb * kBlk;
      gf32x16 g[2] = {gf32x16{}, gf32x16{}}, u[2] = {gf32x16{}, gf32x16{}};
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        products(blk + kc * kFrag, lane, x, kc, g);
        products(blk + (KC + kc) * kFrag, lane, x, kc, u);
      }
      const float *w3 = (const float *)blk + 2 * KC * kFrag + (lane >> 5) * 16;
      float y[2] = {0.0f, 0.0f};   // (of a block by itself: 16 + 8 additions in a row for 256 units, not 128)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = w3[r];
#pragma unroll
        for (int i = 0; i < 2; ++i) y[i] = fmaf(w, g[i][r] * sigmoid(g[i][r]) * u[i][r], y[i]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) z[i] += y[i];
    }
    // lanes 32.. of the first block's sums for lanes ..31 of the second's
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, z[0]), __builtin_bit_cast(uint32_t, z[1]),
                                                    false, false);
    return __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]) +
           ((const float *)lds)[OFF_B3];
  }
};

}  // namespace gated
}  // namespace ks
