// The AdamW step over many tensors (ks.h): one launch for 200 of them, their
// table in the kernel arguments, a workgroup per 1024 elements of one tensor.
//
// Every element is read and written once, so bytes bound it: 28 per element with
// states in 32 bits, 16 with states in 8 bits (m e4m3, v e5m2, one power of two
// per 64 elements), 2 more with the bf16 copy.  A lane takes four consecutive
// elements, so 64 elements are a row of 16 lanes: a block's largest value is
// four lane moves away and no state goes through LDS.
//
// 600 tensors, 25M elements, with copies: 101 us in 8 bits (4.5 TB/s; a 4 GiB copy
// reaches 4.8), 152 us in 32 (4.9).  With 48 tensors to a launch 188 us (each launch's
// start and end); with workgroups of 2048, 4096 and 8192 elements 111, 117 and 123.
#include <hip/hip_runtime.h>

#include "ks_internal.h"

namespace ks {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
static_assert(kAdamChunk == 4 * kThreads, "a workgroup's elements, four per lane");

// the largest of a row of 16 lanes, in each of them
template <int CTRL>
__device__ __forceinline__ float row_max_step(float v) {
  const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false);
  return fmaxf(v, __builtin_bit_cast(float, o));
}
__device__ __forceinline__ float row_max(float v) {
  v = row_max_step<0x121>(v);   // row_ror:1, 2, 4, 8
  v = row_max_step<0x122>(v);
  v = row_max_step<0x124>(v);
  return row_max_step<0x128>(v);
}

__device__ __forceinline__ float pow2(uint32_t e) { return __builtin_bit_cast(float, e << 23); }   // 2^(e - 127)

// four values and the block's exponent byte as states of 8 bits.  V: e5m2 (the
// second moment), else e4m3.
template <bool V>
__device__ __forceinline__ uint32_t encode(const f32x4 &v, uint32_t &e) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(v[i]) < __builtin_inff() ? fabsf(v[i]) : 0.0f);
  top = row_max(top);
  constexpr int kLift = V ? 14 : 7;
  e = (uint32_t)max((int)(__builtin_bit_cast(uint32_t, top) >> 23) - kLift, 1);
  const float inv = pow2(254 - e);
  f32x4 q = v * inv;
  if constexpr (V) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = v[i] > 0.0f ? fmaxf(q[i], 0x1p-16f) : q[i];
  }
  uint32_t c;
  if constexpr (V) {
    c = __builtin_amdgcn_cvt_pk_bf8_f32(q[0], q[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_bf8_f32(q[2], q[3], c, true);
  } else {
    c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
  }
  // infinities and NaN, whatever the conversion makes of them
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (fabsf(v[i]) < __builtin_inff()) continue;
    const uint32_t code = V && v[i] == __builtin_inff() ? 0x7Cu : 0x7Fu;
    c = (c & ~(0xFFu << (8 * i))) | code << (8 * i);
  }
  return c;
}

template <bool V>
__device__ __forceinline__ f32x4 decode(uint32_t c, uint32_t e) {
  f32x2 lo, hi;
  if constexpr (V) {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8(c, false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8(c, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  }
  const float s = pow2(e);
  return f32x4{lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
}

__device__ __forceinline__ uint16_t bf16_of(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

template <bool EIGHT>
__global__ __launch_bounds__(kThreads) void k_adamw(AdamParams a) {
  int lo = 0, hi = a.n_tensors;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (blockIdx.x >= a.chunk_off[mid]) lo = mid;
    else hi = mid;
  }
  const AdamTensor &t = a.t[lo];
  float step_size = a.step_size, inv_sqrt = a.inv_sqrt;
  if (a.step_dev) {
    // 1 - beta^t without cancellation at small t
    const float n = (float)(*a.step_dev + 1u);
    step_size = a.lr / -expm1f(n * a.log_b1);
    inv_sqrt = 1.0f / sqrtf(-expm1f(n * a.log_b2));
  }
  const bool vec = t.flags & kAdamVec, g16 = t.flags & kAdamGrad16;
  const int64_t at = (int64_t)(blockIdx.x - a.chunk_off[lo]) * kAdamChunk + 4 * (int)threadIdx.x;
  if ((at & ~(int64_t)63) >= t.n) return;   // (the same for the 16 lanes of a block)
  const int left = (int)(t.n - at < 4 ? (t.n > at ? t.n - at : 0) : 4);
  f32x4 p = {0, 0, 0, 0}, g = p, m = p, v = p;
  uint32_t cm = 0, cv = 0;
  const bool quad = vec && left == 4;
  if (quad) {
    p = *(const f32x4 *)(t.p + at);
    if (g16) {
      const u32x2 h = *(const u32x2 *)((const uint16_t *)t.g + at);
      g = f32x4{__builtin_bit_cast(float, h[0] << 16), __builtin_bit_cast(float, h[0] & 0xFFFF0000u),
                __builtin_bit_cast(float, h[1] << 16), __builtin_bit_cast(float, h[1] & 0xFFFF0000u)};
    } else {
      g = *(const f32x4 *)((const float *)t.g + at);
    }
    if constexpr (EIGHT) {
      cm = *(const uint32_t *)((const uint8_t *)t.m + at);
      cv = *(const uint32_t *)((const uint8_t *)t.v + at);
    } else {
      m = *(const f32x4 *)((const float *)t.m + at);
      v = *(const f32x4 *)((const float *)t.v + at);
    }
  } else {
    for (int i = 0; i < left; ++i) {
      p[i] = t.p[at + i];
      g[i] = g16 ? __builtin_bit_cast(float, (uint32_t)((const uint16_t *)t.g)[at + i] << 16) : ((const float *)t.g)[at + i];
      if constexpr (EIGHT) {
        cm |= (uint32_t)((const uint8_t *)t.m)[at + i] << (8 * i);
        cv |= (uint32_t)((const uint8_t *)t.v)[at + i] << (8 * i);
      } else {
        m[i] = ((const float *)t.m)[at + i];
        v[i] = ((const float *)t.v)[at + i];
      }
    }
  }
  if constexpr (EIGHT) {
    m = decode<false>(cm, t.m_exp[at >> 6]);
    v = decode<true>(cv, t.v_exp[at >> 6]);
  }
  {
    // each product and sum rounded by itself: the 8-bit states then do not
    // depend on how the compiler fuses them
#pragma clang fp contract(off)
    g = g * a.grad_scale;
    m = m * a.b1 + g * a.c1;
    v = v * a.b2 + (g * a.c2) * g;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = p[i] * t.decay - step_size * (m[i] / (sqrtf(v[i]) * inv_sqrt + a.eps));
  uint32_t em, ev;
  if constexpr (EIGHT) {
    cm = encode<false>(m, em);
    cv = encode<true>(v, ev);
    if ((threadIdx.x & 15) == 0) {
      t.m_exp[at >> 6] = (uint8_t)em;
      t.v_exp[at >> 6] = (uint8_t)ev;
    }
  }
  if (quad) {
    *(f32x4 *)(t.p + at) = p;
    if constexpr (EIGHT) {
      *(uint32_t *)((uint8_t *)t.m + at) = cm;
      *(uint32_t *)((uint8_t *)t.v + at) = cv;
    } else {
      *(f32x4 *)((float *)t.m + at) = m;
      *(f32x4 *)((float *)t.v + at) = v;
    }
    if (t.copy)
      *(u32x2 *)(t.copy + at) = u32x2{bf16_of(p[0]) | (uint32_t)bf16_of(p[1]) << 16, bf16_of(p[2]) | (uint32_t)bf16_of(p[3]) << 16};
  } else {
    for (int i = 0; i < left; ++i) {
      t.p[at + i] = p[i];
      if constexpr (EIGHT) {
        ((uint8_t *)t.m)[at + i] = (uint8_t)(cm >> (8 * i));
        ((uint8_t *)t.v)[at + i] = (uint8_t)(cv >> (8 * i));
      } else {
        ((float *)t.m)[at + i] = m[i];
        ((float *)t.v)[at + i] = v[i];
      }
      if (t.copy) t.copy[at + i] = bf16_of(p[i]);
    }
  }
}

__global__ void k_adamw_count(uint32_t *step) { *step += 1u; }

}  // namespace

hipError_t launch_adamw(const AdamParams &p, bool eight, hipStream_t s) {
  const dim3 grid(p.chunk_off[p.n_tensors]), block(kThreads);
  if (grid.x == 0) return hipSuccess;
  if (eight) hipLaunchKernelGGL((k_adamw<true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((k_adamw<false>), grid, block, 0, s, p);
  return hipGetLastError();
}

hipError_t launch_adamw_count(uint32_t *step, hipStream_t s) {
  hipLaunchKernelGGL(k_adamw_count, dim3(1), dim3(1), 0, s, step);
  return hipGetLastError();
}

}  // namespace ks
