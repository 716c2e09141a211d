// Host stand-ins for the launches of the fitting entry points (see fake_device.cpp).
// TEST INFRASTRUCTURE ONLY.  Each writes what its kernel writes, so that an address
// outside a buffer or two regions over one another show up:
//   launch_gated_forward   adds 1 to each row's z, dz_out and loss sums
//   launch_gated_sums      a workgroup's sums: its number of rows, in every element;
//                          the loss's too
//   launch_gated_rows      adds 1 to each element of the rows' gradients
//   launch_gated_reduce    each gradient and loss: the sum of its family's workgroups
//   launch_adamw           adds 1 to every element of a tensor
//   launch_features        adds 1 to every element of the feature rows and rooflines
#include <hip/hip_runtime_api.h>

#include "ks_internal.h"

namespace ks {

namespace {

int family_of(const int32_t (&off)[KS_NFAM + 1], int wg) {
  int f = 0;
  while (wg >= off[f + 1]) ++f;
  return f;
}

// row(wg, i) for each row i of each workgroup
template <class F>
void each_row(const GatedParams &p, const int32_t (&off)[KS_NFAM + 1], int64_t rows, F &&row) {
  for (int wg = 0; wg < off[KS_NFAM]; ++wg) {
    const int f = family_of(off, wg);
    const int64_t begin = p.fam_off[f] + (wg - off[f]) * rows;
    for (int64_t i = begin; i < begin + rows && i < p.fam_off[f + 1]; ++i) row(wg, i);
  }
}

template <class T>
void add(void *p, int64_t i) { static_cast<T *>(p)[i] += T(1); }

}  // namespace

hipError_t launch_gated_forward(const GatedParams &p, hipStream_t) {
  if (p.loss_part)
    for (int wg = 0; wg < p.fwd_wg[KS_NFAM]; ++wg) p.loss_part[2 * wg] = p.loss_part[2 * wg + 1] = 0.0;
  each_row(p, p.fwd_wg, 64 * (int64_t)p.fwd_tiles, [&](int wg, int64_t i) {
    if (p.z) p.z[i] += 1.0f;
    if (p.dz_out) p.dz_out[i] = 1.0f;
    if (p.loss_part) p.loss_part[2 * wg] += 1.0, p.loss_part[2 * wg + 1] += 1.0;
  });
  return hipSuccess;
}

hipError_t launch_gated_sums(const GatedParams &p, bool loss, hipStream_t) {
  const int size = gated_part_size(p.hidden, p.in_dim);
  for (int wg = 0; wg < p.bwd_wg[KS_NFAM]; ++wg) {
    for (int e = 0; e < size; ++e) p.part[(size_t)wg * size + e] = 0.0f;
    if (loss) p.loss_part[2 * wg] = p.loss_part[2 * wg + 1] = 0.0;
  }
  each_row(p, p.bwd_wg, p.bwd_rows, [&](int wg, int64_t i) {
    const float dz = loss ? 1.0f : p.dz[i];
    if (loss && p.z) p.z[i] += 1.0f;
    if (loss) p.loss_part[2 * wg] += 1.0, p.loss_part[2 * wg + 1] += 1.0;
    p.part[(size_t)wg * size] += dz;
  });
  for (int wg = 0; wg < p.bwd_wg[KS_NFAM]; ++wg)
    for (int e = 1; e < size; ++e) p.part[(size_t)wg * size + e] = p.part[(size_t)wg * size];
  return hipSuccess;
}

hipError_t launch_gated_rows(const GatedParams &p, hipStream_t) {
  each_row(p, p.row_wg, p.row_rows, [&](int, int64_t i) {
    for (int d = 0; d < p.in_dim; ++d) {
      if (p.bf16) add<uint16_t>(p.g_x, i * p.g_ldx + d);
      else add<float>(p.g_x, i * p.g_ldx + d);
    }
  });
  return hipSuccess;
}

hipError_t launch_gated_reduce(const GatedParams &p, hipStream_t) {
  const int size = gated_part_size(p.hidden, p.in_dim);
  for (int f = 0; f < KS_NFAM; ++f) {
    if (p.eta) {
      double a = 0.0, b = 0.0;
      for (int wg = p.loss_wg[f]; wg < p.loss_wg[f + 1]; ++wg) a += p.loss_part[2 * wg], b += p.loss_part[2 * wg + 1];
      p.loss[f] = (float)(a + b);
    }
    if (!p.g_w1) continue;
    float first = 0.0f, last = 0.0f;
    for (int wg = p.bwd_wg[f]; wg < p.bwd_wg[f + 1]; ++wg) {
      first += p.part[(size_t)wg * size];
      last += p.part[(size_t)wg * size + size - 1];
    }
    for (int e = 0; e < p.hidden * p.in_dim; ++e) p.g_w1[f * p.hidden * p.in_dim + e] = p.g_w2[f * p.hidden * p.in_dim + e] = first;
    for (int e = 0; e < p.hidden; ++e) p.g_w3[f * p.hidden + e] = first;
    p.g_b3[f] = last;
  }
  return hipSuccess;
}

hipError_t launch_adamw(const AdamParams &p, bool eight, hipStream_t) {
  for (int i = 0; i < p.n_tensors; ++i) {
    const AdamTensor &t = p.t[i];
    for (uint32_t c = p.chunk_off[i]; c < p.chunk_off[i + 1]; ++c)
      for (int64_t e = (int64_t)(c - p.chunk_off[i]) * kAdamChunk; e < (int64_t)(c + 1 - p.chunk_off[i]) * kAdamChunk && e < t.n; ++e) {
        add<float>(t.p, e);
        if (eight) {
          add<uint8_t>(t.m, e), add<uint8_t>(t.v, e);
          if (e % 64 == 0) add<uint8_t>(t.m_exp, e / 64), add<uint8_t>(t.v_exp, e / 64);
        } else {
          add<float>(t.m, e), add<float>(t.v, e);
        }
        if (t.copy) add<uint16_t>(t.copy, e);
      }
  }
  return hipSuccess;
}

hipError_t launch_adamw_count(uint32_t *step, hipStream_t) {
  *step += 1;
  return hipSuccess;
}

hipError_t launch_features(const EvalParams &p, int in_dim, bool bf16, void *x, int64_t ldx, float *t_roof, hipStream_t) {
  const int64_t pairs = (int64_t)p.n_specs * p.fam_off[KS_NFAM];
  for (int64_t i = 0; i < pairs; ++i) {
    for (int d = 0; d < in_dim; ++d) {
      if (bf16) add<uint16_t>(x, i * ldx + d);
      else add<float>(x, i * ldx + d);
    }
    if (t_roof) t_roof[i] += 1.0f;
  }
  return hipSuccess;
}

}  // namespace ks
