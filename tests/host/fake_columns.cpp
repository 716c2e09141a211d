// Host stand-ins for the launches of the learned columns' entry points (see
// fake_device.cpp).  TEST INFRASTRUCTURE ONLY.  Each reads and writes what its kernels
// read and write, so that an address outside a buffer or two regions over one another show
// up:
//   launch_embed        adds 1 to every element of dst, reads every element of the row of src
//   launch_embed_back   goes through the places and columns as the workgroups do, leaves every
//                       part's sums, and writes each element of the gradient: how often its
//                       id's rows were taken (from the parts), or 0 (an id without rows)
//   launch_order        the order; every count, total and key between the passes
//   launch_eta_loss     each row's dz: 1, each family's loss: its rows, through the
//                       workgroups' sums
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <numeric>
#include <vector>

#include "ks_columns.h"

namespace ks {

namespace {

uint32_t columns(const Cols &c, uint32_t width, uint32_t block) {
  return c.rem && block + 1 == c.blocks ? c.rem : width;
}

volatile float seen;
void read(const void *p, int64_t i, bool b16) {
  seen = b16 ? (float)static_cast<const uint16_t *>(p)[i] : static_cast<const float *>(p)[i];
}

}  // namespace

hipError_t launch_embed(const EmbedParams &p, bool src16, bool dst16, hipStream_t) {
  for (int64_t i = 0; i < p.n_rows; ++i) {
    const int64_t id = p.ids ? (int64_t)p.ids[i] : i;
    for (uint32_t b = 0; b < p.cols.blocks; ++b)
      for (uint32_t j = 0; j < columns(p.cols, 8, b); ++j) {
        if (!p.ids || id < p.n_ids) read(p.src, id * p.src_ld + 8 * b + j, src16);
        const int64_t at = i * p.dst_ld + 8 * b + j;
        if (dst16) static_cast<uint16_t *>(p.dst)[at] += 1;
        else static_cast<float *>(p.dst)[at] += 1.0f;
      }
  }
  return hipSuccess;
}

hipError_t launch_embed_back(const EmbedBackParams &p, bool dy16, hipStream_t) {
  const uint32_t n = std::min<uint32_t>(p.off[p.n_ids], (uint32_t)p.n_rows), groups = kBackThreads / p.wide;
  const size_t slot = (size_t)p.cols.blocks * 8;
  if (p.each * groups != p.run) return hipErrorInvalidValue;
  for (int64_t i = 0; i < 2 * (int64_t)p.runs * (int64_t)slot; ++i) p.part[i] = 0.0f;
  std::vector<uint32_t> taken(p.n_ids, 0);
  for (uint32_t part = 0; part < p.runs; ++part)
    for (uint32_t g = 0; g < groups; ++g) {
      const uint32_t p0 = std::min(part * p.run + g * p.each, n), p1 = std::min(p0 + p.each, n);
      for (uint32_t q = p0; q < p1; ++q) {
        ++taken[p.id[q]];
        for (uint32_t b = 0; b < p.cols.blocks; ++b)
          for (uint32_t j = 0; j < columns(p.cols, 8, b); ++j) read(p.dy, (int64_t)p.row[q] * p.ld + 8 * b + j, dy16);
      }
    }
  if ((uint64_t)p.tiles * p.wide < p.cols.blocks) return hipErrorInvalidValue;
  const int64_t quads = p.fill_wgs * kBackThreads * kBackFill;
  if (quads < (int64_t)p.n_ids * p.quads.blocks) return hipErrorInvalidValue;
  for (int64_t v = 0; v < p.n_ids; ++v)
    for (uint32_t q = 0; q < p.quads.blocks; ++q)
      for (uint32_t j = 0; j < columns(p.quads, 4, q); ++j) p.grad[v * p.grad_ld + 4 * q + j] = (float)taken[v];
  return hipSuccess;
}

hipError_t launch_order(const OrderParams &p, hipStream_t) {
  if (p.n_rows && (uint64_t)p.chunk * p.chunks < p.n_rows) return hipErrorInvalidValue;
  if ((uint64_t(1) << std::min(p.bits * p.passes, 63)) <= p.n_ids) return hipErrorInvalidValue;
  for (size_t i = 0; i < (size_t)p.chunks << p.bits; ++i) p.hist[i] = 0;
  for (size_t i = 0; i < size_t(1) << p.bits; ++i) p.total[i] = 0;
  std::vector<uint32_t> row(p.n_rows);
  std::iota(row.begin(), row.end(), 0u);
  auto key = [&](uint32_t i) { return std::min(p.ids[i], p.n_ids); };
  std::stable_sort(row.begin(), row.end(), [&](uint32_t a, uint32_t b) { return key(a) < key(b); });
  for (uint32_t i = 0; i < p.n_rows; ++i) {
    if (p.passes > 1) p.tmp_id[i] = p.tmp_row[i] = 0;
    p.row[i] = row[i];
    p.id[i] = key(row[i]);
  }
  uint32_t at = 0;
  for (uint32_t v = 0; v <= p.n_ids; ++v) {
    while (at < p.n_rows && p.id[at] < v) ++at;
    p.off[v] = at;
  }
  return hipSuccess;
}

hipError_t launch_eta_loss(const EtaParams &p, hipStream_t) {
  auto rows = [&](int64_t begin, int64_t end) {
    for (int64_t i = begin; i < end; ++i) {
      seen = p.z[i] + p.eta[i] + (p.weight ? p.weight[i] : 0.0f);
      p.dz[i] = 1.0f;
    }
    return (double)(end - begin);
  };
  for (int f = 0; f < KS_NFAM; ++f) {
    double sum = 0.0;
    if (p.wg[KS_NFAM] == 0) sum = rows(p.fam_off[f], p.fam_off[f + 1]);
    for (int wg = p.wg[f]; wg < p.wg[f + 1]; ++wg) {
      const int64_t begin = p.fam_off[f] + (wg - p.wg[f]) * p.rows;
      p.part[2 * wg] = rows(begin, std::min(begin + p.rows, p.fam_off[f + 1]));
      p.part[2 * wg + 1] = 0.0;
      sum += p.part[2 * wg];
    }
    p.loss[f] = (float)sum;
  }
  return hipSuccess;
}

}  // namespace ks
