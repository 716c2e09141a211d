// Host side of the fitting entry points (ks.h): gated heads over feature rows,
// the feature rows themselves and the AdamW step.  Argument checks, the split of
// the rows over workgroups and the launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <utility>
#include <vector>

#include "ks.h"
#include "ks_internal.h"

using ks::set_error;

namespace {

ks_status hip_error(hipError_t e, const char *what) {
  return e == hipSuccess ? KS_OK : set_error(KS_EHIP, "%s: %s", what, hipGetErrorString(e));
}

constexpr size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// sizes and offsets only
ks_status check_rows(const ks_heads *h, const ks_rows *r) {
  if (!r) return set_error(KS_EINVAL, "rows is NULL");
  if (r->n_rows < 0 || r->n_rows >= (int64_t(1) << 31))
    return set_error(KS_ERANGE, "rows.n_rows %lld outside [0, 2^31)", (long long)r->n_rows);
  if (r->fam_off[0] != 0) return set_error(KS_EINVAL, "rows.fam_off[0] must be 0");
  for (int f = 0; f < KS_NFAM; ++f)
    if (r->fam_off[f + 1] < r->fam_off[f]) return set_error(KS_EINVAL, "rows.fam_off decreases at family %d", f);
  if (r->fam_off[KS_NFAM] != r->n_rows)
    return set_error(KS_EINVAL, "rows.fam_off[KS_NFAM] = %lld != n_rows = %lld", (long long)r->fam_off[KS_NFAM],
                     (long long)r->n_rows);
  if (r->ldx < h->in_dim || r->ldx > (int64_t(1) << 20))
    return set_error(KS_EINVAL, "rows.ldx %lld outside in_dim %d .. 2^20", (long long)r->ldx, h->in_dim);
  return KS_OK;
}

// Rows over workgroups; the split depends on sizes alone, so results do not depend on
// the device.  Gradients: all workgroups resident at once, families' last ones
// included, so that each brings its weights once and none waits for another to end; two
// per CU, or one for the rows' and with fp32 heads of 32 inputs (with multiples of 128
// rows and remainders on top, 1,000,003 rows of fp32 32-256 took 427 us, so 363; 65,536
// rows 64, so 46).  Forward the same where the weights leave room for one workgroup per
// CU (fp32, 32 inputs, over 128 units: 163 us, so 154; 100,003 rows 31, so 23), else
// about 1024 (three or four per CU; three of fp32 16-256: 109 us, 113 with 768).
// The loss takes both passes in one launch up to about a workgroup per CU (and each
// family's last one): a launch, the weights' way to the registers and dz's way through
// memory are saved, but that kernel has two waves per SIMD, where the gradients alone
// have four except with fp32 heads of 32 inputs.  fp32 16-64, 4099 rows: 16 us in one
// launch, 19 in two; bf16 32-256, 32,000 rows 36 and 45, 100,000 rows 68 and 64,
// 500,000 rows 184 and 161; fp32 32-256, 500,000 rows 261 and 297, 2,000,003 rows
// 976 and 1000.
constexpr int32_t kOneLaunch = 256 + KS_NFAM;

// The least rows a workgroup takes, a multiple of unit and at least least, with which
// wgs workgroups (or one per family) are enough; off: their numbers.
int32_t split(const ks_rows *r, int64_t least, int64_t unit, int64_t wgs, int32_t (&off)[KS_NFAM + 1]) {
  int64_t rows = std::max(least, ((r->n_rows + wgs - 1) / wgs + unit - 1) / unit * unit);
  for (;; rows += unit) {
    off[0] = 0;
    for (int f = 0; f < KS_NFAM; ++f) off[f + 1] = off[f] + (int32_t)((r->fam_off[f + 1] - r->fam_off[f] + rows - 1) / rows);
    if (off[KS_NFAM] <= wgs) return (int32_t)rows;
  }
}

void plan(ks::GatedParams &p, const ks_heads *h, const ks_rows *r) {
  const bool wide = h->precision == KS_F32 && h->in_dim == 32;
  p.fwd_tiles = split(r, 256, 256, wide && h->hidden > 128 ? 256 : 1024, p.fwd_wg) / 64;   // 64 rows for each of four waves
  // 32 rows for each of its row groups, a step at least
  const int groups = (h->hidden + ks::kGatedGroup - 1) / ks::kGatedGroup, row_groups = groups > 4 ? 1 : groups > 2 ? 2 : 4;
  p.bwd_rows = split(r, ks::kGatedStep, 32 * row_groups, wide ? 256 : 512, p.bwd_wg);
  p.row_rows = split(r, 256, 256, 256, p.row_wg);   // 32 rows for each of its eight waves
}

// Workspace: the backward workgroups' sums, then (the loss) the sums of those that
// take the forward pass, and each row's dz.
struct Room {
  size_t loss, dz, total;
};
Room room_of(const ks::GatedParams &p) {
  Room o;
  o.loss = align256((size_t)p.bwd_wg[KS_NFAM] * ks::gated_part_size(p.hidden, p.in_dim) * sizeof(float));
  o.dz = o.loss + align256((size_t)std::max(p.fwd_wg[KS_NFAM], p.bwd_wg[KS_NFAM]) * 2 * sizeof(double));
  o.total = o.dz + align256((size_t)p.fam_off[KS_NFAM] * sizeof(float));
  return o;
}

void fill(ks::GatedParams &p, const ks_heads *h, const ks_rows *r) {
  std::memset(&p, 0, sizeof p);
  p.x = r->x;
  p.ldx = r->ldx;
  p.bf16 = h->precision == KS_BF16;
  const size_t e = p.bf16 ? 2 : 4;
  p.vec = aligned(r->x, 16) && (size_t)r->ldx * e % 16 == 0;
  for (int f = 0; f <= KS_NFAM; ++f) p.fam_off[f] = r->fam_off[f];
  p.in_dim = h->in_dim;
  p.hidden = h->hidden;
  p.w1 = h->w1;
  p.w2 = h->w2;
  p.w3 = h->w3;
  p.b3 = h->b3;
  plan(p, h, r);
}

ks_status check_all(const ks_heads *h, const ks_rows *r) {
  ks_status st = ks::check_gated(h);
  if (st != KS_OK) return st;
  st = check_rows(h, r);
  if (st != KS_OK) return st;
  if (r->n_rows > 0 && !r->x) return set_error(KS_EINVAL, "rows.x is NULL");
  if (!aligned(r->x, h->precision == KS_BF16 ? 2 : 4)) return set_error(KS_EINVAL, "rows.x is not aligned to its type");
  return KS_OK;
}

ks_status check_room(const ks::GatedParams &p, void *ws, size_t ws_bytes, Room *room) {
  *room = room_of(p);
  if (!ws) return set_error(KS_EWORKSPACE, "workspace is NULL");
  if (ws_bytes < room->total)
    return set_error(KS_EWORKSPACE, "workspace %zu bytes < %zu required", ws_bytes, room->total);
  if (!aligned(ws, 256)) return set_error(KS_EWORKSPACE, "workspace not 256-byte aligned");
  return KS_OK;
}

ks_status take_grad(ks::GatedParams &p, const ks_gated_grad *g) {
  const int n = (g->w1 != nullptr) + (g->w2 != nullptr) + (g->w3 != nullptr) + (g->b3 != nullptr);
  if (n != 0 && n != 4) return set_error(KS_EINVAL, "grad: some of w1, w2, w3, b3 are NULL and some not");
  if (!aligned(g->w1, 4) || !aligned(g->w2, 4) || !aligned(g->w3, 4) || !aligned(g->b3, 4))
    return set_error(KS_EINVAL, "grad: a pointer is not aligned to its type");
  p.g_w1 = g->w1;
  p.g_w2 = g->w2;
  p.g_w3 = g->w3;
  p.g_b3 = g->b3;
  return KS_OK;
}

// whether n rows of width bytes each lda bytes apart share any with n rows ldb apart
bool overlap(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t n, int64_t width) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  if (x >= y + (n - 1) * ldb + width || y >= x + (n - 1) * lda + width) return false;
  // columns of one buffer: apart in every period of the stride
  const uint64_t at = lda == ldb ? (x > y ? x - y : lda - (y - x) % lda) % lda : 0;
  return lda != ldb || at < (uint64_t)width || at + width > (uint64_t)lda;
}

}  // namespace

extern "C" {

ks_status ks_gated_forward(const ks_heads *heads, const ks_rows *rows, float *z, hipStream_t stream) {
  const ks_status st = check_all(heads, rows);
  if (st != KS_OK) return st;
  if (rows->n_rows == 0) return KS_OK;
  if (!z || !aligned(z, 4)) return set_error(KS_EINVAL, "z is NULL or not aligned to its type");
  ks::GatedParams p;
  fill(p, heads, rows);
  p.z = z;
  return hip_error(ks::launch_gated_forward(p, stream), "gated forward launch");
}

size_t ks_gated_workspace_bytes(const ks_heads *heads, const ks_rows *rows) {
  // (weights and rows need not be there yet)
  if (!heads || heads->mode != KS_ETA_GATED) return set_error(KS_EINVAL, "heads is NULL or not gated"), 0;
  if (heads->precision != KS_F32 && heads->precision != KS_BF16)
    return set_error(KS_EINVAL, "heads.precision %d unknown", heads->precision), 0;
  if (heads->hidden < 1 || heads->hidden > 256 || (heads->in_dim != 16 && heads->in_dim != 32))
    return set_error(KS_EINVAL, "heads.hidden %d or in_dim %d not supported", heads->hidden, heads->in_dim), 0;
  if (check_rows(heads, rows) != KS_OK) return 0;
  ks::GatedParams p;
  fill(p, heads, rows);
  const size_t n = room_of(p).total;
  return n ? n : 256;
}

ks_status ks_gated_backward(const ks_heads *heads, const ks_rows *rows, const float *dz, const ks_gated_grad *grad,
                            void *ws, size_t ws_bytes, hipStream_t stream) {
  ks_status st = check_all(heads, rows);
  if (st != KS_OK) return st;
  if (!grad) return set_error(KS_EINVAL, "grad is NULL");
  if (rows->n_rows > 0 && (!dz || !aligned(dz, 4))) return set_error(KS_EINVAL, "dz is NULL or not aligned to its type");
  ks::GatedParams p;
  fill(p, heads, rows);
  st = take_grad(p, grad);
  if (st != KS_OK) return st;
  Room room;
  st = check_room(p, ws, ws_bytes, &room);
  if (st != KS_OK) return st;
  if (grad->x) {
    const int64_t e = p.bf16 ? 2 : 4;
    if (grad->ldx < heads->in_dim || grad->ldx > (int64_t(1) << 20))
      return set_error(KS_EINVAL, "grad.ldx %lld outside in_dim %d .. 2^20", (long long)grad->ldx, heads->in_dim);
    if (!aligned(grad->x, e)) return set_error(KS_EINVAL, "grad.x is not aligned to its type");
    if (rows->n_rows > 0 && overlap(grad->x, grad->ldx * e, rows->x, rows->ldx * e, rows->n_rows, heads->in_dim * e))
      return set_error(KS_EINVAL, "grad.x overlaps rows.x");
    p.g_x = grad->x;
    p.g_ldx = grad->ldx;
    p.g_vec = aligned(grad->x, 4 * e) && grad->ldx % 4 == 0;
  }
  p.dz = dz;
  p.part = static_cast<float *>(ws);
  if (p.g_w1) {
    hipError_t e = ks::launch_gated_sums(p, false, stream);
    if (e == hipSuccess) e = ks::launch_gated_reduce(p, stream);
    if (e != hipSuccess) return hip_error(e, "gated backward launch");
  }
  if (p.g_x) return hip_error(ks::launch_gated_rows(p, stream), "gated rows' gradient launch");
  return KS_OK;
}

ks_status ks_gated_loss(const ks_heads *heads, const ks_rows *rows, const ks_eta_target *target, float *loss, float *z,
                        const ks_gated_grad *grad, void *ws, size_t ws_bytes, hipStream_t stream) {
  ks_status st = check_all(heads, rows);
  if (st != KS_OK) return st;
  if (!target) return set_error(KS_EINVAL, "target is NULL");
  if (rows->n_rows > 0 && !target->eta) return set_error(KS_EINVAL, "target.eta is NULL");
  if (!(target->huber > 0.0)) return set_error(KS_EINVAL, "target.huber %g not above 0", target->huber);
  if (!loss) return set_error(KS_EINVAL, "loss is NULL");
  if (!aligned(target->eta, 4) || !aligned(target->weight, 4) || !aligned(loss, 4) || !aligned(z, 4))
    return set_error(KS_EINVAL, "a pointer is not aligned to its type");
  ks::GatedParams p;
  fill(p, heads, rows);
  if (grad) {
    if (grad->x) return set_error(KS_EINVAL, "grad.x: the loss has no gradient for the rows");
    st = take_grad(p, grad);
    if (st != KS_OK) return st;
  }
  Room room;
  st = check_room(p, ws, ws_bytes, &room);
  if (st != KS_OK) return st;
  char *w = static_cast<char *>(ws);
  p.z = z;
  // (any non-null value without rows: the reduce kernel goes by it)
  p.eta = rows->n_rows > 0 ? target->eta : loss;
  p.weight = target->weight;
  p.huber = (float)target->huber;
  if (!(p.huber > 0.0f)) return set_error(KS_EINVAL, "target.huber %g not above 0 in fp32", target->huber);
  p.loss = loss;
  p.loss_part = reinterpret_cast<double *>(w + room.loss);
  p.part = reinterpret_cast<float *>(w);
  const bool one = p.g_w1 && p.bwd_wg[KS_NFAM] <= kOneLaunch;
  std::memcpy(p.loss_wg, one ? p.bwd_wg : p.fwd_wg, sizeof p.loss_wg);
  if (p.g_w1 && !one) p.dz_out = reinterpret_cast<float *>(w + room.dz);
  p.dz = p.dz_out;
  hipError_t e = one ? hipSuccess : ks::launch_gated_forward(p, stream);
  if (e == hipSuccess && p.g_w1) e = ks::launch_gated_sums(p, one, stream);
  if (e == hipSuccess) e = ks::launch_gated_reduce(p, stream);
  return hip_error(e, "gated loss launch");
}

ks_status ks_features(const ks_desc *desc, const ks_spec *specs, int32_t n_specs, int32_t in_dim, int32_t precision,
                      void *x, int64_t ldx, float *t_roof, void *ws, size_t ws_bytes, hipStream_t stream) {
  if (in_dim != 16 && in_dim != 32) return set_error(KS_EINVAL, "in_dim %d not 16 or 32", in_dim);
  if (precision != KS_F32 && precision != KS_BF16) return set_error(KS_EINVAL, "precision %d unknown", precision);
  if (ldx < in_dim || ldx > (int64_t(1) << 31))
    return set_error(KS_EINVAL, "ldx %lld outside in_dim %d .. 2^31", (long long)ldx, in_dim);
  if (!desc) return set_error(KS_EINVAL, "desc is NULL");
  if (desc->n_rows > 0 && (!x || !aligned(x, precision == KS_BF16 ? 2 : 4)))
    return set_error(KS_EINVAL, "x is NULL or not aligned to its type");
  if (!aligned(t_roof, 4)) return set_error(KS_EINVAL, "t_roof is not aligned to its type");
  if (n_specs > 0 && desc->n_rows >= ((int64_t(1) << 31) + n_specs - 1) / n_specs)
    return set_error(KS_ERANGE, "%lld records for %d specs: 2^31 or more rows", (long long)desc->n_rows, n_specs);
  ks::EvalParams p;
  const ks_status st = ks::feature_prologue(desc, specs, n_specs, ws, ws_bytes, &p, stream);
  if (st != KS_OK) return st;
  return hip_error(ks::launch_features(p, in_dim, precision == KS_BF16, x, ldx, t_roof, stream), "feature rows launch");
}

ks_status ks_adamw(const ks_adamw_config *c, const ks_tensor *tensors, int32_t n_tensors, hipStream_t stream) {
  if (!c) return set_error(KS_EINVAL, "config is NULL");
  if (n_tensors < 0) return set_error(KS_EINVAL, "n_tensors %d below 0", n_tensors);
  if (n_tensors > 0 && !tensors) return set_error(KS_EINVAL, "tensors is NULL");
  if (c->state_bits != 8 && c->state_bits != 32) return set_error(KS_EINVAL, "state_bits %d not 8 or 32", c->state_bits);
  if (!std::isfinite((float)c->lr) || c->lr < 0.0) return set_error(KS_EINVAL, "lr %g not finite and 0 or more", c->lr);
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0))
    return set_error(KS_EINVAL, "beta1 %g or beta2 %g outside [0, 1)", c->beta1, c->beta2);
  if (!((float)c->eps > 0.0f) || !std::isfinite((float)c->eps)) return set_error(KS_EINVAL, "eps %g not above 0", c->eps);
  if (!std::isfinite((float)c->grad_scale)) return set_error(KS_EINVAL, "grad_scale %g not finite", c->grad_scale);
  if (!c->step_dev && c->step < 1) return set_error(KS_EINVAL, "step %lld below 1", (long long)c->step);
  if (!aligned(c->step_dev, 4)) return set_error(KS_EINVAL, "step_dev is not aligned to its type");
  const bool eight = c->state_bits == 8;
  for (int i = 0; i < n_tensors; ++i) {
    const ks_tensor &t = tensors[i];
    if (t.n < 0 || t.n > (int64_t(1) << 33)) return set_error(KS_ERANGE, "tensor %d: n %lld outside 0..2^33", i, (long long)t.n);
    if (t.grad_type != KS_F32 && t.grad_type != KS_BF16) return set_error(KS_EINVAL, "tensor %d: grad_type %d unknown", i, t.grad_type);
    if (!std::isfinite((float)(1.0 - c->lr * (double)t.weight_decay)))
      return set_error(KS_EINVAL, "tensor %d: weight_decay %g not finite, or too large for lr", i, t.weight_decay);
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v) return set_error(KS_EINVAL, "tensor %d: a pointer is NULL", i);
    if (eight ? !t.m_exp || !t.v_exp : t.m_exp || t.v_exp)
      return set_error(KS_EINVAL, "tensor %d: m_exp and v_exp go with states of 8 bits, and only with them", i);
    if (!aligned(t.param, 4) || !aligned(t.grad, t.grad_type == KS_F32 ? 4 : 2) || !aligned(t.copy, 2) ||
        (!eight && (!aligned(t.m, 4) || !aligned(t.v, 4))))
      return set_error(KS_EINVAL, "tensor %d: a pointer is not aligned to its type", i);
  }
  try {
    std::vector<std::pair<uintptr_t, uintptr_t>> at;   // [begin, end)
    at.reserve(n_tensors);
    for (int i = 0; i < n_tensors; ++i)
      if (tensors[i].n > 0) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(tensors[i].param);
        at.emplace_back(p, p + (uintptr_t)tensors[i].n * sizeof(float));
      }
    std::sort(at.begin(), at.end());
    for (size_t i = 1; i < at.size(); ++i)
      if (at[i].first < at[i - 1].second) return set_error(KS_EINVAL, "two tensors share elements of a param");
  } catch (...) {
    return set_error(KS_EINVAL, "no host memory for %d tensors", n_tensors);
  }

  ks::AdamParams p;
  std::memset(&p, 0, sizeof p);
  p.b1 = (float)c->beta1;
  p.c1 = (float)(1.0 - c->beta1);
  p.b2 = (float)c->beta2;
  p.c2 = (float)(1.0 - c->beta2);
  p.eps = (float)c->eps;
  p.grad_scale = (float)c->grad_scale;
  p.lr = (float)c->lr;
  p.step_dev = c->step_dev;
  if (c->step_dev) {
    p.log_b1 = (float)std::log(c->beta1);   // -infinity for 0: beta^t = 0
    p.log_b2 = (float)std::log(c->beta2);
  } else {
    p.step_size = (float)(c->lr / (1.0 - std::pow(c->beta1, (double)c->step)));
    p.inv_sqrt = (float)(1.0 / std::sqrt(1.0 - std::pow(c->beta2, (double)c->step)));
  }
  int64_t chunks = 0;
  auto flush = [&]() {
    p.chunk_off[p.n_tensors] = (uint32_t)chunks;
    const hipError_t e = p.n_tensors ? ks::launch_adamw(p, eight, stream) : hipSuccess;
    p.n_tensors = 0;
    chunks = 0;
    return e;
  };
  for (int i = 0; i < n_tensors; ++i) {
    const ks_tensor &t = tensors[i];
    const int64_t n = (t.n + ks::kAdamChunk - 1) / ks::kAdamChunk;
    if (n == 0) continue;
    if (p.n_tensors == ks::kAdamTensors || chunks + n > (int64_t(1) << 23)) {
      const hipError_t e = flush();
      if (e != hipSuccess) return hip_error(e, "AdamW launch");
    }
    ks::AdamTensor &o = p.t[p.n_tensors];
    o.p = t.param;
    o.g = t.grad;
    o.m = t.m;
    o.v = t.v;
    o.m_exp = t.m_exp;
    o.v_exp = t.v_exp;
    o.copy = t.copy;
    o.n = t.n;
    o.decay = (float)(1.0 - c->lr * (double)t.weight_decay);
    const bool g16 = t.grad_type == KS_BF16;
    const bool vec = aligned(t.param, 16) && aligned(t.grad, g16 ? 8 : 16) && aligned(t.m, eight ? 4 : 16) &&
                     aligned(t.v, eight ? 4 : 16) && aligned(t.copy, 8);
    o.flags = (vec ? ks::kAdamVec : 0u) | (g16 ? ks::kAdamGrad16 : 0u);
    p.chunk_off[p.n_tensors++] = (uint32_t)chunks;
    chunks += n;
  }
  hipError_t e = flush();
  if (e == hipSuccess && c->step_dev) e = ks::launch_adamw_count(c->step_dev, stream);
  return hip_error(e, "AdamW launch");
}

}  // extern "C"
