// Host side of the learned columns' entry points (ks.h): lookup, dropout, the order of
// ids, the table's gradient and the loss at given z.  Argument checks, the split of the
// work over workgroups and the launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "ks.h"
#include "ks_columns.h"

using ks::set_error;

namespace {

ks_status hip_error(hipError_t e, const char *what) {
  return e == hipSuccess ? KS_OK : set_error(KS_EHIP, "%s: %s", what, hipGetErrorString(e));
}

constexpr size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

int64_t size_of(int32_t type) { return type == KS_BF16 ? 2 : 4; }

// sizes and type only
ks_status check_sizes(const ks_matrix *m, const char *name) {
  if (!m) return set_error(KS_EINVAL, "%s is NULL", name);
  if (m->type != KS_F32 && m->type != KS_BF16) return set_error(KS_EINVAL, "%s.type %d unknown", name, m->type);
  if (m->n_rows < 0 || m->n_rows >= (int64_t(1) << 31))
    return set_error(KS_ERANGE, "%s.n_rows %lld outside [0, 2^31)", name, (long long)m->n_rows);
  if (m->n_cols < 1 || m->n_cols > (int64_t(1) << 20))
    return set_error(KS_ERANGE, "%s.n_cols %lld outside 1 .. 2^20", name, (long long)m->n_cols);
  if (m->ld < m->n_cols || m->ld > (int64_t(1) << 20))
    return set_error(KS_EINVAL, "%s.ld %lld outside n_cols %lld .. 2^20", name, (long long)m->ld, (long long)m->n_cols);
  return KS_OK;
}

ks_status check_matrix(const ks_matrix *m, const char *name) {
  const ks_status st = check_sizes(m, name);
  if (st != KS_OK) return st;
  if (m->n_rows > 0 && !m->p) return set_error(KS_EINVAL, "%s.p is NULL", name);
  if (!aligned(m->p, size_of(m->type))) return set_error(KS_EINVAL, "%s.p is not aligned to its type", name);
  return KS_OK;
}

// an address range [p, p + bytes)
struct Span {
  uintptr_t begin, end;
  Span(const void *p, int64_t bytes) : begin(reinterpret_cast<uintptr_t>(p)), end(begin + (uintptr_t)bytes) {}
  explicit Span(const ks_matrix *m)
      : Span(m->p, m->n_rows > 0 ? ((m->n_rows - 1) * m->ld + m->n_cols) * size_of(m->type) : 0) {}
  bool meets(const Span &o) const { return begin < end && o.begin < o.end && begin < o.end && o.begin < end; }
};

// whether two matrices share an element: rows of one stride may be columns of one buffer
bool overlap(const ks_matrix *a, const ks_matrix *b) {
  const Span x(a), y(b);
  if (!x.meets(y)) return false;
  const int64_t s = a->ld * size_of(a->type);
  if (s != b->ld * size_of(b->type)) return true;
  // b's first column behind a's, in a period of the stride
  const int64_t at = (int64_t)(y.begin >= x.begin ? (y.begin - x.begin) % (uintptr_t)s
                                                  : ((uintptr_t)s - (x.begin - y.begin) % (uintptr_t)s) % (uintptr_t)s);
  return at < a->n_cols * size_of(a->type) || at + b->n_cols * size_of(b->type) > s;
}

ks_status check_drop(const ks_drop *d) {
  if (!d) return KS_OK;
  if (!(d->p >= 0.0 && d->p <= 1.0)) return set_error(KS_EINVAL, "drop.p %g outside 0 .. 1", d->p);
  if (!aligned(d->step_dev, 4)) return set_error(KS_EINVAL, "drop.step_dev is not aligned to its type");
  return KS_OK;
}

// the kernels' form, and what stays is multiplied by
ks::Drop drop_of(const ks_drop *d, double *up) {
  ks::Drop o;
  std::memset(&o, 0, sizeof o);
  *up = 1.0;
  if (!d) return o;
  o.least = (uint32_t)std::floor(d->p * 65536.0 + 0.5);
  o.key0 = (uint32_t)d->seed;
  o.key1 = (uint32_t)(d->seed >> 32);
  o.site = d->site;
  o.step = d->step;
  o.step_dev = d->step_dev;
  // (all dropped: no draw stays, whatever the factor)
  if (o.least < 65536u) *up = 65536.0 / (65536.0 - o.least);
  return o;
}

ks::Cols cols_of(int64_t n, int64_t width = 8) {
  ks::Cols c;
  c.blocks = (uint32_t)((n + width - 1) / width);
  c.rem = (uint32_t)(n % width);
  c.magic = c.blocks > 1 ? (uint32_t)(((uint64_t(1) << 32) + c.blocks - 1) / c.blocks) : 0;
  return c;
}

ks_status check_scale(double scale) {
  return std::isfinite((float)scale) ? KS_OK : set_error(KS_EINVAL, "scale %g not finite", scale);
}

ks_status check_room(void *ws, size_t have, size_t need) {
  if (!ws) return set_error(KS_EWORKSPACE, "workspace is NULL");
  if (have < need) return set_error(KS_EWORKSPACE, "workspace %zu bytes < %zu required", have, need);
  if (!aligned(ws, 256)) return set_error(KS_EWORKSPACE, "workspace not 256-byte aligned");
  return KS_OK;
}

ks_status check_order_sizes(const ks_id_order *o) {
  if (!o) return set_error(KS_EINVAL, "order is NULL");
  if (o->n_rows < 0 || o->n_rows >= (int64_t(1) << 31))
    return set_error(KS_ERANGE, "order.n_rows %lld outside [0, 2^31)", (long long)o->n_rows);
  if (o->n_ids < 1 || o->n_ids >= (int64_t(1) << 31))
    return set_error(KS_ERANGE, "order.n_ids %lld outside [1, 2^31)", (long long)o->n_ids);
  return KS_OK;
}

ks_status check_order(const ks_id_order *o) {
  const ks_status st = check_order_sizes(o);
  if (st != KS_OK) return st;
  if (!o->off || (o->n_rows > 0 && (!o->row || !o->id))) return set_error(KS_EINVAL, "order: a pointer is NULL");
  if (!aligned(o->row, 4) || !aligned(o->id, 4) || !aligned(o->off, 4))
    return set_error(KS_EINVAL, "order: a pointer is not aligned to its type");
  return KS_OK;
}

// Chunks of the keys: at most 512, so that the counts of a digit stay short, while that is
// no more than 2^20 keys in each
void plan(ks::OrderParams &p, const ks_id_order *o) {
  std::memset(&p, 0, sizeof p);
  p.n_rows = (uint32_t)o->n_rows;
  p.n_ids = (uint32_t)o->n_ids;
  int bits = 0;
  while (bits < 32 && (uint64_t)o->n_ids >> bits) ++bits;   // (n_ids is a key too)
  p.passes = (bits + ks::kOrderBits - 1) / ks::kOrderBits;
  p.bits = std::max(ks::kOrderFew, (bits + p.passes - 1) / p.passes);
  const int64_t most = int64_t(512) * ks::kOrderKeys;
  p.chunk = (uint32_t)(ks::kOrderKeys * std::min<int64_t>(512, std::max<int64_t>(1, (o->n_rows + most - 1) / most)));
  p.chunks = (uint32_t)((o->n_rows + p.chunk - 1) / p.chunk);
}

struct OrderRoom {
  size_t total, id, row, end;
};
OrderRoom room_of(const ks::OrderParams &p) {
  OrderRoom r;
  r.total = align256(((size_t)p.chunks << p.bits) * sizeof(uint32_t));
  r.id = r.total + align256((sizeof(uint32_t)) << p.bits);
  const size_t keys = p.passes > 1 ? align256((size_t)p.n_rows * sizeof(uint32_t)) : 0;
  r.row = r.id + keys;
  r.end = r.row + keys;
  return r;
}

// Four places of the order for each group of lanes, more where that is over `most` places,
// 4096 at most (64 runs of 64 additions).  Few places are a short way through a small call
// (4099 rows of 16 columns: 11 us with 4, 13 with 8, 19 with 16).  More workgroups leave
// more sums of ids that go on for the join, wide ones above all; fewer do not fill the card:
// with 512, 1024, 2048 workgroups 16,381 rows of 2048 bf16 columns 67, 72, 75 us (of 1024 44,
// 46, 50), 300,007 of 256 38, 36, 40, of 67 28, 27, 27, 2,000,003 of 16 fp32 57, 52, 49.
// Up to twelve places where they make one workgroup, and no join: 1000 rows of 16 columns
// 8 us, 10 with the join; 1400 9 and 10; with sixteen places 2000 rows 12 and 10.
void plan(ks::EmbedBackParams &p, const ks_id_order *o, int64_t n_cols) {
  std::memset(&p, 0, sizeof p);
  p.n_rows = o->n_rows;
  p.n_ids = (uint32_t)o->n_ids;
  p.cols = cols_of(n_cols);
  p.quads = cols_of(n_cols, 4);
  p.wide = std::min<uint32_t>(p.cols.blocks, ks::kBackThreads);
  p.tiles = (p.cols.blocks + p.wide - 1) / p.wide;
  const int64_t fill = ks::kBackThreads * ks::kBackFill, groups = ks::kBackThreads / p.wide;
  const int64_t most = (p.wide > 64 ? 512 : p.wide > 4 ? 1024 : 2048) * 4 * groups;
  p.fill_wgs = (o->n_ids * (int64_t)p.quads.blocks + fill - 1) / fill;
  p.each = (uint32_t)std::min<int64_t>(4 * std::max<int64_t>(1, (o->n_rows * p.tiles + most - 1) / most), 4096);
  if (o->n_rows <= 12 * groups) p.each = std::max<uint32_t>((uint32_t)((o->n_rows + groups - 1) / groups), 4);
  p.run = p.each * (uint32_t)groups;
  p.runs = (uint32_t)((o->n_rows + p.run - 1) / p.run);
}

// Nontemporal stores for the zeros of a gradient that the caches do not keep for its reader
// anyway.  With an AdamW step that reads the gradient, 262 MB on the 16-byte grid 397 us, with
// ordinary stores 406 (16,381 rows of 2048 bf16 columns by themselves 72 and 85); but
// 51 MB 74 and 73, 8 MB 29 and 28, and off the grid zeros for 1,000,000 x 67 61 and 58.
constexpr int64_t kPast = int64_t(1) << 27;
bool past_caches(const ks_matrix *grad) {
  return grad->n_rows * grad->n_cols * (int64_t)sizeof(float) > kPast && (uintptr_t)grad->p % 16 == 0 && grad->ld % 4 == 0;
}

size_t part_bytes(const ks::EmbedBackParams &p) {
  return align256((size_t)p.runs * 2 * p.cols.blocks * 8 * sizeof(float));
}

ks_status check_offsets(const int64_t *off) {
  if (!off) return set_error(KS_EINVAL, "fam_off is NULL");
  if (off[0] != 0) return set_error(KS_EINVAL, "fam_off[0] must be 0");
  for (int f = 0; f < KS_NFAM; ++f)
    if (off[f + 1] < off[f]) return set_error(KS_EINVAL, "fam_off decreases at family %d", f);
  if (off[KS_NFAM] >= (int64_t(1) << 31))
    return set_error(KS_ERANGE, "fam_off[KS_NFAM] = %lld: 2^31 or more rows", (long long)off[KS_NFAM]);
  return KS_OK;
}

void plan(ks::EtaParams &p, const int64_t *off) {
  std::memset(&p, 0, sizeof p);
  std::copy(off, off + KS_NFAM + 1, p.fam_off);
  int64_t most = 0;
  for (int f = 0; f < KS_NFAM; ++f) most = std::max(most, off[f + 1] - off[f]);
  if (most <= 8 * ks::kEtaWide) return;
  p.rows = std::max<int64_t>(1024, (off[KS_NFAM] + 1023) / 1024);
  for (int f = 0; f < KS_NFAM; ++f) p.wg[f + 1] = p.wg[f] + (int32_t)((off[f + 1] - off[f] + p.rows - 1) / p.rows);
}
size_t eta_bytes(const ks::EtaParams &p) { return align256((size_t)std::max(p.wg[KS_NFAM], 1) * 2 * sizeof(double)); }

}  // namespace

extern "C" {

ks_status ks_dropout(const ks_drop *drop, const ks_matrix *x, const ks_matrix *y, hipStream_t stream) {
  if (!drop) return set_error(KS_EINVAL, "drop is NULL");
  ks_status st = check_drop(drop);
  if (st == KS_OK) st = check_matrix(x, "x");
  if (st == KS_OK) st = check_matrix(y, "y");
  if (st != KS_OK) return st;
  if (x->n_rows != y->n_rows || x->n_cols != y->n_cols || x->type != y->type)
    return set_error(KS_EINVAL, "x and y are not of one shape and type");
  if (x->n_rows == 0) return KS_OK;
  if ((x->p != y->p || x->ld != y->ld) && overlap(x, y)) return set_error(KS_EINVAL, "y overlaps x and is not x itself");
  if (Span(y).meets(Span(drop->step_dev, drop->step_dev ? 4 : 0))) return set_error(KS_EINVAL, "y overlaps drop.step_dev");
  ks::EmbedParams p;
  std::memset(&p, 0, sizeof p);
  double up;
  p.drop = drop_of(drop, &up);
  p.src = x->p;
  p.dst = y->p;
  p.src_ld = x->ld;
  p.dst_ld = y->ld;
  p.n_rows = y->n_rows;
  p.n_ids = 1;
  p.factor = (float)up;
  p.cols = cols_of(y->n_cols);
  return hip_error(ks::launch_embed(p, x->type == KS_BF16, y->type == KS_BF16, stream), "dropout launch");
}

ks_status ks_embed(const ks_matrix *table, double scale, const uint32_t *ids, const ks_drop *drop, const ks_matrix *y,
                   hipStream_t stream) {
  ks_status st = check_matrix(table, "table");
  if (st == KS_OK) st = check_matrix(y, "y");
  if (st == KS_OK) st = check_scale(scale);
  if (st == KS_OK) st = check_drop(drop);
  if (st != KS_OK) return st;
  if (table->n_cols != y->n_cols)
    return set_error(KS_EINVAL, "table has %lld columns, y %lld", (long long)table->n_cols, (long long)y->n_cols);
  if (y->n_rows == 0) return KS_OK;
  if (!ids || !aligned(ids, 4)) return set_error(KS_EINVAL, "ids is NULL or not aligned to its type");
  const Span to(y);
  if (overlap(table, y)) return set_error(KS_EINVAL, "y overlaps table");
  if (to.meets(Span(ids, y->n_rows * 4)) || (drop && to.meets(Span(drop->step_dev, drop->step_dev ? 4 : 0))))
    return set_error(KS_EINVAL, "y overlaps ids or drop.step_dev");
  ks::EmbedParams p;
  std::memset(&p, 0, sizeof p);
  double up;
  p.drop = drop_of(drop, &up);
  p.src = table->p;
  p.dst = y->p;
  p.src_ld = table->ld;
  p.dst_ld = y->ld;
  p.n_rows = y->n_rows;
  p.ids = ids;
  p.n_ids = (uint32_t)table->n_rows;
  p.factor = (float)(scale * up);
  if (!std::isfinite(p.factor)) return set_error(KS_EINVAL, "scale %g / (1 - p) not finite in fp32", scale);
  p.cols = cols_of(y->n_cols);
  return hip_error(ks::launch_embed(p, table->type == KS_BF16, y->type == KS_BF16, stream), "lookup launch");
}

size_t ks_embed_sort_workspace_bytes(const ks_id_order *order) {
  if (check_order_sizes(order) != KS_OK) return 0;
  ks::OrderParams p;
  plan(p, order);
  return room_of(p).end;
}

ks_status ks_embed_sort(const uint32_t *ids, const ks_id_order *order, void *ws, size_t ws_bytes, hipStream_t stream) {
  ks_status st = check_order(order);
  if (st != KS_OK) return st;
  if (order->n_rows > 0 && (!ids || !aligned(ids, 4))) return set_error(KS_EINVAL, "ids is NULL or not aligned to its type");
  ks::OrderParams p;
  plan(p, order);
  const OrderRoom room = room_of(p);
  st = check_room(ws, ws_bytes, room.end);
  if (st != KS_OK) return st;
  const int64_t n = 4 * order->n_rows;
  const Span all[] = {Span(order->row, n), Span(order->id, n), Span(order->off, 4 * (order->n_ids + 1)),
                      Span(ws, (int64_t)room.end), Span(ids, n)};
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (all[i].meets(all[j])) return set_error(KS_EINVAL, "ids, order or workspace overlap");
  char *w = static_cast<char *>(ws);
  p.ids = ids;
  p.row = order->row;
  p.id = order->id;
  p.off = order->off;
  p.hist = reinterpret_cast<uint32_t *>(w);
  p.total = reinterpret_cast<uint32_t *>(w + room.total);
  if (p.passes > 1) {
    p.tmp_id = reinterpret_cast<uint32_t *>(w + room.id);
    p.tmp_row = reinterpret_cast<uint32_t *>(w + room.row);
  }
  return hip_error(ks::launch_order(p, stream), "order launch");
}

size_t ks_embed_backward_workspace_bytes(const ks_id_order *order, const ks_matrix *dy) {
  if (check_order_sizes(order) != KS_OK || check_sizes(dy, "dy") != KS_OK) return 0;
  ks::EmbedBackParams p;
  plan(p, order, dy->n_cols);
  return std::max<size_t>(part_bytes(p), 256);
}

ks_status ks_embed_backward(const ks_id_order *order, double scale, const ks_matrix *dy, const ks_drop *drop,
                            const ks_matrix *grad, void *ws, size_t ws_bytes, hipStream_t stream) {
  ks_status st = check_order(order);
  if (st == KS_OK) st = check_matrix(dy, "dy");
  if (st == KS_OK) st = check_matrix(grad, "grad");
  if (st == KS_OK) st = check_scale(scale);
  if (st == KS_OK) st = check_drop(drop);
  if (st != KS_OK) return st;
  if (dy->n_rows != order->n_rows)
    return set_error(KS_EINVAL, "dy has %lld rows, order %lld", (long long)dy->n_rows, (long long)order->n_rows);
  if (grad->n_rows != order->n_ids || grad->n_cols != dy->n_cols || grad->type != KS_F32)
    return set_error(KS_EINVAL, "grad is not KS_F32 [%lld][%lld]", (long long)order->n_ids, (long long)dy->n_cols);
  ks::EmbedBackParams p;
  plan(p, order, dy->n_cols);
  st = check_room(ws, ws_bytes, std::max<size_t>(part_bytes(p), 256));
  if (st != KS_OK) return st;
  const int64_t n = 4 * order->n_rows;
  const Span room(ws, (int64_t)part_bytes(p)), to(grad);
  const Span read[] = {Span(order->row, n), Span(order->id, n), Span(order->off, 4 * (order->n_ids + 1)),
                       Span(drop ? drop->step_dev : nullptr, drop && drop->step_dev ? 4 : 0)};
  for (const Span &s : read)
    if (to.meets(s) || room.meets(s)) return set_error(KS_EINVAL, "grad or workspace overlaps what the call reads");
  if (overlap(grad, dy) || room.meets(Span(dy)) || room.meets(to))
    return set_error(KS_EINVAL, "grad, dy or workspace overlap");
  double up;
  p.drop = drop_of(drop, &up);
  p.dy = dy->p;
  p.ld = dy->ld;
  p.row = order->row;
  p.id = order->id;
  p.off = order->off;
  p.grad = static_cast<float *>(grad->p);
  p.grad_ld = grad->ld;
  p.past = past_caches(grad);
  p.factor = (float)(scale * up);
  if (!std::isfinite(p.factor)) return set_error(KS_EINVAL, "scale %g / (1 - p) not finite in fp32", scale);
  p.part = static_cast<float *>(ws);
  return hip_error(ks::launch_embed_back(p, dy->type == KS_BF16, stream), "table's gradient launch");
}

size_t ks_eta_loss_workspace_bytes(const int64_t fam_off[KS_NFAM + 1]) {
  if (check_offsets(fam_off) != KS_OK) return 0;
  ks::EtaParams p;
  plan(p, fam_off);
  return eta_bytes(p);
}

ks_status ks_eta_loss(const int64_t fam_off[KS_NFAM + 1], const float *z, const ks_eta_target *target, float *loss,
                      float *dz, void *ws, size_t ws_bytes, hipStream_t stream) {
  ks_status st = check_offsets(fam_off);
  if (st != KS_OK) return st;
  const int64_t n = 4 * fam_off[KS_NFAM];
  if (!target) return set_error(KS_EINVAL, "target is NULL");
  if (n > 0 && !target->eta) return set_error(KS_EINVAL, "target.eta is NULL");
  const float huber = (float)target->huber;
  if (!(target->huber > 0.0) || !(huber > 0.0f)) return set_error(KS_EINVAL, "target.huber %g not above 0 in fp32", target->huber);
  if (!loss) return set_error(KS_EINVAL, "loss is NULL");
  if (n > 0 && (!z || !dz)) return set_error(KS_EINVAL, "z or dz is NULL");
  if (!aligned(target->eta, 4) || !aligned(target->weight, 4) || !aligned(loss, 4) || !aligned(z, 4) || !aligned(dz, 4))
    return set_error(KS_EINVAL, "a pointer is not aligned to its type");
  ks::EtaParams p;
  plan(p, fam_off);
  st = check_room(ws, ws_bytes, eta_bytes(p));
  if (st != KS_OK) return st;
  const Span write[] = {Span(loss, 4 * KS_NFAM), Span(dz, n), Span(ws, (int64_t)eta_bytes(p))};
  const Span read[] = {Span(target->eta, n), Span(target->weight, target->weight ? n : 0), Span(z, n)};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < i; ++j)
      if (write[i].meets(write[j])) return set_error(KS_EINVAL, "loss, dz or workspace overlap");
    for (int j = 0; j < 3; ++j)
      if (write[i].meets(read[j]) && !(i == 1 && j == 2 && dz == z))
        return set_error(KS_EINVAL, "loss, dz or workspace overlaps what the call reads");
  }
  p.z = z;
  p.eta = target->eta;
  p.weight = target->weight;
  p.huber = huber;
  p.loss = loss;
  p.dz = dz;
  p.part = static_cast<double *>(ws);
  return hip_error(ks::launch_eta_loss(p, stream), "loss launch");
}

}  // extern "C"
