// CPU driver of the learned columns' host code, built with g++ under AddressSanitizer and
// UndefinedBehaviorSanitizer against host stand-ins of the launches (fake_device.cpp,
// fake_fit.cpp, fake_columns.cpp).  TEST INFRASTRUCTURE ONLY.  Reads calls on stdin, one
// per line, and prints "ok" or what was wrong for each:
//
//   columns <rows> <ids> <columns> <padding> <bf16>   dropout, lookup, order, gradient
//   loss <rows> <weights> <offsets 1..9>              the loss at given z
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

#include "ks.h"

namespace {

struct Room {   // 256-byte aligned, of the asked size to the byte (a multiple of 256)
  void *p;
  explicit Room(size_t n) : p(std::aligned_alloc(256, n)) { std::memset(p, 0xFF, n); }
  ~Room() { std::free(p); }
  Room(const Room &) = delete;
  Room &operator=(const Room &) = delete;
};

#define NEED(c) \
  if (!(c)) return #c

struct Matrix {   // to the byte
  std::vector<char> room;
  ks_matrix m;
  Matrix(int64_t n, int64_t cols, int64_t ld, int32_t type) {
    const size_t e = type == KS_BF16 ? 2 : 4;
    room.assign(n ? ((n - 1) * ld + cols) * e : 0, 0);
    m = {n ? room.data() : nullptr, n, cols, ld, type, 0};
  }
  double at(int64_t i, int64_t j) const {
    const int64_t k = i * m.ld + j;
    return m.type == KS_BF16 ? reinterpret_cast<const uint16_t *>(room.data())[k] : reinterpret_cast<const float *>(room.data())[k];
  }
  bool all(double v) const {   // ... and nothing between the columns
    for (int64_t i = 0; i < m.n_rows; ++i)
      for (int64_t j = 0; j < (i + 1 < m.n_rows ? m.ld : m.n_cols); ++j)
        if (at(i, j) != (j < m.n_cols ? v : 0.0)) return false;
    return true;
  }
};

const char *run_columns(std::istream &in) {
  int64_t n, v, cols, pad;
  int bf16;
  in >> n >> v >> cols >> pad >> bf16;
  const int32_t type = bf16 ? KS_BF16 : KS_F32;
  Matrix x(n, cols, cols + pad, type), y(n, cols, cols + pad, type), table(v, cols, cols + pad, type), looked(n, cols, cols, KS_F32);
  const ks_drop drop = {0.25, 7, 1, 2, nullptr};
  NEED(ks_dropout(&drop, &x.m, &y.m, nullptr) == KS_OK);
  NEED(y.all(1.0));
  std::vector<uint32_t> ids(n), row(n), id(n), off(v + 1);
  std::vector<uint32_t> count(v, 0);
  for (int64_t i = 0; i < n; ++i) {
    ids[i] = (uint32_t)(i * 2654435761u % (uint64_t)(v + v / 4 + 2));
    if (ids[i] > v) ids[i] = 0xFFFFFFFFu;
    if (ids[i] < v) ++count[ids[i]];
  }
  NEED(ks_embed(&table.m, 2.0, ids.data(), &drop, &looked.m, nullptr) == KS_OK);
  NEED(looked.all(1.0));
  const ks_id_order order = {n, v, row.data(), id.data(), off.data()};
  const size_t need = ks_embed_sort_workspace_bytes(&order);
  NEED(need > 0 && need % 256 == 0);
  Room ws(need);
  NEED(ks_embed_sort(ids.data(), &order, ws.p, need - 1, nullptr) == KS_EWORKSPACE);
  NEED(ks_embed_sort(ids.data(), &order, ws.p, need, nullptr) == KS_OK);
  for (int64_t i = 0; i < v; ++i) NEED(off[i + 1] - off[i] == count[i]);
  Matrix grad(v, cols, cols + pad, KS_F32);
  const size_t room = ks_embed_backward_workspace_bytes(&order, &x.m);
  NEED(room > 0 && room % 256 == 0);
  Room back(room);
  NEED(ks_embed_backward(&order, 2.0, &x.m, &drop, &grad.m, back.p, room - 1, nullptr) == KS_EWORKSPACE);
  NEED(ks_embed_backward(&order, 2.0, &x.m, &drop, &grad.m, back.p, room, nullptr) == KS_OK);
  for (int64_t i = 0; i < v; ++i)
    for (int64_t j = 0; j < cols; ++j) NEED(grad.at(i, j) == count[i]);
  return nullptr;
}

const char *run_loss(std::istream &in) {
  int64_t n, off[KS_NFAM + 1] = {0};
  int weights;
  in >> n >> weights;
  for (int f = 1; f < KS_NFAM; ++f) in >> off[f];
  off[KS_NFAM] = n;
  std::vector<float> z(n, 0.0f), eta(n, 2.0f), w(n, 1.0f), dz(n, 0.0f), loss(KS_NFAM, -1.0f);
  const ks_eta_target target = {eta.data(), weights ? w.data() : nullptr, 1.0};
  const size_t need = ks_eta_loss_workspace_bytes(off);
  NEED(need > 0 && need % 256 == 0);
  Room ws(need);
  NEED(ks_eta_loss(off, z.data(), &target, loss.data(), dz.data(), ws.p, need - 1, nullptr) == KS_EWORKSPACE);
  NEED(ks_eta_loss(off, z.data(), &target, loss.data(), dz.data(), ws.p, need, nullptr) == KS_OK);
  for (float d : dz) NEED(d == 1.0f);
  for (int f = 0; f < KS_NFAM; ++f) NEED(loss[f] == (float)(off[f + 1] - off[f]));
  return nullptr;
}

}  // namespace

int main() {
  std::string line, word;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    in >> word;
    const char *wrong = word == "columns" ? run_columns(in) : word == "loss" ? run_loss(in) : "unknown call";
    if (wrong) std::cout << line << ": " << wrong << " (" << ks_last_error() << ")\n";
    else std::cout << "ok\n";
  }
}
