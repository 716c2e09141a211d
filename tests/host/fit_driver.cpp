// CPU driver of the fitting entry points' host code, built with g++ under
// AddressSanitizer and UndefinedBehaviorSanitizer against host stand-ins of the launches
// (fake_device.cpp, fake_fit.cpp).  TEST INFRASTRUCTURE ONLY.  Reads calls on stdin, one
// per line, and prints "ok" or what was wrong for each:
//
//   rows <n> <in_dim> <hidden> <bf16> <padding> <offsets 1..9>   forward, backward, loss
//   adam <bits> <bf16 gradients> <shift> <sizes...>              one step over tensors
//   features <records> <specs> <in_dim> <bf16> <padding>
//   args                                                         statuses, a line each
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <iostream>
#include <memory>
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

alignas(16) float weight[4];   // never read by the stand-ins

ks_heads heads_of(int in_dim, int hidden, int bf16) {
  ks_heads h;
  std::memset(&h, 0, sizeof h);
  h.mode = KS_ETA_GATED;
  h.in_dim = in_dim;
  h.hidden = hidden;
  h.precision = bf16 ? KS_BF16 : KS_F32;
  h.w1 = h.w2 = h.w3 = h.b3 = weight;
  return h;
}

const char *fail(const char *what) { return what; }
#define NEED(c) \
  if (!(c)) return fail(#c)

const char *run_rows(std::istream &in) {
  int64_t n, pad;
  int in_dim, hidden, bf16;
  in >> n >> in_dim >> hidden >> bf16 >> pad;
  const ks_heads h = heads_of(in_dim, hidden, bf16);
  ks_rows r;
  r.n_rows = n;
  r.ldx = in_dim + pad;
  r.fam_off[0] = 0;
  for (int f = 1; f < KS_NFAM; ++f) in >> r.fam_off[f];
  r.fam_off[KS_NFAM] = n;
  const size_t e = bf16 ? 2 : 4;
  std::vector<char> x(n ? ((n - 1) * r.ldx + in_dim) * e : 0);
  r.x = n ? x.data() : nullptr;
  const size_t need = ks_gated_workspace_bytes(&h, &r);
  NEED(need > 0 && need % 256 == 0);
  Room ws(need);
  std::vector<float> z(n, 0.0f), dz(n, 1.0f), w1(KS_NFAM * hidden * in_dim), w2(w1.size()), w3(KS_NFAM * hidden), b3(KS_NFAM);
  NEED(ks_gated_forward(&h, &r, z.data(), nullptr) == KS_OK);
  for (float v : z) NEED(v == 1.0f);
  auto rows = [&](int f) { return (float)(r.fam_off[f + 1] - r.fam_off[f]); };
  auto sums = [&]() {
    for (int f = 0; f < KS_NFAM; ++f) {
      for (int i = 0; i < hidden * in_dim; ++i)
        if (w1[f * hidden * in_dim + i] != rows(f) || w2[f * hidden * in_dim + i] != rows(f)) return false;
      for (int i = 0; i < hidden; ++i)
        if (w3[f * hidden + i] != rows(f)) return false;
      if (b3[f] != rows(f)) return false;
      b3[f] = w3[f * hidden] = -1.0f;
    }
    return true;
  };
  std::vector<char> gx(x.size());
  ks_gated_grad g{w1.data(), w2.data(), w3.data(), b3.data(), n ? gx.data() : nullptr, r.ldx};
  NEED(ks_gated_backward(&h, &r, n ? dz.data() : nullptr, &g, ws.p, need, nullptr) == KS_OK);
  NEED(sums());
  for (int64_t i = 0; i < n; ++i)
    for (int64_t d = 0; d < r.ldx && i * r.ldx + d < (int64_t)(gx.size() / e); ++d) {
      const int64_t at = i * r.ldx + d;
      const float v = bf16 ? (float)((uint16_t *)gx.data())[at] : ((float *)gx.data())[at];
      NEED(v == (d < in_dim ? 1.0f : 0.0f));
    }
  g.x = nullptr;
  std::vector<float> eta(n, 2.0f), loss(KS_NFAM), z2(n, 0.0f);
  const ks_eta_target t{eta.data(), nullptr, INFINITY};
  NEED(ks_gated_loss(&h, &r, &t, loss.data(), z2.data(), &g, ws.p, need, nullptr) == KS_OK);
  NEED(sums());
  for (int f = 0; f < KS_NFAM; ++f) NEED(loss[f] == 2 * rows(f));
  for (float v : z2) NEED(v == 1.0f);
  NEED(ks_gated_loss(&h, &r, &t, loss.data(), nullptr, nullptr, ws.p, need, nullptr) == KS_OK);
  for (int f = 0; f < KS_NFAM; ++f) NEED(loss[f] == 2 * rows(f));
  return "ok";
}

const char *run_adam(std::istream &in) {
  int bits, g16, shift;
  in >> bits >> g16 >> shift;
  const bool eight = bits == 8;
  struct T {
    std::vector<float> p;
    std::vector<char> g, m, v;
    std::vector<uint8_t> me, ve;
    std::vector<uint16_t> copy;
    int64_t n;
  };
  std::vector<std::unique_ptr<T>> ts;
  std::vector<ks_tensor> arr;
  for (int64_t n; in >> n;) {
    auto t = std::make_unique<T>();
    const size_t s = eight ? 1 : 4, at = n + shift;
    t->n = n;
    t->p.resize(at);
    t->g.resize(at * (g16 ? 2 : 4));
    t->m.resize(at * s), t->v.resize(at * s);
    t->copy.resize(at);
    t->me.resize((n + 63) / 64), t->ve.resize((n + 63) / 64);
    ks_tensor k;
    std::memset(&k, 0, sizeof k);
    k.n = n;
    k.param = t->p.data() + shift;
    k.grad = t->g.data() + shift * (g16 ? 2 : 4);
    k.m = t->m.data() + shift * s, k.v = t->v.data() + shift * s;
    if (eight) k.m_exp = t->me.data(), k.v_exp = t->ve.data();
    k.copy = ts.size() % 2 ? t->copy.data() + shift : nullptr;
    k.grad_type = g16 ? KS_BF16 : KS_F32;
    if (n == 0) k.param = nullptr, k.grad = nullptr, k.m = k.v = nullptr, k.m_exp = k.v_exp = nullptr, k.copy = nullptr;
    ts.push_back(std::move(t));
    arr.push_back(k);
  }
  uint32_t count = 4;
  const ks_adamw_config c{1e-3, 0.9, 0.999, 1e-8, 1.0, bits, 0, 1, &count};
  NEED(ks_adamw(&c, arr.data(), (int32_t)arr.size(), nullptr) == KS_OK);
  NEED(count == 5);
  for (size_t j = 0; j < ts.size(); ++j) {
    const T &t = *ts[j];
    for (int64_t i = 0; i < t.n + shift; ++i) {
      const bool in_it = i >= shift;
      NEED(t.p[i] == (in_it ? 1.0f : 0.0f));
      NEED(t.copy[i] == (in_it && j % 2 ? 1 : 0));
      NEED((eight ? (float)(uint8_t)t.m[i] : ((const float *)t.m.data())[i]) == (in_it ? 1.0f : 0.0f));
      NEED((eight ? (float)(uint8_t)t.v[i] : ((const float *)t.v.data())[i]) == (in_it ? 1.0f : 0.0f));
    }
    for (uint8_t v : t.me) NEED(v == (eight ? 1 : 0));
    for (uint8_t v : t.ve) NEED(v == (eight ? 1 : 0));
  }
  return "ok";
}

const char *run_features(std::istream &in) {
  int64_t n, pad;
  int specs, in_dim, bf16;
  in >> n >> specs >> in_dim >> bf16 >> pad;
  std::vector<uint32_t> zero(n, 0), req_off{0, 1}, one{1}, hist{5};
  ks_desc d;
  std::memset(&d, 0, sizeof d);
  d.n_rows = n;
  for (int f = 0; f <= KS_NFAM; ++f) d.fam_off[f] = n * f / KS_NFAM;
  d.step = d.m = d.n = d.k = d.a = d.b = zero.data();
  d.n_steps = 1;
  d.req_off = req_off.data();
  d.req_q = one.data();
  d.req_h = hist.data();
  d.n_req = 1;
  d.elem_bytes = 2;
  std::vector<ks_spec> sp(specs, ks_spec{1e15, 4e12, 3e-6, 5e7, 8e-6, 2e-6, 3e11, 64u, 0u});
  const size_t need = ks_workspace_bytes(&d, specs);
  NEED(need > 0);
  Room ws((need + 255) / 256 * 256);
  const int64_t ldx = in_dim + pad, pairs = n * specs;
  std::vector<char> x(pairs ? ((pairs - 1) * ldx + in_dim) * (bf16 ? 2 : 4) : 0);
  std::vector<float> roof(pairs);
  NEED(ks_features(&d, sp.data(), specs, in_dim, bf16 ? KS_BF16 : KS_F32, n ? x.data() : nullptr, ldx, roof.data(), ws.p, need,
                   nullptr) == KS_OK);
  for (float v : roof) NEED(v == 1.0f);
  return "ok";
}

void report(const char *name, ks_status st) {
  std::printf("%s %d\n", name, (int)st);
  if (st != KS_OK && std::strlen(ks_last_error()) == 0) std::printf("%s empty-message\n", name);
}

// Rows and their gradients in one buffer: rows at 0, gradients `at` elements behind.
void columns(const char *name, int64_t n, int64_t ldx, int64_t at, int64_t ldg) {
  const ks_heads h = heads_of(16, 8, 0);
  std::vector<float> buf(4096), dz(n, 1.0f), w(KS_NFAM * 8 * 16);
  ks_rows r;
  r.n_rows = n;
  for (int f = 0; f <= KS_NFAM; ++f) r.fam_off[f] = n * f / KS_NFAM;
  r.x = buf.data() + 1024;
  r.ldx = ldx;
  const size_t need = ks_gated_workspace_bytes(&h, &r);
  Room ws(need);
  const ks_gated_grad g{nullptr, nullptr, nullptr, nullptr, buf.data() + 1024 + at, ldg};
  report(name, ks_gated_backward(&h, &r, dz.data(), &g, ws.p, need, nullptr));
}

void run_args() {
  columns("columns_apart", 20, 40, 16, 40);
  columns("columns_apart_before", 20, 40, -16, 40);
  columns("columns_far_apart", 20, 40, 24 + 40, 40);
  columns("columns_of_other_rows", 20, 32, 16 + 32 * 5, 32);
  columns("columns_meet", 20, 40, 15, 40);
  columns("columns_meet_before", 20, 40, -15, 40);
  columns("columns_run_into_the_next_row", 20, 40, 25, 40);
  columns("columns_of_other_strides", 20, 40, 16, 48);
  columns("same_rows", 20, 16, 0, 16);
  columns("one_row_apart", 1, 16, 16, 16);
  columns("one_row_meets", 1, 40, 15, 40);
  columns("behind_the_last", 20, 16, 16 * 20, 16);
  ks_heads h = heads_of(16, 64, 0);
  ks_rows r;
  std::memset(&r, 0, sizeof r);
  r.ldx = 16;
  std::printf("workspace %d\n", ks_gated_workspace_bytes(&h, &r) > 0);
  h.precision = 2;
  std::printf("workspace_of_unknown_precision %d\n", ks_gated_workspace_bytes(&h, &r) > 0);
}

}  // namespace

int main() {
  for (std::string line; std::getline(std::cin, line);) {
    std::istringstream in(line);
    std::string what;
    in >> what;
    if (what == "rows") std::printf("%s\n", run_rows(in));
    else if (what == "adam") std::printf("%s\n", run_adam(in));
    else if (what == "features") std::printf("%s\n", run_features(in));
    else if (what == "args") run_args();
    else return 2;
  }
  return 0;
}
