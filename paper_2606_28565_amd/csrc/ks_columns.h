// Internal interface between the host code of the learned columns (ks_columns.cpp) and
// their kernels.  Not installed; not part of the ABI.
#pragma once

#include "ks_internal.h"

namespace ks {

// ---- learned columns, dropout (ks_embed.hip) and the order of ids (ks_order.hip)
// Eight columns of one row (a block of ks_drop's draws) are a lane's work; `blocks` of
// them make a row, whose last one has `rem` columns (0: eight).
struct Cols {
  uint32_t blocks, rem;
  uint32_t magic;                    // ceil(2^32 / blocks); 0: one block
};
struct Drop {
  uint32_t key0, key1, site, step;
  const uint32_t *step_dev;          // nullable
  uint32_t least;                    // T: a draw at least this stays; 0: no dropout
};
struct EmbedParams {
  const void *src;                   // x, or the table
  void *dst;
  int64_t src_ld, dst_ld, n_rows;
  const uint32_t *ids;               // null: row i of src is i
  uint32_t n_ids;                    // (1 without ids)
  float factor;
  Cols cols;
  Drop drop;
  uint64_t first;                    // of a launch (set by it): its first block of all,
  int64_t row0;                      // that one's row
  uint32_t block0;                   // and block there
};
hipError_t launch_embed(const EmbedParams &p, bool src16, bool dst16, hipStream_t s);

// A workgroup of k_embed_back takes `run` places of the order, `each` of them for each of
// its 256 / wide groups of lanes, and leaves a sum of the id that began before its places
// (0) and of the one that began in them and goes on behind (1).
constexpr int kBackThreads = 256, kBackFill = 4;   // quads of columns a thread, for ids without rows
struct EmbedBackParams {
  const void *dy;
  int64_t ld, n_rows;
  const uint32_t *row, *id, *off;
  uint32_t n_ids;
  float *grad;
  int64_t grad_ld;
  float factor;
  Cols cols, quads;                  // quads: of four columns
  Drop drop;
  uint32_t wide, each, run, runs, tiles;   // runs parts of the order, tiles of `wide` blocks
  int64_t fill_wgs;                  // ... and for the ids without rows
  bool past;                         // their zeros are not kept in the caches
  float *part;                       // [runs][2][8 blocks]
  int64_t wg0, fill_wg0, fill_row0;  // of a launch (set by it): its first workgroup, the first
  uint32_t fill_quad0;               // for ids without rows, and where that one begins
};
hipError_t launch_embed_back(const EmbedBackParams &p, bool dy16, hipStream_t s);

constexpr int kOrderThreads = 512;   // of a workgroup that ranks keys
constexpr int kOrderKeys = 2048;     // keys ranked at a time
constexpr int kOrderFew = 8, kOrderBits = 10;   // of a digit: the fewest that take no more passes
struct OrderParams {
  const uint32_t *ids;
  uint32_t n_rows, n_ids;
  uint32_t *row, *id, *off;
  uint32_t *tmp_row, *tmp_id;        // [n_rows]; null with one pass
  uint32_t *hist, *total;            // [chunks][2^bits], [2^bits]
  uint32_t chunk, chunks;            // keys of a workgroup, a multiple of kOrderKeys
  int32_t bits, passes;
};
hipError_t launch_order(const OrderParams &p, hipStream_t s);

// ---- the loss at given z (ks_eta.hip)
constexpr int kEtaWide = 1024;        // threads of a workgroup that takes a whole family
struct EtaParams {
  int64_t fam_off[KS_NFAM + 1];
  int64_t rows;                      // of a workgroup
  int32_t wg[KS_NFAM + 1];           // none: a workgroup for each family
  const float *z, *eta, *weight;
  float huber;
  float *loss, *dz;
  double *part;                      // [workgroups][2]
};
hipError_t launch_eta_loss(const EtaParams &p, hipStream_t s);

}  // namespace ks
