// Attention of rows of queries with rules on their scores on the matrix instructions: what its translation units share.
//
// Maps that read the same key head and the same latent group form a cell (mpc of them); the rows of a cell are the (token, map)
// pairs of a sequence, token by token, and a workgroup takes a tile of BQ of them.  A tile's keys can be shared out over several
// pieces, which leave un-normalised fp32 sums, their maximum (in units of log 2) and their weight in a slot of scratch memory.
#pragma once
#include <algorithm>

#include "gta_rules.h"

namespace gta {

struct Piece { int b, tile, piece, pieces, slot, pad[3]; };   // slot: of the tile's first piece, where pieces > 1

struct RowsArgs {
  const void *q, *k, *c;            // c, k: packed rows, or the prefix's caches
  int64_t qs, ks, cs;               // row strides in elements
  void *L;                          // [tokens, n_q * d_l]
  const int32_t *cu;
  int per_seq, batch;
  int nq, mpc, cells, kdiv, cdiv;   // cells of a key head, of a latent group
  int dl, slices;                   // slices of a cell's latent columns, one per workgroup
  Rules rules;
  const Piece *list;                // work, in the order it is started; NULL: every tile of every sequence, whole
  const int32_t *count;
  int tiles;                        // of the launch
  float *pacc; float2 *pml;         // [slot, cell, BQ, d_l], [slot, cell, BQ]
  // keys from one slot of a cache (prefix): tokens are sequences, which see its rows; `pieces` of every tile
  CacheView prefix, own;
  int prefix_slot, pieces, ps_shift;
};

inline int gcd_of(int a, int b) { return b ? gcd_of(b, a % b) : a; }
inline int maps_per_cell(const Dims &d) { return gcd_of(d.qpk, d.qpc); }

// What a query row of a prefix call sees of the prefix's P rows, and its position
__device__ __forceinline__ void prefix_seen(const RowsArgs &a, int b, int P, int &lo, int &hi, int &own) {
  const int slot = a.own.slots ? a.own.slots[b] : b;
  own = (int)((int64_t)P + slot_rows(a.own, slot) - 1);
  seen_by(a.rules, b, own, own + 1, lo, hi);
  hi = min(hi, P - 1);
}

// bf16 (gta_masked_bf16.hip)
bool rows_bf16_ok(const Dims &d);
bool rows_operands_ok(const void *p, int64_t stride, int esize);
bool masked_bf16_fits(const Dims &d, int batch, int64_t total);
size_t masked_bf16_bytes(const Dims &d, int batch, int64_t total);
int launch_masked_bf16(const Dims &d, const MaskedArgs &m, void *ws, hipStream_t st);

// The prefix's rows: rows of a tile for `rows` query rows of a cell, workgroups that share its latent columns, launch
int prefix_tile_rows(const Dims &d, int rows);
int prefix_slices(const Dims &d, int bq);
void launch_prefix_rows(const Dims &d, const RowsArgs &a, int bq, hipStream_t st);

// gta_prefix_decode.hip
bool prefix_tuned(const Dims &d);   // with pages of a power of two of at least 16 rows
bool prefix_fits(const Dims &d, int batch, int prefix_max, int max_seq);
bool prefix_layout_ok(const gta_cache &prefix, const gta_cache &own);
size_t prefix_bytes(const Dims &d, int batch, int prefix_max, int max_seq);
int launch_prefix(const Dims &d, const PrefixArgs &x, void *ws, hipStream_t st);

}  // namespace gta
