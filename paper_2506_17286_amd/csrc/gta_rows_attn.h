// Attention of rows of queries with rules on their scores on the matrix instructions: what its translation units share.
//
// Maps that read the same key head and the same latent group form a cell (mpc of them); the rows of a cell are the (token, map)
// pairs of a sequence, token by token, and a workgroup takes a tile of BQ of them.  A tile's keys can be shared out over several
// pieces, which leave fp32 averages over their keys, and per row a maximum m (in units of log 2) and a weight l, in a slot of scratch
// memory: the piece counts as l 2^m.  Averages do not depend on what their weights referred to, so that whichever workgroup or wave of a row's
// columns goes through its keys again (wave_row) leaves what the row's one (m, l) fits.
// Keys whose scores are -infinity have the weight 0 and take part with it, as what they hold may not be finite; l = -1 marks a row without
// averages.
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
  float *pacc; float2 *pml;         // averages [slot, cell, BQ, d_l], (m, l) [slot, cell, BQ]
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

// One row of queries over keys lo .. hi by one wave, a key a lane for the scores, columns lane, lane + 64, .. for the averages; rows(j): pool
// row of key j, k and c: the row's key head and columns, rows ks and cs apart.  Returns the row's weight (0: sees none, or scores of
// -infinity only).  For waves whose sums are not finite: what is not seen is not read, and averages over the keys so far stay in the range
// of the latents where sums of thousands of large ones do not.
template <typename T, int COLS, class F>
__device__ float wave_row(const Rules &rules, const T *q, int dh, const T *k, int64_t ks, const T *c, int64_t cs, float slope, int own, int lo,
                           int hi, F rows, float (&avg)[COLS]) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < COLS; ++i) avg[i] = 0.f;
#pragma unroll 1
  for (int64_t j0 = lo; j0 <= hi; j0 += 64) {
    const int cnt = (int)min((int64_t)64, hi - j0 + 1);
    float sc = -INFINITY;
    int64_t row = 0;
    if (lane < cnt) {
      row = rows((int)j0 + lane);
      const T *kr = k + row * ks;
      float dot = 0.f;
#pragma unroll 1
      for (int i = 0; i < dh; ++i) dot = fmaf((float)kr[i], (float)q[i], dot);
      sc = ruled_score(rules, dot, slope, fabsf((float)(own - ((int)j0 + lane))));
    }
    float mx = sc;
    for (int i = 32; i; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
    const float mn = fmaxf(m, mx), ref = mn > -INFINITY ? mn : 0.f, before = l * __builtin_amdgcn_exp2f(m - ref);
    const float p = lane < cnt ? __builtin_amdgcn_exp2f(sc - ref) : 0.f;
    float sum = p;
    for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
    m = mn;
    l = before + sum;
    const float per = l > 0.f ? 1.f / l : 0.f, kept = before * per;
#pragma unroll
    for (int i = 0; i < COLS; ++i) avg[i] *= kept;
#pragma unroll 1
    for (int t = 0; t < cnt; ++t) {
      const float pt = __shfl(p, t) * per;
      const int64_t at = ((int64_t)__shfl((int)(row >> 32), t) << 32) | (unsigned)__shfl((int)row, t);
      const T *cr = c + at * cs;
#pragma unroll
      for (int i = 0; i < COLS; ++i) avg[i] = fmaf(pt, (float)cr[i * 64 + lane], avg[i]);
    }
  }
  if (l != l) {   // a score that is NaN
#pragma unroll
    for (int i = 0; i < COLS; ++i) avg[i] = l;
  }
  return l;
}

// bf16 (gta_masked_bf16.hip)
bool rows_bf16_ok(const Dims &d);
int masked_bf16_columns(const Dims &d);   // latent columns of a workgroup of 128 rows
void launch_masked_bf16(const Dims &d, const RowsArgs &a, hipStream_t st);
// fp32 (gta_masked_f32.hip): rows of 32 per tile
bool rows_f32_ok(const Dims &d);
int rows_f32_columns(const Dims &d);
bool launch_rows_f32(const Dims &d, const RowsArgs &a, bool cache, hipStream_t st);   // false: nothing was launched
// either (gta_masked_plan.hip)
bool masked_tuned(const Dims &d);
bool masked_fits(const Dims &d, int batch, int64_t total);
bool rows_operands_ok(const void *p, int64_t stride, int esize);
size_t masked_bytes(const Dims &d, int batch, int64_t total);        // of a call
size_t masked_bytes_up_to(const Dims &d, int batch, int64_t total);  // of any of as many sequences and tokens or fewer
int launch_masked(const Dims &d, const MaskedArgs &m, void *ws, hipStream_t st);

// The prefix's rows: rows of a tile for `rows` query rows of a cell, workgroups that share its latent columns, launch
int prefix_tile_rows(const Dims &d, int rows);
int prefix_slices(const Dims &d, int bq, int prefix_max);
void launch_prefix_rows(const Dims &d, const RowsArgs &a, int bq, hipStream_t st);

// gta_prefix_decode.hip
bool prefix_tuned(const Dims &d);   // with pages of a power of two of at least 16 rows
bool prefix_fits(const Dims &d, int batch);
bool prefix_layout_ok(const gta_cache &prefix, const gta_cache &own);
size_t prefix_bytes(const Dims &d, int batch, int prefix_max, int max_seq);
size_t prefix_bytes_up_to(const Dims &d, int batch, int prefix_max, int max_seq);
int launch_prefix(const Dims &d, const PrefixArgs &x, void *ws, hipStream_t st);

}  // namespace gta
