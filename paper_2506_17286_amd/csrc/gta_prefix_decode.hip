// One new token per sequence over a prefix that the batch shares and over the sequence's own cached rows, with rules on the scores
// (gta_score_rules):
//   1. the prefix is read once for all: the batch's queries are the rows of rows_attn_kernel (bf16) and rows_attn_f32_kernel, which
//      leave un-normalised sums of pieces of the prefix;
//   2. stream_kernel reads every sequence's own rows once for all its maps, in pieces, too;
//   3. prefix_join_kernel weighs the sums by their maxima.
#include <math.h>

#include <type_traits>

#include "gta_lds_load.h"
#include "gta_rows_attn.h"

namespace gta {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

struct StreamArgs {
  const void *q;
  CacheView prefix, own;
  int prefix_slot, batch, nq, qpk, qpc, dh, dl, kw, cw;
  Rules rules;
  int maps, blocks;            // maps of a workgroup, workgroups of a latent group's maps
  int heads;                   // key heads that a workgroup's maps read at most
  int pieces, ps_shift;
  int rows, stages, stage_bytes, k_instr, instr;   // of a tile: rows, load instructions of its keys and in all (1 KiB each)
  float *pacc; float2 *pml;    // [batch, pieces, n_q, d_l], [batch, pieces, n_q]
};

__device__ __forceinline__ int load_uniform(const int32_t *p) {
  int v;
  asm volatile("s_load_dword %0, %1, 0x0\n\ts_waitcnt lgkmcnt(0)" : "=s"(v) : "s"(p));
  return v;
}

// Waits until at most n of the wave's loads are in flight (fewer where n is between two of the cases).
__device__ __forceinline__ void wait_loads(int n) {
  if (n >= 32) asm volatile("s_waitcnt vmcnt(32)" ::: "memory");
  else if (n >= 24) asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
  else if (n >= 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  else if (n >= 12) asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
  else if (n >= 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else if (n >= 6) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
  else if (n >= 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
  else if (n >= 3) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
  else if (n >= 2) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
  else if (n >= 1) asm volatile("s_waitcnt vmcnt(1)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

constexpr float kLazy = 8.0f;        // log2 units by which a score may pass the maximum that weights refer to
constexpr int kMaxInstr = 16;        // load instructions of a wave and tile

// A workgroup has up to 16 maps of one latent group of a sequence and NF * 64 of its latent columns.  Tiles of 16 or 32 rows,
// keys and latents, go from memory straight into LDS, `stages` of them, one barrier a tile; every wave has the scores of all maps
// (16 columns of a 16 x 16 product, its own head's kept) and sums up a quarter of the columns:
//   S[row][map] = K q^T: lane (x = l % 16, h = l / 16) ends up with map x, rows 4 h .. 4 h + 3;
//   L[column][map] += C^T p: which is what the second operand of the other product wants from it.
// Bound by memory: every row is read once (once per head or slice where a layer's rows are wider than a workgroup's, from L2).
// bf16 weights are rounded for the second product, as in the kernel of the prefix, and so is their sum.  (Two parts of 16 bits would
// cost nothing here, but an infinite latent times the second, which may be 0 or less, is no infinity.)
// Rows in front of the first that is seen are cleared in LDS, rows behind the last read as zeros: what is masked has the weight 0, and
// that times a latent that is not finite would not be.
template <typename T, int DH, int NF>
__global__ __launch_bounds__(256, NF > 8 ? 1 : 2) void stream_kernel(StreamArgs a) {
  constexpr int ES = sizeof(T), KS = DH * ES / 64, KCH = DH * ES / 16;   // 64-byte steps and chunks of a key head
  constexpr int SW = NF * 64, CP = SW * ES, CCH = CP / 16;               // latent columns, their bytes and chunks a row
  constexpr int PM = CCH / 2 < 8 ? CCH / 2 - 1 : 7;                      // pairs of chunks that rows are swapped over (bf16)
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = blockIdx.z, piece = blockIdx.x, slices = a.dl / SW;
  const int slice = blockIdx.y % slices, rest = blockIdx.y / slices, block = rest % a.blocks, cgrp = rest / a.blocks;
  const int g0 = cgrp * a.qpc + block * a.maps, gn = min(a.maps, a.qpc - block * a.maps);   // maps g0 .. g0 + gn - 1
  const int kh0 = g0 / a.qpk, heads = (g0 + gn - 1) / a.qpk - kh0 + 1;
  const int slot = a.own.slots ? a.own.slots[b] : b, P = slot_rows(a.prefix, a.prefix_slot), n = slot_rows(a.own, slot);
  const int own = (int)((int64_t)P + n - 1);
  int lo, hi;
  seen_by(a.rules, b, own, own + 1, lo, hi);
  lo = __builtin_amdgcn_readfirstlane(max(lo - P, 0));      // rows of the sequence itself
  hi = __builtin_amdgcn_readfirstlane(hi - P);
  const int64_t at = ((int64_t)b * a.pieces + piece) * a.nq + g0;
  const int t_lo = lo / a.rows, tiles = hi < lo ? 0 : hi / a.rows - t_lo + 1;
  const int t0 = t_lo + (int)((int64_t)tiles * piece / a.pieces), t1 = t_lo + (int)((int64_t)tiles * (piece + 1) / a.pieces);
  if (t0 >= t1) {
    if (slice == 0 && tid < gn) a.pml[at + tid] = make_float2(-INFINITY, 0.f);
    return;
  }
  const int g = min(g0 + x, g0 + gn - 1), head = g / a.qpk - kh0;   // this lane's map (lanes without one repeat the last)
  const float slope = a.rules.slopes ? a.rules.slopes[g] : 0.f;

  const int us = __builtin_amdgcn_readfirstlane(slot);
  const int32_t *table = a.own.pm.table ? a.own.pm.table + (int64_t)us * a.own.pm.pages_per_slot : nullptr;
  const int64_t row0 = table ? 0 : (int64_t)us * a.own.max_seq;
  const char *Kb = (const char *)((const T *)a.own.k + row0 * a.kw + (int64_t)kh0 * DH);
  const char *Cb = (const char *)((const T *)a.own.c + row0 * a.cw + (int64_t)cgrp * a.dl + slice * SW);
  const unsigned kws = (unsigned)a.kw * ES, cws = (unsigned)a.cw * ES;
  const int KP = a.heads * DH * ES, kch = KP / 16;

  // This wave's load instructions of a tile are wave, wave + 4, ..; slot s of a row holds the row's chunk s, swapped with others so
  // that 16 rows' reads of one chunk fall into different banks.
  unsigned voff[kMaxInstr];
#pragma unroll
  for (int i = 0; i < kMaxInstr; ++i) {
    const int in = wave + 4 * i;
    if (in < a.k_instr) {
      const int s = in * 64 + lane, row = s / kch, c = s % kch ^ (row & 7);
      voff[i] = c * 16 < heads * DH * ES ? row * kws + c * 16 : ~0u - 15u;   // (fewer heads than others' maps read: nothing)
    } else {
      const int s = (in - a.k_instr) * 64 + lane, row = s / CCH;
      int c = s % CCH;
      if constexpr (ES == 2) c = ((c >> 1) ^ (row & PM)) * 2 + (c & 1);
      else c = ((c >> 2) ^ ((row >> 2) & 3)) * 4 + (c & 3);
      voff[i] = row * cws + c * 16;
    }
  }
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  const int k_half = a.k_instr * 16 / a.rows, c_half = (a.instr - a.k_instr) * 16 / a.rows;   // instructions of 16 rows
  auto issue = [&](int t, int st) __attribute__((always_inline)) {
    const int j0 = t * a.rows, rows = min(hi + 1 - j0, a.rows);
    const unsigned kbytes = rows > 0 ? (rows - 1) * kws + heads * DH * ES : 0u, cbytes = rows > 0 ? (rows - 1) * cws + CP : 0u;
    int64_t p0 = j0, p1 = j0;
    if (table) {   // 16 rows lie in one page
      auto find = [&](int j) {
        int pg = load_uniform(table + __builtin_amdgcn_readfirstlane(j >> a.ps_shift));
        pg = (unsigned)pg >= (unsigned)a.own.pm.num_pages ? 0 : pg;
        return ((int64_t)pg << a.ps_shift) + (j & (a.own.pm.page_size - 1));
      };
      p0 = find(min(j0, hi & ~15));
      p1 = a.rows > 16 ? find(min(j0 + 16, hi & ~15)) - 16 : p0;
    }
    const u32x4 k0 = uniform_buffer_of(Kb + p0 * kws, kbytes), k1 = uniform_buffer_of(Kb + p1 * kws, kbytes);
    const u32x4 c0 = uniform_buffer_of(Cb + p0 * cws, cbytes), c1 = uniform_buffer_of(Cb + p1 * cws, cbytes);
    const unsigned to = lds0 + st * a.stage_bytes;
#pragma unroll
    for (int i = 0; i < kMaxInstr; ++i) {
      const int in = wave + 4 * i;
      if (in < a.instr) {
        if (in < a.k_instr) load_to_lds(in < k_half ? k0 : k1, voff[i], to + in * 1024);
        else load_to_lds(in - a.k_instr < c_half ? c0 : c1, voff[i], to + in * 1024);
      }
    }
  };
  const int per_tile = (a.instr - wave + 3) / 4;

  f32x4 qf[KS];   // 64 bytes' worth of a step, 16 of them per lane
  {
    const f32x4 *qp = reinterpret_cast<const f32x4 *>((const T *)a.q + ((int64_t)b * a.nq + g) * DH) + h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = qp[ks * 4];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
  }
  f32x4 acc[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  for (int s = 0; s < a.stages - 1; ++s) issue(t0 + s, s);   // (steps past the last read zeros)
  int st = 0, fill = a.stages - 1;
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    wait_loads((a.stages - 2) * per_tile);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    issue(t + a.stages - 1, fill);
    fill = fill + 1 == a.stages ? 0 : fill + 1;
    const char *kt = smem + st * a.stage_bytes, *ct = kt + a.k_instr * 1024;
    st = st + 1 == a.stages ? 0 : st + 1;
    const int j0 = t * a.rows;
    if (j0 < lo) {   // clear what is in front of the first row
      for (int i = tid; i < (lo - j0) * CCH; i += 256) *reinterpret_cast<u32x4 *>(smem + (ct - smem) + i * 16) = u32x4{0u, 0u, 0u, 0u};
      __syncthreads();
    }
#pragma unroll 1
    for (int r0 = 0; r0 < a.rows; r0 += 16) {
      f32x4 s{0.f, 0.f, 0.f, 0.f};
      const char *kr = kt + (r0 + x) * KP;
#pragma unroll 1
      for (int kk = 0; kk < heads; ++kk) {
        f32x4 d{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const f32x4 kf = *reinterpret_cast<const f32x4 *>(kr + ((kk * KCH + ks * 4 + h) ^ (x & 7)) * 16);
          if constexpr (ES == 2) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[ks]), d, 0, 0, 0);
          else {
#pragma unroll
            for (int e = 0; e < 4; ++e) d = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[ks][e], d, 0, 0, 0);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = head == kk ? d[e] : s[e];
      }
      float p[4];
      float mt = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = j0 + r0 + 4 * h + e;
        const float v = ruled_score(a.rules, s[e], slope, (float)(n - 1 - j));
        p[e] = j >= lo && j <= hi ? v : -INFINITY;
        mt = fmaxf(mt, p[e]);
      }
      mt = fmaxf(mt, __shfl_xor(mt, 16));
      mt = fmaxf(mt, __shfl_xor(mt, 32));
      const float mn = mt > m + kLazy ? mt : m, ref = mn > -INFINITY ? mn : 0.f;
      const float corr = __builtin_amdgcn_exp2f(m - ref);
      if (__builtin_amdgcn_ballot_w64(mn != m) != 0) {
        l *= corr;
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[f] *= corr;
      }
      m = mn;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = __builtin_amdgcn_exp2f(p[e] - ref);
        if constexpr (ES == 2) p[e] = (float)(__bf16)p[e];
        l += p[e];
      }
      if constexpr (ES == 2) {
        bf16x4 p1;
#pragma unroll
        for (int e = 0; e < 4; ++e) p1[e] = (__bf16)p[e];
        const int row = r0 + 4 * h + (x >> 2);
        const char *cr = ct + row * CP + (x & 1) * 8;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const int pair = (wave * NF + f) ^ (row & PM);   // 16 columns are a pair of chunks
          const s16x4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(cr + (pair * 2 + ((x >> 1) & 1)) * 16));
          acc[f] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(c, __builtin_bit_cast(s16x4, p1), acc[f], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = r0 + 4 * h + e, blk = (wave * NF + f) ^ ((row >> 2) & 3);   // 16 columns are a block of 64 bytes
            const float c = *reinterpret_cast<const float *>(ct + row * CP + blk * 64 + x * 4);
            acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(c, p[e], acc[f], 0, 0, 0);
          }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land behind the workgroup's end
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (x < gn) {
    float *to = a.pacc + (at + x) * a.dl + slice * SW + wave * NF * 16 + 4 * h;
#pragma unroll
    for (int f = 0; f < NF; ++f) *reinterpret_cast<f32x4 *>(to + f * 16) = acc[f];
    if (slice == 0 && wave == 0 && h == 0) a.pml[at + x] = make_float2(m, l);
  }
}

struct JoinArgs {
  StreamArgs s;
  RowsArgs r;      // the prefix's pieces
  int bq;
  void *l_out;
};

// One (sequence, map): the sums of the prefix's and the sequence's own pieces, weighed by 2^(maximum - the largest).
constexpr int kMaxPieces = 512;
template <typename T>
__global__ __launch_bounds__(256) void prefix_join_kernel(JoinArgs j) {
  __shared__ float weight[kMaxPieces];
  __shared__ float red[8];
  const int b = blockIdx.x, g = blockIdx.y, tid = threadIdx.x, S = j.r.pieces, all = S + j.s.pieces;
  const int cell = g / j.r.mpc, row = b * j.r.mpc + g % j.r.mpc, tile = row / j.bq;
  auto shared_at = [&](int i) { return ((int64_t)(tile * S + i) * j.r.cells + cell) * j.bq + row % j.bq; };
  auto own_at = [&](int i) { return ((int64_t)b * j.s.pieces + i) * j.s.nq + g; };
  float2 ml[kMaxPieces / 256];
  float mx = -INFINITY;
#pragma unroll
  for (int v = 0; v < kMaxPieces / 256; ++v) {
    const int i = v * 256 + tid;
    ml[v] = make_float2(-INFINITY, 0.f);
    if (i < all) ml[v] = i < S ? j.r.pml[shared_at(i)] : j.s.pml[own_at(i - S)];
    mx = fmaxf(mx, ml[v].x);
  }
  for (int i = 32; i; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
  if ((tid & 63) == 0) red[tid >> 6] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float ref = mx > -INFINITY ? mx : 0.f;
  float sum = 0.f;
#pragma unroll
  for (int v = 0; v < kMaxPieces / 256; ++v) {
    const int i = v * 256 + tid;
    // a piece that sees nothing has left no sums; NaN scores have a weight that is NaN and no maximum
    const float w = ml[v].y != ml[v].y ? ml[v].y : ml[v].y != 0.f ? __builtin_amdgcn_exp2f(ml[v].x - ref) : 0.f;
    if (i < all) weight[i] = w;
    if (w != 0.f) sum = fmaf(w, ml[v].y, sum);
  }
  for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
  if ((tid & 63) == 0) red[4 + (tid >> 6)] = sum;
  __syncthreads();
  sum = (red[4] + red[5]) + (red[6] + red[7]);
  const int slot = j.s.own.slots ? j.s.own.slots[b] : b;
  const int own = (int)((int64_t)slot_rows(j.s.prefix, j.s.prefix_slot) + slot_rows(j.s.own, slot) - 1);
  int lo, hi;
  seen_by(j.s.rules, b, own, own + 1, lo, hi);
  const bool sees = lo <= hi;
  for (int col = tid * 4; col < j.s.dl; col += 1024) {
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < all; ++i) {
      const float w = weight[i];
      if (w == 0.f) continue;
      const float *from = i < S ? j.r.pacc + shared_at(i) * j.s.dl : j.s.pacc + own_at(i - S) * j.s.dl;
      const f32x4 p = *reinterpret_cast<const f32x4 *>(from + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(w, p[e], v[e]);
    }
    T *to = (T *)j.l_out + ((int64_t)b * j.s.nq + g) * j.s.dl + col;
    const float inv = 1.f / sum;   // (sees something: NaN where all scores are -infinity or one is NaN)
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = (T)(sees ? v[e] * inv : 0.f);
  }
}

// How own rows are cut: which maps and columns a workgroup has, rows of a tile, pieces of a sequence.
struct StreamPlan { int nf, maps, blocks, heads, rows, stages, pieces, lds; };

StreamPlan stream_plan(const Dims &d, int batch, int max_seq) {
  const int es = d.esize();
  StreamPlan p{};
  p.maps = std::min(d.qpc, 16);
  p.nf = d.dl % 1024 == 0 ? 16 : d.dl % 512 == 0 ? 8 : d.dl % 256 == 0 ? 4 : d.dl % 128 == 0 ? 2 : 1;
  auto heads_of = [&](int maps) {   // key heads that `maps` maps from a multiple of them on lie in at most
    int most = 1;
    for (int c = 0; c < d.nc; ++c)
      for (int i = 0; i < d.qpc; i += maps) {
        const int first = c * d.qpc + i, last = c * d.qpc + std::min(i + maps, d.qpc) - 1;
        most = std::max(most, last / d.qpk - first / d.qpk + 1);
      }
    return most;
  };
  auto row_bytes = [&]() { return (heads_of(p.maps) * d.dh + p.nf * 64) * es; };
  // two tiles of 16 rows of 4 KiB fill the LDS; wider rows in parts of maps or columns, whichever take more of them
  while (row_bytes() > 4096 && (p.maps > 1 || p.nf > 1)) {
    if (p.nf > 1 && (heads_of(p.maps) * d.dh <= p.nf * 64 || p.maps == 1)) p.nf /= 2;
    else p.maps = (p.maps + 1) / 2;
  }
  p.heads = heads_of(p.maps);
  p.blocks = (d.qpc + p.maps - 1) / p.maps;
  const int row = row_bytes();
  p.rows = row <= 2048 ? 32 : 16;
  const int tile = p.rows * row;
  p.stages = tile <= 16384 ? 3 : std::max(2, std::min(4, 155648 / tile));
  p.lds = p.stages * tile;
  const int64_t per = (int64_t)batch * d.nc * p.blocks * (d.dl / (p.nf * 64));
  p.pieces = (int)std::max<int64_t>(1, std::min<int64_t>({(512 + per - 1) / per, (max_seq + 127) / 128, 64}));
  return p;
}

// Prefix: rows of a tile, slices, pieces.
struct PrefixPlan { int bq, mpc, cells, tiles, pieces; };

PrefixPlan prefix_plan(const Dims &d, int batch, int prefix_max) {
  PrefixPlan p{};
  p.mpc = maps_per_cell(d);
  p.cells = d.nq / p.mpc;
  p.bq = d.dtype == GTA_BF16 ? prefix_tile_rows(d, batch * p.mpc) : 32;
  p.tiles = (int)(((int64_t)batch * p.mpc + p.bq - 1) / p.bq);
  const int64_t per = (int64_t)p.tiles * p.cells * (d.dtype == GTA_BF16 ? prefix_slices(d, p.bq) : d.dl / rows_f32_columns(d));
  p.pieces = (int)std::max<int64_t>(1, std::min<int64_t>({(256 + per - 1) / per, ((int64_t)prefix_max + 255) / 256, 256}));
  return p;
}

struct PrefixWs { float *pacc, *oacc; float2 *pml, *oml; size_t bytes; };

PrefixWs carve_prefix(const Dims &d, int batch, const PrefixPlan &p, const StreamPlan &s, void *base) {
  PrefixWs w{};
  size_t off = 0;
  auto take = [&](size_t n) { void *q = base ? (char *)base + off : nullptr; off += align_up(n); return q; };
  const size_t prows = (size_t)p.tiles * p.pieces * p.cells * p.bq, orows = (size_t)batch * s.pieces * d.nq;
  w.pml = (float2 *)take(prows * 8);
  w.oml = (float2 *)take(orows * 8);
  w.pacc = (float *)take(prows * d.dl * 4);
  w.oacc = (float *)take(orows * d.dl * 4);
  w.bytes = off;
  return w;
}

template <typename T, int DH, int NF>
void launch_stream_of(const StreamArgs &a, int slices, int groups, int lds, hipStream_t st) {
  allow_dynamic_lds((const void *)stream_kernel<T, DH, NF>, lds);
  stream_kernel<T, DH, NF><<<dim3((unsigned)a.pieces, (unsigned)(slices * a.blocks * groups), (unsigned)a.batch), 256, lds, st>>>(a);
}

template <typename T, int DH>
void launch_stream(const StreamArgs &a, int nf, int groups, int lds, hipStream_t st) {
  const int slices = a.dl / (nf * 64);
  switch (nf) {
    case 1: launch_stream_of<T, DH, 1>(a, slices, groups, lds, st); break;
    case 2: launch_stream_of<T, DH, 2>(a, slices, groups, lds, st); break;
    case 4: launch_stream_of<T, DH, 4>(a, slices, groups, lds, st); break;
    case 8: launch_stream_of<T, DH, 8>(a, slices, groups, lds, st); break;
    default: launch_stream_of<T, DH, 16>(a, slices, groups, lds, st);
  }
}

}  // namespace

// Page sizes of a power of two from 16 rows on
static bool pages_ok(const gta_cache &c) { return !c.block_table || (c.page_size >= 16 && !(c.page_size & (c.page_size - 1))); }

bool prefix_tuned(const Dims &d) { return rows_bf16_ok(d) || (rows_f32_ok(d) && d.dh >= 64); }
bool prefix_fits(const Dims &d, int batch, int prefix_max, int max_seq) {
  const int mpc = maps_per_cell(d);
  return prefix_tuned(d) && (int64_t)batch * mpc < (1 << 24) && d.nq <= 512 && (int64_t)d.wk_w * d.esize() * 32 < (1 << 30) &&
         (int64_t)d.wc_w * d.esize() * 32 < (1 << 30);
}

size_t prefix_bytes(const Dims &d, int batch, int prefix_max, int max_seq) {
  if (!prefix_fits(d, batch, prefix_max, max_seq)) return 0;
  return carve_prefix(d, batch, prefix_plan(d, batch, prefix_max), stream_plan(d, batch, max_seq), nullptr).bytes;
}

bool prefix_layout_ok(const gta_cache &prefix, const gta_cache &own) { return pages_ok(prefix) && pages_ok(own); }

int launch_prefix(const Dims &d, const PrefixArgs &x, void *ws, hipStream_t st) {
  const PrefixPlan p = prefix_plan(d, x.batch, x.prefix.max_seq);
  const StreamPlan s = stream_plan(d, x.batch, x.own.max_seq);
  const PrefixWs w = carve_prefix(d, x.batch, p, s, ws);
  auto shift_of = [](const PageMap &pm) { int n = 0; while (pm.table && (1 << n) < pm.page_size) ++n; return n; };
  RowsArgs r{};
  r.q = x.q; r.k = x.prefix.k; r.c = x.prefix.c; r.qs = d.wq_w; r.ks = d.wk_w; r.cs = d.wc_w; r.batch = x.batch;
  r.nq = d.nq; r.mpc = p.mpc; r.cells = p.cells; r.kdiv = d.qpk / p.mpc; r.cdiv = d.qpc / p.mpc; r.dl = d.dl; r.rules = x.rules;
  r.tiles = p.tiles * p.pieces; r.pacc = w.pacc; r.pml = w.pml; r.prefix = x.prefix; r.own = x.own; r.prefix_slot = x.prefix_slot;
  r.pieces = p.pieces; r.ps_shift = shift_of(x.prefix.pm);
  if (d.dtype == GTA_BF16) launch_prefix_rows(d, r, p.bq, st);
  else launch_rows_f32(d, r, true, st);
  StreamArgs a{};
  a.q = x.q; a.prefix = x.prefix; a.own = x.own; a.prefix_slot = x.prefix_slot; a.batch = x.batch; a.nq = d.nq; a.qpk = d.qpk; a.qpc = d.qpc;
  a.dh = d.dh; a.dl = d.dl; a.kw = d.wk_w; a.cw = d.wc_w; a.rules = x.rules; a.maps = s.maps; a.blocks = s.blocks; a.heads = s.heads;
  a.pieces = s.pieces; a.ps_shift = shift_of(x.own.pm); a.rows = s.rows; a.stages = s.stages;
  a.k_instr = s.rows * s.heads * d.dh * d.esize() / 1024; a.instr = a.k_instr + s.rows * s.nf * 64 * d.esize() / 1024;
  a.stage_bytes = a.instr * 1024; a.pacc = w.oacc; a.pml = w.oml;
  if (d.dtype == GTA_BF16) {
    if (d.dh == 64) launch_stream<__bf16, 64>(a, s.nf, d.nc, s.lds, st);
    else launch_stream<__bf16, 128>(a, s.nf, d.nc, s.lds, st);
  } else {
    if (d.dh == 64) launch_stream<float, 64>(a, s.nf, d.nc, s.lds, st);
    else launch_stream<float, 128>(a, s.nf, d.nc, s.lds, st);
  }
  const JoinArgs j{a, r, p.bq, x.l_out};
  const dim3 grid((unsigned)x.batch, (unsigned)d.nq);
  if (d.dtype == GTA_BF16) prefix_join_kernel<__bf16><<<grid, 256, 0, st>>>(j);
  else prefix_join_kernel<float><<<grid, 256, 0, st>>>(j);
  return check_launch();
}

}  // namespace gta
