// One new token per sequence over a prefix that the batch shares and over the sequence's own cached rows, with rules on the scores
// (gta_score_rules):
//   1. the prefix is read once for all: the batch's queries are the rows of rows_attn_kernel (bf16) and rows_attn_f32_kernel, which
//      leave averages over pieces of the prefix;
//   2. stream_kernel reads every sequence's own rows once for all its maps, in pieces, too;
//   3. prefix_join_kernel weighs the averages by what their pieces count.
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
  int prefix_slot, batch, nq, qpk, qpc, dl, kw, cw;
  Rules rules;
  int maps, blocks;            // maps of a workgroup, workgroups of a latent group's maps
  int heads;                   // key heads that a workgroup's maps read at most
  int wave_lds, ps_shift;      // bytes of a wave
  int share, each;             // workgroups that a batch's tiles are shared out to; or (> 0) pieces of every sequence
  int32_t *first;              // [batch + 1] pieces in front of each sequence
  float *pacc; float2 *pml;    // averages [pieces, n_q, d_l], maximum and weight [pieces, n_q]
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
// Sequences of a batch whose tiles are shared out evenly, a lane each.  Shared out / in as many pieces for every sequence: 64 of 20 to 1500 rows of the
// 1B shape 36 / 43 us, 20 to 4096 66 / 75, 4096 each 111 / 114, 32 of the wide shape 73 / 95; 64 of the paper's layer 22 / 21.
constexpr int kShared = 64;

// Rows lo .. hi of the sequence itself that its new token sees (none: hi < lo); n of them are cached, `own` is the token's position
__device__ __forceinline__ void own_rows(const StreamArgs &a, int b, int &slot, int &n, int &own, int &lo, int &hi) {
  slot = a.own.slots ? a.own.slots[b] : b;
  const int P = slot_rows(a.prefix, a.prefix_slot);
  n = slot_rows(a.own, slot);
  own = (int)((int64_t)P + n - 1);
  seen_by(a.rules, b, own, own + 1, lo, hi);
  lo = max(lo - P, 0);
  hi -= P;
}


// inclusive sums over the lanes of a wave
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast 15, 31
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// Pieces in front of and of sequence b (lane b) and how many there are, where a batch is shared out: a round is what a workgroup's
// waves take at a time, and T rounds make a piece, T the least of a growing series with which there are no more pieces than
// workgroups, all at once on the chip.  (With more than half as many sequences as those, there may be no such T: about twice as many pieces
// then, dealt out as workgroups end.)
template <int NWV>
__device__ __forceinline__ int share_out(const StreamArgs &a, int &before, int &mine) {
  const int b = threadIdx.x & 63;
  int rounds = 0;
  if (b < a.batch) {
    int slot, n, own, lo, hi;
    own_rows(a, b, slot, n, own, lo, hi);
    if (lo <= hi) rounds = min(((hi >> 4) - (lo >> 4) + NWV) / NWV, 1 << 24);   // (64 of them fit 32 bits)
  }
  const int total = __builtin_amdgcn_readlane(wave_scan(rounds), 63), some = __popcll(__ballot(rounds > 0));
  int t = max(1, (total + a.share - 1) / a.share);
  if (2 * some > a.share) t = max(1, (total + 2 * a.share - 1) / (2 * a.share));
  else
#pragma unroll 1
    while (__builtin_amdgcn_readlane(wave_scan((rounds + t - 1) / t), 63) > a.share) t += (t + 7) / 8;
  mine = (rounds + t - 1) / t;
  const int run = wave_scan(mine);
  before = run - mine;
  return __builtin_amdgcn_readlane(run, 63);
}

// A workgroup has a piece of one sequence's rows, up to 16 maps of one latent group and SW = NF * 64 of its latent columns.  A wave takes
// tiles of 16 rows, keys and latents, by itself: they go from memory straight into LDS of its own, the next tile's keys as this
// one's have been read, its latents likewise, so that about a tile per wave is on its way at any time, and no barrier is met before the
// waves' sums are joined.
//   S[row][map] = K q^T: lane (x = l % 16, h = l / 16) ends up with map x, rows 4 h .. 4 h + 3 (of each key head; its own is kept);
//   L[column][map] += C^T p: which is what the second operand wants from that lane.
// Bound by memory: every row is read once (once per block of maps or slice where a layer's rows are wider than 4 KiB, then from L2).
// 64 sequences of 20 to 1500 rows of 2 KiB 20.0 us, 5 TB/s; 32 of 100 to 4000 rows of 4 KiB in pages of 64 62 us, 4.6 TB/s; a few short ones 5 us,
// a chain of lengths, page, keys, latents and the waves' join.
// bf16 weights are rounded for the second product, as in the kernel of the prefix, and so is their sum.  (Two parts of 16 bits would
// cost nothing here, but an infinite latent times the second, which may be 0 or less, is no infinity.)
// Sums of finite latents may pass the range: a workgroup whose averages are not finite in the end goes through its tiles once more, with
// weights that are lowered by a power of two so that they are at most 1 in all.  (Lowered from the start, they lose what large latents of
// little weight count: those below 2^(lift - 126), lift 25 for 32768 rows.)
// Rows in front of the first that is seen are cleared in LDS, rows behind the last read as zeros: what is masked has the weight 0, and
// that times a latent that is not finite would not be.
template <typename T, int DH, int NF, int NWV>
__global__ __launch_bounds__(NWV * 64, NF >= 8 ? 1 : 2) void stream_kernel(StreamArgs a) {
  constexpr int ES = sizeof(T), KS = DH * ES / 64, KCH = DH * ES / 16;   // 64-byte steps and 16-byte chunks of a key head
  constexpr int SW = NF * 64, CP = SW * ES, CCH = CP / 16, NFR = NF * 4;  // latent columns, their bytes and chunks a row, blocks of 16
  constexpr int PM = CCH / 2 < 8 ? CCH / 2 - 1 : 7;                      // pairs of chunks that rows are swapped over (bf16)
  constexpr int KI = KCH / 4, CI = CCH / 4;                              // load instructions (1 KiB) of a head's, of the latents' 16 rows
  constexpr int KR = 64 / KCH, CR = CCH < 64 ? 64 / CCH : 1;             // rows of an instruction
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float2 stats[NWV][16];
  const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int slices = a.dl / SW, slice = blockIdx.y % slices, rest = blockIdx.y / slices, block = rest % a.blocks, cgrp = rest / a.blocks;
  const int g0 = cgrp * a.qpc + block * a.maps, gn = min(a.maps, a.qpc - block * a.maps);   // maps g0 .. g0 + gn - 1
  const int kh0 = g0 / a.qpk, heads = (g0 + gn - 1) / a.qpk - kh0 + 1;
  int b, piece, pieces;
  const int id = blockIdx.x;
  if (a.each) {
    b = id / a.each; piece = id - b * a.each; pieces = a.each;
    if (id == 0 && blockIdx.y == 0)
      for (int i = tid; i <= a.batch; i += NWV * 64) a.first[i] = i * a.each;
  } else {
    int before, mine;
    const int all = share_out<NWV>(a, before, mine);
    if (id == 0 && blockIdx.y == 0 && tid <= a.batch) a.first[tid] = tid < a.batch ? before : all;   // (a.batch < 64 or this lane has `all`)
    if (id == 0 && blockIdx.y == 0 && tid == 0) a.first[a.batch] = all;
    if (id >= all) return;
    b = 63 - __builtin_clzll(__ballot(lane < a.batch && mine > 0 && before <= id));
    piece = id - __shfl(before, b);
    pieces = __shfl(mine, b);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  piece = __builtin_amdgcn_readfirstlane(piece);
  pieces = __builtin_amdgcn_readfirstlane(pieces);
  int slot, n, own, lo, hi;
  own_rows(a, b, slot, n, own, lo, hi);
  slot = __builtin_amdgcn_readfirstlane(slot);
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  n = __builtin_amdgcn_readfirstlane(n);
  const int64_t at = (int64_t)id * a.nq + g0;
  const int t_lo = lo >> 4, tiles = hi < lo ? 0 : (hi >> 4) - t_lo + 1;
  const int t0 = t_lo + (int)((int64_t)tiles * piece / pieces), t1 = t_lo + (int)((int64_t)tiles * (piece + 1) / pieces);
  if (t0 >= t1) {
    if (slice == 0 && tid < gn) a.pml[at + tid] = make_float2(-INFINITY, -1.f);
    return;
  }
  const int g = min(g0 + x, g0 + gn - 1), head = g / a.qpk - kh0;   // this lane's map (lanes without one repeat the last)
  const float slope = a.rules.slopes ? a.rules.slopes[g] : 0.f;

  const int32_t *table = a.own.pm.table ? a.own.pm.table + (int64_t)slot * a.own.pm.pages_per_slot : nullptr;
  const int64_t row0 = table ? 0 : (int64_t)slot * a.own.max_seq;
  const char *Kb = (const char *)((const T *)a.own.k + row0 * a.kw + (int64_t)kh0 * DH);
  const char *Cb = (const char *)((const T *)a.own.c + row0 * a.cw + (int64_t)cgrp * a.dl + slice * SW);
  const unsigned kws = (unsigned)a.kw * ES, cws = (unsigned)a.cw * ES;

  // Slot s of a row in LDS holds its chunk s, swapped with others so that 16 rows' reads of one chunk fall into different banks: keys
  // s ^ (row % 8), bf16 latents pairs of chunks ^ row, fp32 latents blocks of four chunks ^ row / 4.  A lane's part of that and of the
  // offset here, an instruction's where it is issued.
  const unsigned klane = (lane / KCH) * kws, kchunk = lane % KCH ^ (lane / KCH & 7);
  const int clr = CCH < 64 ? lane / CCH : 0;
  const unsigned clane = clr * cws, cchunk = (CCH < 64 ? lane % CCH : lane) ^ (ES == 2 ? (clr & PM) * 2 : 0);
  char *mem = smem + wave * a.wave_lds;
  const unsigned klds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)mem, clds = klds + a.heads * KI * 1024;
  const char *kmem = mem;
  char *cmem = mem + a.heads * KI * 1024;
  int64_t p0 = 0;   // pool row of the tile in work on
  auto find = [&](int t) {   // its 16 rows lie in one page
    const int j = min(t * 16, hi & ~15);
    if (!table) return (int64_t)j;
    int pg = load_uniform(table + __builtin_amdgcn_readfirstlane(j >> a.ps_shift));
    pg = (unsigned)pg >= (unsigned)a.own.pm.num_pages ? 0 : pg;
    return ((int64_t)pg << a.ps_shift) + (j & (a.own.pm.page_size - 1));
  };
  auto rows_of = [&](int t) { return t < t1 ? min(hi + 1 - t * 16, 16) : 0; };
  auto issue_k = [&](int t) __attribute__((always_inline)) {
    const int rows = rows_of(t);
    const u32x4 r = uniform_buffer_of(Kb + p0 * kws, rows > 0 ? (rows - 1) * kws + heads * DH * ES : 0u);
    unsigned to = klds;
#pragma unroll 1
    for (int kk = 0; kk < heads; ++kk) {
#pragma unroll
      for (int i = 0; i < KI; ++i, to += 1024) load_to_lds(r, klane + (kchunk ^ (i * KR & 7)) * 16 + (i * KR * kws + kk * DH * ES), to);
    }
  };
  auto issue_c = [&](int t) __attribute__((always_inline)) {
    const int rows = rows_of(t);
    const u32x4 r = uniform_buffer_of(Cb + p0 * cws, rows > 0 ? (rows - 1) * cws + CP : 0u);
#pragma unroll
    for (int i = 0; i < CI; ++i) {
      const int row = CCH <= 64 ? i * CR : i / (CCH / 64), sub = CCH <= 64 ? 0 : i % (CCH / 64);
      const unsigned swap = ES == 2 ? (row & PM) * 2 : (row >> 2 & 3) * 4;
      load_to_lds(r, clane + (cchunk ^ swap) * 16 + (row * cws + sub * 1024), clds + i * 1024);
    }
  };

  f32x4 qf[KS];   // 64 bytes' worth of a step, 16 of them per lane
  {
    const f32x4 *qp = reinterpret_cast<const f32x4 *>((const T *)a.q + ((int64_t)b * a.nq + g) * DH) + h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = qp[ks * 4];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
  }
  f32x4 acc[NFR];
#pragma unroll
  for (int f = 0; f < NFR; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f, lift = 0.f;   // lift: by how many powers of two weights are lowered
  while (true) {
    int t = t0 + wave;
    p0 = find(t);
    issue_k(t);
    issue_c(t);
#pragma unroll 1
    for (; t < t1; t += NWV) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CI) : "memory");   // the keys are there
      f32x4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int kk = 0; kk < heads; ++kk) {
        const char *kr = kmem + kk * KI * 1024 + x * KCH * 16;
        f32x4 d{0.f, 0.f, 0.f, 0.f}, kf[KS], part[3];   // fp32: four sums of a quarter of the products each, off by half as much as one
        if constexpr (ES == 4) part[0] = part[1] = part[2] = d;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = *reinterpret_cast<const f32x4 *>(kr + ((ks * 4 + h) ^ (x & 7)) * 16);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          if constexpr (ES == 2) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[ks]), __builtin_bit_cast(bf16x8, qf[ks]), d, 0, 0, 0);
          else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              f32x4 &to = e == 0 ? d : part[e - 1];
              to = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[ks][e], qf[ks][e], to, 0, 0, 0);
            }
          }
        }
        if constexpr (ES == 4) d = (d + part[0]) + (part[1] + part[2]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = head == kk ? d[e] : s[e];
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // and have been read
      p0 = find(t + NWV);
      issue_k(t + NWV);
      const int j0 = t * 16;
      float p[4], mt = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = j0 + 4 * h + e;
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
        for (int f = 0; f < NFR; ++f) acc[f] *= corr;
      }
      m = mn;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = __builtin_amdgcn_exp2f(p[e] - (ref + lift));
        if constexpr (ES == 2) p[e] = (float)(__bf16)p[e];
        l += p[e];
      }
      wait_loads(heads * KI);                                      // the latents are there
      if (j0 < lo) {   // clear what is in front of the first row
        for (int i = lane; i < (lo - j0) * CCH; i += 64) *reinterpret_cast<u32x4 *>(cmem + i * 16) = u32x4{0u, 0u, 0u, 0u};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      if constexpr (ES == 2) {
        bf16x4 p1;
#pragma unroll
        for (int e = 0; e < 4; ++e) p1[e] = (__bf16)p[e];
        const int row = 4 * h + (x >> 2);
        const char *cr = cmem + row * CP + (x & 1) * 8 + (x >> 1 & 1) * 16;
#pragma unroll
        for (int f = 0; f < NFR; ++f) {   // 16 columns are a pair of chunks
          const s16x4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(cr + (f ^ (row & PM)) * 32));
          acc[f] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(c, __builtin_bit_cast(s16x4, p1), acc[f], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int f = 0; f < NFR; ++f)     // and a block of 64 bytes
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float c = *reinterpret_cast<const float *>(cmem + (4 * h + e) * CP + (f ^ h) * 64 + x * 4);
            acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(c, p[e], acc[f], 0, 0, 0);
          }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      issue_c(t + NWV);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    int id0 = tid;
    asm volatile("" : "+v"(id0));   // (addresses of what follows are worked out here and not kept through the tiles)
    // join the waves' sums: [map][column] in each one's LDS
    const int xo = id0 & 15, ho = id0 >> 4 & 3;
    if (ho == 0) stats[wave][xo] = make_float2(m + lift, l);
#pragma unroll
    for (int f = 0; f < NFR; ++f) *reinterpret_cast<f32x4 *>(mem + xo * (SW * 4) + ((f * 16 + 4 * ho) ^ (xo & 7) * 4) * 4) = acc[f];
    __syncthreads();
    bool odd = false;   // an average is not finite
    for (int i = id0; i < gn * (SW / 4); i += NWV * 64) {
      const int map = i / (SW / 4), col = i % (SW / 4) * 4;
      float mx = -INFINITY;
#pragma unroll
      for (int w = 0; w < NWV; ++w) mx = fmaxf(mx, stats[w][map].x);
      const float ref = mx > -INFINITY ? mx : 0.f;
      f32x4 v{0.f, 0.f, 0.f, 0.f};
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < NWV; ++w) {
        const float2 ml = stats[w][map];
        const float wt = ml.y != ml.y ? ml.y : __builtin_amdgcn_exp2f(ml.x - ref);
        const f32x4 c = *reinterpret_cast<const f32x4 *>(smem + w * a.wave_lds + map * (SW * 4) + (col ^ (map & 7) * 4) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(wt, c[e], v[e]);
        sum = fmaf(wt, ml.y, sum);
      }
      const float inv = sum == 0.f ? 0.f : ES == 4 ? 1.f / sum : __builtin_amdgcn_rcpf(sum);
      *reinterpret_cast<f32x4 *>(a.pacc + (at + map) * a.dl + slice * SW + col) = v * inv;
      if (slice == 0 && col == 0) a.pml[at + map] = make_float2(mx, sum);
      odd |= (v[0] * 0.f + v[1] * 0.f) + (v[2] * 0.f + v[3] * 0.f) != 0.f;
    }
    if (__builtin_expect(!__syncthreads_or(odd) || lift > 0.f, 1)) return;
    lift = kLazy + 5.f + (float)(32 - __builtin_clz(t1 - t0));   // 2^(lift - kLazy) > 16 (t1 - t0): the waves' sums together are below the largest latent
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int f = 0; f < NFR; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

struct JoinArgs {
  StreamArgs s;
  RowsArgs r;      // the prefix's pieces
  int bq;
  void *l_out;
};

// One (sequence, map) and 128 of its columns: the averages of the prefix's and the sequence's own pieces, weighed by weight * 2^(maximum -
// the largest).  Eight groups of 32 lanes take every eighth piece, four columns a lane, so that most of what is read is asked for at once.
// Bound by latency: 4.7 us for two sequences, 6.8 for 64 of the 1B shape with 32 pieces of the prefix each.
constexpr int kMaxPieces = 1280;   // 256 of the prefix, 4 workgroups per CU
template <typename T>
__global__ __launch_bounds__(256) void prefix_join_kernel(JoinArgs j) {
  __shared__ float weight[kMaxPieces];
  __shared__ float red[8];
  __shared__ f32x4 part[8][32];
  const int b = blockIdx.x, g = blockIdx.y, tid = threadIdx.x, S = j.r.pieces;
  const int first = j.s.first[b], all = min(S + j.s.first[b + 1] - first, kMaxPieces);
  const int cell = g / j.r.mpc, row = b * j.r.mpc + g % j.r.mpc, tile = row / j.bq;
  auto shared_at = [&](int i) { return ((int64_t)(tile * S + i) * j.r.cells + cell) * j.bq + row % j.bq; };
  auto own_at = [&](int i) { return (int64_t)(first + i) * j.s.nq + g; };
  float mx = -INFINITY;
  float2 ml[kMaxPieces / 256];
#pragma unroll
  for (int v = 0; v < kMaxPieces / 256; ++v) {
    const int i = v * 256 + tid;
    ml[v] = make_float2(-INFINITY, -1.f);
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
    // a piece that sees nothing has left no averages (weight -1); one of weight 0 takes part: its averages may not be finite.  NaN scores
    // have a weight that is NaN and no maximum
    const bool none = ml[v].y < 0.f;
    const float w = ml[v].y != ml[v].y ? ml[v].y : none ? -1.f : __builtin_amdgcn_exp2f(ml[v].x - ref) * ml[v].y;
    if (i < all) weight[i] = w;
    if (!none) sum += w;
  }
  for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
  if ((tid & 63) == 0) red[4 + (tid >> 6)] = sum;
  __syncthreads();
  sum = (red[4] + red[5]) + (red[6] + red[7]);
  const float inv = __builtin_amdgcn_rcpf(sum);   // (something is seen: NaN in the end where all scores are -infinity or one is NaN)
  const int group = tid >> 5, col = blockIdx.z * 128 + (tid & 31) * 4;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
  if (col < j.s.dl) {
#pragma unroll 4
    for (int i = group; i < all; i += 8) {
      const float w = weight[i];
      const float *from = i < S ? j.r.pacc + shared_at(i) * j.s.dl : j.s.pacc + own_at(i - S) * j.s.dl;
      if (!(w < 0.f)) {
        const f32x4 p = *reinterpret_cast<const f32x4 *>(from + col);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(w * inv, p[e], v[e]);   // (averages: a sum of them may pass the range)
      }
    }
  }
  part[group][tid & 31] = v;
  __syncthreads();
  if (group || col >= j.s.dl) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) v += part[i][tid];
  int slot, n, own, lo, hi;
  own_rows(j.s, b, slot, n, own, lo, hi);
  seen_by(j.s.rules, b, own, own + 1, lo, hi);
  T *to = (T *)j.l_out + ((int64_t)b * j.s.nq + g) * j.s.dl + col;
#pragma unroll
  for (int e = 0; e < 4; ++e) to[e] = (T)(lo <= hi ? v[e] : 0.f);
}

// How own rows are cut: which maps and columns a workgroup has, its waves and their LDS, pieces.
constexpr int kFour = 38 * 1024, kThree = 50 * 1024;   // LDS of a wave that four, three of a workgroup have room for
struct StreamPlan { int nf, maps, blocks, heads, waves, wave_lds, share, each, grid; };

StreamPlan stream_plan(const Dims &d, int batch, int max_seq) {
  const int es = d.esize();
  StreamPlan p{};
  p.maps = std::min(d.qpc, 16);
  p.nf = d.dl % 512 == 0 ? 8 : d.dl % 256 == 0 ? 4 : d.dl % 128 == 0 ? 2 : 1;
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
  p.wave_lds = std::max(16 * row_bytes(), 16 * p.nf * 64 * 4);   // a tile; the wave's sums in the end
  p.waves = p.wave_lds > kThree ? 2 : p.wave_lds > kFour ? 3 : 4;
  const int per = d.nc * p.blocks * (d.dl / (p.nf * 64)), at_once = std::min(4, 160 * 1024 / (p.waves * p.wave_lds + 1024));
  if (batch <= kShared) {
    p.share = std::max(1, 256 * std::max(at_once, 1) / per);
    p.grid = 2 * batch > p.share ? 2 * p.share + batch : p.share;
    const int64_t most = (int64_t)batch * ((max_seq + 15) / 16);   // pieces of a tile each
    p.grid = (int)std::min<int64_t>(p.grid, most);
  } else {
    p.each = (int)std::max<int64_t>(1, std::min<int64_t>((512 + (int64_t)batch * per - 1) / ((int64_t)batch * per), (max_seq + 127) / 128));
    p.grid = batch * p.each;
  }
  return p;
}

// Prefix: rows of a tile, slices, pieces, 256 in all, of 128 rows at least.  With 512 and with 128 in all: 64 sequences of the 1B shape behind 8192
// rows 35.6 us (512: 37.3, 128: 36.2), 256 46.7 (52.4, 56.3), 32 of the wide shape behind 32768 80 (85, 120), fp32 64 of the paper's layer behind 2048
// 24.1 (24.1, 27.1), two in bf16 behind 32768 28.5 (28.3, 25.1).
struct PrefixPlan { int bq, mpc, cells, tiles, pieces; };

PrefixPlan prefix_plan(const Dims &d, int batch, int prefix_max) {
  PrefixPlan p{};
  p.mpc = maps_per_cell(d);
  p.cells = d.nq / p.mpc;
  p.bq = d.dtype == GTA_BF16 ? prefix_tile_rows(d, batch * p.mpc) : 32;
  p.tiles = (int)(((int64_t)batch * p.mpc + p.bq - 1) / p.bq);
  const int64_t per = (int64_t)p.tiles * p.cells * (d.dtype == GTA_BF16 ? prefix_slices(d, p.bq, prefix_max) : d.dl / rows_f32_columns(d));
  p.pieces = (int)std::max<int64_t>(1, std::min<int64_t>({(256 + per - 1) / per, ((int64_t)prefix_max + 127) / 128, 256}));
  return p;
}

struct PrefixWs { float *pacc, *oacc; float2 *pml, *oml; int32_t *first; size_t bytes; };

// prows: rows of pieces of the prefix in all cells; opieces: pieces of own rows
PrefixWs carve_prefix(const Dims &d, int batch, size_t prows, size_t opieces, void *base) {
  PrefixWs w{};
  size_t off = 0;
  auto take = [&](size_t n) { void *q = base ? (char *)base + off : nullptr; off += align_up(n); return q; };
  const size_t orows = opieces * d.nq;
  w.first = (int32_t *)take(((size_t)batch + 1) * 4);
  w.pml = (float2 *)take(prows * 8);
  w.oml = (float2 *)take(orows * 8);
  w.pacc = (float *)take(prows * d.dl * 4);
  w.oacc = (float *)take(orows * d.dl * 4);
  w.bytes = off;
  return w;
}
PrefixWs carve_prefix(const Dims &d, int batch, const PrefixPlan &p, const StreamPlan &s, void *base) {
  return carve_prefix(d, batch, (size_t)p.tiles * p.pieces * p.cells * p.bq, (size_t)s.grid, base);
}

// (false: nothing was launched)
template <typename T, int DH, int NF>
bool launch_stream_of(const StreamArgs &a, const StreamPlan &p, unsigned y, hipStream_t st) {
  auto run = [&](auto kernel) {
    allow_dynamic_lds((const void *)kernel, p.waves * p.wave_lds);
    kernel<<<dim3((unsigned)p.grid, y), p.waves * 64, p.waves * p.wave_lds, st>>>(a);
    return true;
  };
  // what stream_plan comes to: one key head leaves room for four waves but in fp32 rows of 128 + 512, sixteen may take it
  constexpr int LEAST = 16 * (DH + NF * 64) * (int)sizeof(T), MOST = std::min(16 * (16 * DH + NF * 64) * (int)sizeof(T), 65536);
  if constexpr (LEAST <= kFour) {
    if (p.waves == 4) return run(stream_kernel<T, DH, NF, 4>);
  }
  if constexpr (MOST > kFour) {
    if (p.waves == 3) return run(stream_kernel<T, DH, NF, 3>);
  }
  if constexpr (MOST > kThree) {
    if (p.waves == 2) return run(stream_kernel<T, DH, NF, 2>);
  }
  return false;
}

template <typename T, int DH>
bool launch_stream(const StreamArgs &a, const StreamPlan &p, int groups, hipStream_t st) {
  const unsigned y = (unsigned)(a.dl / (p.nf * 64) * p.blocks * groups);
  switch (p.nf) {
    case 1:
      if constexpr (DH == 64 || sizeof(T) == 4) return launch_stream_of<T, DH, 1>(a, p, y, st);   // bf16 heads of 128 have latents in units of 128
      return false;
    case 2: return launch_stream_of<T, DH, 2>(a, p, y, st);
    case 4: return launch_stream_of<T, DH, 4>(a, p, y, st);
    default: return launch_stream_of<T, DH, 8>(a, p, y, st);
  }
}

}  // namespace

// Page sizes of a power of two from 16 rows on
static bool pages_ok(const gta_cache &c) { return !c.block_table || (c.page_size >= 16 && !(c.page_size & (c.page_size - 1))); }

bool prefix_tuned(const Dims &d) { return rows_bf16_ok(d) || (rows_f32_ok(d) && d.dh >= 64); }
// sequences that a launch takes
static int most_sequences(const Dims &d) {
  const bool any = prefix_tuned(d) && d.nq <= 512 && (int64_t)d.wk_w * d.esize() * 32 < (1 << 30) && (int64_t)d.wc_w * d.esize() * 32 < (1 << 30);
  return any ? ((1 << 24) - 1) / maps_per_cell(d) : 0;
}
bool prefix_fits(const Dims &d, int batch) { return batch <= most_sequences(d); }

size_t prefix_bytes(const Dims &d, int batch, int prefix_max, int max_seq) {
  if (!prefix_fits(d, batch)) return 0;
  return carve_prefix(d, batch, prefix_plan(d, batch, prefix_max), stream_plan(d, batch, max_seq), nullptr).bytes;
}

// What is enough for any batch of up to `batch` sequences (as many of them as a launch takes): fewer may be cut into more pieces, or into larger tiles' worth of them.
size_t prefix_bytes_up_to(const Dims &d, int batch, int prefix_max, int max_seq) {
  batch = std::min(batch, most_sequences(d));
  if (!batch) return 0;
  const int mpc = maps_per_cell(d);
  size_t prows = 0;
  for (int rows : {32, 64, INT_MAX}) {   // where prefix_tile_rows changes
    const int b = std::min(batch, rows / mpc);
    if (b == 0) continue;
    const PrefixPlan p = prefix_plan(d, b, prefix_max);
    const size_t tiles = (size_t)p.tiles * p.cells, slices = d.dtype == GTA_BF16 ? prefix_slices(d, p.bq, prefix_max) : d.dl / rows_f32_columns(d);
    prows = std::max(prows, std::min(tiles + 256 / slices, tiles * std::max<size_t>(1, ((size_t)prefix_max + 127) / 128)) * p.bq);
  }
  const StreamPlan s = stream_plan(d, batch, max_seq);
  size_t opieces = (size_t)s.grid;
  if (batch > kShared) {
    const size_t per = (size_t)d.nc * s.blocks * (d.dl / (s.nf * 64));
    opieces = std::max<size_t>(opieces, std::min<size_t>(512 / per + batch, (size_t)batch * (((size_t)max_seq + 127) / 128)));
    opieces = std::max<size_t>(opieces, (size_t)stream_plan(d, kShared, max_seq).grid);
  }
  return std::max(carve_prefix(d, batch, prows, opieces, nullptr).bytes, prefix_bytes(d, batch, prefix_max, max_seq));
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
  else if (!launch_rows_f32(d, r, true, st)) return GTA_ERR_UNSUPPORTED;
  StreamArgs a{};
  a.q = x.q; a.prefix = x.prefix; a.own = x.own; a.prefix_slot = x.prefix_slot; a.batch = x.batch; a.nq = d.nq; a.qpk = d.qpk; a.qpc = d.qpc;
  a.dl = d.dl; a.kw = d.wk_w; a.cw = d.wc_w; a.rules = x.rules; a.maps = s.maps; a.blocks = s.blocks; a.heads = s.heads;
  a.wave_lds = s.wave_lds; a.ps_shift = shift_of(x.own.pm); a.share = s.share; a.each = s.each; a.first = w.first; a.pacc = w.oacc; a.pml = w.oml;
  bool streamed;
  if (d.dtype == GTA_BF16) streamed = d.dh == 64 ? launch_stream<__bf16, 64>(a, s, d.nc, st) : launch_stream<__bf16, 128>(a, s, d.nc, st);
  else streamed = d.dh == 64 ? launch_stream<float, 64>(a, s, d.nc, st) : launch_stream<float, 128>(a, s, d.nc, st);
  if (!streamed) return GTA_ERR_UNSUPPORTED;   // the join would read piece counts that nobody has written
  const JoinArgs j{a, r, p.bq, x.l_out};
  const dim3 grid((unsigned)x.batch, (unsigned)d.nq, (unsigned)((d.dl + 127) / 128));
  if (d.dtype == GTA_BF16) prefix_join_kernel<__bf16><<<grid, 256, 0, st>>>(j);
  else prefix_join_kernel<float><<<grid, 256, 0, st>>>(j);
  return check_launch();
}

}  // namespace gta
