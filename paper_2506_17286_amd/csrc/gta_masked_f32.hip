// fp32 attention of rows of queries with rules on their scores, on fp32 matrix instructions (gta_rows_attn.h): a workgroup has a tile
// of 32 rows and up to 128 latent columns, its four waves every fourth block of 32 keys each, with statistics and sums of their own
// that are joined in LDS at the end.  Both products are transposed, S^T = K Q^T and L^T += C^T P^T: weights go from one's
// accumulators into the other.  Keys and latents come from memory straight into registers, the next block's as this one's come free.
// Bound by the matrix instructions (64 cycles for 2048 products) and by how evenly tiles fall on the CUs: 4 x 1024 tokens of the paper's
// layer with a bias 62.5 us a call (64 TFLOP/s of the 153 that a large matrix product reaches), 5.4 of it the list; 640 workgroups, two on a
// CU, and a wave has up to 8 steps between filling its registers and joining its sums.
//
// A masked weight is 0, but 0 times a latent that is not finite is NaN, and sums of finite ones may pass the range: a tile whose sums are not
// finite in the end is gone through once more, row by row, over the keys that each row sees (wave_row).
#include <math.h>

#include "gta_rows_attn.h"

namespace gta {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float pair_max(float v) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int i = 32; i; i >>= 1) v = min(v, __shfl_xor(v, i));
  return __builtin_amdgcn_readfirstlane(v);
}

template <int DH, int DLW, bool CACHE>
__global__ __launch_bounds__(256, DH + DLW < 256 || !CACHE ? 2 : 1) void rows_attn_f32_kernel(RowsArgs a) {
  constexpr int NT = DLW / 32, OP = DLW + 4, BQ = 32;
  // A score's products are added up 32 at a time: one sum over a head of 128 is off by twice as much (one sequence of 3000 keys, error of its
  // row 1.3e-6 and 0.7e-6).  (Two sums where registers are short; four spill 31 of them.)
  // Queries in LDS, so that two workgroups share a CU's registers: 1B shape, 4 x 1024 tokens 268 -> 231 us, 464 tokens 125 -> 105, 60 tokens 13.9 -> 14.8.
  // Not on caches, whose addresses take more of them: 16 sequences of the wide shape behind 8000 rows 114 -> 160.
  constexpr bool QLDS = DH + DLW == 256 && !CACHE;
  constexpr int SUMS = DH == 128 && DLW == 64 ? 2 : DH / 32;
  typedef float cvec __attribute__((ext_vector_type(NT)));
  extern __shared__ __attribute__((aligned(16))) float dyn[];
  float (*lacc)[32][OP] = reinterpret_cast<float (*)[32][OP]>(dyn);   // [4][32][OP]
  __shared__ float sm[4][32], sl[4][32];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, ln = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int per = a.cells * a.slices, u = (int)blockIdx.x / per, r_ = (int)blockIdx.x - u * per;
  int b, tile, piece, pieces, slot;
  if constexpr (CACHE) {
    b = 0; tile = u / a.pieces; piece = u - tile * a.pieces; pieces = a.pieces; slot = tile * a.pieces;
  } else {
    if (a.list) {
      if (u >= a.count[0]) return;
      const Piece e = a.list[u];
      b = e.b; tile = e.tile; piece = e.piece; pieces = e.pieces; slot = e.slot;
    } else {   // every tile of every sequence
      const int lvl = u / a.batch;
      b = u - lvl * a.batch; tile = a.tiles / a.batch - 1 - lvl;
      piece = slot = 0; pieces = 1;
    }
  }
  const int slice = r_ % a.slices, cell = r_ / a.slices;
  int64_t start = 0;
  int Tb = CACHE ? a.batch : a.per_seq, keys;
  if constexpr (CACHE) keys = slot_rows(a.prefix, a.prefix_slot);
  else {
    start = a.cu ? a.cu[b] : (int64_t)b * a.per_seq;
    if (a.cu) Tb = a.cu[b + 1] - (int)start;
    keys = Tb;
  }
  if (!CACHE && tile * BQ >= Tb * a.mpc) return;
  const int R = Tb * a.mpc, r0 = tile * BQ, row = min(r0 + ln, R - 1);   // (rows past the last repeat it and are not stored)
  const int tok = row / a.mpc, g = cell * a.mpc + (row - tok * a.mpc);
  int lo, hi, own;
  if constexpr (CACHE) prefix_seen(a, tok, keys, lo, hi, own);
  else {
    own = tok;
    seen_by(a.rules, start + tok, tok, keys, lo, hi);
  }
  const float slope = a.rules.slopes ? a.rules.slopes[g] : 0.f;
  const bool sees = lo <= hi;
  const int wlo = wave_min(sees ? lo : INT_MAX), whi = -wave_min(sees ? -hi : 1);   // none: whi = -1
  const int base = whi < 0 ? 0 : wlo >> 5, blocks = whi < 0 ? 0 : (whi >> 5) - base + 1;
  const int b0 = base + (int)((int64_t)blocks * piece / pieces), b1 = base + (int)((int64_t)blocks * (piece + 1) / pieces);

  const float *kcol = (const float *)a.k + (cell / a.kdiv) * DH, *ccol = (const float *)a.c + (int64_t)(cell / a.cdiv) * a.dl + slice * DLW;
  const int32_t *table = nullptr;
  int64_t krow0 = start;
  if constexpr (CACHE) {
    krow0 = a.prefix.pm.table ? 0 : (int64_t)a.prefix_slot * a.prefix.max_seq;
    if (a.prefix.pm.table) table = a.prefix.pm.table + (int64_t)a.prefix_slot * a.prefix.pm.pages_per_slot;
  }
  // rows of key j's two runs of 16, less j's own number: key k of the block is row k + (first or second of them).  Keys past the last
  // repeat it; they are masked.
  auto runs = [&](int blk, int64_t &p0, int64_t &p1) {
    if (CACHE && table) {
      const int last = max(keys - 1, 0), j0 = min(blk * 32, last & ~15), j1 = min(j0 + 16, last & ~15);
      auto find = [&](int j) {
        int pg = table[j >> a.ps_shift];
        pg = (unsigned)pg >= (unsigned)a.prefix.pm.num_pages ? 0 : pg;
        return ((int64_t)pg << a.ps_shift) + (j & (a.prefix.pm.page_size - 1)) - j;
      };
      p0 = find(j0);
      p1 = find(j1);
    } else p0 = p1 = krow0;
  };
  f32x4 qf[QLDS ? 1 : DH / 8];
  f32x4 *ql = reinterpret_cast<f32x4 *>(dyn) + lane;   // [DH / 8][64], until the waves are joined
  {
    const float *qp = (const float *)a.q + (start + tok) * a.qs + g * DH + h * 4;
    if constexpr (QLDS) {
#pragma unroll
      for (int c = wave * (DH / 32); c < (wave + 1) * (DH / 32); ++c) ql[c * 64] = *reinterpret_cast<const f32x4 *>(qp + c * 8);
      __syncthreads();
    } else {
#pragma unroll
      for (int c = 0; c < DH / 8; ++c) qf[c] = *reinterpret_cast<const f32x4 *>(qp + c * 8);
    }
  }
  f32x16 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  f32x4 kf[DH / 8];
  cvec cf[16];
  int64_t p0 = 0, p1 = 0;
  // Packed rows: a block's first row is uniform, its rows are within 32 bits of it (heads of 64, 4 x 1024 tokens with a bias 68.4 -> 63.7 us; heads of
  // 128, where registers are shorter, 231 -> 275)
  constexpr bool UNIFORM = !CACHE && DH <= 64;
  const unsigned ks = (unsigned)a.ks, cs = (unsigned)a.cs;
  auto kload = [&](int blk) {
    if constexpr (UNIFORM) {
      const char *base = (const char *)(kcol + (start + blk * 32) * a.ks);
      const unsigned off = ((unsigned)min(ln, keys - 1 - blk * 32) * ks + h * 4) * 4;
#pragma unroll
      for (int c = 0; c < DH / 8; ++c) kf[c] = *reinterpret_cast<const f32x4 *>(base + (off + c * 32));
      return;
    }
    const int key = min(blk * 32 + ln, keys - 1);
    const float *p = kcol + ((ln < 16 || key < blk * 32 + 16 ? p0 : p1) + key) * a.ks + h * 4;
#pragma unroll
    for (int c = 0; c < DH / 8; ++c) kf[c] = *reinterpret_cast<const f32x4 *>(p + c * 8);
  };
  auto cload = [&](int blk, int e) {
    if constexpr (UNIFORM) {
      const char *base = (const char *)(ccol + (start + blk * 32) * a.cs);
      const unsigned off = ((unsigned)min(8 * (e >> 2) + 4 * h + (e & 3), keys - 1 - blk * 32) * cs + ln * NT) * 4;
      cf[e] = *reinterpret_cast<const cvec *>(base + off);
      return;
    }
    const int key = min(blk * 32 + 8 * (e >> 2) + 4 * h + (e & 3), keys - 1);
    cf[e] = *reinterpret_cast<const cvec *>(ccol + ((e < 8 || key < blk * 32 + 16 ? p0 : p1) + key) * a.cs + ln * NT);
  };
  int blk = b1 - 1 - wave;
  if (blk >= b0) {
    runs(blk, p0, p1);
    kload(blk);
#pragma unroll
    for (int e = 0; e < 16; ++e) cload(blk, e);
  }
#pragma unroll 1
  for (; blk >= b0; blk -= 4) {
    const int next = max(blk - 4, b0);   // (behind the last one: loaded, not used)
    f32x16 s;
    if constexpr (QLDS) asm volatile("" ::: "memory");   // the queries are read again in every step
#pragma unroll
    for (int i = 0; i < SUMS; ++i) {
      f32x16 part;
#pragma unroll
      for (int e = 0; e < 16; ++e) part[e] = 0.f;
#pragma unroll
      for (int c = i * (DH / 8 / SUMS); c < (i + 1) * (DH / 8 / SUMS); ++c) {
        f32x4 q;
        if constexpr (QLDS) q = ql[c * 64];
        else q = qf[c];
#pragma unroll
        for (int j = 0; j < 4; ++j) part = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[c][j], q[j], part, 0, 0, 0);
      }
      s = i ? s + part : part;
    }
    runs(next, p0, p1);
    kload(next);
    const int from = lo - blk * 32 - 4 * h, to = hi - blk * 32 - 4 * h;
    const float d0 = (float)(own - blk * 32 - 4 * h);
    float bm = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int key = 8 * (e >> 2) + (e & 3);
      const float v = ruled_score(a.rules, s[e], slope, fabsf(d0 - (float)key));
      s[e] = key < from || key > to ? -INFINITY : v;
      bm = fmaxf(bm, s[e]);
    }
    // the running maximum moves only when a block passes it by 2^8: fp32 weights carry any such scale
    const float mc = pair_max(bm), mn = mc > m + 8.f ? mc : m, ref = mn > -INFINITY ? mn : 0.f;
    const float corr = __builtin_amdgcn_exp2f(m - ref);
    m = mn;
    float ps = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f(s[e] - ref);
      ps += s[e];
    }
    l = fmaf(l, corr, ps);
    if (__builtin_amdgcn_ballot_w64(corr != 1.f) != 0) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= corr;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(cf[e][t], s[e], acc[t], 0, 0, 0);
      cload(next, e);
    }
  }
  // join the waves: tile t, register e of a lane is column (8 (e / 4) + 4 h + e % 4) * NT + t of its row
  l = pair_sum(l);
  if (h == 0) { sm[wave][ln] = m; sl[wave][ln] = l; }
  __syncthreads();
  float mx = sm[0][ln];
#pragma unroll
  for (int w = 1; w < 4; ++w) mx = fmaxf(mx, sm[w][ln]);
  const float ref = mx > -INFINITY ? mx : 0.f, ws = __builtin_amdgcn_exp2f(m - ref);
  const bool used = l != 0.f;   // (NaN too)
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    cvec v;
#pragma unroll
    for (int t = 0; t < NT; ++t) v[t] = used ? acc[t][e] * (l != l ? l : ws) : acc[t][e] * 0.f;   // (sums of weight 0 that are not finite show)
    *reinterpret_cast<cvec *>(&lacc[wave][ln][(8 * (e >> 2) + 4 * h + (e & 3)) * NT]) = v;
  }
  __syncthreads();
  const bool split = CACHE || pieces > 1;
  const int64_t at = ((int64_t)(slot + piece) * a.cells + cell) * BQ;
  auto weight_of = [&](int rr, float &top) {
    top = fmaxf(fmaxf(sm[0][rr], sm[1][rr]), fmaxf(sm[2][rr], sm[3][rr]));
    const float ref = top > -INFINITY ? top : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (sl[w][rr] != 0.f) sum += sl[w][rr] * (sl[w][rr] != sl[w][rr] ? 1.f : __builtin_amdgcn_exp2f(sm[w][rr] - ref));
    return sum;
  };
  bool odd = false;   // a sum is not finite
  constexpr int PER = 32 * (DLW / 4) / 256;   // four columns of a row each
  f32x4 sums[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at4 = i * 256 + tid, rr = at4 / (DLW / 4), col = at4 % (DLW / 4) * 4;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) v += *reinterpret_cast<const f32x4 *>(&lacc[w][rr][col]);
    sums[i] = v;
    odd |= (v[0] * 0.f + v[1] * 0.f) + (v[2] * 0.f + v[3] * 0.f) != 0.f;
  }
  const bool again = __syncthreads_or(odd);
  if (split && slice == 0 && tid < BQ && r0 + tid < R) {   // (the first wave has the first 32 rows in its lanes)
    float top;
    const float sum = weight_of(tid, top);
    a.pml[at + tid] = sees ? make_float2(top, sum) : make_float2(-INFINITY, -1.f);
  }
  if (__builtin_expect(again, 0)) {
#pragma unroll 1
    for (int i = wave * 8; i < wave * 8 + 8 && r0 + i < R; ++i) {
      constexpr int COLS = DLW / 64;
      const int tk = (r0 + i) / a.mpc, gg = cell * a.mpc + (r0 + i - tk * a.mpc);
      const int from = max(__shfl(lo, i), b0 * 32), to = min(__shfl(hi, i), min(b1 * 32, keys) - 1);
      float avg[COLS];
      const float w = wave_row(a.rules, (const float *)a.q + (start + tk) * a.qs + gg * DH, DH, kcol, a.ks, ccol, a.cs, __shfl(slope, i), __shfl(own, i),
                               from, to, [&](int j) { return CACHE ? cache_row_clamped(a.prefix.pm, a.prefix.max_seq, a.prefix_slot, j) : start + j; }, avg);
      float *to_row = split ? a.pacc + (at + i) * a.dl : (float *)a.L + ((start + tk) * a.nq + gg) * (int64_t)a.dl;
      const bool any = __shfl(sees ? 1 : 0, i), none = w == 0.f && !split;   // (a piece may have none of the keys that a row sees)
#pragma unroll
      for (int e = 0; e < COLS; ++e) to_row[slice * DLW + e * 64 + lane] = !any ? 0.f : none ? NAN : avg[e];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at4 = i * 256 + tid, rr = at4 / (DLW / 4), col = at4 % (DLW / 4) * 4;
    const bool any = __shfl(sees ? 1 : 0, rr) != 0;
    if (r0 + rr >= R) continue;
    float top;
    const float sum = weight_of(rr, top);
    const float inv = any && !(split && sum == 0.f) ? 1.f / sum : 0.f;
    f32x4 v = sums[i] * inv;
    if (!any) v = f32x4{0.f, 0.f, 0.f, 0.f};
    if (split) *reinterpret_cast<f32x4 *>(a.pacc + (at + rr) * a.dl + slice * DLW + col) = v;
    else {
      const int tk = (r0 + rr) / a.mpc;
      *reinterpret_cast<f32x4 *>((float *)a.L + ((start + tk) * a.nq + cell * a.mpc + (r0 + rr - tk * a.mpc)) * (int64_t)a.dl + slice * DLW + col) = v;
    }
  }
}

template <int DH, int DLW>
bool launch_of(const RowsArgs &a, bool cache, hipStream_t st) {
  constexpr int LDS = 4 * 32 * (DLW + 4) * 4;
  const unsigned grid = (unsigned)((int64_t)a.tiles * a.cells * a.slices);
  if (!cache) {
    allow_dynamic_lds((const void *)rows_attn_f32_kernel<DH, DLW, false>, LDS);
    rows_attn_f32_kernel<DH, DLW, false><<<grid, 256, LDS, st>>>(a);
    return true;
  }
  if constexpr (DH >= 64) {   // (what prefix_tuned lets through)
    allow_dynamic_lds((const void *)rows_attn_f32_kernel<DH, DLW, true>, LDS);
    rows_attn_f32_kernel<DH, DLW, true><<<grid, 256, LDS, st>>>(a);
    return true;
  }
  return false;
}

}  // namespace

bool rows_f32_ok(const Dims &d) { return d.dtype == GTA_F32 && (d.dh == 32 || d.dh == 64 || d.dh == 128) && d.dl % 64 == 0; }
int rows_f32_columns(const Dims &d) { return d.dl % 128 == 0 ? 128 : 64; }

bool launch_rows_f32(const Dims &d, const RowsArgs &args, bool cache, hipStream_t st) {
  RowsArgs a = args;
  const bool wide = rows_f32_columns(d) == 128;
  a.slices = d.dl / rows_f32_columns(d);
  if (d.dh == 32) return wide ? launch_of<32, 128>(a, cache, st) : launch_of<32, 64>(a, cache, st);
  if (d.dh == 64) return wide ? launch_of<64, 128>(a, cache, st) : launch_of<64, 64>(a, cache, st);
  return wide ? launch_of<128, 128>(a, cache, st) : launch_of<128, 64>(a, cache, st);
}

}  // namespace gta
