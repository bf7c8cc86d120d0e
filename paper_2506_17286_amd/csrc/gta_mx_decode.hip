// Attention of one new token per sequence over a cache of 8-bit rows (Sec. 3.3, App. B.1.3):
//   L_g = sum_t Softmax_t(q_g . K_t / sqrt(d_h)) C_t
// with the context split over workgroups, each of which leaves an un-normalised sum, its maximum and its weight; a second
// launch joins them.
#include <type_traits>

#include "gta_mx.h"

namespace gta {
namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

struct MxAttnArgs {
  const void *q;
  MxView cv;
  int nq, qpk, qpc, dh, dl, kw, cw, batch, splits, share, ps_shift, maps;   // maps: of a workgroup
  float scale_log2e;
  float *pacc, *pml;   // [pieces, n_q, d_l], [pieces, n_q, 2]
  int32_t *prefix;     // [batch + 1] pieces in front of each sequence (matrix-instruction kernel)
  void *l_out;
};

// rows of the slot that take part
__device__ __forceinline__ int mx_rows(const MxView &cv, int b, int &slot) {
  slot = cv.slots ? cv.slots[b] : b;
  return slot >= 0 && slot < cv.max_batch ? min(max(cv.seq_lens[slot], 0), cv.max_seq) : 0;
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__bf16 v) { return (float)v; }

constexpr int kAnyMaxHead = 1024, kAnyMaxLatent = 4096;

// Any page sizes, heads of more than 512: a workgroup per (split, map, sequence), a row per thread for the scores, four latents per
// thread for the sums, which are averages over the rows so far: the largest finite latents stay finite.
template <typename T>
__global__ __launch_bounds__(256) void mx_attn_any_kernel(MxAttnArgs a) {
  __shared__ float qs[kAnyMaxHead];
  __shared__ float ps[256];
  __shared__ int64_t rowid[256];
  __shared__ float red[4], red2[4];
  __shared__ float accs[256 * 4];
  const int s = blockIdx.x, g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  int slot, j0, j1;
  const int n = mx_rows(a.cv, b, slot);
  j0 = (int)((int64_t)n * s / a.splits);
  j1 = (int)((int64_t)n * (s + 1) / a.splits);
  const int kcol = g / a.qpk * a.dh, ccol = g / a.qpc * a.dl, nb = a.dh / kMxBlock;
  for (int i = tid; i < a.dh; i += 256) qs[i] = to_f(((const T *)a.q)[((int64_t)b * a.nq + g) * a.dh + i]);
  const int quads = a.dl / 4, lanes = min(quads, 256), groups = 256 / lanes;   // row groups where there are few latents
  const int my = tid % lanes, grp = tid / lanes;
  float m = -INFINITY, l = 0.f, acc[kAnyMaxLatent / 1024][4] = {};
  __syncthreads();
  for (int jb = j0; jb < j1; jb += 256) {
    const int cnt = min(256, j1 - jb);
    float sc = -INFINITY;
    if (tid < cnt) {
      const int64_t row = cache_row_clamped(a.cv.pm, a.cv.max_seq, slot, jb + tid);
      rowid[tid] = row;
      const uint8_t *kr = a.cv.k + row * a.kw + kcol, *sr = a.cv.ks + row * (a.kw / kMxBlock) + kcol / kMxBlock;
      float sum = 0.f;
      for (int i = 0; i < nb; ++i) {
        float part = 0.f;
        for (int w = 0; w < 8; ++w) {
          const int code = reinterpret_cast<const int *>(kr)[i * 8 + w];
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(code, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(code, true);
          const float *qq = qs + i * 32 + w * 4;
          part = fmaf(lo[0], qq[0], fmaf(lo[1], qq[1], fmaf(hi[0], qq[2], fmaf(hi[1], qq[3], part))));
        }
        sum = fmaf(part, mx_scale(sr[i]), sum);
      }
      sc = sum * a.scale_log2e;
    }
    float mx = sc;
    for (int i = 32; i; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float mn = fmaxf(m, mx), ref = mn > -INFINITY ? mn : 0.f;
    const float p = tid < cnt ? exp2f(sc - ref) : 0.f, corr = exp2f(m - ref);
    ps[tid] = p;
    float sum = p;
    for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
    if ((tid & 63) == 0) red2[tid >> 6] = sum;
    __syncthreads();
    const float before = l * corr;
    l = before + (red2[0] + red2[1]) + (red2[2] + red2[3]);
    m = mn;
    const float per = l > 0.f ? 1.f / l : 0.f, kept = before * per;
    for (int v = 0; v * 256 + my < quads; ++v)
      for (int e = 0; e < 4; ++e) acc[v][e] *= kept;
    if (grp < groups)
      for (int r = grp; r < cnt; r += groups) {
        const float pr = ps[r] * per;
        const int64_t row = rowid[r];
        for (int v = 0; v * 256 + my < quads; ++v) {
          const int col = ccol + (v * 256 + my) * 4;
          const int code = *reinterpret_cast<const int *>(a.cv.c + row * a.cw + col);
          const float ws = pr * mx_scale(a.cv.cs[row * (a.cw / kMxBlock) + col / kMxBlock]);
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(code, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(code, true);
          acc[v][0] = fmaf(ws, lo[0], acc[v][0]); acc[v][1] = fmaf(ws, lo[1], acc[v][1]);
          acc[v][2] = fmaf(ws, hi[0], acc[v][2]); acc[v][3] = fmaf(ws, hi[1], acc[v][3]);
        }
      }
    __syncthreads();
  }
  const int64_t at = ((int64_t)b * a.splits + s) * a.nq + g;   // every split writes, those without rows too
  float *out = a.pacc + at * a.dl;
  if (groups == 1) {
    for (int v = 0; grp == 0 && v * 256 + my < quads; ++v)   // (threads over: 129 to 255 quads)
      for (int e = 0; e < 4; ++e) out[(v * 256 + my) * 4 + e] = acc[v][e];
  } else {
    for (int e = 0; e < 4; ++e) accs[tid * 4 + e] = acc[0][e];
    __syncthreads();
    if (grp == 0)
      for (int e = 0; e < 4; ++e) {
        float v = 0.f;
        for (int r = 0; r < groups; ++r) v += accs[(r * lanes + my) * 4 + e];
        out[my * 4 + e] = v;
      }
  }
  if (tid == 0) { a.pml[at * 2] = m; a.pml[at * 2 + 1] = l; }
}

// ---- matrix-instruction kernel ------------------------------------------------------------------
// A wave takes tiles of 32 rows and keeps everything of a tile in registers, codes included; the loads of the next tile go out
// piece by piece as the registers of this one come free, so that about a tile per wave is on its way at any time (96 to 128 KiB
// of a CU).  No barrier until the waves' sums are joined, but for the one a tile of waves that work in pairs.  What is left is
// memory: in the loop 64 x 8192 rows of 1056 bytes come in at 6.6 TB/s, rows of 2112 at 6.0 (a bare read: 6.8 to 7.05).
//
//   scores  S[t][g] = K q: rows t are the 16 rows of the first operand (lane x = l % 16 has row x, 16 bytes of every 64-byte
//           piece of it from h = l / 16 on), maps g the 16 columns of the second.  Codes become bf16 with their block's scale
//           in one instruction for two, exactly.  A lane ends up with the scores of map x for rows 4h .. 4h+3.
//   sums    L[d][g] = C^T p: the second operand wants, in lane (x, h), the weights of map x for rows 4h .. 4h+3 (of each half
//           tile): what the lane has.  For the first, lane (x, h) loads those same rows, LC bytes of each from x * LC on, and
//           turns pairs of rows into pairs of bf16; product j of a chunk has latents x * LC + j.
// The order of the rows and columns inside a product is free, which is what lets codes go from memory to the matrix unit
// without passing through LDS or another lane.
//
// Key heads get sums of their own, from which each column keeps those of its head: with zeros in the second operand instead,
// a NaN among one head's keys would reach the maps of all.  Weights are taken in two bf16 parts (16 bits; three for fp32),
// fp32 queries in three (24 bits); codes are exact in bf16, so that products are exact and sums fp32.
// Weights are 2^(score - ref) with ref the maximum of the wave's first tile: what they refer to changes no digit of them, only
// their range.  A wave that meets a score more than 40 above (28 in units of the natural exponent) goes through its rows once
// more with the maximum it has found by then.  Rescaling the sums in the loop instead keeps two copies of them in registers
// (64 latents of 256 and 1 key of 64: 125 registers spilled).
// Sums of weights and latents stay below 2^127 as long as latents do below 2^57: a weight is at most 2^40, rows are 2^30.  A piece
// with larger ones, which its scale bytes tell, is gone through once more, too, with weights of at most 2^-32 and sums below 2^126:
// the average of finite latents is finite.  (Such weights are good to 2^-18, the rounding of an exponent of 32 and more.)
template <typename T> struct Parts { static constexpr int Q = 1, P = 2; };
template <> struct Parts<float> { static constexpr int Q = 3, P = 3; };

// v in N bf16 parts that add up to it
template <int N>
__device__ __forceinline__ void split_parts(float v, __bf16 (&out)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    out[i] = (__bf16)v;
    const float r = v - (float)out[i];
    v = fabsf((float)out[i]) < INFINITY ? r : 0.f;
  }
}

__device__ __forceinline__ unsigned cvt_lo(unsigned w, float s) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false)); }
__device__ __forceinline__ unsigned cvt_hi(unsigned w, float s) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)); }

template <int BYTES> struct Word;
template <> struct Word<8> { typedef u32x2 type; };
template <> struct Word<16> { typedef u32x4 type; };

constexpr float kLowest = -3e38f;   // stands for "no score yet" where a difference is taken
constexpr float kMostAbove = 40.f;
constexpr unsigned kLargeScale = 127 + 48;   // latents of blocks below it are less than 2^57
constexpr float kLower = 32.f;               // how far such a piece's weights are lowered

constexpr int kTile = 32;           // rows of a tile
// A larger batch has a workgroup per sequence.  1024 and 1025 sequences of 256 rows of the paper's layer 24.6 and 14.0 us (1B shape 60.8 and
// 53.7), one of 16384 among others of 64 23.5 and 104.7: the cut is for lengths that differ.
constexpr int kShareBatch = 1024;

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

// How a batch is cut into pieces, one per workgroup.  A round is what a workgroup's waves take at a time; a sequence of r rounds
// becomes ceil(r / T) pieces of about as many rounds.  T is the least of eight values, between the rounds that each of `share`
// workgroups has if nothing is lost and those with which every batch fits, with which there are no more pieces than workgroups:
// all run at once, and the longest ends no later than it must.  Batches of many sequences are cut finer than the chip needs at
// once, and the pieces dealt out as workgroups end.  (Workgroups that go on into the next sequence instead have to set out twice,
// 5 to 10 us: 64 x 8192 rows of 1024 bytes 104 us against 93.)
constexpr int kCutTries = 8;
struct Cut {
  int prefix[kShareBatch + 1], rows[kShareBatch];   // pieces in front of each sequence, its rows
  int sums[4][kCutTries], found;
};

__device__ __forceinline__ int rounds_of(int n, int per_round) { return (n + per_round - 1) / per_round; }

// Returns the number of pieces.  splits > 0: that many of each sequence that has the rounds.
__device__ __forceinline__ int cut_batch(const MxView &cv, int batch, int per_round, int splits, int share, Cut &cut) {
  constexpr int PER = kShareBatch / 256, NT = kCutTries;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int r[PER], total = 0, some = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    r[i] = 0;
    const int b = tid + 256 * i;
    if (256 * i < batch && b < batch) {
      int slot;
      const int n = mx_rows(cv, b, slot);
      cut.rows[b] = n;
      r[i] = rounds_of(n, per_round);
      total += r[i];
      some += n > 0;
    }
  }
  int t = 1;
  if (!splits) {
    total = wave_scan(total);
    some = wave_scan(some);
    if (lane == 63) { cut.sums[wave][0] = total; cut.sums[wave][1] = some; }
    __syncthreads();
    total = cut.sums[0][0] + cut.sums[1][0] + cut.sums[2][0] + cut.sums[3][0];
    some = cut.sums[0][1] + cut.sums[1][1] + cut.sums[2][1] + cut.sums[3][1];
    total = __builtin_amdgcn_readfirstlane(total);
    some = __builtin_amdgcn_readfirstlane(some);
    __syncthreads();
    if (2 * some > share) {
      t = max(1, (total + 2 * share - 1) / (2 * share));
    } else {
      const int lo = max(1, (total + share - 1) / share), hi = max(lo, (total + share - some - 1) / (share - some));
      auto candidate = [&](int i) { return lo + (int)((int64_t)(hi - lo) * i / (NT - 1)); };
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const int tc = candidate(c);
        int k = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (256 * i < batch) k += rounds_of(r[i], tc);
        k = wave_scan(k);
        if (lane == 63) cut.sums[wave][c] = k;
      }
      __syncthreads();
      t = hi;
#pragma unroll
      for (int c = NT - 2; c >= 0; --c)
        if (cut.sums[0][c] + cut.sums[1][c] + cut.sums[2][c] + cut.sums[3][c] <= share) t = candidate(c);
      t = __builtin_amdgcn_readfirstlane(t);
      __syncthreads();
    }
  }
  int before = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (256 * i >= batch) break;
    const int b = tid + 256 * i, k = splits ? min(splits, r[i]) : rounds_of(r[i], t);
    int run = wave_scan(k);
    if (lane == 63) cut.sums[wave][i] = run;   // (a column of its own each time)
    __syncthreads();
    const int w0 = cut.sums[0][i], w1 = cut.sums[1][i], w2 = cut.sums[2][i];
    run += before + (wave > 0 ? w0 : 0) + (wave > 1 ? w1 : 0) + (wave > 2 ? w2 : 0);
    if (b < batch) cut.prefix[b + 1] = run;
    before += w0 + w1 + w2 + cut.sums[3][i];
  }
  if (tid == 0) cut.prefix[0] = 0;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(before);
}

// The same for up to 64 sequences, a lane each, by every wave for itself: no LDS and no barrier (2 us less at the start of a launch).
// Lane b: pieces in front of and of sequence b, its rows.  Returns the number of pieces.
__device__ __forceinline__ int cut_lanes(const MxView &cv, int batch, int per_round, int splits, int share, int &before, int &mine, int &rows) {
  const int b = threadIdx.x & 63;
  int slot;
  rows = b < batch ? mx_rows(cv, b, slot) : 0;
  const int r = rounds_of(rows, per_round);
  int t = 1;
  if (!splits) {
    const int total = __builtin_amdgcn_readlane(wave_scan(r), 63), some = __popcll(__ballot(rows > 0));
    if (2 * some > share) {
      t = max(1, (total + 2 * share - 1) / (2 * share));
    } else {
      const int lo = max(1, (total + share - 1) / share), hi = max(lo, (total + share - some - 1) / (share - some));
      t = lo;
#pragma unroll 1
      for (int c = 1; c < kCutTries && __builtin_amdgcn_readlane(wave_scan(rounds_of(r, t)), 63) > share; ++c)
        t = lo + (int)((int64_t)(hi - lo) * c / (kCutTries - 1));
    }
  }
  mine = splits ? min(splits, r) : rounds_of(r, t);
  const int run = wave_scan(mine);
  before = run - mine;
  return __builtin_amdgcn_readlane(run, 63);
}

// KB bytes of a key row, CS latent columns of a workgroup.  WPT: from 512 columns on two waves take a tile together; each has the
// scores of its half of the rows, hands them to the other through LDS, and the sums of its half of the columns.  With 1024 the
// sums alone would fill the accumulation registers (rows of 2112 bytes: 95 us against 67 for 8 x 8000..32768); with 512 one wave
// can do it, but twice the waves for half the registers fill and drain sooner (one sequence of 8192 rows 17.3 -> 15.4 us, 64
// of them the same).
// EDGE: rows of other widths than KB and CS, more than 16 maps, heads that end inside a piece.  A workgroup then has a.maps maps
// from g0 on and reads the columns of their key heads and latents (blockIdx.z: which maps, blockIdx.y: which CS of their latents);
// a head begins a piece of its own, and lanes without columns ask for what lies behind the buffer, zeros that cost nothing.  (64 x
// 8192 rows of 5 keys of 64 and 512 latents for 15 maps: 2215 us in mx_attn_any_kernel, 94 here.)  Rows of the widths KB and CS go
// without: one scale byte a load in place of four alone takes 182 us for 32 x 16384 of 1024 + 1024 to 207.  With and without, 64 x 8192
// bf16 rows: 64 + 128 26.2 / 25.5 us, + 256 42.3 / 35.4, + 512 69.5 / 69.0; 128 + 128 32.4 / 30.2, + 256 45.7 / 39.0, + 512 71.9 / 67.7; 256 + 256
// 56.6 / 49.5, + 512 85.9 / 85.5, + 1024 131.9 / 130.6; 512 + 512 113.5 / 112.0, + 1024 163.7 / 161.5; 1024 + 1024 247 / 205; 64 x 1024 and one of 4096
// rows 3 to 20 % apart, but for one of 1024 + 1024 (17.9 / 19.1).
template <typename T, int KB, int CS, int WPT, int OCC, bool SHARED, bool EDGE>
__global__ __launch_bounds__(256, OCC) void mx_attn_kernel(MxAttnArgs a) {
  constexpr int NQP = Parts<T>::Q, NPP = Parts<T>::P;
  constexpr int HF = 2, KH = HF / WPT, KP = KB / 64;                     // half tiles, those this wave scores, key pieces
  constexpr int CW = CS / WPT, LC = CW >= 256 ? 16 : CW / 16, NCH = CW / (16 * LC);   // this wave's columns, bytes per lane and load, chunks
  constexpr int KW = EDGE ? KP : KB >= 128 ? KB / 128 : 1;               // scale words of a key row: four bytes (two for one piece; EDGE: a byte each)
  constexpr int NS = 4 / WPT;                                            // tiles worked on at a time
  constexpr bool QREG = KB * NQP <= 192;
  typedef typename Word<LC>::type CWord;
  __shared__ std::conditional_t<SHARED, Cut, int> cut;
  __shared__ float sm[NS][16], sl[NS][16];
  typedef f32x4 Handed[NS][2][64];
  extern __shared__ __attribute__((aligned(16))) char lds[];   // the queries and, behind them, the scores that pairs of waves hand over; then the waves' sums
  Handed *const handed = reinterpret_cast<Handed *>(lds + (QREG ? 0 : KB * NQP * 32));
  const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), stream = wave / WPT, role = wave % WPT;
  const int z = blockIdx.y;
  const int g0 = EDGE ? blockIdx.z * a.maps : 0, nq = EDGE ? min(a.maps, a.nq - g0) : a.nq;
  const int kh0 = EDGE ? g0 / a.qpk : 0, kheads = EDGE ? (g0 + nq - 1) / a.qpk - kh0 + 1 : 0;
  const int latent0 = EDGE ? g0 / a.qpc * a.dl : 0, latents = EDGE ? ((g0 + nq - 1) / a.qpc + 1) * a.dl - latent0 : 0;
  if (EDGE && z * CS >= latents) return;   // (other maps have more of them)
  const bool first_here = z == 0 && (!EDGE || blockIdx.z == 0);

  // ---- this workgroup's piece: rows [j0, j1) of sequence b
  int b = blockIdx.x, slot, j0 = 0, j1, n;
  bool whole = true;
  if constexpr (SHARED) {
    const int wg = blockIdx.x;
    int first, k;
    if (a.batch <= 64) {
      int before, mine, rows;
      const int pieces = cut_lanes(a.cv, a.batch, kTile * NS, a.splits, a.share, before, mine, rows);
      if (wg == 0 && first_here && wave == 0) {
        if (lane < a.batch) a.prefix[lane + 1] = before + mine;
        if (lane == 0) a.prefix[0] = 0;
      }
      if (wg >= pieces) return;
      b = __builtin_amdgcn_readfirstlane(__ffsll(__ballot(before + mine > wg)) - 1);
      first = __builtin_amdgcn_readlane(before, b);
      k = __builtin_amdgcn_readlane(mine, b);
      n = __builtin_amdgcn_readlane(rows, b);
    } else {
      const int pieces = cut_batch(a.cv, a.batch, kTile * NS, a.splits, a.share, cut);
      if (wg == 0 && first_here)
        for (int i = tid; i <= a.batch; i += 256) a.prefix[i] = cut.prefix[i];
      if (wg >= pieces) return;
      for (int i = tid; i < a.batch; i += 256)
        if (cut.prefix[i] <= wg && wg < cut.prefix[i + 1]) cut.found = i;
      __syncthreads();
      b = __builtin_amdgcn_readfirstlane(cut.found);
      n = __builtin_amdgcn_readfirstlane(cut.rows[b]);
      first = __builtin_amdgcn_readfirstlane(cut.prefix[b]);
      k = __builtin_amdgcn_readfirstlane(cut.prefix[b + 1]) - first;
    }
    slot = a.cv.slots ? a.cv.slots[b] : b;
    const int r = rounds_of(n, kTile * NS), q = r / k, more = r % k, i = wg - first;   // one round more for the first of them
    j0 = (i * q + min(i, more)) * (kTile * NS);
    j1 = min(n, j0 + (q + (i < more)) * (kTile * NS));
    whole = k == 1;
  } else {
    n = mx_rows(a.cv, b, slot);
    j1 = n;
    if (n == 0) {
      for (int i = tid; i < nq * CS; i += 256) {
        const int g = g0 + i / CS, col = latent0 + z * CS + i % CS - g / a.qpc * a.dl;
        if (col >= 0 && col < a.dl) ((T *)a.l_out)[((int64_t)b * a.nq + g) * a.dl + col] = (T)0.f;
      }
      return;
    }
  }
  const int64_t part = (int64_t)blockIdx.x * a.nq + g0;   // where a piece that is not the whole sequence goes
  const int nt = (j1 - j0 + kTile - 1) / kTile;

  // Where the rows of tile t are: the pool row of the first row of each half, and how many rows the half has.  Page numbers are
  // asked for (constant memory, a scalar load that waits for no other) some time before they are used.
  typedef const __attribute__((address_space(4))) int32_t *Table;
  const bool paged = a.cv.pm.table != nullptr;   // contiguous slots: one page, of number 0, at the slot's first row
  const Table pages = paged ? (Table)a.cv.pm.table + (int64_t)slot * a.cv.pm.pages_per_slot : (Table)a.cv.seq_lens;
  const int64_t slot_row = paged ? 0 : (int64_t)slot * a.cv.max_seq;
  const int in_page = paged ? (1 << a.ps_shift) - 1 : INT32_MAX, any_page = paged ? -1 : 0, num_pages = paged ? a.cv.pm.num_pages : 0;
  struct Pages { int page[HF]; };
  struct At { int64_t row[HF]; int rows[HF]; };
  auto ask = [&](int t) {
    Pages r;
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) r.page[hf] = pages[(min(j0 + t * kTile + hf * 16, j1 - 1) >> a.ps_shift) & any_page];
    return r;
  };
  auto settle = [&](int t, const Pages &r) {
    At at;
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) {
      const int jb = j0 + t * kTile + hf * 16, pg = (unsigned)r.page[hf] < (unsigned)num_pages ? r.page[hf] : 0;
      // (the compiler does not see that these are the same in all lanes)
      at.rows[hf] = __builtin_amdgcn_readfirstlane(min(max(j1 - jb, 0), 16));
      const int64_t row = slot_row + ((int64_t)pg << a.ps_shift) + (jb & in_page);
      at.row[hf] = (int64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)row) | (int64_t)__builtin_amdgcn_readfirstlane((int)(row >> 32)) << 32;
    }
    return at;
  };

  // Loads through buffers that end with the half's rows: what lies behind reads as zeros and costs nothing, in the last tile of
  // a share and in the tiles that a wave asks for behind it.
  u32x4 kb[KH][KP];
  unsigned ks[KH][KW];
  CWord cb[HF][4][NCH];
  unsigned cs[HF][4][NCH];
  const int col0 = latent0 + z * CS + role * CW, mine = EDGE ? latents - z * CS - role * CW : 0;   // columns of this wave
  const int key0 = EDGE ? kh0 * a.dh : 0, kwidth = EDGE ? a.kw : KB;
  const int ppk = (a.dh + 63) / 64;   // pieces of a key head
  const unsigned koff = x * kwidth + h * 16, ksoff = x * (kwidth / 32) + (EDGE ? h >> 1 : 0);
  // EDGE: column of a key piece in the row's window, and what to add to the offset of lanes that have none (of a piece of no head; in
  // the second half of a head's last): beyond any buffer, whose 16 rows have at most 2^18 columns.
  constexpr unsigned kNone = 0x40000000;
  unsigned key_at[EDGE ? KP : 1], key_end[EDGE ? KP : 1], late = 0, none[EDGE ? NCH : 1];
  if constexpr (EDGE) {
    late = a.dh % 64 && h >= 2 ? kNone : 0;
    int head = 0, piece = 0;
#pragma unroll
    for (int p = 0; p < KP; ++p) {
      key_at[p] = head * a.dh + piece * 64;
      key_end[p] = (head < kheads ? 0 : kNone) + (piece == ppk - 1 ? late : 0);
      if (++piece == ppk) { piece = 0; ++head; }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) none[c] = c * 16 * LC + x * (int)LC >= mine ? kNone : 0;
  }
  unsigned coff[4], csoff[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    coff[j] = (4 * h + j) * a.cw + x * LC;
    csoff[j] = (4 * h + j) * (a.cw / 32) + x * LC / 32;
  }
  auto buffer = [&](const uint8_t *pool, const At &at, int hf, int width, int skip) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)(pool + at.row[hf] * width + skip), 0, max(at.rows[hf] * width - skip, 0), 0x00020000);
  };
  // Latents are streamed past the caches; keys and scale bytes are not, whose lines are asked for more than once (64 bytes of a
  // row's 128 at a time, one scale byte per lane).  All streamed: 32 x 16384 rows of 2112 bytes 217 us against 191, 64 x 8192 of
  // 1056 95 against 92; none: 207 and 101.
  constexpr int kPast = 2;
  auto my_half = [&](const At &at, int kh) {   // of the rows that this wave scores
    if constexpr (WPT == 1) return at;
    At r{};
    r.row[kh] = role ? at.row[1] : at.row[0];
    r.rows[kh] = role ? at.rows[1] : at.rows[0];
    return r;
  };
  auto load_key_scales = [&](const At &at) {
#pragma unroll
    for (int hf = 0; hf < KH; ++hf) {
      const auto r = buffer(a.cv.ks, my_half(at, hf), hf, kwidth / 32, key0 / 32);
#pragma unroll
      for (int i = 0; i < KW; ++i) {
        if constexpr (EDGE) ks[hf][i] = __builtin_amdgcn_raw_buffer_load_b8(r, ksoff + key_at[i] / 32 + key_end[i], 0, 0);
        else if constexpr (KB >= 128) ks[hf][i] = __builtin_amdgcn_raw_buffer_load_b32(r, ksoff + i * 4, 0, 0);
        else ks[hf][i] = __builtin_amdgcn_raw_buffer_load_b16(r, ksoff, 0, 0);
      }
    }
  };
  auto load_keys = [&](const At &at, int p) {
#pragma unroll
    for (int hf = 0; hf < KH; ++hf)
      kb[hf][p] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer(a.cv.k, my_half(at, hf), hf, kwidth, key0),
                                                                                  EDGE ? koff + key_at[p] + key_end[p] : koff + p * 64, 0, 0));
  };
  auto load_latents = [&](const At &at, int c) {
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) {
      const auto r = buffer(a.cv.c, at, hf, a.cw, col0), rs = buffer(a.cv.cs, at, hf, a.cw / 32, col0 / 32);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned o = coff[j] + c * 16 * LC + (EDGE ? none[c] : 0);
        if constexpr (LC == 16) cb[hf][j][c] = __builtin_bit_cast(CWord, __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, kPast));
        else cb[hf][j][c] = __builtin_bit_cast(CWord, __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, kPast));
        cs[hf][j][c] = __builtin_amdgcn_raw_buffer_load_b8(rs, csoff[j] + c * LC / 2 + (EDGE ? none[c] : 0), 0, 0);
      }
    }
  };

  // the queries are asked for first, then the first tile's rows: these are on their way while the queries are laid out
  const int kg = x < nq ? (g0 + x) / a.qpk - kh0 : -1;
  constexpr int PER = 16 / (int)sizeof(T);   // in words of 16 bytes, which is what queries are aligned to
  typedef __attribute__((ext_vector_type(PER))) T QWord;
  struct Eight { QWord w[8 / PER]; };
  constexpr int QF = QREG ? KP * 2 : KP / 2;   // fragments this wave lays out: all of them, or every fourth
  Eight qv[QF];
#pragma unroll
  for (int i = 0; i < QF; ++i) {   // second operand for half a piece: dimensions h * 16 + (f & 1) * 8 .. of the piece
    const int f = QREG ? i : wave + 4 * i, p = f >> 1, d0 = p % ppk * 64 + h * 16;
    const T *from = (const T *)a.q + ((int64_t)b * a.nq + g0 + (kg == p / ppk ? x : 0)) * a.dh + (EDGE && d0 >= a.dh ? 0 : d0) + (f & 1) * 8;
#pragma unroll
    for (int w = 0; w < 8 / PER; ++w) qv[i].w[w] = reinterpret_cast<const QWord *>(from)[w];
  }
  At nxt{};
  auto start = [&]() {
    const Pages now = ask(stream), later = ask(stream + NS);
    const At first = settle(stream, now);
    load_key_scales(first);
#pragma unroll
    for (int p = 0; p < KP; ++p) load_keys(first, p);
#pragma unroll
    for (int c = 0; c < NCH; ++c) load_latents(first, c);
    nxt = settle(stream + NS, later);
  };
  __builtin_amdgcn_sched_barrier(0);
  start();
  __builtin_amdgcn_sched_barrier(0);
  bf16x8 qr[QREG ? KP * 2 : 1][NQP];
  bf16x8 *qs = reinterpret_cast<bf16x8 *>(lds);   // [KP * 2][NQP][64]
#pragma unroll
  for (int i = 0; i < QF; ++i) {
    const int f = QREG ? i : wave + 4 * i;
    bf16x8 out[NQP];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      __bf16 v[NQP];
      split_parts<NQP>(kg == (f >> 1) / ppk && (!EDGE || (f >> 1) % ppk * 64 + h * 16 < a.dh) ? to_f(qv[i].w[e / PER][e % PER]) : 0.f, v);
#pragma unroll
      for (int j = 0; j < NQP; ++j) out[j][e] = v[j];
    }
#pragma unroll
    for (int j = 0; j < NQP; ++j) {
      if constexpr (QREG) qr[i][j] = out[j];
      else qs[(f * NQP + j) * 64 + lane] = out[j];
    }
  }
  if constexpr (!QREG) __syncthreads();

  f32x4 acc[NCH][LC];
  float m = -INFINITY, l = 0.f, seen = -INFINITY;   // what weights refer to, their sum, the largest score of this lane's rows
  unsigned most = 0;   // largest scale byte of its latents

  auto tile = [&](int t, int turn) {
    // ---- scores; a piece's query fragments are asked for a piece ahead, its sums are taken a piece later
    f32x4 sc[HF], before[KH];
#pragma unroll
    for (int hf = 0; hf < KH; ++hf) sc[hf] = before[hf] = f32x4{0.f, 0.f, 0.f, 0.f};
    unsigned kscale[KH][KW];
#pragma unroll
    for (int hf = 0; hf < KH; ++hf)
#pragma unroll
      for (int i = 0; i < KW; ++i) kscale[hf][i] = EDGE ? ks[hf][i] : ks[hf][i] >> (8 * (h >> 1));
    load_key_scales(nxt);
    auto fragments = [&](int p, bf16x8 (&out)[2][NQP]) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < NQP; ++i) {
          if constexpr (QREG) out[half][i] = qr[p * 2 + half][i];
          else out[half][i] = qs[((p * 2 + half) * NQP + i) * 64 + lane];
        }
    };
    auto take = [&](int p) {
      const bool of_map = kg == p / ppk;
#pragma unroll
      for (int hf = 0; hf < KH; ++hf)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[hf][i] += of_map ? before[hf][i] : 0.f;
    };
    bf16x8 qf[2][NQP], qn[2][NQP];
    fragments(0, qf);
#pragma unroll
    for (int p = 0; p < KP; ++p) {
      if (p + 1 < KP) fragments(p + 1, qn);
      f32x4 d[KH];
#pragma unroll
      for (int hf = 0; hf < KH; ++hf) d[hf] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int hf = 0; hf < KH; ++hf) {
          const unsigned w = kscale[hf][EDGE ? p : p / 2];
          const float s = __uint_as_float((!EDGE && p & 1 ? w << 7 : w << 23) & 0x7f800000u);
          const u32x4 k4 = {cvt_lo(kb[hf][p][2 * half], s), cvt_hi(kb[hf][p][2 * half], s), cvt_lo(kb[hf][p][2 * half + 1], s),
                            cvt_hi(kb[hf][p][2 * half + 1], s)};
#pragma unroll
          for (int i = 0; i < NQP; ++i)
            d[hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k4), qf[half][i], d[hf], 0, 0, 0);
        }
      load_keys(nxt, p);
      if (p) take(p - 1);
#pragma unroll
      for (int hf = 0; hf < KH; ++hf) before[hf] = d[hf];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < NQP; ++i) qf[half][i] = qn[half][i];
      __builtin_amdgcn_sched_barrier(0);   // one piece at a time: conversions taken up early would need registers
    }
    take(KP - 1);
    if constexpr (WPT > 1) {
      handed[turn][stream][role][lane] = sc[0];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_barrier();   // (two sets of places: the one written here is read no later than in front of the next)
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
      sc[0] = handed[turn][stream][0][lane];
      sc[1] = handed[turn][stream][1][lane];
    }
    // ---- weights
    const int left = j1 - (j0 + t * kTile);   // rows of this tile
    float mx = -INFINITY;
#pragma unroll
    for (int hf = 0; hf < HF; ++hf)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[hf][i] = hf * 16 + 4 * h + i < left ? sc[hf][i] * a.scale_log2e : -INFINITY;
        mx = fmaxf(mx, sc[hf][i]);
      }
    seen = fmaxf(seen, mx);
    if (t == stream && m == -INFINITY) {
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      m = fmaxf(mx, __shfl_xor(mx, 32));
    }
    const float ref = fmaxf(m, kLowest);
    unsigned pp[NPP][HF * 2];   // pairs of rows
#pragma unroll
    for (int hf = 0; hf < HF; ++hf)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float p0 = __builtin_amdgcn_exp2f(sc[hf][2 * r] - ref), p1 = __builtin_amdgcn_exp2f(sc[hf][2 * r + 1] - ref);
        l += p0 + p1;
#pragma unroll
        for (int i = 0; i < NPP; ++i) {
          const bf16x2 v = {(__bf16)p0, (__bf16)p1};
          pp[i][hf * 2 + r] = __builtin_bit_cast(unsigned, v);
          p0 -= (float)v[0];
          p1 -= (float)v[1];
        }
      }
    // ---- sums; the scale bytes first (looked at among the products: 64 x 2048 fp32 rows of the paper's layer 13.8 -> 14.1 us)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int hf = 0; hf < HF; ++hf)
#pragma unroll
        for (int j = 0; j < 4; ++j) most = max(most, cs[hf][j][c]);
    const Pages then = ask(t + 2 * NS);   // (no LDS is read from here on, whose waits would be waits for these loads)
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
#pragma unroll
      for (int w = 0; w < LC / 4; ++w) {
        unsigned op[4][HF * 2];   // [latent of the word][pairs of rows]
#pragma unroll
        for (int hf = 0; hf < HF; ++hf)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const unsigned w0 = cb[hf][2 * r][c][w], w1 = cb[hf][2 * r + 1][c][w];
            const float s0 = mx_scale(cs[hf][2 * r][c]), s1 = mx_scale(cs[hf][2 * r + 1][c]);
            const unsigned a0 = cvt_lo(w0, s0), a1 = cvt_hi(w0, s0), b0 = cvt_lo(w1, s1), b1 = cvt_hi(w1, s1);
            op[0][hf * 2 + r] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
            op[1][hf * 2 + r] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
            op[2][hf * 2 + r] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
            op[3][hf * 2 + r] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
          }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < NPP; ++i) {
            f32x4 &d = acc[c][w * 4 + e];
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{op[e][0], op[e][1], op[e][2], op[e][3]}),
                                                        __builtin_bit_cast(bf16x8, u32x4{pp[i][0], pp[i][1], pp[i][2], pp[i][3]}), d, 0, 0, 0);
          }
      }
      load_latents(nxt, c);
      __builtin_amdgcn_sched_barrier(0);
    }
    nxt = settle(t + 2 * NS, then);
  };

  bool lowered = false;
  while (true) {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < LC; ++j) acc[c][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
    if constexpr (WPT == 1) {
      for (int t = stream; t < nt; t += NS) tile(t, 0);
    } else {   // all waves go through as many tiles: they meet in each
      for (int t = stream; t - stream < nt; t += NS) tile(t, ((t - stream) / NS) & 1);
    }
    seen = fmaxf(seen, __shfl_xor(seen, 16));
    seen = fmaxf(seen, __shfl_xor(seen, 32));
    bool large = !lowered && __any(most >= kLargeScale);
    bool again = large || __any(seen > m + kMostAbove);   // (never a second time)
    if constexpr (WPT > 1) again = __syncthreads_or(again);
    if (!again) break;
    if constexpr (WPT > 1) large = __syncthreads_or(large);   // (a pair's waves have the same scores, but different latents)
    m = fmaxf(m, seen) + (large ? kLower : 0.f);
    lowered |= large;
    start();
  }

  // ---- the four waves' sums, through LDS
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (lane < 16 && role == 0) { sm[stream][x] = m; sl[stream][x] = l; }
  __syncthreads();   // (queries are not read any more, either)
  float *buf = reinterpret_cast<float *>(lds);   // [NS][n_q][ROW]
  auto highest = [&](int g) {
    float v = sm[0][g];
#pragma unroll
    for (int w = 1; w < NS; ++w) v = fmaxf(v, sm[w][g]);
    return v;
  };
  const float top = highest(x);
  const float f = __builtin_amdgcn_exp2f(fmaxf(m, kLowest) - fmaxf(top, kLowest));
  auto joined = [&](int g, float &mg) {   // sum of the weights of map g
    mg = highest(g);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < NS; ++w) v += sl[w][g] * __builtin_amdgcn_exp2f(fmaxf(sm[w][g], kLowest) - fmaxf(mg, kLowest));
    return v;
  };
  if (!whole && z == 0 && tid < nq) {
    float mg;
    const float lg = joined(tid, mg);
    a.pml[(part + tid) * 2] = mg;
    a.pml[(part + tid) * 2 + 1] = lg;
  }
  // Rows of n_q maps, CS columns in words of 16 bytes; a word's place is turned by the lane group that wrote it and rows are
  // padded, so that the lanes of a store meet different banks.
  constexpr int ROW = CS + 16;
  auto place = [](int col) { return col ^ (((col / (4 * LC)) & 3) * 4); };
  if (x < nq) {
    float *dst = buf + (stream * nq + x) * ROW;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < LC; j += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4 *>(dst + place(role * CW + c * 16 * LC + (4 * h + i) * LC + j)) =
              f32x4{acc[c][j][i] * f, acc[c][j + 1][i] * f, acc[c][j + 2][i] * f, acc[c][j + 3][i] * f};
        __builtin_amdgcn_sched_barrier(0);   // not all of them out of the accumulation registers at once
      }
  }
  __syncthreads();
  for (int i = tid; i < nq * (CS / 4); i += 256) {
    const int g = i / (CS / 4), cc = i % (CS / 4) * 4, col = latent0 + z * CS + cc - (g0 + g) / a.qpc * a.dl;   // latent of the map's group
    if (col < 0 || col >= a.dl) continue;
    f32x4 v = *reinterpret_cast<const f32x4 *>(buf + g * ROW + place(cc));
#pragma unroll
    for (int w = 1; w < NS; ++w) v += *reinterpret_cast<const f32x4 *>(buf + (w * nq + g) * ROW + place(cc));
    if (whole) {
      float mg;
      const float lg = joined(g, mg);
      T *o = (T *)a.l_out + ((int64_t)b * a.nq + g0 + g) * a.dl + col;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (T)(v[e] / lg);
    } else {
      *reinterpret_cast<f32x4 *>(a.pacc + (part + g) * a.dl + col) = v;
    }
  }
}

// Joins the pieces of a map: a workgroup per (map, sequence, 256 latents), four latents per thread and the pieces dealt to as
// many groups of threads as there are.  SHARED: the pieces that mx_attn_kernel left (it has written sequences of one piece itself); otherwise
// a.splits of them for every sequence, which are averages.
constexpr int kMaxPieces = 2560;   // of a sequence: at most twice the workgroups that the chip holds, and one, or 1024 splits

template <typename T, bool SHARED>
__global__ __launch_bounds__(256) void mx_join_kernel(MxAttnArgs a) {
  __shared__ float wt[kMaxPieces];
  __shared__ float red[4], red2[4];
  __shared__ f32x4 sums[256];
  const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  T *out = (T *)a.l_out + ((int64_t)b * a.nq + g) * a.dl;
  int first, pieces;
  bool none;
  if constexpr (SHARED) {
    first = a.prefix[b];
    pieces = a.prefix[b + 1] - first;
    none = pieces == 0;
    if (pieces == 1) return;
  } else {
    int slot;
    none = mx_rows(a.cv, b, slot) == 0;
    pieces = a.splits;
    first = b * a.splits;
  }
  if (none) {
    const int i = blockIdx.z * 256 + tid;
    if (i < a.dl) out[i] = (T)0.f;
    return;
  }
  auto at = [&](int i) { return ((int64_t)first + i) * a.nq + g; };
  float m = -INFINITY;
  for (int i = tid; i < pieces; i += 256) {
    const float v = a.pml[at(i) * 2];
    wt[i] = v;
    m = fmaxf(m, v);
  }
#pragma unroll
  for (int i = 32; i; i >>= 1) m = fmaxf(m, __shfl_xor(m, i));
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), kLowest);
  float l = 0.f;
  for (int i = tid; i < pieces; i += 256) {
    const float w = __builtin_amdgcn_exp2f(fmaxf(wt[i], kLowest) - m);
    wt[i] = w;
    l = fmaf(a.pml[at(i) * 2 + 1], w, l);
  }
#pragma unroll
  for (int i = 32; i; i >>= 1) l += __shfl_xor(l, i);
  if ((tid & 63) == 0) red2[tid >> 6] = l;
  __syncthreads();
  l = (red2[0] + red2[1]) + (red2[2] + red2[3]);
  if constexpr (!SHARED) {
    for (int i = tid; i < pieces; i += 256) wt[i] = wt[i] * a.pml[at(i) * 2 + 1] / l;
    __syncthreads();
    l = 1.f;
  }
  // 64 threads for 256 latents (fewer where there are fewer), the pieces dealt to the others
  const int c0 = blockIdx.z * 256, lanes = min(a.dl - c0, 256) / 4, groups = 256 / lanes, my = tid % lanes, grp = tid / lanes;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (grp < groups) {
#pragma unroll 8
    for (int i = grp; i < pieces; i += groups) v += *reinterpret_cast<const f32x4 *>(a.pacc + at(i) * a.dl + c0 + my * 4) * wt[i];
  }
  sums[tid] = v;
  __syncthreads();
  if (grp) return;
  for (int r = 1; r < groups; ++r) v += sums[r * lanes + my];
#pragma unroll
  for (int e = 0; e < 4; ++e) out[c0 + my * 4 + e] = (T)(v[e] / l);   // scores of nothing but -inf: 0 / 0
}

}  // namespace

bool mx_decode_dims_ok(const Dims &d) { return mx_widths_ok(d) && d.dh <= kAnyMaxHead && d.dl <= kAnyMaxLatent && d.nq <= 65535; }

// How the matrix-instruction kernel takes a shape.  Rows of instantiated widths and up to 16 maps in whole pieces of 64 go in one, or
// in slices of their latents.  Anything else (EDGE) is cut into blocks of up to 16 maps, each with the key heads and latents that it
// reads, by the fewest columns in all, padding included.  No blocks: heads of more than 512.
struct MxPlan { int kb, cs, maps, blocks, slices; bool edge; };

static MxPlan mx_plan(const Dims &d) {
  int cs = 1024;
  while (cs >= 128 && !(d.wc_w % cs == 0 && (d.wc_w == cs || cs >= 512))) cs /= 2;
  const int kb = d.wk_w;
  if (d.dh % 64 == 0 && d.nq <= 16 && cs >= 128 &&
      ((kb == 64 && cs <= 512) || (kb == 128 && cs <= 512) || (kb == 256 && cs >= 256) || (kb == 512 && cs >= 512) || (kb == 1024 && cs == 1024)))
    return MxPlan{kb, cs, d.nq, 1, d.wc_w / cs, false};
  const int ppk = (d.dh + 63) / 64;
  auto heads = [](int maps, int per, int most) { return std::min(most, maps % per == 0 ? maps / per : per % maps == 0 ? 1 : (maps + per - 2) / per + 1); };
  MxPlan best{};
  int64_t least = INT64_MAX;
  for (int m = std::min(d.nq, 16); m >= 1; --m) {
    const int pieces = heads(m, d.qpk, d.nk) * ppk, wide = heads(m, d.qpc, d.nc) * d.dl;
    if (pieces > 8) continue;   // (1024 columns of keys: 114 registers spilled)
    MxPlan p{64, 0, m, (d.nq + m - 1) / m, 1, true};
    while (p.kb < pieces * 64) p.kb *= 2;
    p.cs = wide <= 128 && p.kb <= 128 ? 128 : wide <= 512 || (wide % 1024 && wide % 512 == 0) ? 512 : 1024;
    p.slices = (wide + p.cs - 1) / p.cs;
    const int64_t cost = (int64_t)p.blocks * p.slices * (p.kb + p.cs);
    if (cost < least) { least = cost; best = p; }
  }
  return best;
}

bool mx_decode_tuned(const Dims &d) { return mx_plan(d).blocks > 0; }

// Pages that the matrix-instruction kernel takes: a power of two of at least half a tile.
static bool mx_layout_tuned(const MxView &cv) {
  return !cv.pm.table || (cv.pm.page_size >= 16 && (cv.pm.page_size & (cv.pm.page_size - 1)) == 0);
}

// Workgroups per CU, by the registers that a wave's sums, its codes and the rest take.
constexpr int mx_occupancy(int cs) { return cs >= 1024 ? 1 : cs >= 256 ? 2 : 3; }

// Workgroups that the chip holds at once.
static int mx_share(const MxPlan &p) { return std::max(2, 256 * mx_occupancy(p.cs) / (p.slices * p.blocks)); }

// Most pieces of a batch (Cut).
static int64_t mx_most_pieces(int batch, int share, int requested) {
  return requested > 0 ? (int64_t)batch * std::min(requested, 1024) : 2 * batch > share ? 2 * (int64_t)share + batch : share;
}

static int mx_equal_splits(const Dims &d, int batch, int max_seq, int requested) {
  if (requested > 0) return std::min(requested, 1024);
  const int64_t maps = (int64_t)batch * d.nq, want = (1024 + maps - 1) / maps;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, max_seq / 256), 256));
}

static size_t piece_bytes(const Dims &d) { return (size_t)d.nq * ((size_t)d.dl + 2) * 4; }
static size_t prefix_bytes(int batch) { return batch <= kShareBatch ? align_up(((size_t)batch + 1) * 4) : 0; }

size_t mx_decode_bytes(const Dims &d, int batch, int max_seq, int requested) {
  // the call picks the kernel by the page size too: enough for either
  size_t n = piece_bytes(d) * batch * mx_equal_splits(d, batch, max_seq, requested);
  const MxPlan p = mx_plan(d);
  if (p.blocks && batch <= kShareBatch) n = std::max(n, prefix_bytes(batch) + piece_bytes(d) * mx_most_pieces(batch, mx_share(p), requested));
  return n;
}

template <typename T, int KB, int CS, bool EDGE>
static void launch_tuned(const MxAttnArgs &a, const MxPlan &p, int pieces, hipStream_t st) {
  constexpr int WPT = CS >= 512 ? 2 : 1;
  constexpr int OCC = mx_occupancy(CS);
  const int handed = WPT > 1 ? 2 * 4 / WPT * 2 * 64 * 16 : 0;
  const int lds = std::max(KB * Parts<T>::Q * 32 + handed, 4 / WPT * p.maps * (CS + 16) * 4);   // (16 maps, 512 columns: two workgroups per CU)
  if (pieces) {
    if (lds > 40 * 1024) allow_dynamic_lds((const void *)mx_attn_kernel<T, KB, CS, WPT, OCC, true, EDGE>, lds);
    mx_attn_kernel<T, KB, CS, WPT, OCC, true, EDGE><<<dim3(pieces, p.slices, p.blocks), 256, lds, st>>>(a);
    mx_join_kernel<T, true><<<dim3(a.nq, a.batch, (a.dl + 255) / 256), 256, 0, st>>>(a);
  } else {
    if (lds > 40 * 1024) allow_dynamic_lds((const void *)mx_attn_kernel<T, KB, CS, WPT, OCC, false, EDGE>, lds);
    mx_attn_kernel<T, KB, CS, WPT, OCC, false, EDGE><<<dim3(a.batch, p.slices, p.blocks), 256, lds, st>>>(a);
  }
}

template <typename T>
static void launch_decode(const Dims &d, const MxAttnArgs &a, bool tuned, const MxPlan &p, int pieces, hipStream_t st) {
  if (!tuned) {
    mx_attn_any_kernel<T><<<dim3(a.splits, d.nq, a.batch), 256, 0, st>>>(a);
    mx_join_kernel<T, false><<<dim3(d.nq, a.batch, (d.dl + 255) / 256), 256, 0, st>>>(a);
    return;
  }
  const int which = p.kb * 4096 + p.cs;
  if (p.edge) {
    switch (which) {
      case 64 * 4096 + 128: return launch_tuned<T, 64, 128, true>(a, p, pieces, st);
      case 64 * 4096 + 512: return launch_tuned<T, 64, 512, true>(a, p, pieces, st);
      case 64 * 4096 + 1024: return launch_tuned<T, 64, 1024, true>(a, p, pieces, st);
      case 128 * 4096 + 128: return launch_tuned<T, 128, 128, true>(a, p, pieces, st);
      case 128 * 4096 + 512: return launch_tuned<T, 128, 512, true>(a, p, pieces, st);
      case 128 * 4096 + 1024: return launch_tuned<T, 128, 1024, true>(a, p, pieces, st);
      case 256 * 4096 + 512: return launch_tuned<T, 256, 512, true>(a, p, pieces, st);
      case 256 * 4096 + 1024: return launch_tuned<T, 256, 1024, true>(a, p, pieces, st);
      case 512 * 4096 + 512: return launch_tuned<T, 512, 512, true>(a, p, pieces, st);
      case 512 * 4096 + 1024: return launch_tuned<T, 512, 1024, true>(a, p, pieces, st);
    }
    return;
  }
  switch (which) {
    case 64 * 4096 + 128: return launch_tuned<T, 64, 128, false>(a, p, pieces, st);
    case 64 * 4096 + 256: return launch_tuned<T, 64, 256, false>(a, p, pieces, st);
    case 64 * 4096 + 512: return launch_tuned<T, 64, 512, false>(a, p, pieces, st);
    case 128 * 4096 + 128: return launch_tuned<T, 128, 128, false>(a, p, pieces, st);
    case 128 * 4096 + 256: return launch_tuned<T, 128, 256, false>(a, p, pieces, st);
    case 128 * 4096 + 512: return launch_tuned<T, 128, 512, false>(a, p, pieces, st);
    case 256 * 4096 + 256: return launch_tuned<T, 256, 256, false>(a, p, pieces, st);
    case 256 * 4096 + 512: return launch_tuned<T, 256, 512, false>(a, p, pieces, st);
    case 256 * 4096 + 1024: return launch_tuned<T, 256, 1024, false>(a, p, pieces, st);
    case 512 * 4096 + 512: return launch_tuned<T, 512, 512, false>(a, p, pieces, st);
    case 512 * 4096 + 1024: return launch_tuned<T, 512, 1024, false>(a, p, pieces, st);
    case 1024 * 4096 + 1024: return launch_tuned<T, 1024, 1024, false>(a, p, pieces, st);
  }
}

int launch_mx_decode(const Dims &d, const void *q, const MxView &cv, int batch, int requested, void *ws, size_t ws_bytes, void *l_out,
                     hipStream_t st) {
  const MxPlan plan = mx_plan(d);
  const bool tuned = plan.blocks && mx_layout_tuned(cv);
  // row numbers and their sums over a batch that is cut stay well inside 32 bits
  if (cv.max_seq > (1 << 30) || (batch <= kShareBatch && (int64_t)batch * cv.max_seq >= ((int64_t)1 << 36))) return GTA_ERR_UNSUPPORTED;
  const size_t head = tuned ? prefix_bytes(batch) : 0;
  const int64_t fit = ws_bytes > head ? (int64_t)((ws_bytes - head) / piece_bytes(d)) : 0;
  int share = 0, splits = 0;
  int64_t pieces = 0;
  if (ws_bytes < head) return GTA_ERR_WORKSPACE;
  if (tuned && batch <= kShareBatch) {
    share = mx_share(plan);
    splits = std::min(requested, 1024);
    pieces = mx_most_pieces(batch, share, requested);
    if (fit < pieces) {   // a smaller workspace: as many pieces as it holds, or whole sequences
      if (requested > 0) return GTA_ERR_WORKSPACE;
      share = (int)fit;
      splits = share < 2 * batch ? 1 : 0;
      pieces = splits ? batch : share;
    }
  } else if (!tuned) {
    splits = mx_equal_splits(d, batch, cv.max_seq, requested);
    if (fit < (int64_t)batch * splits) {
      if (requested > 0 || fit < batch) return GTA_ERR_WORKSPACE;
      splits = (int)(fit / batch);
    }
    pieces = (int64_t)batch * splits;
  }
  int shift = 0;
  if (cv.pm.table) while ((1 << shift) < cv.pm.page_size && shift < 30) ++shift;
  float *acc = (float *)((char *)ws + head);
  const MxAttnArgs a{q, cv, d.nq, d.qpk, d.qpc, d.dh, d.dl, d.wk_w, d.wc_w, batch, splits, share, shift, plan.maps, d.scale * 1.4426950408889634f,
                     acc, acc + std::min(pieces, fit) * d.nq * d.dl, (int32_t *)ws, l_out};
  if (d.dtype == GTA_BF16) launch_decode<__bf16>(d, a, tuned, plan, (int)pieces, st);
  else launch_decode<float>(d, a, tuned, plan, (int)pieces, st);
  return check_launch();
}

}  // namespace gta
