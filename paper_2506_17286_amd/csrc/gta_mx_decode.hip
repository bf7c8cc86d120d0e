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
typedef __attribute__((ext_vector_type(4))) short s16x4;

struct MxAttnArgs {
  const void *q;
  MxView cv;
  int nq, qpk, qpc, dh, dl, kw, cw, splits, ps_shift;
  float scale_log2e;
  float *pacc, *pml;   // [batch, splits, n_q, d_l], [batch, splits, n_q, 2]
  void *l_out;         // the result itself where there is one split, or NULL
};

// rows of the slot that take part
__device__ __forceinline__ int mx_rows(const MxView &cv, int b, int &slot) {
  slot = cv.slots ? cv.slots[b] : b;
  return slot >= 0 && slot < cv.max_batch ? min(max(cv.seq_lens[slot], 0), cv.max_seq) : 0;
}

// rows [j0, j1) of split s of n rows, in units of `unit` rows
__device__ __forceinline__ void mx_slice(int n, int s, int splits, int unit, int &j0, int &j1) {
  const int64_t units = (n + unit - 1) / unit;
  j0 = (int)min((int64_t)n, units * s / splits * unit);
  j1 = (int)min((int64_t)n, units * (s + 1) / splits * unit);
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__bf16 v) { return (float)v; }

constexpr int kAnyMaxHead = 1024, kAnyMaxLatent = 4096;

// Any widths and page sizes: a workgroup per (split, map, sequence), a row per thread for the scores, four latents per
// thread for the sums.
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
  mx_slice(n, s, a.splits, 1, j0, j1);
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
    l = l * corr + (red2[0] + red2[1]) + (red2[2] + red2[3]);
    m = mn;
    for (int v = 0; v * 256 + my < quads; ++v)
      for (int e = 0; e < 4; ++e) acc[v][e] *= corr;
    if (grp < groups)
      for (int r = grp; r < cnt; r += groups) {
        const float pr = ps[r];
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
  const int64_t at = ((int64_t)b * a.splits + s) * a.nq + g;
  float *out = a.pacc + at * a.dl;
  if (groups == 1) {
    for (int v = 0; v * 256 + my < quads; ++v)
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
// A wave takes tiles of TT rows and keeps everything of a tile in registers, codes included: no barrier until the waves'
// sums are joined, and the loads of the next tile go out piece by piece as the registers of this one come free.
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

template <typename T, int KB, int CS, int TT, int OCC>
__global__ __launch_bounds__(256, OCC) void mx_attn_kernel(MxAttnArgs a) {
  constexpr int NQP = Parts<T>::Q, NPP = Parts<T>::P;
  constexpr int HF = TT / 16, KP = KB / 64;                          // half tiles, key pieces
  constexpr int LC = CS >= 256 ? 16 : CS / 16, NCH = CS / (16 * LC);   // bytes per lane and load, chunks
  constexpr int KW = KB >= 128 ? KB / 128 : 1;                       // scale words of a key row: four bytes (two for one piece)
  constexpr bool QREG = KB * NQP <= 256;
  typedef typename Word<LC>::type CWord;
  extern __shared__ char lds[];
  const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s = blockIdx.x, z = blockIdx.y, b = blockIdx.z;
  int slot, j0, j1;
  const int n = mx_rows(a.cv, b, slot);
  mx_slice(n, s, a.splits, TT, j0, j1);
  const int64_t part = ((int64_t)b * a.splits + s) * a.nq;
  if (j0 >= j1) {
    if (a.l_out) {
      for (int i = tid; i < a.nq * CS; i += 256) {
        const int g = i / CS, col = z * CS + i % CS;
        if (col / a.dl == g / a.qpc) ((T *)a.l_out)[((int64_t)b * a.nq + g) * a.dl + col % a.dl] = (T)0.f;
      }
    } else if (z == 0 && tid < a.nq) {
      a.pml[(part + tid) * 2] = -INFINITY;
      a.pml[(part + tid) * 2 + 1] = 0.f;
    }
    return;
  }
  const int nt = (j1 - j0 + TT - 1) / TT;

  // pool row of the first row of half tile hf of tile t, and the last row of that half that exists; a half behind the slice's
  // end takes the rows of the last one that is not
  auto half_at = [&](int t, int hf, int &lim) -> int64_t {
    int jb = j0 + t * TT + hf * 16;
    jb = min(jb, (j1 - 1) & ~15);
    lim = min(15, j1 - 1 - jb);
    if (!a.cv.pm.table) return (int64_t)slot * a.cv.max_seq + jb;
    // (constant memory: a scalar load that waits for no other load)
    typedef const __attribute__((address_space(4))) int32_t *Table;
    int pg = ((Table)a.cv.pm.table)[(int64_t)slot * a.cv.pm.pages_per_slot + (jb >> a.ps_shift)];
    pg = (unsigned)pg >= (unsigned)a.cv.pm.num_pages ? 0 : pg;
    return ((int64_t)pg << a.ps_shift) + (jb & ((1 << a.ps_shift) - 1));
  };

  u32x4 kb[HF][KP];
  unsigned ks[HF][KW];
  CWord cb[HF][4][NCH];
  unsigned cs[HF][4][NCH];
  struct At { int64_t row[HF]; int lim[HF]; };
  auto at_tile = [&](int t) { At r; 
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) r.row[hf] = half_at(t, hf, r.lim[hf]);
    return r; };
  auto load_key_scales = [&](const At &at) {
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) {
      const uint8_t *base = a.cv.ks + at.row[hf] * (KB / 32);
#pragma unroll
      for (int i = 0; i < KW; ++i) {
        const uint8_t *p = base + (unsigned)(min(x, at.lim[hf]) * (KB / 32) + i * 4);
        if constexpr (KB >= 128) ks[hf][i] = __builtin_nontemporal_load(reinterpret_cast<const unsigned *>(p));
        else ks[hf][i] = __builtin_nontemporal_load(reinterpret_cast<const unsigned short *>(p));
      }
    }
  };
  auto load_keys = [&](const At &at, int p) {
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) {
      const uint8_t *base = a.cv.k + at.row[hf] * KB;
      kb[hf][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(base + (unsigned)(min(x, at.lim[hf]) * KB + h * 16 + p * 64)));
    }
  };
  auto load_latents = [&](const At &at, int c) {
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) {
      const uint8_t *base = a.cv.c + at.row[hf] * a.cw + z * CS;
      const uint8_t *sb = a.cv.cs + at.row[hf] * (a.cw / 32) + z * (CS / 32);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = min(4 * h + j, at.lim[hf]);
        cb[hf][j][c] = __builtin_nontemporal_load(reinterpret_cast<const CWord *>(base + (unsigned)(r * a.cw + x * LC + c * 16 * LC)));
        cs[hf][j][c] = __builtin_nontemporal_load(sb + (unsigned)(r * (a.cw / 32) + x * LC / 32 + c * 16 * LC / 32));
      }
    }
  };

  // the first tile's rows are on their way while the queries are laid out
  At nxt{};
  auto start = [&]() {
    const At first = at_tile(wave);
    load_key_scales(first);
#pragma unroll
    for (int p = 0; p < KP; ++p) load_keys(first, p);
#pragma unroll
    for (int c = 0; c < NCH; ++c) load_latents(first, c);
    nxt = at_tile(min(wave + 4, nt - 1));
  };
  if (wave < nt) start();
  const int ppk = a.dh / 64;   // pieces of a key head
  const int kg = x < a.nq ? x / a.qpk : -1;
  auto query_fragment = [&](int f, bf16x8 (&out)[NQP]) {   // second operand for half a piece: dimensions h * 16 + (f & 1) * 8 ..
    const int p = f >> 1;
    const bool mine = kg == p / ppk;
    typedef __attribute__((ext_vector_type(8))) T Eight;
    const Eight src = *reinterpret_cast<const Eight *>((const T *)a.q + ((int64_t)b * a.nq + (mine ? x : 0)) * a.dh + (p % ppk) * 64 + h * 16 + (f & 1) * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      __bf16 v[NQP];
      split_parts<NQP>(mine ? to_f(src[e]) : 0.f, v);
#pragma unroll
      for (int i = 0; i < NQP; ++i) out[i][e] = v[i];
    }
  };
  bf16x8 qr[QREG ? KP * 2 : 1][NQP];
  bf16x8 *qs = reinterpret_cast<bf16x8 *>(lds);   // [KP * 2][NQP][64]
  if constexpr (QREG) {
#pragma unroll
    for (int f = 0; f < KP * 2; ++f) query_fragment(f, qr[f]);
  } else {
    for (int f = wave; f < KP * 2; f += 4) {
      bf16x8 v[NQP];
      query_fragment(f, v);
#pragma unroll
      for (int i = 0; i < NQP; ++i) qs[(f * NQP + i) * 64 + lane] = v[i];
    }
    __syncthreads();
  }

  f32x4 acc[NCH][LC];
  float m = -INFINITY, l = 0.f, seen = -INFINITY;   // what weights refer to, their sum, the largest score of this lane's rows

  auto tile = [&](int t, auto more) {
    constexpr bool MORE = decltype(more)::value;
    // ---- scores
    f32x4 sc[HF];
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) sc[hf] = f32x4{0.f, 0.f, 0.f, 0.f};
    unsigned kscale[HF][KW];
#pragma unroll
    for (int hf = 0; hf < HF; ++hf)
#pragma unroll
      for (int i = 0; i < KW; ++i) kscale[hf][i] = ks[hf][i] >> (8 * (h >> 1));
    if constexpr (MORE) load_key_scales(nxt);
#pragma unroll
    for (int p = 0; p < KP; ++p) {
      f32x4 d[HF];
#pragma unroll
      for (int hf = 0; hf < HF; ++hf) d[hf] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 qf[NQP];
#pragma unroll
        for (int i = 0; i < NQP; ++i) {
          if constexpr (QREG) qf[i] = qr[p * 2 + half][i];
          else qf[i] = qs[((p * 2 + half) * NQP + i) * 64 + lane];
        }
#pragma unroll
        for (int hf = 0; hf < HF; ++hf) {
          const unsigned w = kscale[hf][p / 2];
          const float sl = __uint_as_float((p & 1 ? w << 7 : w << 23) & 0x7f800000u);
          const u32x4 k4 = {cvt_lo(kb[hf][p][2 * half], sl), cvt_hi(kb[hf][p][2 * half], sl), cvt_lo(kb[hf][p][2 * half + 1], sl),
                            cvt_hi(kb[hf][p][2 * half + 1], sl)};
#pragma unroll
          for (int i = 0; i < NQP; ++i)
            d[hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k4), qf[i], d[hf], 0, 0, 0);
        }
      }
      if constexpr (MORE) load_keys(nxt, p);
      const bool mine = kg == p / ppk;
#pragma unroll
      for (int hf = 0; hf < HF; ++hf)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[hf][i] += mine ? d[hf][i] : 0.f;
      __builtin_amdgcn_sched_barrier(0);   // one piece at a time: conversions taken up early would need registers
    }
    // ---- weights
    const int left = j1 - (j0 + t * TT);   // rows of this tile
    float mx = -INFINITY;
#pragma unroll
    for (int hf = 0; hf < HF; ++hf)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[hf][i] = hf * 16 + 4 * h + i < left ? sc[hf][i] * a.scale_log2e : -INFINITY;
        mx = fmaxf(mx, sc[hf][i]);
      }
    seen = fmaxf(seen, mx);
    if (t == wave && m == -INFINITY) {
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
    // ---- sums
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
            if constexpr (HF == 2)
              d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{op[e][0], op[e][1], op[e][2], op[e][3]}),
                                                          __builtin_bit_cast(bf16x8, u32x4{pp[i][0], pp[i][1], pp[i][2], pp[i][3]}), d, 0, 0, 0);
            else
              d = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, u32x2{op[e][0], op[e][1]}),
                                                            __builtin_bit_cast(s16x4, u32x2{pp[i][0], pp[i][1]}), d, 0, 0, 0);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (MORE) load_latents(nxt, c);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  while (true) {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < LC; ++j) acc[c][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
    int t = wave;
    for (; t + 4 < nt; t += 4) {
      const At after = at_tile(min(t + 8, nt - 1));
      tile(t, std::true_type{});
      nxt = after;
    }
    if (t < nt) tile(t, std::false_type{});
    seen = fmaxf(seen, __shfl_xor(seen, 16));
    seen = fmaxf(seen, __shfl_xor(seen, 32));
    if (!__any(seen > m + kMostAbove)) break;   // (always the second time)
    m = fmaxf(m, seen);
    start();
  }

  // ---- the four waves' sums, chunk by chunk through LDS
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  __syncthreads();   // queries are not read any more
  float *sm = reinterpret_cast<float *>(lds), *sl = sm + 64, *buf = sm + 128;   // [4][16], [4][16], [4][n_q][16 * LC]
  if (lane < 16) { sm[wave * 16 + x] = m; sl[wave * 16 + x] = l; }
  __syncthreads();
  float top = fmaxf(fmaxf(sm[x], sm[16 + x]), fmaxf(sm[32 + x], sm[48 + x]));
  const float f = __builtin_amdgcn_exp2f(fmaxf(m, kLowest) - fmaxf(top, kLowest));
  auto joined = [&](int g, float &mg) {   // sum of the weights of map g
    mg = fmaxf(fmaxf(sm[g], sm[16 + g]), fmaxf(sm[32 + g], sm[48 + g]));
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) v += sl[w * 16 + g] * __builtin_amdgcn_exp2f(fmaxf(sm[w * 16 + g], kLowest) - fmaxf(mg, kLowest));
    return v;
  };
  if (!a.l_out && z == 0 && tid < a.nq) {
    float mg;
    const float lg = joined(tid, mg);
    a.pml[(part + tid) * 2] = mg;
    a.pml[(part + tid) * 2 + 1] = lg;
  }
  constexpr int CW = 16 * LC;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    if (c) __syncthreads();
    if (x < a.nq) {
      float *dst = buf + (wave * a.nq + x) * CW;
#pragma unroll
      for (int j = 0; j < LC; j += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4 *>(dst + (4 * h + i) * LC + j) =
              f32x4{acc[c][j][i] * f, acc[c][j + 1][i] * f, acc[c][j + 2][i] * f, acc[c][j + 3][i] * f};
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();
    for (int i = tid; i < a.nq * (CW / 4); i += 256) {
      const int g = i / (CW / 4), cc = i % (CW / 4) * 4, col = z * CS + c * CW + cc;
      if (col / a.dl != g / a.qpc) continue;
      f32x4 v = *reinterpret_cast<const f32x4 *>(buf + g * CW + cc);
#pragma unroll
      for (int w = 1; w < 4; ++w) v += *reinterpret_cast<const f32x4 *>(buf + (w * a.nq + g) * CW + cc);
      if (a.l_out) {
        float mg;
        const float inv = 1.f / joined(g, mg);
        T *o = (T *)a.l_out + ((int64_t)b * a.nq + g) * a.dl + col % a.dl;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (T)(v[e] * inv);
      } else {
        *reinterpret_cast<f32x4 *>(a.pacc + (part + g) * a.dl + col % a.dl) = v;
      }
    }
  }
}

// Joins the splits: a thread per latent of a map.
template <typename T>
__global__ __launch_bounds__(256) void mx_join_kernel(MxView cv, const float *pacc, const float *pml, int splits, int nq, int dl, T *l_out) {
  const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  if (i >= nq * dl) return;
  int slot;
  const int n = mx_rows(cv, b, slot);
  const int g = i / dl;
  const int64_t base = (int64_t)b * splits * nq;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int s = 0; s < splits; ++s) m = fmaxf(m, pml[(base + s * nq + g) * 2]);
  for (int s = 0; s < splits; ++s) {
    const int64_t at = base + s * nq + g;
    const float ls = pml[at * 2 + 1];
    if (ls == 0.f) continue;                        // a split without rows
    const float ms = pml[at * 2];
    const float w = ms == m ? 1.f : exp2f(ms - m);   // (-inf) - (-inf): scores of nothing but NaN
    l = fmaf(ls, w, l);
    acc = fmaf(pacc[at * dl + i % dl], w, acc);
  }
  l_out[(int64_t)b * nq * dl + i] = (T)(n == 0 ? 0.f : acc / l);   // scores of nothing but -inf: 0 / 0
}

}  // namespace

bool mx_decode_dims_ok(const Dims &d) { return mx_widths_ok(d) && d.dh <= kAnyMaxHead && d.dl <= kAnyMaxLatent && d.nq <= 65535; }

// Widths of a latent slice: one workgroup's columns of a latent row.
static int mx_slice_width(const Dims &d) {
  for (int cs = 1024; cs >= 128; cs /= 2)
    if (d.wc_w % cs == 0 && (d.wc_w == cs || cs >= 512)) return cs;
  return 0;
}

// The matrix-instruction kernel takes heads of whole pieces of 64, up to 16 maps, and the rows that are instantiated.
bool mx_decode_tuned(const Dims &d) {
  const int cs = mx_slice_width(d), kb = d.wk_w;
  if (d.dh % 64 || d.nq > 16 || cs == 0) return false;
  return (kb == 64 && cs <= 512) || (kb == 128 && cs <= 512) || (kb == 256 && cs >= 256) || (kb == 512 && cs >= 512) || (kb == 1024 && cs == 1024);
}

static bool mx_layout_tuned(const MxView &cv) {
  return !cv.pm.table || (cv.pm.page_size >= 16 && (cv.pm.page_size & (cv.pm.page_size - 1)) == 0);
}

int mx_decode_splits(const Dims &d, int batch, int max_seq) {
  if (mx_decode_tuned(d)) {
    const int z = d.wc_w / mx_slice_width(d);
    const int target = d.wk_w + mx_slice_width(d) >= 1024 ? 256 : d.wk_w + mx_slice_width(d) >= 512 ? 512 : 1024;
    const int want = target / (batch * z), cap = max_seq / 128;
    return std::max(1, std::min(std::min(want, cap), 256));
  }
  const int want = (1024 + batch * d.nq - 1) / (batch * d.nq), cap = max_seq / 256;
  return std::max(1, std::min(std::min(want, cap), 256));
}

template <typename T, int KB, int CS>
static void launch_tuned(const MxAttnArgs &a, int z, int batch, hipStream_t st) {
  constexpr int TT = KB + CS > 512 ? 16 : 32;
  constexpr int OCC = CS >= 1024 ? 1 : KB + CS >= 512 ? 2 : KB + CS > 192 ? 3 : 4;
  constexpr int LC = CS >= 256 ? 16 : CS / 16;
  const int lds = std::max(KB * Parts<T>::Q * 32, 512 + 4 * a.nq * 16 * LC * 4);
  if (lds > 65536) allow_dynamic_lds((const void *)mx_attn_kernel<T, KB, CS, TT, OCC>, lds);
  mx_attn_kernel<T, KB, CS, TT, OCC><<<dim3(a.splits, z, batch), 256, lds, st>>>(a);
}

template <typename T>
static void launch_decode(const Dims &d, MxAttnArgs a, int batch, hipStream_t st) {
  const int splits = a.splits;
  T *out = (T *)a.l_out;
  if (mx_decode_tuned(d) && mx_layout_tuned(a.cv)) {
    const int cs = mx_slice_width(d), z = d.wc_w / cs;
    if (splits > 1) a.l_out = nullptr;
    switch (d.wk_w * 4096 + cs) {
      case 64 * 4096 + 128: launch_tuned<T, 64, 128>(a, z, batch, st); break;
      case 64 * 4096 + 256: launch_tuned<T, 64, 256>(a, z, batch, st); break;
      case 64 * 4096 + 512: launch_tuned<T, 64, 512>(a, z, batch, st); break;
      case 128 * 4096 + 128: launch_tuned<T, 128, 128>(a, z, batch, st); break;
      case 128 * 4096 + 256: launch_tuned<T, 128, 256>(a, z, batch, st); break;
      case 128 * 4096 + 512: launch_tuned<T, 128, 512>(a, z, batch, st); break;
      case 256 * 4096 + 256: launch_tuned<T, 256, 256>(a, z, batch, st); break;
      case 256 * 4096 + 512: launch_tuned<T, 256, 512>(a, z, batch, st); break;
      case 256 * 4096 + 1024: launch_tuned<T, 256, 1024>(a, z, batch, st); break;
      case 512 * 4096 + 512: launch_tuned<T, 512, 512>(a, z, batch, st); break;
      case 512 * 4096 + 1024: launch_tuned<T, 512, 1024>(a, z, batch, st); break;
      case 1024 * 4096 + 1024: launch_tuned<T, 1024, 1024>(a, z, batch, st); break;
    }
    if (splits == 1) return;
  } else {
    mx_attn_any_kernel<T><<<dim3(splits, d.nq, batch), 256, 0, st>>>(a);
  }
  mx_join_kernel<T><<<dim3((d.nq * d.dl + 255) / 256, batch), 256, 0, st>>>(a.cv, a.pacc, a.pml, splits, d.nq, d.dl, out);
}

int launch_mx_decode(const Dims &d, const void *q, const MxView &cv, int batch, int splits, float *part, void *l_out, hipStream_t st) {
  int shift = 0;
  if (cv.pm.table) while ((1 << shift) < cv.pm.page_size && shift < 30) ++shift;
  const MxAttnArgs a{q, cv, d.nq, d.qpk, d.qpc, d.dh, d.dl, d.wk_w, d.wc_w, splits, shift, d.scale * 1.4426950408889634f,
                     part, part + (int64_t)batch * splits * d.nq * d.dl, l_out};
  if (d.dtype == GTA_BF16) launch_decode<__bf16>(d, a, batch, st);
  else launch_decode<float>(d, a, batch, st);
  return check_launch();
}

}  // namespace gta
