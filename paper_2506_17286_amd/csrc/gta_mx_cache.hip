// 8-bit cache rows written and read back.
//   append: block exponent e = least integer with amax <= 448 * 2^e (amax: largest finite magnitude of the 32 elements),
//           kept in [-117, 119]; code = x * 2^-e rounded to e4m3 (to nearest, ties to even).  The scaling is by a power of
//           two and exact, so a code is the one rounding there is.  NaN and infinities become the NaN code.
//   read:   code * 2^e, exact in bf16 and fp32.
#include <type_traits>

#include "gta_mx.h"

namespace gta {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

typedef __attribute__((ext_vector_type(4))) float f32x4;

// eight consecutive elements; VEC: on 16 bytes
template <bool VEC>
__device__ __forceinline__ f32x8 load8(const float *p) {
  if constexpr (VEC) return __builtin_shufflevector(*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4), 0, 1, 2, 3, 4, 5, 6, 7);
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = p[i];
  return v;
}
template <bool VEC>
__device__ __forceinline__ f32x8 load8(const __bf16 *p) {
  if constexpr (VEC) return __builtin_convertvector(*reinterpret_cast<const bf16x8 *>(p), f32x8);
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)p[i];
  return v;
}

// A workgroup's rows as words of ELEMS elements, keys first: `per_row` of them a row, and an inverse of it for divisions (exact for
// the numbers that come up: below 2^11, or below per_row <= 2^16).
struct Words {
  int kw, cw, per_row;
  unsigned inverse;
};
// Most words of a sequence that one workgroup stores, setting the length as well, in place of a launch of many and one behind it for
// the lengths: 1 to 64 sequences of 2048 words (32 rows of 1024 elements) 6.7 to 7.4 us against 9.1, half as much again level,
// of 4096 words 10.2 to 14.4 against 8.8 to 9.4; 300 sequences of 1024 words 6.8 to 7.5 against 9.1, of 2048 10.7 to 11.5 against 9.1 to 12.6.
constexpr int kMostWords = 2048;

// Where word i of the workgroup lies: its row there, its column, whether it is a key's.
struct Place { int row, at, width; bool key; };
template <int ELEMS>
__device__ __forceinline__ Place place_of(const Words &w, int i) {
  Place p;
  p.row = (int)__umulhi((unsigned)i, w.inverse);
  const int col = (i - p.row * w.per_row) * ELEMS;
  p.key = col < w.kw;
  p.at = p.key ? col : col - w.kw;
  p.width = p.key ? w.kw : w.cw;
  return p;
}

// Exponent of a block by its largest finite magnitude: 448 = 1.75 * 2^8.
__device__ __forceinline__ int mx_exponent(float amax) {
  const unsigned u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kMxMinExp), kMxMaxExp);
}

// Sixteen elements of a block, two lanes to a block: codes, and the block's exponent.
__device__ __forceinline__ u32x4 quantise16(const f32x8 (&x)[2], int &e) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) { const float m = fabsf(x[i >> 3][i & 7]); amax = fmaxf(amax, m < INFINITY ? m : 0.f); }
  amax = fmaxf(amax, __shfl_xor(amax, 1));
  e = mx_exponent(amax);
  const float inv = __uint_as_float((unsigned)(127 - e) << 23);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = x[i >> 1][(i & 1) * 4 + j];
      const float s = fminf(fmaxf(v * inv, -448.f), 448.f);   // beyond 448 only where e is at its upper end
      y[j] = fabsf(v) < INFINITY ? s : __builtin_nanf("");
    }
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
  }
  return w;
}

// What sequence b adds, or why it does not: rows (0: nothing to do), slot, first row.
struct AppendPlan { int n, slot, p; bool full; };

__device__ __forceinline__ AppendPlan append_plan(const MxView &cv, const int32_t *cu_new, int b, int max_new) {
  AppendPlan a{0, -1, 0, false};
  const int n = cu_new[b + 1] - cu_new[b];
  const int slot = cv.slots ? cv.slots[b] : b;
  if (n <= 0 || slot < 0 || slot >= cv.max_batch) return a;
  a.slot = slot;
  a.n = n;
  if (n > max_new) return a;
  a.p = cv.seq_lens[slot];
  a.full = a.p < 0 || (int64_t)a.p + n > cv.max_seq || !rows_backed_wave(cv.pm, slot, a.p, a.p + n);
  return a;
}

// rows_per_wg rows of sequence blockIdx.y from blockIdx.x * rows_per_wg on, a thread to sixteen elements and two threads to a block:
// a whole 16-byte word of codes to store (eight elements a thread: 16 sequences of 300..2048 rows of 2048 elements 39 us against 31).
// Bound by memory, and by the chain of loads in front (lengths, slot, pages) where there are few rows; with a second word on its
// way per thread it took as long.  Codes of prompts go past the caches whatever their size: below 20 MB that takes as long as keeping
// them, an attention over the rows right behind included (8 x 512 rows of 1024 elements 13.3 us, with it 21.7 against 22.0); fp32 prompts
// of 35 to 70 MB 30 to 65 us against 35 to 72.
// COMMIT: the workgroup has the whole sequence and sets its length as well.
template <typename T, bool COMMIT, bool VEC>
__global__ __launch_bounds__(256) void mx_append_kernel(MxView cv, const T *k_new, int64_t k_stride, const T *c_new, int64_t c_stride,
                                                        const int32_t *cu_new, Words w, int max_new, int rows_per_wg) {
  const int b = blockIdx.y;
  const AppendPlan a = append_plan(cv, cu_new, b, max_new);
  if (a.slot < 0) return;
  if (a.n <= max_new && !a.full) {
    const int j0 = blockIdx.x * rows_per_wg, words = min(max(a.n - j0, 0), rows_per_wg) * w.per_row;   // (behind the last row: 0, no product that wraps)
    const int64_t src0 = (int64_t)cu_new[b] + j0;
    for (int i = threadIdx.x; i < words; i += 256) {
      const Place p = place_of<16>(w, i);
      const T *src = p.key ? k_new + (src0 + p.row) * k_stride + p.at : c_new + (src0 + p.row) * c_stride + p.at;
      const f32x8 x[2] = {load8<VEC>(src), load8<VEC>(src + 8)};
      const int64_t dst = cache_row(cv.pm, cv.max_seq, a.slot, a.p + j0 + p.row);
      int e;
      const u32x4 codes = quantise16(x, e);
      store16<!COMMIT>(reinterpret_cast<u32x4 *>((p.key ? cv.k : cv.c) + dst * p.width + p.at), codes);   // (prompts: past the caches, at any size)
      if ((p.at & 31) == 0) (p.key ? cv.ks : cv.cs)[dst * (p.width / kMxBlock) + p.at / kMxBlock] = (uint8_t)(e + 127);
    }
  }
  if (COMMIT) {
    __syncthreads();
    if (threadIdx.x == 0) {
      if (a.n > max_new) cv.status[a.slot] = GTA_ERR_SHAPE;
      else if (a.full) cv.status[a.slot] = GTA_ERR_CACHE_FULL;
      else cv.seq_lens[a.slot] = a.p + a.n;
    }
  }
}

// a wave per sequence
__global__ __launch_bounds__(256) void mx_append_commit_kernel(MxView cv, const int32_t *cu_new, int batch, int max_new) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b >= batch) return;
  const AppendPlan a = append_plan(cv, cu_new, b, max_new);
  if (a.slot < 0 || (threadIdx.x & 63)) return;
  if (a.n > max_new) cv.status[a.slot] = GTA_ERR_SHAPE;   // caller's bound was wrong: nothing stored
  else if (a.full) cv.status[a.slot] = GTA_ERR_CACHE_FULL;
  else cv.seq_lens[a.slot] = a.p + a.n;
}

// A thread has the elements of one 16-byte word to store, next to its neighbours': stores past the caches want that (with two words
// a thread, 32 bytes apart, 41 000 rows took 46 us against 25).  Two words of codes on their way per thread.
constexpr int kAtOnce = 2;
template <typename T> constexpr int kReadElems = 16 / (int)sizeof(T);

template <typename T, bool NT>
__global__ __launch_bounds__(256) void mx_read_kernel(MxView cv, const int32_t *first, const int32_t *cu_rows, Words w, int max_rows,
                                                      int rows_per_wg, T *k_out, T *c_out) {
  const int b = blockIdx.y, n = cu_rows[b + 1] - cu_rows[b];
  const int slot = cv.slots ? cv.slots[b] : b;
  const bool slot_ok = slot >= 0 && slot < cv.max_batch;
  if (n > max_rows) {   // caller's bound was wrong: nothing read
    if (slot_ok && blockIdx.x == 0 && threadIdx.x == 0) cv.status[slot] = GTA_ERR_SHAPE;
    return;
  }
  const int j0 = blockIdx.x * rows_per_wg, words = min(max(max(n, 0) - j0, 0), rows_per_wg) * w.per_row;
  const int have = slot_ok ? min(cv.seq_lens[slot], cv.max_seq) : 0;
  const int64_t row0 = (int64_t)(first ? first[b] : 0) + j0, dst0 = (int64_t)cu_rows[b] + j0;
  constexpr int E = kReadElems<T>;
  for (int i0 = threadIdx.x; i0 < words; i0 += 256 * kAtOnce) {
    unsigned codes[kAtOnce][E / 4];
    float scale[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = i0 + 256 * u;
      if (i >= words) break;
      const Place p = place_of<E>(w, i);
      const int64_t row = row0 + p.row, src = row >= 0 && row < have ? cache_row(cv.pm, cv.max_seq, slot, (int)row) : -1;
#pragma unroll
      for (int h = 0; h < E / 4; ++h) codes[u][h] = 0u;   // rows that are not there read as zeros
      scale[u] = 0.f;
      if (src >= 0) {
        const uint8_t *at = (p.key ? cv.k : cv.c) + src * p.width + p.at;
        if constexpr (E == 8) {
          const u32x2 c = *reinterpret_cast<const u32x2 *>(at);
          codes[u][0] = c.x;
          codes[u][1] = c.y;
        } else {
          codes[u][0] = *reinterpret_cast<const unsigned *>(at);
        }
        scale[u] = mx_scale((p.key ? cv.ks : cv.cs)[src * (p.width / kMxBlock) + p.at / kMxBlock]);
      }
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = i0 + 256 * u;
      if (i >= words) break;
      const Place p = place_of<E>(w, i);
      typedef __attribute__((ext_vector_type(E))) float Vf;
      typedef __attribute__((ext_vector_type(E))) T Vt;
      Vf v;
#pragma unroll
      for (int h = 0; h < E / 4; ++h) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[u][h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[u][h], true);
        v[4 * h] = lo[0] * scale[u]; v[4 * h + 1] = lo[1] * scale[u]; v[4 * h + 2] = hi[0] * scale[u]; v[4 * h + 3] = hi[1] * scale[u];
      }
      store16<NT>(reinterpret_cast<Vt *>((p.key ? k_out : c_out) + (dst0 + p.row) * p.width + p.at), __builtin_convertvector(v, Vt));
    }
  }
}

}  // namespace

// Rows of a workgroup: about `words` words of them.
static int rows_per_workgroup(const Words &w, int words) { return std::max(1, words / w.per_row); }

static Words words_of(const Dims &d, int elems) {
  const int per_row = (d.wk_w + d.wc_w) / elems;
  return Words{d.wk_w, d.wc_w, per_row, (unsigned)(((uint64_t)1 << 32) / per_row + 1)};
}

int launch_mx_append(const Dims &d, const MxView &cv, const void *k_new, int64_t k_stride, const void *c_new, int64_t c_stride,
                     const int32_t *cu_new, int batch, int max_new, hipStream_t st) {
  const Words w = words_of(d, 16);
  const int most = std::min(max_new, cv.max_seq);   // a sequence of more rows than a slot has stores none
  // few rows: a workgroup per sequence; otherwise the lengths need a launch behind this one (every workgroup reads the old one)
  const bool one = (int64_t)most * w.per_row <= kMostWords;
  const int rows = one ? std::max(most, 1) : rows_per_workgroup(w, 512);
  const dim3 grid(one ? 1u : (unsigned)(((int64_t)most + rows - 1) / rows), batch);
  if (grid.x >= (1u << 24)) return GTA_ERR_UNSUPPORTED;   // launch size
  auto run = [&](auto t) {
    using T = decltype(t);
    const T *k = (const T *)k_new, *c = (const T *)c_new;
    const int64_t per = 16 / (int)sizeof(T);
    const bool vec = k_stride % per == 0 && c_stride % per == 0 && (((uintptr_t)k | (uintptr_t)c) & 15u) == 0;
    auto go = [&](auto commit, auto v) {
      mx_append_kernel<T, decltype(commit)::value, decltype(v)::value><<<grid, 256, 0, st>>>(cv, k, k_stride, c, c_stride, cu_new, w, max_new, rows);
    };
    if (one) { if (vec) go(std::true_type{}, std::true_type{}); else go(std::true_type{}, std::false_type{}); }
    else { if (vec) go(std::false_type{}, std::true_type{}); else go(std::false_type{}, std::false_type{}); }
    if (!one) mx_append_commit_kernel<<<(batch + 3) / 4, 256, 0, st>>>(cv, cu_new, batch, max_new);
  };
  if (d.dtype == GTA_BF16) run(__bf16{}); else run(float{});
  return check_launch();
}

int launch_mx_read(const Dims &d, const MxView &cv, const int32_t *first, const int32_t *cu_rows, int batch, int max_rows,
                   void *k_out, void *c_out, hipStream_t st) {
  const Words w = words_of(d, d.dtype == GTA_BF16 ? kReadElems<__bf16> : kReadElems<float>);
  const int rows = rows_per_workgroup(w, 1024);
  const dim3 grid((unsigned)(((int64_t)max_rows + rows - 1) / rows), batch);
  if (grid.x == 0) return GTA_OK;
  if (grid.x >= (1u << 24)) return GTA_ERR_UNSUPPORTED;   // launch size
  auto run = [&](auto t, auto nt) {
    using T = decltype(t);
    mx_read_kernel<T, decltype(nt)::value><<<grid, 256, 0, st>>>(cv, first, cu_rows, w, max_rows, rows, (T *)k_out, (T *)c_out);
  };
  if (stream_past_caches((int64_t)batch * max_rows * (d.wk_w + d.wc_w) * d.esize())) {
    if (d.dtype == GTA_BF16) run(__bf16{}, std::true_type{}); else run(float{}, std::true_type{});
  } else {
    if (d.dtype == GTA_BF16) run(__bf16{}, std::false_type{}); else run(float{}, std::false_type{});
  }
  return check_launch();
}

}  // namespace gta
