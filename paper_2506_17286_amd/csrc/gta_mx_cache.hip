// 8-bit cache rows written and read back.
//   append: block exponent e = least integer with amax <= 448 * 2^e (amax: largest finite magnitude of the 32 elements),
//           kept in [-117, 119]; code = x * 2^-e rounded to e4m3 (to nearest, ties to even).  The scaling is by a power of
//           two and exact, so a code is the one rounding there is.  NaN and infinities become the NaN code.
//   read:   code * 2^e, exact in bf16 and fp32.
#include "gta_mx.h"

namespace gta {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

__device__ __forceinline__ f32x8 load8(const float *p) { f32x8 v; for (int i = 0; i < 8; ++i) v[i] = p[i]; return v; }
__device__ __forceinline__ f32x8 load8(const __bf16 *p) { f32x8 v; for (int i = 0; i < 8; ++i) v[i] = (float)p[i]; return v; }

// Exponent of a block by its largest finite magnitude: 448 = 1.75 * 2^8.
__device__ __forceinline__ int mx_exponent(float amax) {
  const unsigned u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kMxMinExp), kMxMaxExp);
}

// Eight elements of a block, four lanes to a block: codes, and the block's exponent.
__device__ __forceinline__ u32x2 quantise8(const f32x8 &x, int &e) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) { const float m = fabsf(x[i]); amax = fmaxf(amax, m < INFINITY ? m : 0.f); }
  amax = fmaxf(amax, __shfl_xor(amax, 1));
  amax = fmaxf(amax, __shfl_xor(amax, 2));
  e = mx_exponent(amax);
  const float inv = __uint_as_float((unsigned)(127 - e) << 23);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool finite = fabsf(x[i]) < INFINITY;
    const float s = fminf(fmaxf(x[i] * inv, -448.f), 448.f);   // beyond 448 only where e is at its upper end
    y[i] = finite ? s : __builtin_nanf("");
  }
  unsigned w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], r, true);
  }
  return u32x2{w[0], w[1]};
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

// Lanes of a row: one per 8 elements, keys first.  rows_per_wg rows of sequence blockIdx.y from blockIdx.x * rows_per_wg on.
// COMMIT: the workgroup has the whole sequence and sets its length as well.
template <typename T, bool COMMIT>
__global__ __launch_bounds__(256) void mx_append_kernel(MxView cv, const T *k_new, int64_t k_stride, const T *c_new, int64_t c_stride,
                                                        const int32_t *cu_new, int kw, int cw, int max_new, int rows_per_wg) {
  const int b = blockIdx.y;
  const AppendPlan a = append_plan(cv, cu_new, b, max_new);
  if (a.slot < 0) return;
  if (a.n <= max_new && !a.full) {
    const int per_row = (kw + cw) / 8, j0 = blockIdx.x * rows_per_wg, j1 = min(a.n, j0 + rows_per_wg);
    for (int i = threadIdx.x; i < (j1 - j0) * per_row; i += 256) {
      const int j = j0 + i / per_row, col = i % per_row * 8;
      const int64_t src = (int64_t)cu_new[b] + j, dst = cache_row(cv.pm, cv.max_seq, a.slot, a.p + j);
      const bool key = col < kw;
      const int at = key ? col : col - kw, width = key ? kw : cw;
      int e;
      const u32x2 codes = quantise8(key ? load8(k_new + src * k_stride + at) : load8(c_new + src * c_stride + at), e);
      *reinterpret_cast<u32x2 *>((key ? cv.k : cv.c) + dst * width + at) = codes;
      if ((at & 31) == 0) (key ? cv.ks : cv.cs)[dst * (width / kMxBlock) + at / kMxBlock] = (uint8_t)(e + 127);
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

__device__ __forceinline__ void store8(float *p, const f32x8 &v) { for (int i = 0; i < 8; ++i) p[i] = v[i]; }
__device__ __forceinline__ void store8(__bf16 *p, const f32x8 &v) { for (int i = 0; i < 8; ++i) p[i] = (__bf16)v[i]; }

template <typename T>
__global__ __launch_bounds__(256) void mx_read_kernel(MxView cv, const int32_t *first, const int32_t *cu_rows, int kw, int cw,
                                                      int max_rows, int rows_per_wg, T *k_out, T *c_out) {
  const int b = blockIdx.y, n = cu_rows[b + 1] - cu_rows[b];
  const int slot = cv.slots ? cv.slots[b] : b;
  const bool slot_ok = slot >= 0 && slot < cv.max_batch;
  if (n > max_rows) {   // caller's bound was wrong: nothing read
    if (slot_ok && blockIdx.x == 0 && threadIdx.x == 0) cv.status[slot] = GTA_ERR_SHAPE;
    return;
  }
  const int per_row = (kw + cw) / 8, j0 = blockIdx.x * rows_per_wg, j1 = min(n, j0 + rows_per_wg);
  const int have = slot_ok ? min(cv.seq_lens[slot], cv.max_seq) : 0, f = first ? first[b] : 0;
  for (int i = threadIdx.x; i < (j1 - j0) * per_row; i += 256) {
    const int j = j0 + i / per_row, col = i % per_row * 8;
    const bool key = col < kw;
    const int at = key ? col : col - kw, width = key ? kw : cw;
    const int64_t row = (int64_t)f + j;
    const int64_t src = row >= 0 && row < have ? cache_row(cv.pm, cv.max_seq, slot, (int)row) : -1;
    f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (src >= 0) {
      const u32x2 w = *reinterpret_cast<const u32x2 *>((key ? cv.k : cv.c) + src * width + at);
      const float s = mx_scale((key ? cv.ks : cv.cs)[src * (width / kMxBlock) + at / kMxBlock]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
        v[4 * h] = lo[0] * s; v[4 * h + 1] = lo[1] * s; v[4 * h + 2] = hi[0] * s; v[4 * h + 3] = hi[1] * s;
      }
    }
    const int64_t dst = (int64_t)cu_rows[b] + j;
    store8((key ? k_out : c_out) + dst * width + at, v);
  }
}

}  // namespace

int launch_mx_append(const Dims &d, const MxView &cv, const void *k_new, int64_t k_stride, const void *c_new, int64_t c_stride,
                     const int32_t *cu_new, int batch, int max_new, hipStream_t st) {
  const int rows = 16;
  const dim3 grid((unsigned)((max_new + rows - 1) / rows), batch);
  auto run = [&](auto t) {
    using T = decltype(t);
    const T *k = (const T *)k_new, *c = (const T *)c_new;
    if (grid.x <= 1) {
      mx_append_kernel<T, true><<<dim3(1, batch), 256, 0, st>>>(cv, k, k_stride, c, c_stride, cu_new, d.wk_w, d.wc_w, max_new, rows);
      return;
    }
    mx_append_kernel<T, false><<<grid, 256, 0, st>>>(cv, k, k_stride, c, c_stride, cu_new, d.wk_w, d.wc_w, max_new, rows);
    mx_append_commit_kernel<<<(batch + 3) / 4, 256, 0, st>>>(cv, cu_new, batch, max_new);
  };
  if (d.dtype == GTA_BF16) run(__bf16{}); else run(float{});
  return check_launch();
}

int launch_mx_read(const Dims &d, const MxView &cv, const int32_t *first, const int32_t *cu_rows, int batch, int max_rows,
                   void *k_out, void *c_out, hipStream_t st) {
  const int rows = 16;
  const dim3 grid((unsigned)((max_rows + rows - 1) / rows), batch);
  if (grid.x == 0) return GTA_OK;
  if (d.dtype == GTA_BF16)
    mx_read_kernel<__bf16><<<grid, 256, 0, st>>>(cv, first, cu_rows, d.wk_w, d.wc_w, max_rows, rows, (__bf16 *)k_out, (__bf16 *)c_out);
  else
    mx_read_kernel<float><<<grid, 256, 0, st>>>(cv, first, cu_rows, d.wk_w, d.wc_w, max_rows, rows, (float *)k_out, (float *)c_out);
  return check_launch();
}

}  // namespace gta
