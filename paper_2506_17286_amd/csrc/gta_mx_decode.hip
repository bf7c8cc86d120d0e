// Attention of one new token per sequence over a cache of 8-bit rows (Sec. 3.3, App. B.1.3):
//   L_g = sum_t Softmax_t(q_g . K_t / sqrt(d_h)) C_t
// with the context split over workgroups, each of which leaves an un-normalised sum, its maximum and its weight; a second
// launch joins them.
#include "gta_mx.h"

namespace gta {
namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2;

struct MxAttnArgs {
  const void *q;
  MxView cv;
  int nq, qpk, qpc, dh, dl, kw, cw, splits;
  float scale_log2e;
  float *pacc, *pml;   // [batch, splits, n_q, d_l], [batch, splits, n_q, 2]
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

// Joins the splits: a thread per latent of a map.
template <typename T>
__global__ __launch_bounds__(256) void mx_join_kernel(const float *pacc, const float *pml, int splits, int nq, int dl, T *l_out) {
  const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  if (i >= nq * dl) return;
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
  l_out[(int64_t)b * nq * dl + i] = (T)(l == 0.f ? 0.f : acc / l);
}

}  // namespace

bool mx_decode_dims_ok(const Dims &d) { return mx_widths_ok(d) && d.dh <= kAnyMaxHead && d.dl <= kAnyMaxLatent && d.nq <= 65535; }

int mx_decode_splits(const Dims &d, int batch, int max_seq) {
  const int want = (1024 + batch * d.nq - 1) / (batch * d.nq), cap = max_seq / 256;
  return std::max(1, std::min(std::min(want, cap), 256));
}

int launch_mx_decode(const Dims &d, const void *q, const MxView &cv, int batch, int splits, float *part, void *l_out, hipStream_t st) {
  float *pml = part + (int64_t)batch * splits * d.nq * d.dl;
  const MxAttnArgs a{q, cv, d.nq, d.qpk, d.qpc, d.dh, d.dl, d.wk_w, d.wc_w, splits, d.scale * 1.4426950408889634f, part, pml};
  const dim3 grid(splits, d.nq, batch), join((d.nq * d.dl + 255) / 256, batch);
  if (d.dtype == GTA_BF16) {
    mx_attn_any_kernel<__bf16><<<grid, 256, 0, st>>>(a);
    mx_join_kernel<__bf16><<<join, 256, 0, st>>>(part, pml, splits, d.nq, d.dl, (__bf16 *)l_out);
  } else {
    mx_attn_any_kernel<float><<<grid, 256, 0, st>>>(a);
    mx_join_kernel<float><<<join, 256, 0, st>>>(part, pml, splits, d.nq, d.dl, (float *)l_out);
  }
  return check_launch();
}

}  // namespace gta
