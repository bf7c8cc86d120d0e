// Attention with rules on its scores for any shape, stride and alignment: a workgroup per (token, map) walks the keys that the
// token sees, 256 at a time, a key a thread for the scores and a latent (or several) a thread for the averages.  Every row is read
// once for every map: the measure of the other kernels, not a fast one.  Bound by the latency of its scalar products: 4 x 4096 tokens of
// packed documents, 1B shape, 17 ms where the matrix instructions take 88 us.
#include <algorithm>

#include "gta_rules.h"

namespace gta {
namespace {

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__bf16 v) { return (float)v; }

// rows j0 .. j0 + rows - 1 of the keys that a token may see
template <typename T>
struct Rows {
  const T *k, *c;
  int64_t ks, cs, row0;
  PageMap pm;
  int slot, max_seq;
  __device__ int64_t row(int i) const { return pm.table ? cache_row_clamped(pm, max_seq, slot, i) : row0 + i; }
};

// One (token, map): keys lo .. hi, of which the first `cut` are rows of `a` and the others rows 0 .. of `b`.  Keys past the wanted
// ones are not read.
template <typename T>
__device__ void attend_row(const Dims &d, const Rules &rules, const T *q, int g, const Rows<T> &a, const Rows<T> &b, int cut, int lo, int hi,
                           int own, T *out) {
  __shared__ float qs[kRulesMaxHead], ps[256], red[4], red2[4];
  __shared__ int64_t at[256];
  const int tid = threadIdx.x, kcol = g / d.qpk * d.dh, ccol = g / d.qpc * d.dl;
  const float slope = rules.slopes ? rules.slopes[g] : 0.f;
  for (int i = tid; i < d.dh; i += 256) qs[i] = to_f(q[i]);
  float m = -INFINITY, l = 0.f, acc[kRulesMaxLatent / 256] = {};
  __syncthreads();
  for (int64_t j0 = lo; j0 <= hi; j0 += 256) {
    const int cnt = (int)min((int64_t)256, hi - j0 + 1);
    float sc = -INFINITY;
    if (tid < cnt) {
      const int j = (int)j0 + tid;
      const bool first = j < cut;
      const int64_t row = first ? a.row(j) : b.row(j - cut);
      at[tid] = row;
      const T *kr = (first ? a.k + row * a.ks : b.k + row * b.ks) + kcol;
      float dot = 0.f;
      for (int i = 0; i < d.dh; ++i) dot = fmaf(to_f(kr[i]), qs[i], dot);
      sc = ruled_score(rules, dot, slope, fabsf((float)(own - j)));
    }
    float mx = sc;
    for (int i = 32; i; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    const float mn = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]))), ref = mn > -INFINITY ? mn : 0.f;
    const float p = tid < cnt ? exp2f(sc - ref) : 0.f, corr = exp2f(m - ref);
    ps[tid] = p;
    float sum = p;
    for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
    if ((tid & 63) == 0) red2[tid >> 6] = sum;
    __syncthreads();
    const float before = l * corr;
    l = before + ((red2[0] + red2[1]) + (red2[2] + red2[3]));
    m = mn;
    const float per = l > 0.f ? 1.f / l : 0.f, kept = before * per;   // averages: sums of large latents would pass the range
    for (int v = 0, col = tid; col < d.dl; ++v, col += 256) {
      float s = acc[v] * kept;
      for (int r = 0; r < cnt; ++r) {
        const T *cr = j0 + r < cut ? a.c + at[r] * a.cs : b.c + at[r] * b.cs;
        s = fmaf(ps[r] * per, to_f(cr[ccol + col]), s);
      }
      acc[v] = s;
    }
    __syncthreads();
  }
  for (int v = 0, col = tid; col < d.dl; ++v, col += 256) out[col] = (T)(lo > hi ? 0.f : l > 0.f ? acc[v] : NAN);
}

// The sequence of a packed token: the last b with cu[b] <= t.
__device__ __forceinline__ int sequence_of(const int32_t *cu, int batch, int64_t t) {
  int lo = 0, hi = batch;   // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <typename T>
__device__ void masked_row(const Dims &d, const MaskedArgs &m, int64_t t, int g) {
  const int64_t per = m.total / m.batch;
  int64_t start;
  int len;
  if (m.cu) {
    if (t < m.cu[0] || t >= m.cu[m.batch]) return;   // rows of no sequence
    const int b = sequence_of(m.cu, m.batch, t);
    start = m.cu[b];
    len = m.cu[b + 1] - (int)start;
  } else {
    start = t / per * per;
    len = (int)per;
  }
  const Rows<T> rows{(const T *)m.k, (const T *)m.c, m.k_stride, m.c_stride, start, PageMap{}, 0, 0};
  const int own = (int)(t - start);
  int lo, hi;
  seen_by(m.rules, t, own, len, lo, hi);
  attend_row<T>(d, m.rules, (const T *)m.q + t * m.q_stride + (int64_t)g * d.dh, g, rows, rows, INT_MAX, lo, hi, own,
                (T *)m.l_out + (t * d.nq + g) * d.dl);
}

template <typename T>
__global__ __launch_bounds__(256) void masked_any_kernel(Dims d, MaskedArgs m) {
  for (int64_t t = blockIdx.x; t < m.total; t += gridDim.x) masked_row<T>(d, m, t, blockIdx.y);
}

template <typename T>
__global__ __launch_bounds__(256) void prefix_any_kernel(Dims d, PrefixArgs p) {
  const int b = blockIdx.x, g = blockIdx.y, slot = p.own.slots ? p.own.slots[b] : b;
  const int shared = slot_rows(p.prefix, p.prefix_slot), mine = slot_rows(p.own, slot);
  const Rows<T> first{(const T *)p.prefix.k, (const T *)p.prefix.c, d.wk_w, d.wc_w, (int64_t)p.prefix_slot * p.prefix.max_seq,
                      p.prefix.pm, p.prefix_slot, p.prefix.max_seq};
  const Rows<T> then{(const T *)p.own.k, (const T *)p.own.c, d.wk_w, d.wc_w, (int64_t)slot * p.own.max_seq, p.own.pm, slot, p.own.max_seq};
  const int own = (int)((int64_t)shared + mine - 1);
  int lo, hi;
  seen_by(p.rules, b, own, own + 1, lo, hi);
  attend_row<T>(d, p.rules, (const T *)p.q + ((int64_t)b * d.nq + g) * d.dh, g, first, then, shared, lo, hi, own,
                (T *)p.l_out + ((int64_t)b * d.nq + g) * d.dl);
}

}  // namespace

int launch_masked_any(const Dims &d, const MaskedArgs &m, hipStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>(m.total, 1 << 23), (unsigned)d.nq);   // a launch has fewer than 2^32 threads along x
  if (d.dtype == GTA_BF16) masked_any_kernel<__bf16><<<grid, 256, 0, st>>>(d, m);
  else masked_any_kernel<float><<<grid, 256, 0, st>>>(d, m);
  return check_launch();
}

int launch_prefix_any(const Dims &d, const PrefixArgs &p, hipStream_t st) {
  const dim3 grid((unsigned)p.batch, (unsigned)d.nq);
  if (d.dtype == GTA_BF16) prefix_any_kernel<__bf16><<<grid, 256, 0, st>>>(d, p);
  else prefix_any_kernel<float><<<grid, 256, 0, st>>>(d, p);
  return check_launch();
}

}  // namespace gta
