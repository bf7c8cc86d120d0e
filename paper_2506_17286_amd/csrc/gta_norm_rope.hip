// RMS norm of every query and key head with its rotation (App. B.1.1) in the same pass:
//   y_j = x_j / sqrt(mean_i x_i^2 + eps) * gain_j,   then (y_j, y_{j + d/2}) turned by position * base^(-2j/d).
// Sums, the norm and the rotation are fp32 (angles fp64); the only rounding to 16 bits is that of the result.
#include "gta_mx.h"
#include "gta_rope.h"

namespace gta {
namespace {

struct NormRopeArgs {
  const void *q, *k, *q_gain, *k_gain;
  int64_t q_stride, k_stride;
  const int32_t *positions;
  void *q_out, *k_out;
  int64_t total;
  int nq, nk, dh, rope;
  float eps;
  double base;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__bf16 v) { return (float)v; }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int i = 32; i; i >>= 1) v += __shfl_xor(v, i);
  return v;
}

// Any head width, stride and alignment: a wave per (token, head), element by element.
template <typename T>
__global__ __launch_bounds__(256) void norm_rope_any_kernel(NormRopeArgs a) {
  const int heads = a.nq + a.nk, lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= a.total * heads) return;
  const int64_t t = item / heads;
  const int h = (int)(item % heads);
  const bool is_q = h < a.nq;
  const T *x = is_q ? (const T *)a.q + t * a.q_stride + (int64_t)h * a.dh : (const T *)a.k + t * a.k_stride + (int64_t)(h - a.nq) * a.dh;
  T *y = is_q ? (T *)a.q_out + (t * a.nq + h) * a.dh : (T *)a.k_out + (t * a.nk + h - a.nq) * a.dh;
  const T *gain = (const T *)(is_q ? a.q_gain : a.k_gain);
  float ss = 0.f;
  for (int j = lane; j < a.dh; j += 64) { const float v = to_f(x[j]); ss = fmaf(v, v, ss); }
  const float r = rsqrtf(wave_sum(ss) / (float)a.dh + a.eps);
  auto normed = [&](int j) { return to_f(x[j]) * r * (gain ? to_f(gain[j]) : 1.f); };
  if (!a.rope) {
    for (int j = lane; j < a.dh; j += 64) y[j] = (T)normed(j);
    return;
  }
  const int half = a.dh / 2, p = a.positions ? a.positions[t] : (int)t;
  for (int j = lane; j < half; j += 64) {
    const float lo = normed(j), hi = normed(j + half);
    const float2 cs = rope_cos_sin_any(p, pow(a.base, -2.0 * j / a.dh));
    y[j] = (T)(lo * cs.x - hi * cs.y);
    y[j + half] = (T)(hi * cs.x + lo * cs.y);
  }
}

}  // namespace

int launch_qk_norm_rope(const Dims &d, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *q_gain,
                        const void *k_gain, float eps, const int32_t *positions, int64_t total, void *q_out, void *k_out,
                        hipStream_t st) {
  const NormRopeArgs a{q, k, q_gain, k_gain, q_stride, k_stride, positions, q_out, k_out, total, d.nq, d.nk, d.dh, d.rope, eps,
                       d.rope_base};
  const int64_t items = total * (d.nq + d.nk);
  const dim3 grid((unsigned)((items + 3) / 4));
  if (d.dtype == GTA_BF16) norm_rope_any_kernel<__bf16><<<grid, 256, 0, st>>>(a);
  else norm_rope_any_kernel<float><<<grid, 256, 0, st>>>(a);
  return check_launch();
}

}  // namespace gta
