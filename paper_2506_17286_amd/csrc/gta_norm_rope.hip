// RMS norm of every query and key head with its rotation (App. B.1.1) in the same pass:
//   y_j = x_j / sqrt(mean_i x_i^2 + eps) * gain_j,   then (y_j, y_{j + d/2}) turned by position * base^(-2j/d).
// Sums, the norm and the rotation are fp32, sines of fp32 rows are rounded once from fp64, those of bf16 rows are fp32; the only
// rounding to 16 bits is that of the result.
#include <math.h>

#include <type_traits>

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
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < a.total * heads; item += (int64_t)gridDim.x * 4) {
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
      continue;
    }
    const int half = a.dh / 2, p = a.positions ? a.positions[t] : (int)t;
    for (int j = lane; j < half; j += 64) {
      const float lo = normed(j), hi = normed(j + half);
      const float2 cs = rope_cos_sin_any(p, pow(a.base, -2.0 * j / a.dh));
      y[j] = (T)(lo * cs.x - hi * cs.y);
      y[j + half] = (T)(hi * cs.x + lo * cs.y);
    }
  }
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
__device__ __forceinline__ f32x8 load8(const __bf16 *p) { return __builtin_convertvector(*reinterpret_cast<const bf16x8 *>(p), f32x8); }
__device__ __forceinline__ f32x8 load8(const float *p) {
  return __builtin_shufflevector(*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4), 0, 1, 2, 3, 4, 5, 6, 7);
}

template <bool NT>
__device__ __forceinline__ void store8(__bf16 *p, const f32x8 &v) { store16<NT>(reinterpret_cast<bf16x8 *>(p), __builtin_convertvector(v, bf16x8)); }
template <bool NT>
__device__ __forceinline__ void store8(float *p, const f32x8 &v) {
  static_assert(!NT, "two words a thread");
  *reinterpret_cast<f32x4 *>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
  *reinterpret_cast<f32x4 *>(p + 4) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}

// What one position turns pair j < d_h/2 by, from the host: 64-bit fractions of a turn for bf16 rows, radians for fp32 rows.
template <typename T> struct Angles { uint64_t at[128]; };
template <> struct Angles<float> { double at[128]; };
__device__ __forceinline__ float2 cos_sin_of(int p, uint64_t turn) { return rope_cos_sin_turn(p, turn); }
__device__ __forceinline__ float2 cos_sin_of(int p, double freq) { return rope_cos_sin(p, freq); }

// Heads of 16 * LANES elements, rows and rows' starts in whole 16 bytes.  A lane has eight elements j.. and their partners
// j + d_h/2 of HEADS heads of one token: their sines are the same and worked out once, a head's sum of squares is taken over
// LANES neighbours, and loads and stores are 16 bytes.  Bound by memory where there are many tokens and by the launch where there
// are few.
template <typename T, int LANES, int HEADS, bool NT>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormRopeArgs a, Angles<T> angles) {
  constexpr int DH = 16 * LANES, HALF = DH / 2;
  const int heads = a.nq + a.nk, groups = (heads + HEADS - 1) / HEADS;
  const unsigned item = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, row = item / groups;   // token and group of heads
  const int j = threadIdx.x % LANES * 8;
  const int64_t t = row;
  if (t >= a.total) return;
  const int h0 = (int)(item - row * groups) * HEADS;
  const int p = a.rope ? (a.positions ? a.positions[t] : (int)t) : 0;
  const T *qg = (const T *)a.q_gain, *kg = (const T *)a.k_gain;
  f32x8 lo[HEADS], hi[HEADS];
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int h = min(h0 + i, heads - 1);   // (a last group may be short: it repeats a head and stores nothing for it)
    const T *x = h < a.nq ? (const T *)a.q + t * a.q_stride + h * DH : (const T *)a.k + t * a.k_stride + (h - a.nq) * DH;
    lo[i] = load8(x + j);
    hi[i] = load8(x + j + HALF);
  }
  f32x8 cs, sn;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float2 c = make_float2(1.f, 0.f);
    if (a.rope) c = cos_sin_of(p, angles.at[j + e]);
    cs[e] = c.x;
    sn[e] = c.y;
  }
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int h = h0 + i;
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(lo[i][e], lo[i][e], fmaf(hi[i][e], hi[i][e], ss));
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) ss += __shfl_xor(ss, m);
    const float r = rsqrtf(ss * (1.f / DH) + a.eps);
    const T *gain = h < a.nq ? qg : kg;
    lo[i] *= r;
    hi[i] *= r;
    if (gain) {
      lo[i] *= load8(gain + j);
      hi[i] *= load8(gain + j + HALF);
    }
    if (h < heads) {
      T *y = h < a.nq ? (T *)a.q_out + (t * a.nq + h) * DH : (T *)a.k_out + (t * a.nk + h - a.nq) * DH;
      store8<NT>(y + j, lo[i] * cs - hi[i] * sn);
      store8<NT>(y + j + HALF, hi[i] * cs + lo[i] * sn);
    }
  }
}

}  // namespace

template <typename T, int LANES>
static void launch_vector(const NormRopeArgs &a, hipStream_t st) {
  Angles<T> angles{};
  if (a.rope) {
    if constexpr (sizeof(T) == 4) rope_freqs(a.base, a.dh, a.dh / 2, angles.at);
    else rope_turns(a.base, a.dh, a.dh / 2, angles.at);
  }
  const int heads = a.nq + a.nk;
  auto run = [&](auto n, auto nt) {
    constexpr int HEADS = decltype(n)::value;
    const int64_t threads = a.total * ((heads + HEADS - 1) / HEADS) * LANES;
    norm_rope_kernel<T, LANES, HEADS, decltype(nt)::value><<<dim3((unsigned)((threads + 255) / 256)), 256, 0, st>>>(a, angles);
  };
  // few tokens: a head to every group of lanes, so that its load is the only one waited for
  if (a.total * heads * LANES < (1 << 17)) run(std::integral_constant<int, 1>{}, std::false_type{});
  else if (sizeof(T) == 2 && stream_past_caches(a.total * heads * a.dh * 2)) run(std::integral_constant<int, 4>{}, std::bool_constant<sizeof(T) == 2>{});
  else run(std::integral_constant<int, 4>{}, std::false_type{});
}

// Heads of 32, 64, 128 or 256 and 16-byte rows; fp32 rows as far as their angles stay in the reduction's range.
template <typename T>
static bool try_vector(const NormRopeArgs &a, hipStream_t st) {
  if (sizeof(T) == 4 && !rope_angles_small(a.rope, a.base)) return false;
  const int64_t per = 16 / (int)sizeof(T);
  if (a.q_stride % per || a.k_stride % per || (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.q_gain | (uintptr_t)a.k_gain) & 15u))
    return false;
  if (a.total * ((a.nq + a.nk + 3) / 4) * (a.dh / 16) >= ((int64_t)1 << 32) - 256) return false;   // threads of a launch
  switch (a.dh) {
    case 32: launch_vector<T, 2>(a, st); return true;
    case 64: launch_vector<T, 4>(a, st); return true;
    case 128: launch_vector<T, 8>(a, st); return true;
    case 256: launch_vector<T, 16>(a, st); return true;
    default: return false;
  }
}

int launch_qk_norm_rope(const Dims &d, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *q_gain,
                        const void *k_gain, float eps, const int32_t *positions, int64_t total, void *q_out, void *k_out,
                        hipStream_t st) {
  const NormRopeArgs a{q, k, q_gain, k_gain, q_stride, k_stride, positions, q_out, k_out, total, d.nq, d.nk, d.dh, d.rope, eps,
                       d.rope_base};
  if (d.dtype == GTA_BF16 ? try_vector<__bf16>(a, st) : try_vector<float>(a, st)) return check_launch();
  const int64_t items = total * (d.nq + d.nk);
  const dim3 grid((unsigned)std::min<int64_t>((items + 3) / 4, 1 << 20));
  if (d.dtype == GTA_BF16) norm_rope_any_kernel<__bf16><<<grid, 256, 0, st>>>(a);
  else norm_rope_any_kernel<float><<<grid, 256, 0, st>>>(a);
  return check_launch();
}

}  // namespace gta
