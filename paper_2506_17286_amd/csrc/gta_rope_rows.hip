// Rotary positions of projected queries and keys (App. B.1.1 with the pairs, the part of the head and the frequencies of
// gta_rope_spec): pair j of a head, (a, b), becomes m (a cos t - b sin t, b cos t + a sin t), t = position * f_j.  fp32 arithmetic,
// one rounding; sines as in the norm's kernels: fp32 for bf16 rows, rounded once from fp64 for fp32 rows.
#include <math.h>

#include <algorithm>

#include "gta_rope.h"
#include "gta_rules.h"

namespace gta {
namespace {

struct RopeSide { const void *in; void *out; int64_t in_stride, out_stride; int heads; };   // queries or keys
struct RopeArgs {
  RopeSide q, k;
  const int32_t *positions;
  int64_t total;
  int dh, r, interleaved, back;
  float magnitude;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__bf16 v) { return (float)v; }
__device__ __forceinline__ float2 cos_sin(__bf16, int p, uint64_t turn) { return rope_cos_sin_turn(p, turn); }
__device__ __forceinline__ float2 cos_sin(float, int p, uint64_t turn) { return rope_cos_sin_turn_f64(p, turn); }

// Any widths, strides and alignment: a wave per (token, head), a pair or a copied element per lane.
template <typename T>
__global__ __launch_bounds__(256) void rope_any_kernel(RopeArgs a, gta_rotation rot) {
  const int heads = a.q.heads + a.k.heads, lane = threadIdx.x & 63, pairs = a.r / 2;
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < a.total * heads; item += (int64_t)gridDim.x * 4) {
    const int64_t t = item / heads;
    const int h = (int)(item % heads), hk = h - a.q.heads;
    const T *x = hk < 0 ? (const T *)a.q.in + t * a.q.in_stride + (int64_t)h * a.dh : (const T *)a.k.in + t * a.k.in_stride + (int64_t)hk * a.dh;
    T *y = hk < 0 ? (T *)a.q.out + t * a.q.out_stride + (int64_t)h * a.dh : (T *)a.k.out + t * a.k.out_stride + (int64_t)hk * a.dh;
    const int p = a.positions ? a.positions[t] : (int)t;
    for (int j = lane; j < pairs; j += 64) {
      const int lo = a.interleaved ? 2 * j : j, hi = a.interleaved ? 2 * j + 1 : j + pairs;
      float2 cs = cos_sin(T(), p, rot.turn[j]);
      if (a.back) cs.y = -cs.y;
      const float u = to_f(x[lo]), v = to_f(x[hi]);
      y[lo] = (T)((u * cs.x - v * cs.y) * a.magnitude);
      y[hi] = (T)((v * cs.x + u * cs.y) * a.magnitude);
    }
    if (x != y)
      for (int j = a.r + lane; j < a.dh; j += 64) y[j] = x[j];
  }
}

}  // namespace

int make_rotation(const Dims &d, const gta_rope_spec &s, gta_rotation *out) {
  if (s.layout != GTA_ROPE_HALF && s.layout != GTA_ROPE_INTERLEAVED) return GTA_ERR_DTYPE;
  if (s.scaling < GTA_ROPE_PLAIN || s.scaling > GTA_ROPE_GIVEN) return GTA_ERR_DTYPE;
  const int r = s.rotary_dim ? s.rotary_dim : d.dh, pairs = r / 2;
  if (r <= 0 || r % 2 || r > d.dh) return GTA_ERR_SHAPE;
  if (pairs > GTA_ROPE_MAX_PAIRS) return GTA_ERR_UNSUPPORTED;
  const float m = s.magnitude == 0.f ? 1.f : s.magnitude;
  auto positive = [](float v) { return v > 0.f && v <= 3e38f; };
  if (!positive(m)) return GTA_ERR_SHAPE;
  if (s.scaling == GTA_ROPE_GIVEN ? !s.frequency : !positive(s.base)) return s.scaling == GTA_ROPE_GIVEN ? GTA_ERR_NULL : GTA_ERR_SHAPE;
  const bool scaled = s.scaling == GTA_ROPE_LINEAR || s.scaling == GTA_ROPE_BASE || s.scaling == GTA_ROPE_BANDS;
  if (scaled && !positive(s.factor)) return GTA_ERR_SHAPE;
  if (s.scaling == GTA_ROPE_BASE && r <= 2) return GTA_ERR_SHAPE;
  if (s.scaling == GTA_ROPE_BANDS && !(positive(s.trained_len) && positive(s.slow_turns) && positive(s.fast_turns) && s.slow_turns < s.fast_turns))
    return GTA_ERR_SHAPE;
  gta_rotation rot{};
  rot.layout = s.layout; rot.rotary_dim = r; rot.magnitude = m;
  const long double per_radian = 0.15915494309189533576888376337251436203L, two64 = 18446744073709551616.0L, factor = scaled ? s.factor : 1.0L;
  const long double log_base = s.scaling == GTA_ROPE_GIVEN ? 0.0L : logl((long double)s.base) + (s.scaling == GTA_ROPE_BASE ? logl(factor) * r / (r - 2) : 0.0L);
  for (int j = 0; j < pairs; ++j) {
    long double f = s.scaling == GTA_ROPE_GIVEN ? (long double)s.frequency[j] : expl(-2.0L * j / r * log_base);
    if (s.scaling == GTA_ROPE_LINEAR) f /= factor;
    if (s.scaling == GTA_ROPE_BANDS) {
      const long double t = s.trained_len * f * per_radian;
      const long double kept = std::min(std::max((t - s.slow_turns) / ((long double)s.fast_turns - s.slow_turns), 0.0L), 1.0L);
      f = (1.0L - kept) * f / factor + kept * f;
    }
    const long double turns = f * per_radian;
    if (!(fabsl(turns) < 1e15L)) return GTA_ERR_SHAPE;   // not finite, or no digits left behind the point
    const long double part = (turns - floorl(turns)) * two64;
    rot.turn[j] = part >= two64 ? 0 : (uint64_t)part;
  }
  *out = rot;
  return GTA_OK;
}

int launch_qk_rope(const Dims &d, const gta_rotation &r, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                   const int32_t *positions, int64_t total, bool transposed, void *q_out, int64_t q_out_stride, void *k_out,
                   int64_t k_out_stride, hipStream_t st) {
  const RopeArgs a{{q, q_out, q_stride, q_out_stride, q ? d.nq : 0}, {k, k_out, k_stride, k_out_stride, k ? d.nk : 0},
                   positions, total, d.dh, r.rotary_dim, r.layout == GTA_ROPE_INTERLEAVED, transposed, r.magnitude};
  const int64_t items = total * (a.q.heads + a.k.heads);
  const dim3 grid((unsigned)std::min<int64_t>((items + 3) / 4, 1 << 20));
  if (d.dtype == GTA_BF16) rope_any_kernel<__bf16><<<grid, 256, 0, st>>>(a, r);
  else rope_any_kernel<float><<<grid, 256, 0, st>>>(a, r);
  return check_launch();
}

}  // namespace gta
