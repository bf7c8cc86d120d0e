// Rotary positions of projected queries and keys (App. B.1.1 with the pairs, the part of the head and the frequencies of
// gta_rope_spec): pair j of a head, (a, b), becomes m (a cos t - b sin t, b cos t + a sin t), t = position * f_j.  fp32 arithmetic,
// one rounding; sines as in the norm's kernels: fp32 for bf16 rows, rounded once from fp64 for fp32 rows.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "gta_mx.h"
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
  store16<NT>(reinterpret_cast<f32x4 *>(p), __builtin_shufflevector(v, v, 0, 1, 2, 3));
  store16<NT>(reinterpret_cast<f32x4 *>(p + 4), __builtin_shufflevector(v, v, 4, 5, 6, 7));
}

template <int PAIRS> struct Turns { uint64_t at[PAIRS]; };

// Heads and their turning parts in whole units of 16 elements, rows and rows' starts in whole 16 bytes.  A thread has one unit of
// HEADS heads of a token: eight pairs, whose sines it works out once, or 16 elements to copy; loads and stores are 16 bytes, those of
// neighbouring threads next to each other.  Bound by memory where there are many tokens: 21 600 of the 1B shape out of a wide projection, half
// of a head turning by neighbours, 14.3 us, 6.2 TB/s (with 32 bytes a thread next to each other 22); by the launch where there are few.
template <typename T, int PAIRS, int HEADS, bool INTER, bool NT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, Turns<PAIRS> turns) {
  const unsigned heads = a.q.heads + a.k.heads, groups = (heads + HEADS - 1) / HEADS, units = a.dh / 16, per = groups * units;
  const unsigned item = blockIdx.x * 256 + threadIdx.x, row = item / per, rest = item - row * per, grp = rest / units, u = rest - grp * units;
  const int64_t t = row;
  if (t >= a.total) return;
  // Two chunks of eight elements: the halves of eight pairs (u, u + r/2), or, of neighbours in pairs and of what is copied, the thread's
  // own in either half of the head or its rest.  Neighbouring threads have neighbouring chunks in both.
  const unsigned pair_units = a.r / 16, rest_units = units - pair_units;
  const bool halves = !INTER && u < pair_units;
  const int lo = INTER || halves ? u * 8 : a.r + (u - pair_units) * 8, hi = INTER ? lo + a.dh / 2 : halves ? lo + a.r / 2 : lo + rest_units * 8;
  const bool turn_lo = INTER ? lo < a.r : halves, turn_hi = INTER ? hi < a.r : halves;
  const int p = a.positions ? a.positions[t] : (int)t;
  f32x8 x[HEADS], y[HEADS];
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int h = min(grp * HEADS + i, heads - 1), hk = h - a.q.heads;   // (a last group may be short: it repeats a head and stores nothing for it)
    const T *in = hk < 0 ? (const T *)a.q.in + t * a.q.in_stride + h * a.dh : (const T *)a.k.in + t * a.k.in_stride + hk * a.dh;
    x[i] = load8(in + lo);
    y[i] = load8(in + hi);
  }
  f32x8 cs, sn;   // halves: of the eight pairs; neighbours: of four pairs of either chunk
  if (turn_lo || turn_hi) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int pair = !INTER ? lo + e : min(e < 4 ? lo / 2 + e : hi / 2 + e - 4, PAIRS - 1);   // (not used where the chunk is copied)
      const float2 c = cos_sin(T(), p, turns.at[pair]);
      cs[e] = c.x * a.magnitude;
      sn[e] = (a.back ? -c.y : c.y) * a.magnitude;
    }
  }
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int h = grp * HEADS + i, hk = h - a.q.heads;
    if (h >= (int)heads) break;
    T *out = hk < 0 ? (T *)a.q.out + t * a.q.out_stride + h * a.dh : (T *)a.k.out + t * a.k.out_stride + hk * a.dh;
    f32x8 v = x[i], w = y[i];
    if constexpr (INTER) {
      const f32x8 a0 = __builtin_shufflevector(v, w, 0, 2, 4, 6, 8, 10, 12, 14), b0 = __builtin_shufflevector(v, w, 1, 3, 5, 7, 9, 11, 13, 15);
      if (turn_lo || turn_hi) {
        const f32x8 a1 = a0 * cs - b0 * sn, b1 = b0 * cs + a0 * sn;
        if (turn_lo) v = __builtin_shufflevector(a1, b1, 0, 8, 1, 9, 2, 10, 3, 11);
        if (turn_hi) w = __builtin_shufflevector(a1, b1, 4, 12, 5, 13, 6, 14, 7, 15);
      }
    } else if (halves) {
      const f32x8 a0 = v;
      v = a0 * cs - w * sn;
      w = w * cs + a0 * sn;
    }
    store8<NT>(out + lo, v);
    store8<NT>(out + hi, w);
  }
}

template <typename T, int PAIRS>
void launch_vector(const RopeArgs &a, const gta_rotation &r, hipStream_t st) {
  Turns<PAIRS> turns;
  for (int j = 0; j < PAIRS; ++j) turns.at[j] = r.turn[j];
  const int heads = a.q.heads + a.k.heads;
  auto run = [&](auto n, auto nt) {
    constexpr int HEADS = decltype(n)::value;
    constexpr bool NT = decltype(nt)::value;
    const int64_t threads = a.total * ((heads + HEADS - 1) / HEADS) * (a.dh / 16);
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (a.interleaved) rope_kernel<T, PAIRS, HEADS, true, NT><<<grid, 256, 0, st>>>(a, turns);
    else rope_kernel<T, PAIRS, HEADS, false, NT><<<grid, 256, 0, st>>>(a, turns);
  };
  // Few tokens: a head to a thread, so that its load is the only one waited for.  The kernel alone with one head and with four a thread,
  // 1B shape: 1 token 2.2 / 2.8 us, 256 3.4 / 4.0, 1024 3.7 / 4.2, 2048 4.4 / 4.4, 4096 5.9 / 5.1.
  if (a.total * heads * (a.dh / 16) < (1 << 17)) run(std::integral_constant<int, 1>{}, std::false_type{});
  else if (stream_past_caches(a.total * heads * a.dh * sizeof(T))) run(std::integral_constant<int, 4>{}, std::true_type{});
  else run(std::integral_constant<int, 4>{}, std::false_type{});
}

template <typename T>
bool try_vector(const RopeArgs &a, const gta_rotation &r, hipStream_t st) {
  const int64_t per = 16 / (int)sizeof(T);
  if (a.dh % 16 || a.r % 16 || a.r > 512) return false;
  if ((a.q.heads && (a.q.in_stride % per || a.q.out_stride % per)) || (a.k.heads && (a.k.in_stride % per || a.k.out_stride % per))) return false;
  if (((uintptr_t)a.q.in | (uintptr_t)a.q.out | (uintptr_t)a.k.in | (uintptr_t)a.k.out) & 15u) return false;
  if (a.total * (a.q.heads + a.k.heads) * (a.dh / 16) >= ((int64_t)1 << 32) - 256) return false;   // threads of a launch
  if (a.r <= 64) launch_vector<T, 32>(a, r, st);
  else if (a.r <= 128) launch_vector<T, 64>(a, r, st);
  else launch_vector<T, 256>(a, r, st);
  return true;
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
  if (d.dtype == GTA_BF16 ? try_vector<__bf16>(a, r, st) : try_vector<float>(a, r, st)) return check_launch();
  const int64_t items = total * (a.q.heads + a.k.heads);
  const dim3 grid((unsigned)std::min<int64_t>((items + 3) / 4, 1 << 20));
  if (d.dtype == GTA_BF16) rope_any_kernel<__bf16><<<grid, 256, 0, st>>>(a, r);
  else rope_any_kernel<float><<<grid, 256, 0, st>>>(a, r);
  return check_launch();
}

}  // namespace gta
