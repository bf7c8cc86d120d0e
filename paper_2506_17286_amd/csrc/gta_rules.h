// Rotary positions as a model's configuration states them, and attention with rules on its scores (gta_score_rules): a cap by a
// tanh, a bias that falls with the distance, an interval of keys per token.
#pragma once
#include <math.h>

#include <algorithm>

#include "gta_internal.h"

namespace gta {

int make_rotation(const Dims &d, const gta_rope_spec &s, gta_rotation *out);
int launch_qk_rope(const Dims &d, const gta_rotation &r, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                   const int32_t *positions, int64_t total, bool transposed, void *q_out, int64_t q_out_stride, void *k_out,
                   int64_t k_out_stride, hipStream_t st);

constexpr float kLog2e = 1.4426950408889634f;

// The rules as kernels take them: scores leave them in units of log 2.
struct Rules {
  float scale, cap, inv_cap;   // softmax scale; cap and its inverse, 0 where there is none
  // cap * tanh(s / cap) for |s| <= near, s and result in units of log 2 as `scale2` makes them: s times a polynomial in s^2, off by
  // at most 6.9e-6 of the result (the best of its degree for tanh(x) / x up to 1).  `near` is the cap, or where that is more 256 (times
  // log2 e), so that the error is below 2^-9, half of what a rounded weight of 16 bits is off by.  Caps below 2^-10, whose coefficients of up
  // to cap^-8 would leave fp32, have near = -1: no score is.
  float scale2, cap2, near, steep, poly[5];   // cap2: the cap in these units; steep * (q . k) = s / cap, where near = cap2 times 2 log2(e)
  const float *slopes;
  const int32_t *first, *last;
};

inline Rules rules_of(const Dims &d, const gta_score_rules *r) {
  Rules out{};
  out.scale = d.scale;
  out.scale2 = d.scale * kLog2e;
  if (r) {
    const double cap2 = (double)r->cap * 1.4426950408889634;
    const double best[5] = {0.999993088553236, -0.33298064162659136, 0.1303680737376961, -0.044817503256505964, 0.009036401546491156};
    const bool polynomial = r->cap >= 0x1p-10f;
    out.cap2 = (float)cap2;
    out.near = polynomial ? std::min(out.cap2, 256.f * kLog2e) : -1.f;
    out.steep = r->cap > 0.f ? (float)std::min((out.near == out.cap2 ? 2.0 * 1.4426950408889634 : 1.0) * d.scale / r->cap, 3e38) : 0.f;
    for (int i = 0; i < 5 && polynomial; ++i) out.poly[i] = (float)(best[i] * pow(cap2, -2.0 * i));
    out.cap = r->cap;
    out.inv_cap = r->cap > 0.f ? 1.f / r->cap : 0.f;
    out.slopes = r->slopes; out.first = r->first; out.last = r->last;
  }
  return out;
}

// tanh to 3 units in the last place.  Below 5/8 the continued fraction x / (1 + y / (3 + y / (5 + y / (7 + ..)))), y = x^2, cut
// behind the 9, which is the quotient below (off by less than 1e-9 of it there); above, 1 - 2 / (e^2|x| + 1).
__device__ __forceinline__ float tanh_exactly(float x) {
  const float a = fabsf(x), y = x * x;
  const float lo = x * fmaf(y, y + 105.f, 945.f) * __builtin_amdgcn_rcpf(fmaf(y, fmaf(y, 15.f, 420.f), 945.f));
  const float hi = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(2.f * kLog2e * a) + 1.f), x);
  return a < 0.625f ? lo : a >= 0.625f ? hi : x;   // NaN stays
}

// A product q . k to a score in units of log 2; distance = |position - key| (not negative)
__device__ __forceinline__ float ruled_score(const Rules &r, float dot, float slope, float distance) {
  float s = dot * r.scale;
  if (r.cap > 0.f) s = r.cap * tanh_exactly(s * r.inv_cap);
  return fmaf(-slope, distance, s) * kLog2e;
}

// What a token at `own` of `keys` keys sees: lo .. hi, nothing where lo > hi
__device__ __forceinline__ void seen_by(const Rules &r, int64_t token, int own, int keys, int &lo, int &hi) {
  lo = r.first ? max(r.first[token], 0) : 0;
  hi = max(min(r.last ? r.last[token] : own, keys - 1), -1);
}

constexpr int kRulesMaxHead = 1024, kRulesMaxLatent = 4096;
inline bool rules_dims_ok(const Dims &d) { return d.dh <= kRulesMaxHead && d.dl <= kRulesMaxLatent; }

struct MaskedArgs {
  const void *q, *k, *c;
  int64_t q_stride, k_stride, c_stride;
  const int32_t *cu;
  int batch;
  int64_t total;
  int max_len;
  Rules rules;
  void *l_out;
};
struct PrefixArgs {
  const void *q;
  CacheView prefix, own;   // prefix.slots unused
  int prefix_slot, batch;
  Rules rules;
  void *l_out;
};

// any shapes
int launch_masked_any(const Dims &d, const MaskedArgs &m, hipStream_t st);
int launch_prefix_any(const Dims &d, const PrefixArgs &p, hipStream_t st);

// rows of a slot that take part
__device__ __forceinline__ int slot_rows(const CacheView &cv, int slot) {
  return slot >= 0 && slot < cv.max_batch ? min(max(cv.seq_lens[slot], 0), cv.max_seq) : 0;
}

}  // namespace gta
