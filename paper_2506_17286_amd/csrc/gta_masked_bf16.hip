// bf16 attention of rows of queries with rules on their scores (gta_score_rules), on matrix instructions:
//   s = scale q . k,  capped by a tanh,  less slope * |distance|,  keys first .. last,  softmax,  times the latents.
//
// A workgroup has a tile of 128, 64 or 32 rows (gta_rows_attn.h) and 32 keys a step; both products are taken transposed, as
//   S^T[key][row] = K Q^T,   L^T[column][row] += C^T P^T,
// so that a row's statistics live in a pair of lanes, its weights go from the scores' accumulators into the second product
// without leaving registers, and its slope, position and interval are scalars of a lane.  Key and latent tiles go from memory
// straight into LDS through three stages.  Blocks go from the last one seen to the first: with a bias the largest scores come
// first.  A wave skips the blocks none of its rows sees, masks those that some rows see, and takes the others, whose softmax is dealt
// out between the matrix instructions, without looking at their maximum: weights refer to the maximum a row has, whatever their size,
// and a row sum beyond 2^32 sends the wave through the full step.
// Weights are rounded to bf16 for the second product (their sum is that of the rounded ones); everything else is fp32.
// Bound by the softmax's vector arithmetic beside the matrix instructions, which then draw the more power the less they wait.  Whole calls,
// the list of tiles (5 to 10 us) among them: 4 x 4096 tokens of documents of 100 to 2000, 1B shape, 88 us (498 TFLOP/s of what is seen; whole
// sequences, causal, 810); 32 ragged prompts of the paper's layer, a cap, 105 us (572); 2 x 8192 of the wide shape, window, cap and bias
// 1300 us (673; with the scores, which each of four latent tiles works out, 895).  A cap costs 16 to 26 %, a bias 1 to 8.
//
// A masked weight is 0, but 0 times a latent that is not finite is NaN, and sums of finite ones may pass the range: a wave whose sums are not
// finite in the end goes through its rows once more, one by one, over the keys that each sees (wave_row).
#include <math.h>

#include <type_traits>

#include "gta_lds_load.h"
#include "gta_rows_attn.h"

namespace gta {
namespace {

typedef __bf16 bf16;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// QW groups of 32 rows times 4 / QW groups of columns, a wave each.  Layout of a tile in LDS: a load instruction fetches 1 KiB in
// lane order, so rows that it fetches cannot be padded apart and it fetches rows that are not read together: keys a + K_INSTR i
// with instruction a, 16 bytes further per a, every second i with its halves swapped (k_sel); latents 4 a + r with instruction
// 4 b + r, 64 bytes further per r.  Reads then fall into different columns of banks, at one (keys: two) addresses a lane plus
// constants.
template <int DH_, int DLW_, int QW_>
struct Tile {
  static constexpr int DH = DH_, DLW = DLW_, QW = QW_, CG = 4 / QW, BK = 32, BQ = 32 * QW, NW = 4, NT = 256;
  static constexpr int NDLB = DLW / 32 / CG;   // blocks of 32 columns of a wave
  static constexpr int K_ROW = DH * 2, C_ROW = DLW * 2, K_CPR = K_ROW / 16, C_CPR = C_ROW / 16;
  static constexpr int K_INSTR = BK * K_ROW / 1024, C_INSTR = BK * C_ROW / 1024, C_RPI = 1024 / C_ROW;
  static constexpr int K_PITCH = 1024 + 16, C_PITCH = 1024 + 64, C_GROUP = 4 * C_PITCH;
  static constexpr int K_BYTES = K_INSTR * K_PITCH, STAGE = K_BYTES + C_INSTR * C_PITCH, NSTAGE = 3;
  static constexpr int OUT_PITCH = DLW * 2 + 16;
  static constexpr int SMEM = NSTAGE * STAGE > BQ * OUT_PITCH ? NSTAGE * STAGE : BQ * OUT_PITCH;
  // Workgroups of a CU, as the registers are shared out.  (Tiles of 512 columns fill a CU's LDS, but with 512 registers a lane the
  // accumulators go to the half that takes no arithmetic, and are copied out and back every step.)
  static constexpr int BLOCKS = DH == 64 && SMEM <= 53 * 1024 ? 3 : 2;
  static_assert(K_INSTR >= NW && C_INSTR >= NW && C_RPI >= 1 && NDLB >= 1 && SMEM <= 160 * 1024, "tile");
  __device__ static constexpr int k_sel(int i) { return K_CPR == 16 ? i & 1 : (i ^ (i >> 1)) & 1; }
  __device__ static constexpr int c_row(int a) { return a / C_RPI * C_GROUP + a % C_RPI * C_ROW; }
};

constexpr float kLazyThreshold = 8.0f;          // log2 units
constexpr float kRowSumLimit = 4294967296.0f;   // 2^32
enum { kCap = 1, kBias = 2 };

// f(0), .., f(N - 1) as constants: loops over the accumulators.  (Unrolled loops in their place leave accumulators of 256 columns
// in memory: 4 x 4096 tokens of packed documents, 1B shape, 1600 us.)
template <class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void each(F f) { each_of(f, std::make_integer_sequence<int, N>{}); }
#define EACH(i) [&](auto i) __attribute__((always_inline))

__device__ __forceinline__ float pair_max(float v) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ int wave_min(int v) {
  v = min(v, __builtin_amdgcn_update_dpp(INT_MAX, v, 0x111, 0xf, 0xf, false));   // row_shr 1, 2, 4, 8
  v = min(v, __builtin_amdgcn_update_dpp(INT_MAX, v, 0x112, 0xf, 0xf, false));
  v = min(v, __builtin_amdgcn_update_dpp(INT_MAX, v, 0x114, 0xf, 0xf, false));
  v = min(v, __builtin_amdgcn_update_dpp(INT_MAX, v, 0x118, 0xf, 0xf, false));
  v = min(v, __builtin_amdgcn_update_dpp(INT_MAX, v, 0x142, 0xa, 0xf, false));   // row_bcast 15, 31
  v = min(v, __builtin_amdgcn_update_dpp(INT_MAX, v, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_max(int v) { return -wave_min(-v); }

// A scalar load, waited for in place: a vector load would make the compiler wait for every load in flight.
__device__ __forceinline__ int load_uniform(const int32_t *p) {
  int v;
  asm volatile("s_load_dword %0, %1, 0x0\n\ts_waitcnt lgkmcnt(0)" : "=s"(v) : "s"(p));
  return v;
}

template <class T, int MODS, bool CACHE>
__global__ __launch_bounds__(256, T::BLOCKS) void rows_attn_kernel(RowsArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int span[8], sees_from[256], sees_to[256];   // what a lane's row sees, out of the registers of the main loop
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, ln = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), qw = wave % T::QW, cg = wave / T::QW;
  const int per = a.cells * a.slices;
  int u, r;   // which tile (or piece), workgroup of it
  if (a.tiles < (CACHE ? 8 : 64)) { u = (int)blockIdx.x / per; r = (int)blockIdx.x - u * per; }
  else {   // eight tiles at a time, one per XCD: a tile's workgroups read the same keys and latents
    const int at = (int)blockIdx.x >> 3, round = at / per;
    r = at - round * per;
    u = round * 8 + ((int)blockIdx.x & 7);
  }
  if (u >= a.tiles) return;
  int b, tile, piece = 0, pieces = 1, slot = 0;
  if constexpr (CACHE) {
    b = 0; tile = u / a.pieces; piece = u - tile * a.pieces; pieces = a.pieces; slot = tile * a.pieces;
  } else if (a.list) {
    if (u >= load_uniform(a.count)) return;
    const Piece *e = a.list + u;
    b = load_uniform(&e->b); tile = load_uniform(&e->tile); piece = load_uniform(&e->piece); pieces = load_uniform(&e->pieces);
    slot = load_uniform(&e->slot);
  } else {
    const int per_level = a.batch, lvl = u / per_level;
    b = u - lvl * per_level; tile = a.tiles / a.batch - 1 - lvl;
  }
  const int slice = r % a.slices, cell = r / a.slices;
  int64_t start = 0;
  int Tb = CACHE ? a.batch : a.per_seq, keys;
  if constexpr (CACHE) keys = slot_rows(a.prefix, a.prefix_slot);
  else {
    start = (int64_t)b * a.per_seq;
    if (a.cu) {
      start = load_uniform(a.cu + b);
      Tb = load_uniform(a.cu + b + 1) - (int)start;
    }
    keys = Tb;
  }
  const int R = Tb * a.mpc, r0 = tile * T::BQ;               // rows of the sequence, first of this tile
  if (!CACHE && r0 >= R) return;
  const int wr0 = r0 + qw * 32, row = min(wr0 + ln, R - 1);  // (rows past the last repeat it and are not stored)
  const int tok = row / a.mpc, g = cell * a.mpc + (row - tok * a.mpc);
  int lo, hi, own;
  const bool plain = CACHE && !a.rules.first && !a.rules.last;   // every row sees the whole prefix
  if constexpr (CACHE) {
    if (plain && !(MODS & kBias)) { lo = 0; hi = keys - 1; own = 0; }   // (no look at the sequences' lengths)
    else prefix_seen(a, tok, keys, lo, hi, own);
  } else {
    own = tok;
    seen_by(a.rules, start + tok, tok, keys, lo, hi);
  }
  const float slope = MODS & kBias ? a.rules.slopes[g] : 0.f, slope2 = slope * kLog2e;
  const bool sees = lo <= hi;   // (a mask of lanes)
  // blocks of 32 keys: those that some row of the wave sees (w0 .. w1), those that all of them see (i0 .. i1)
  const bool idle = wr0 >= R;
  int w0, w1, ilo, ihi, first, last;
  sees_from[tid] = lo;
  sees_to[tid] = hi;
  if (plain) {
    first = 0; last = (keys - 1) >> 5;   // -1 >> 5 = -1: none
    w0 = idle ? INT_MAX : 0; w1 = idle ? -1 : last;
    ilo = 0; ihi = keys - 1;
  } else {
    const int wlo = wave_min(sees && !idle ? lo : INT_MAX), whi = wave_max(sees && !idle ? hi : -1);
    ilo = wave_max(sees ? lo : 0);
    ihi = wave_min(sees ? hi : INT_MAX);
    w0 = wlo == INT_MAX ? INT_MAX : wlo >> 5;
    w1 = whi >> 5;
    if (lane == 0) { span[wave] = w0; span[4 + wave] = w1; }
    __syncthreads();
    first = min(min(span[0], span[1]), min(span[2], span[3]));
    last = max(max(span[4], span[5]), max(span[6], span[7]));
  }
  const int blocks = __builtin_amdgcn_readfirstlane(last < 0 ? 0 : last - first + 1);
  const int base = __builtin_amdgcn_readfirstlane(last < 0 ? 0 : first);
  const int b0 = base + (int)((int64_t)blocks * piece / pieces), b1 = base + (int)((int64_t)blocks * (piece + 1) / pieces);
  const int nsteps = b1 - b0;                                // step t: block b1 - 1 - t
  const int ta = max(b1 - 1 - w1, 0), tb = w1 < 0 ? -1 : min(b1 - 1 - w0, nsteps - 1);   // this wave's steps

  int64_t krow0 = start;
  const int32_t *table = nullptr;
  if constexpr (CACHE) {
    krow0 = a.prefix.pm.table ? 0 : (int64_t)a.prefix_slot * a.prefix.max_seq;
    if (a.prefix.pm.table) table = a.prefix.pm.table + (int64_t)a.prefix_slot * a.prefix.pm.pages_per_slot;
  }
  const bf16 *kcol = (const bf16 *)a.k + (cell / a.kdiv) * T::DH, *ccol = (const bf16 *)a.c + (int64_t)(cell / a.cdiv) * a.dl + slice * T::DLW;
  const char *Kb = (const char *)(kcol + krow0 * a.ks), *Cb = (const char *)(ccol + krow0 * a.cs);
  const unsigned wk2 = (unsigned)a.ks * 2, wc2 = (unsigned)a.cs * 2;

  bf16x8 qf[T::DH / 16];
  f32x16 acc[T::NDLB];
  each<T::NDLB>(EACH(i) { acc[i] = f32x16{}; });
  float m_run = -INFINITY, l_run = 0.f;

  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  constexpr int KI = T::K_INSTR / T::NW, CI = T::C_INSTR / T::NW;
  // A lane's offsets in instructions `wave`, `wave` + 4, ..: the latter have rows 4 (keys), 4 C_RPI (latents) further on.  Where registers
  // are short that goes into the buffers' addresses instead (a dozen scalar instructions a step: 4 x 4096 tokens of packed documents, 1B
  // shape, 94 -> 104 us; with cap and bias 4 spilled loads a step less, 2 x 8192 of the wide shape 1540 -> 1285).
  constexpr bool FEW = MODS == (kCap | kBias) || (T::NDLB == 8 && MODS != 0);
  unsigned kv[FEW ? 1 : KI], cv[FEW ? 1 : CI];
#pragma unroll
  for (int i = 0; i < (FEW ? 1 : KI); ++i)
    kv[i] = (wave + T::NW * i + T::K_INSTR * (lane / T::K_CPR)) * wk2 + ((lane % T::K_CPR) ^ (T::k_sel(lane / T::K_CPR) * (T::K_CPR / 2))) * 16;
#pragma unroll
  for (int i = 0; i < (FEW ? 1 : CI); ++i) cv[i] = (4 * (i * T::C_RPI + lane / T::C_CPR) + wave) * wc2 + (lane % T::C_CPR) * 16;
  // Request keys, latents of a block; rows past the last key, and blocks past the last step, read as zeros.  Step t reads the keys of
  // the block of step t + 1 and the latents of its own, and asks for the keys of step t + 3's and the latents of step t + 2's: each
  // has this step and the next to arrive in.
  unsigned kfill = lds0, cfill = lds0 + T::K_BYTES;
  int kblk = b1 - 1, cblk = b1 - 1;
  auto rows_at = [&](int blk) { return blk >= b0 ? min(keys - blk * 32, 32) : 0; };
  // `rows` rows (fewer than 1: none) of `row` bytes, `pitch` apart, without the first `skip`
  auto buffer_at = [&](const char *p, int rows, unsigned pitch, unsigned row, int skip) {
    if (!FEW) skip = 0;
    return buffer_of(p + (int64_t)skip * pitch, rows > skip ? (rows - 1 - skip) * pitch + row : 0u);
  };
  auto next_stage = [&](unsigned f, unsigned first) { return f == first + (T::NSTAGE - 1) * T::STAGE ? first : f + T::STAGE; };
  // Pool rows of a block's two runs of 16 rows, each in one page (the second's less 16).  Latents are asked for a step after the keys
  // of their block: the rows are kept.
  int64_t kp0 = 0, kp1 = 0, cp0 = 0, cp1 = 0;
  int page_at = -1, page_is = 0;
  auto page_rows = [&](int j0) __attribute__((always_inline)) {
    const int end = max(keys - 1, 0) & ~15, jt = min(max(j0, 0), end), ju = min(jt + 16, end);
    auto at = [&](int j) {
      const int want = __builtin_amdgcn_readfirstlane(j >> a.ps_shift);
      if (want != page_at) {
        page_at = want;
        page_is = load_uniform(table + want);
        page_is = (unsigned)page_is >= (unsigned)a.prefix.pm.num_pages ? 0 : page_is;
      }
      return ((int64_t)page_is << a.ps_shift) + (j & (a.prefix.pm.page_size - 1));
    };
    kp1 = at(ju) - 16;
    kp0 = at(jt);
  };
  auto issue_k = [&]() __attribute__((always_inline)) {
    const int rows = rows_at(kblk), j0 = kblk * 32;
    if (CACHE && table) {
      page_rows(j0);
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const unsigned to = kfill + (wave + T::NW * i) * T::K_PITCH;
        if (lane < 32) load_to_lds(buffer_at(Kb + kp0 * wk2, rows, wk2, T::K_ROW, 4 * i), kv[FEW ? 0 : i], to);
        else load_to_lds(buffer_at(Kb + kp1 * wk2, rows, wk2, T::K_ROW, 4 * i), kv[FEW ? 0 : i], to);
      }
    } else {
#pragma unroll
      for (int i = 0; i < KI; ++i)
        load_to_lds(buffer_at(Kb + (int64_t)j0 * wk2, rows, wk2, T::K_ROW, 4 * i), kv[FEW ? 0 : i], kfill + (wave + T::NW * i) * T::K_PITCH);
    }
    --kblk;
    kfill = next_stage(kfill, lds0);
  };
  auto issue_c = [&]() __attribute__((always_inline)) {
    const int rows = rows_at(cblk), j0 = cblk * 32;
    if (CACHE && table) {
#pragma unroll
      for (int i = 0; i < CI; ++i) {
        const unsigned to = cfill + (wave + T::NW * i) * T::C_PITCH;
        if constexpr (CI == 1) {
          if (lane < 32) load_to_lds(buffer_at(Cb + cp0 * wc2, rows, wc2, T::C_ROW, 0), cv[0], to);
          else load_to_lds(buffer_at(Cb + cp1 * wc2, rows, wc2, T::C_ROW, 0), cv[0], to);
        } else load_to_lds(buffer_at(Cb + (i < CI / 2 ? cp0 : cp1) * wc2, rows, wc2, T::C_ROW, 4 * T::C_RPI * i), cv[FEW ? 0 : i], to);
      }
    } else {
#pragma unroll
      for (int i = 0; i < CI; ++i)
        load_to_lds(buffer_at(Cb + (int64_t)j0 * wc2, rows, wc2, T::C_ROW, 4 * T::C_RPI * i), cv[FEW ? 0 : i], cfill + (wave + T::NW * i) * T::C_PITCH);
    }
    --cblk;
    cfill = next_stage(cfill, lds0 + T::K_BYTES);
  };
  auto issue = [&]() __attribute__((always_inline)) {   // the latents' block is one behind the keys': its rows are those looked up last
    if (CACHE && table) { cp0 = kp0; cp1 = kp1; }
    issue_c();
    issue_k();
  };
  // all but the last step's requests have landed (with pages there are more of them: a stricter wait), then the waves meet
  auto wait_meet = [&]() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(KI + CI) : "memory"); };

  const int ksel = T::k_sel(ln / T::K_INSTR) * (T::K_ROW / 2);
  const int koff = ln % T::K_INSTR * T::K_PITCH + ln / T::K_INSTR * T::K_ROW + h * 16;
  const int koff_lo = koff + ksel, koff_hi = koff - ksel;
  const int coff = T::K_BYTES + ((lane & 15) >> 2) * T::C_PITCH + h * (T::c_row(1) - T::c_row(0)) +
                   (((lane >> 4) & 1) * 16 + (lane & 3) * 4) * 2 + cg * T::NDLB * 64;
  auto c_frag = [&](int st, int mm, int dlb) {
    const char *p = smem + (st + coff) + T::c_row(4 * mm) + dlb * 64;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + T::c_row(2)));
    const s16x8 c8 = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, c8);
  };
  auto k_frag = [&](int st, int ks) {
    return *reinterpret_cast<const bf16x8 *>(smem + (st + (ks < T::DH / 32 ? koff_lo : koff_hi)) + ks * 32);
  };
  auto scores = [&](int st, f32x16 &s) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    bf16x8 kf[T::DH / 16];
#pragma unroll
    for (int ks = 0; ks < T::DH / 16; ++ks) kf[ks] = k_frag(st, ks);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < T::DH / 16; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
  };
  // register e of a lane: key 8 (e / 4) + 4 h + e % 4 of its block
  auto key_of = [](int e) { return 8 * (e >> 2) + (e & 3); };
  // product to score, plus `plus`, in units of log 2; d0 = position less the block's first key less 4 h.  A cap's tanh is the polynomial
  // for scores up to `near` (Rules; `top` is the largest met).  Where a block has larger ones (far) it is 1 - 2 / (e^2x + 1), off by 2^-23 of
  // the cap, and with caps that this is too much for (those above 256), or that have no polynomial, tanh_exactly.  (With that everywhere,
  // scores above the cap cost a third more: 32 ragged prompts with a cap of 3 142 -> 192 us.)
  struct Consts { float sc2, steep, cap2, poly[5]; };
  const Consts consts{a.rules.scale2, a.rules.steep, a.rules.cap2, {a.rules.poly[0], a.rules.poly[1], a.rules.poly[2], a.rules.poly[3], a.rules.poly[4]}};
  auto score_of = [&](const Consts &k, float s, int e, float d0, float plus, float &top, bool far) __attribute__((always_inline)) {
    if constexpr (MODS & kBias) plus = fmaf(-slope2, fabsf(d0 - (float)key_of(e)), plus);
    if constexpr (MODS & kCap) {
      if (far) return fmaf(-2.f * k.cap2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s * k.steep) + 1.f), k.cap2 + plus);
      const float x = s * k.sc2, y = x * x;
      top = fmaxf(top, fabsf(x));
      return fmaf(x, fmaf(y, fmaf(y, fmaf(y, fmaf(y, k.poly[4], k.poly[3]), k.poly[2]), k.poly[1]), k.poly[0]), plus);
    } else return fmaf(s, k.sc2, plus);
  };
  auto too_far = [&](float top) { return (MODS & kCap) && __builtin_amdgcn_ballot_w64(top > a.rules.near) != 0; };
  auto dist0 = [&](int blk) { return MODS & kBias ? (float)(own - blk * 32 - 4 * h) : 0.f; };
  // the whole step for the scores of a block: rules, mask, running maximum, weights as the second product wants them
  auto softmax = [&](f32x16 &v, int blk, bool masked, bf16x8 (&pn)[2], float &corr) __attribute__((always_inline)) {
    const float d0 = dist0(blk);
    float top = 0.f;
    Consts k = consts;   // (opaque: copies of them in vector registers would be kept through the main loop)
    if (MODS) asm volatile("" : "+s"(k.sc2), "+s"(k.steep), "+s"(k.cap2), "+s"(k.poly[0]), "+s"(k.poly[1]), "+s"(k.poly[2]), "+s"(k.poly[3]), "+s"(k.poly[4]));
    if constexpr (MODS & kCap) {
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(v[e]));
      top *= fabsf(k.sc2);
    }
    if (too_far(top)) {
      if (a.rules.near == k.cap2) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = score_of(k, v[e], e, d0, 0.f, top, true);
      } else {
        float d1 = d0;
        asm volatile("" : "+v"(d1));   // (distances of their own, one after the other: no registers for more)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          v[e] = fmaf(k.cap2, tanh_exactly(v[e] * k.steep), MODS & kBias ? -slope2 * fabsf(d1 - (float)key_of(e)) : 0.f);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = score_of(k, v[e], e, d0, 0.f, top, false);
    }
    if (masked) {
      const int from = sees_from[tid] - blk * 32 - 4 * h, to = sees_to[tid] - blk * 32 - 4 * h;
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = key_of(e) < from || key_of(e) > to ? -INFINITY : v[e];
    }
    float bm = fmaxf(v[0], v[1]);
#pragma unroll
    for (int e = 2; e < 16; e += 2) bm = fmaxf(fmaxf(v[e], v[e + 1]), bm);
    const float m_cand = pair_max(bm), m_new = m_cand > m_run + kLazyThreshold ? fmaxf(m_run, m_cand) : m_run;
    const float ref = m_new > -INFINITY ? m_new : 0.f;
    corr = __builtin_amdgcn_exp2f(m_run - ref);
    m_run = m_new;
    const bf16x2 ones = {(bf16)1.0f, (bf16)1.0f};
    float ps = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      bf16x2 pk;
      pk[0] = (bf16)__builtin_amdgcn_exp2f(v[e] - ref);
      pk[1] = (bf16)__builtin_amdgcn_exp2f(v[e + 1] - ref);
      pn[e >> 3][e & 7] = pk[0]; pn[e >> 3][(e & 7) + 1] = pk[1];
      ps = __builtin_amdgcn_fdot2_f32_bf16(pk, ones, ps, false);   // the row sum uses the rounded values
    }
    l_run = fmaf(l_run, corr, ps);
  };

  bf16x8 pf[2] = {};
  float corr = 1.f;
  issue_k();
  {
    const bf16 *qg = (const bf16 *)a.q + (start + tok) * a.qs + g * T::DH + h * 8;
#pragma unroll
    for (int ks = 0; ks < T::DH / 16; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qg + ks * 16);
#pragma unroll
    for (int ks = 0; ks < T::DH / 16; ++ks) asm volatile("" : "+v"(qf[ks]));   // waited for here and not in the loop
  }
  issue();
  wait_meet();
  auto interior = [&](int t) { const int j = (b1 - 1 - t) * 32; return j >= ilo && j + 31 <= ihi; };
  auto mine = [&](int t) { return t >= ta && t <= tb; };
  int cur = (T::NSTAGE - 1) * T::STAGE, nxt = 0;   // of step -1, which has the scores of block 0
  auto rescale = [&]() {
    if (__builtin_amdgcn_ballot_w64(corr != 1.f) != 0) {   // rare: the running maximum moved
      each<T::NDLB>(EACH(i) { acc[i] *= corr; });
    }
  };
  auto rotate = [&]() {
    wait_meet();
    cur = nxt;
    nxt = nxt == (T::NSTAGE - 1) * T::STAGE ? 0 : nxt + T::STAGE;
  };
  // Steps whose next block all rows see: p0 <= t < p1 <= nsteps.  Every wave takes nsteps of them in all: they meet at each one's end.
  const int p0 = max(ta, b1 - 2 - (ihi - 31 < 0 ? -1 : (ihi - 31) >> 5)), p1 = min(tb, b1 - 1 - ((ilo + 31) >> 5));
  int t = -1;
  // Steps before and behind them, and those of blocks that the wave skips.
  auto plain_until = [&](int end) __attribute__((always_inline)) {
#pragma unroll 1
    for (; t < end; ++t) {
      const bool here = mine(t), next = mine(t + 1);
      issue();
      if (here) rescale();
      f32x16 s;
      bf16x8 pn[2] = {};
      if (next) {
        scores(nxt, s);
        softmax(s, b1 - 2 - t, !interior(t + 1), pn, corr);
      }
      if (here) {
        each<2 * T::NDLB>(EACH(i) {
          constexpr int mm = i / T::NDLB, dlb = i % T::NDLB;
          acc[dlb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c_frag(cur, mm, dlb), pf[mm], acc[dlb], 0, 0, 0);
        });
      }
      pf[0] = pn[0]; pf[1] = pn[1];
      if (!here || !next) corr = 1.f;   // nothing to rescale yet, or nothing left
      rotate();
    }
  };
  plain_until(min(p0, nsteps));
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): a scalar load on its way would make every wait for LDS in the loop one for all of it (87 -> 90 us)
#pragma unroll 1
  for (; t < p1; ++t) {
    // The scores of block t + 1, then the second product of block t with the softmax of block t + 1 between its instructions;
    // fragments are read a few instructions ahead of their use, and the scheduling barriers keep this order.
    constexpr int KS = T::DH / 16, KS1 = KS / 2;
    bf16x8 kf[KS];
#pragma unroll
    for (int ks = 0; ks < KS1; ++ks) kf[ks] = k_frag(nxt, ks);
    __builtin_amdgcn_sched_barrier(0);
    issue();
    rescale();
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks == 1) {
#pragma unroll
        for (int k2 = KS1; k2 < KS; ++k2) kf[k2] = k_frag(nxt, k2);
      }
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    constexpr int NS = 2 * T::NDLB, LA = NS < 3 ? NS : 3;
    auto cread = [&](int i) { return c_frag(cur, i / T::NDLB, i % T::NDLB); };
    bf16x8 cf[NS + LA], pn[2];
#pragma unroll
    for (int i = 0; i < LA; ++i) cf[i] = cread(i);
    float ps = 0.f, top = 0.f;
    const float negm = -m_run, d0 = dist0(b1 - 2 - t);
    const bf16x2 ones = {(bf16)1.0f, (bf16)1.0f};
    auto soft_pair = [&](int e) {
      bf16x2 pk;
      pk[0] = (bf16)__builtin_amdgcn_exp2f(score_of(consts, s[e], e, d0, negm, top, false));
      pk[1] = (bf16)__builtin_amdgcn_exp2f(score_of(consts, s[e + 1], e + 1, d0, negm, top, false));
      pn[e >> 3][e & 7] = pk[0]; pn[e >> 3][(e & 7) + 1] = pk[1];
      ps = __builtin_amdgcn_fdot2_f32_bf16(pk, ones, ps, false);
    };
    each<NS>(EACH(i) {
      if constexpr (i + LA < NS) cf[i + LA] = cread(i + LA);
      acc[i % T::NDLB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cf[i], pf[i / T::NDLB], acc[i % T::NDLB], 0, 0, 0);
#pragma unroll
      for (int e = i * 16 / NS; e < (i + 1) * 16 / NS; ++e)
        if (e % 2 == 0) soft_pair(e);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (__builtin_amdgcn_ballot_w64(!(ps < kRowSumLimit)) != 0 || too_far(top)) {   // rare
      softmax(s, b1 - 2 - t, false, pn, corr);
    } else {
      l_run += ps;
      corr = 1.f;
    }
    pf[0] = pn[0]; pf[1] = pn[1];
    rotate();
  }
  plain_until(nsteps);
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");   // no load may land in what follows

  const float l_all = pair_sum(l_run);
  float z[4] = {};
  each<T::NDLB>(EACH(i) {
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e % 4] = fmaf(acc[i][e], 0.f, z[e % 4]);
  });
  const bool finite = (z[0] + z[1]) + (z[2] + z[3]) == 0.f || !sees || idle;
  const bool split = CACHE || pieces > 1;
  const int64_t at = ((int64_t)(slot + piece) * a.cells + cell) * T::BQ;   // row 0 of the piece's sums
  const int my = qw * 32 + ln;                                            // row of the tile
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(!finite) != 0, 0)) {
    const int c0 = cg * T::NDLB * 32;
    constexpr int COLS = (T::NDLB + 1) / 2;   // of 64 lanes; 32 columns: the upper half of the lanes repeats the lower
#pragma unroll 1
    for (int i = 0; i < 32; ++i) {
      const int rr = wr0 + i;
      if (rr >= R) break;
      const int tk = rr / a.mpc, gg = cell * a.mpc + (rr - tk * a.mpc), l0 = sees_from[wave * 64 + i], l1 = sees_to[wave * 64 + i];
      const int from = max(l0, b0 * 32), to = min(l1, min(b1 * 32, keys) - 1);
      int own_i = tk;
      if constexpr (CACHE) own_i = (int)((int64_t)keys + slot_rows(a.own, a.own.slots ? a.own.slots[tk] : tk) - 1);
      float avg[COLS];
      const bf16 *cc = ccol + c0 - (T::NDLB == 1 && lane >= 32 ? 32 : 0);
      const float w = wave_row(a.rules, (const bf16 *)a.q + (start + tk) * a.qs + gg * T::DH, T::DH, kcol, a.ks, cc, a.cs,
                               MODS & kBias ? a.rules.slopes[gg] : 0.f, own_i, from, to,
                               [&](int j) { return CACHE ? cache_row_clamped(a.prefix.pm, a.prefix.max_seq, a.prefix_slot, j) : start + j; }, avg);
      if (T::NDLB == 1 && lane >= 32) continue;
      if (split) {
#pragma unroll
        for (int e = 0; e < COLS; ++e) a.pacc[(at + qw * 32 + i) * a.dl + slice * T::DLW + c0 + e * 64 + lane] = avg[e];
      } else {
#pragma unroll
        for (int e = 0; e < COLS; ++e)
          *reinterpret_cast<bf16 *>(smem + (qw * 32 + i) * T::OUT_PITCH + (c0 + e * 64 + lane) * 2) = (bf16)(l0 > l1 ? 0.f : w == 0.f ? NAN : avg[e]);
      }
    }
  } else if (split) {
    if (wr0 + ln < R) {
      float *pa = a.pacc + (at + my) * a.dl + slice * T::DLW + cg * T::NDLB * 32 + 4 * h;
      const float inv = l_all == 0.f ? 0.f : __builtin_amdgcn_rcpf(l_all);   // (a piece may have none of the keys that a row sees)
      each<T::NDLB>(EACH(i) { acc[i] *= inv; });
      __builtin_amdgcn_sched_barrier(0);   // every store from registers of its own: one that shares them waits for the one before (27 -> 29 us)
      each<T::NDLB * 4>(EACH(i) {
        constexpr int dlb = i / 4, rq = i % 4;
        *reinterpret_cast<float4 *>(pa + dlb * 32 + rq * 8) = make_float4(acc[dlb][rq * 4], acc[dlb][rq * 4 + 1], acc[dlb][rq * 4 + 2], acc[dlb][rq * 4 + 3]);
      });
    }
  } else {
    const float inv = 1.0f / l_all;
    each<T::NDLB * 4>(EACH(i) {
      constexpr int dlb = i / 4, rq = i % 4;
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16)(sees ? acc[dlb][rq * 4 + e] * inv : 0.f);
      *reinterpret_cast<bf16x4 *>(smem + my * T::OUT_PITCH + (cg * T::NDLB * 32 + dlb * 32 + rq * 8 + 4 * h) * 2) = v;
    });
  }
  if (split) {   // whether the wave went through its rows again or not
    if (h == 0 && slice == 0 && cg == 0 && wr0 + ln < R) a.pml[at + my] = sees ? make_float2(m_run, l_all) : make_float2(-INFINITY, -1.f);
    return;
  }
  __syncthreads();
  constexpr int CPR = T::DLW / 8, RPP = T::NT / CPR;   // 16-byte chunks of a row, rows per pass
  const int rr0 = tid / CPR, ch = tid % CPR;
#pragma unroll 4
  for (int it = 0; it < T::BQ / RPP; ++it) {
    const int rr = it * RPP + rr0, full = r0 + rr;
    if (full < R) {
      const int tk = full / a.mpc;
      bf16 *to = (bf16 *)a.L + ((start + tk) * a.nq + cell * a.mpc + (full - tk * a.mpc)) * (int64_t)a.dl + slice * T::DLW + ch * 8;
      *reinterpret_cast<u32x4 *>(to) = *reinterpret_cast<const u32x4 *>(smem + rr * T::OUT_PITCH + ch * 16);
    }
  }
}

template <class T, int MODS, bool CACHE>
void launch_mods(const RowsArgs &a, unsigned grid, hipStream_t st) {
  allow_dynamic_lds((const void *)rows_attn_kernel<T, MODS, CACHE>, T::SMEM);
  rows_attn_kernel<T, MODS, CACHE><<<grid, T::NT, T::SMEM, st>>>(a);
}

template <class T, bool CACHE>
void launch_tile(RowsArgs a, hipStream_t st) {
  const int64_t tiles = a.tiles < (CACHE ? 8 : 64) ? a.tiles : (a.tiles + 7) / 8 * 8;
  const unsigned grid = (unsigned)(tiles * a.cells * a.slices);
  switch ((a.rules.cap > 0.f ? kCap : 0) | (a.rules.slopes ? kBias : 0)) {
    case 0: launch_mods<T, 0, CACHE>(a, grid, st); break;
    case kCap: launch_mods<T, kCap, CACHE>(a, grid, st); break;
    case kBias: launch_mods<T, kBias, CACHE>(a, grid, st); break;
    default: launch_mods<T, kCap | kBias, CACHE>(a, grid, st);
  }
}

// Latent columns of a workgroup of 128 rows
int wide_tile(const Dims &d) { return d.dh == 128 ? (d.dl % 256 == 0 ? 256 : 128) : (d.dl % 128 == 0 ? 128 : 64); }

template <bool CACHE>
void launch_rows(const Dims &d, RowsArgs a, int dlw, hipStream_t st) {
  a.slices = d.dl / dlw;
  if (d.dh == 64) {
    if (dlw == 128) launch_tile<Tile<64, 128, 4>, CACHE>(a, st);
    else launch_tile<Tile<64, 64, 4>, CACHE>(a, st);
  } else if (dlw == 256) launch_tile<Tile<128, 256, 4>, CACHE>(a, st);
  else launch_tile<Tile<128, 128, 4>, CACHE>(a, st);
}

}  // namespace

bool rows_bf16_ok(const Dims &d) {
  return d.dtype == GTA_BF16 && ((d.dh == 128 && d.dl % 128 == 0) || (d.dh == 64 && d.dl % 64 == 0));
}

// A batch of few rows takes tiles of 64 or 32, whose waves share the columns: scratch memory for as many rows, and less to load where
// a wave would have none.  One call, behind 8192 rows, with and without: 8 sequences of the 1B shape 25.5 / 26.2 us, 32 29.3 / 29.5, 64 35.8 / 35.2,
// 32 of the wide shape 46.2 / 48.0, 64 53.8 / 53.6, 6 of the paper's layer 20.2 / 20.2: level or up to 4 % faster, with a quarter or half
// of the scratch memory.
int prefix_tile_rows(const Dims &d, int rows) {
  if (d.dh == 64) return d.dl % 128 == 0 && rows <= 32 ? 32 : 128;
  return rows <= 32 ? 32 : rows <= 64 && d.dl % 256 == 0 ? 64 : 128;
}
// Latent columns of a workgroup: with 256 two of them share a CU, with 512 the scores are worked out half as often.  One call, 256
// against 512: 64 sequences of the 1B shape behind 1024 rows 24.8 / 29.1 us, 8192 35.5 / 37.9, 32768 47.6 / 49.5; 32 of the wide shape
// 28.4 / 30.8, 44.4 / 42.8, 102.9 / 86.6.  (The line between the two is the bound on the prefix's rows; at 8192 itself the wide shape is on its
// slower side by 4 %.)
static int prefix_columns(const Dims &d, int bq, int prefix_max) {
  if (d.dh == 64 || bq == 128) return wide_tile(d);
  return d.dl % 1024 == 0 && prefix_max > 8192 ? 512 : d.dl % 256 == 0 ? 256 : 128;
}
int prefix_slices(const Dims &d, int bq, int prefix_max) { return d.dl / prefix_columns(d, bq, prefix_max); }

void launch_prefix_rows(const Dims &d, const RowsArgs &args, int bq, hipStream_t st) {
  RowsArgs a = args;
  const int w = prefix_columns(d, bq, a.prefix.max_seq);
  if (bq == 128) { launch_rows<true>(d, a, w, st); return; }
  a.slices = d.dl / w;
  if (d.dh == 64) launch_tile<Tile<64, 128, 1>, true>(a, st);
  else if (bq == 64) {
    if (w == 512) launch_tile<Tile<128, 512, 2>, true>(a, st);
    else launch_tile<Tile<128, 256, 2>, true>(a, st);
  } else if (w == 512) launch_tile<Tile<128, 512, 1>, true>(a, st);
  else if (w == 256) launch_tile<Tile<128, 256, 1>, true>(a, st);
  else launch_tile<Tile<128, 128, 1>, true>(a, st);
}

int masked_bf16_columns(const Dims &d) { return wide_tile(d); }
void launch_masked_bf16(const Dims &d, const RowsArgs &a, hipStream_t st) { launch_rows<false>(d, a, wide_tile(d), st); }

}  // namespace gta
