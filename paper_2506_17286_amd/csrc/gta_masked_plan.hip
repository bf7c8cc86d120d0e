// A batch of packed sequences as a list of tiles of query rows for the kernels of gta_prefill_masked_attention, and the join of tiles
// whose keys were shared out.
#include <math.h>

#include "gta_rows_attn.h"

namespace gta {
namespace {

// Rows of a sequence of n tokens, in tiles
__device__ __forceinline__ int tiles_of(int n, int mpc, int bq) { return n > 0 ? (int)(((int64_t)n * mpc + bq - 1) / bq) : 0; }

struct PlanArgs {
  const int32_t *cu;
  int per_seq, batch, mpc, bq, capacity, max_len;
  const int32_t *first, *last;
  int per, most;      // workgroups of a tile; pieces to cut the batch into at least (0: none is cut)
  int32_t *offsets;   // [batch + 1] tiles in front of each sequence
  Piece *list;        // [capacity]
  int32_t *count;     // pieces, tiles that are cut
  Piece *cut;         // [capacity]
};

// Lists a batch's tiles, most keys first, one workgroup.  What a tile sees is estimated from its first and last token, which is
// exact for intervals whose ends do not fall; the kernel works out its own.  With `most` the tiles of a batch that would leave CUs
// idle are cut into pieces of about as many blocks of keys as make that many.  Bound by its chain of loads, scans and LDS atomics: 5.5 us
// for 4 sequences of 4096 tokens, 9 for 32 ragged ones.
constexpr int kPlanThreads = 1024, kBins = 256, kLeastBlocks = 4, kPlanBatch = 2047, kPlanKept = 4;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  __shared__ int bins[kBins], sums[kPlanThreads / 64], total_s, slots_s, cuts_s;
  __shared__ unsigned long long cost_s;
  __shared__ int offsets_s[kPlanBatch + 1];
  int *offsets = a.batch <= kPlanBatch ? offsets_s : a.offsets;   // the search looks at them again and again
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < kBins; i += kPlanThreads) bins[i] = 0;
  if (tid == 0) { cost_s = 0; slots_s = 0; cuts_s = 0; }
  int before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kPlanThreads) {   // tiles in front of each sequence
    const int b = b0 + tid;
    const int n = b < a.batch ? tiles_of(a.cu ? a.cu[b + 1] - a.cu[b] : a.per_seq, a.mpc, a.bq) : 0;
    int run = n;
    for (int i = 1; i < 64; i <<= 1) { const int v = __shfl_up(run, i); run += lane >= i ? v : 0; }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    int add = before, all = before;
    for (int w = 0; w < kPlanThreads / 64; ++w) { add += w < wave ? sums[w] : 0; all += sums[w]; }
    if (b < a.batch) offsets[b] = add + run - n;
    before = all;
    __syncthreads();
  }
  if (tid == 0) offsets[a.batch] = before;
  __threadfence_block();
  __syncthreads();
  const int tiles = min(before, a.capacity);
  auto look = [&](int t, int &b, int &tile) {
    int lo = 0, hi = a.batch;   // offsets[lo] <= t < offsets[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (offsets[mid] <= t) lo = mid;
      else hi = mid;
    }
    b = lo;
    tile = t - offsets[lo];
    const int64_t start = a.cu ? a.cu[b] : (int64_t)b * a.per_seq;
    const int n = a.cu ? a.cu[b + 1] - (int)start : a.per_seq;
    const int t0 = (int)((int64_t)tile * a.bq / a.mpc), t1 = min((int)(((int64_t)(tile + 1) * a.bq - 1) / a.mpc), n - 1);
    const int from = a.first ? max(a.first[start + t0], 0) : 0, to = min(a.last ? max(a.last[start + t0], a.last[start + t1]) : t1, n - 1);
    return to < from ? 0 : (to >> 5) - (from >> 5) + 1;
  };
  const int widest = (a.max_len + 31) / 32;
  auto bin_of = [&](int blocks) { return kBins - 1 - min((int)((int64_t)blocks * (kBins - 1) / max(widest, 1)), kBins - 1); };   // most first
  // f(tile number, sequence, tile, blocks of keys) for this thread's tiles; the first few are looked up once
  int kept_b[kPlanKept], kept_tile[kPlanKept], kept_blocks[kPlanKept];
#pragma unroll
  for (int i = 0; i < kPlanKept; ++i) {
    const int t = tid + i * kPlanThreads;
    if (t < tiles) kept_blocks[i] = look(t, kept_b[i], kept_tile[i]);
  }
  auto each_tile = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kPlanKept; ++i)
      if (tid + i * kPlanThreads < tiles) f(kept_b[i], kept_tile[i], kept_blocks[i]);
    for (int t = tid + kPlanKept * kPlanThreads; t < tiles; t += kPlanThreads) {
      int b, tile;
      const int blocks = look(t, b, tile);
      f(b, tile, blocks);
    }
  };
  int target = INT_MAX;
  if (a.most) {
    unsigned long long mine = 0;
    each_tile([&](int, int, int blocks) { mine += blocks; });
    if (mine) atomicAdd(&cost_s, mine);
    __syncthreads();
    target = max((int)((cost_s * a.per + a.most - 1) / a.most), kLeastBlocks);
  }
  auto pieces_of = [&](int blocks) { return a.most && blocks > target ? (blocks + target - 1) / target : 1; };
  each_tile([&](int, int, int blocks) {
    const int n = pieces_of(blocks);
    atomicAdd(&bins[bin_of(blocks / n)], n);
  });
  __syncthreads();
  if (wave == 0) {   // four bins a lane
    int v[kBins / 64], sum = 0;
    for (int i = 0; i < kBins / 64; ++i) { v[i] = bins[lane * (kBins / 64) + i]; sum += v[i]; }
    int run = sum;
    for (int i = 1; i < 64; i <<= 1) { const int up = __shfl_up(run, i); run += lane >= i ? up : 0; }
    if (lane == 63) total_s = run;
    run -= sum;
    for (int i = 0; i < kBins / 64; ++i) { bins[lane * (kBins / 64) + i] = run; run += v[i]; }
  }
  __syncthreads();
  each_tile([&](int b, int tile, int blocks) {
    const int n = pieces_of(blocks);
    const int slot = n > 1 ? atomicAdd(&slots_s, n) : 0, at = atomicAdd(&bins[bin_of(blocks / n)], n);
    for (int i = 0; i < n; ++i)
      if (at + i < a.capacity) a.list[at + i] = Piece{b, tile, i, n, slot, {}};
    if (n > 1) {
      const int c = atomicAdd(&cuts_s, 1);
      if (c < a.capacity) a.cut[c] = Piece{b, tile, 0, n, slot, {}};
    }
  });
  __syncthreads();
  if (tid == 0) { a.count[0] = min(total_s, a.capacity); a.count[1] = min(cuts_s, a.capacity); }
}

// Joins the pieces of one row of a tile: weights l 2^(m - max); a wave per (row, cell), four columns a lane and step.
template <typename T>
__global__ __launch_bounds__(256) void join_pieces_kernel(RowsArgs a, const Piece *cut, int bq) {
  if ((int)blockIdx.x >= a.count[1]) return;
  const Piece p = cut[blockIdx.x];
  const int lane = threadIdx.x & 63, cell = blockIdx.z, rr = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int64_t start = a.cu ? a.cu[p.b] : (int64_t)p.b * a.per_seq;
  const int R = (a.cu ? a.cu[p.b + 1] - (int)start : a.per_seq) * a.mpc, full = p.tile * bq + rr;
  if (full >= R) return;
  auto at = [&](int i) { return ((int64_t)(p.slot + i) * a.cells + cell) * bq + rr; };
  float mx = -INFINITY;
  for (int i = 0; i < p.pieces; ++i) mx = fmaxf(mx, a.pml[at(i)].x);
  const float ref = mx > -INFINITY ? mx : 0.f;
  const int tk = full / a.mpc;
  T *to = (T *)a.L + ((start + tk) * a.nq + cell * a.mpc + (full - tk * a.mpc)) * (int64_t)a.dl;
  float l = 0.f;
  for (int i = 0; i < p.pieces; ++i) {
    const float2 ml = a.pml[at(i)];
    if (!(ml.y < 0.f)) l = fmaf(__builtin_amdgcn_exp2f(ml.x - ref), ml.y, l);
  }
  int lo, hi;
  seen_by(a.rules, start + tk, tk, R / a.mpc, lo, hi);
  const float inv = lo <= hi ? 1.f / l : 0.f;
  for (int col = lane * 4; col < a.dl; col += 256) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < p.pieces; ++i) {
      const float2 ml = a.pml[at(i)];
      if (ml.y < 0.f) continue;
      const float w = __builtin_amdgcn_exp2f(ml.x - ref) * ml.y * inv;
      const float4 s = *reinterpret_cast<const float4 *>(a.pacc + at(i) * a.dl + col);
      v.x = fmaf(w, s.x, v.x); v.y = fmaf(w, s.y, v.y); v.z = fmaf(w, s.z, v.z); v.w = fmaf(w, s.w, v.w);
    }
    if (lo <= hi && !(l > 0.f)) v.x = v.y = v.z = v.w = NAN;   // scores of nothing but -infinity, or NaN among them
    to[col] = (T)v.x; to[col + 1] = (T)v.y; to[col + 2] = (T)v.z; to[col + 3] = (T)v.w;
  }
}

// Pieces of a batch that is cut.  Not cut / 256 / 512: 2048 tokens of the paper's layer 46 / 43 / 52 us, 4096 80 / 59 / 63; two prompts of 3000 of the
// 1B shape, which are 384 workgroups, not cut 91, cut for 512 110.
constexpr int kAtOnce = 256;
constexpr int kShort = 1536;   // keys

int tile_rows(const Dims &d) { return d.dtype == GTA_BF16 ? 128 : 32; }
int columns(const Dims &d) { return d.dtype == GTA_BF16 ? masked_bf16_columns(d) : rows_f32_columns(d); }

struct MaskedWs {
  int32_t *offsets, *count;
  Piece *list, *cut;
  float *pacc; float2 *pml;
  int64_t capacity, slots;
  int most;
  size_t bytes;
};

// workgroups of a tile
int per_tile(const Dims &d) { return d.nq / maps_per_cell(d) * (d.dl / columns(d)); }
int64_t tiles_at_most(const Dims &d, int batch, int64_t total) { return total * maps_per_cell(d) / tile_rows(d) + batch; }

// What a launch has room for: row numbers of 32 bits, and 2^32 threads (with a last round of eight tiles, and those that are cut)
constexpr int64_t kMostRows = (int64_t)INT32_MAX - 256;
int64_t most_tiles(const Dims &d) { return ((1 << 24) - 1) / per_tile(d) - 8 - kAtOnce; }

// tiles: of the batch at most; least: slots to have room for at least
MaskedWs carve_masked(const Dims &d, int batch, int64_t tiles, void *base, int64_t least = 0) {
  MaskedWs w{};
  const int bq = tile_rows(d), cells = d.nq / maps_per_cell(d), per = per_tile(d);
  w.most = tiles * per < kAtOnce ? kAtOnce : 0;
  w.slots = std::max(w.most ? tiles + kAtOnce / per + 1 : 0, least);
  w.capacity = std::max(tiles, w.slots);
  size_t off = 0;
  auto take = [&](size_t n) { void *p = base ? (char *)base + off : nullptr; off += align_up(n); return p; };
  w.offsets = (int32_t *)take(((size_t)batch + 1) * 4);
  w.count = (int32_t *)take(8);
  w.list = (Piece *)take((size_t)w.capacity * sizeof(Piece));
  w.cut = (Piece *)take((size_t)w.slots * sizeof(Piece));   // (a batch that is cut has as many slots as its list has entries)
  w.pml = (float2 *)take((size_t)w.slots * cells * bq * 8);
  w.pacc = (float *)take((size_t)w.slots * cells * bq * d.dl * 4);
  w.bytes = off;
  return w;
}

}  // namespace

bool masked_tuned(const Dims &d) { return rows_bf16_ok(d) || rows_f32_ok(d); }

// 16-byte chunks, and 32 rows within the 2 GiB that an offset reaches
bool rows_operands_ok(const void *p, int64_t stride, int esize) {
  return !((uintptr_t)p & 15u) && stride * esize % 16 == 0 && stride * esize * 32 < ((int64_t)1 << 31);
}

bool masked_fits(const Dims &d, int batch, int64_t total) {
  return masked_tuned(d) && total * maps_per_cell(d) < kMostRows && tiles_at_most(d, batch, total) <= most_tiles(d);
}

size_t masked_bytes(const Dims &d, int batch, int64_t total) {
  return masked_fits(d, batch, total) ? carve_masked(d, batch, tiles_at_most(d, batch, total), nullptr).bytes : 0;
}

// More sequences or tokens than a launch takes: as for the most that it takes.
size_t masked_bytes_up_to(const Dims &d, int batch, int64_t total) {
  if (!masked_tuned(d) || most_tiles(d) < 1) return 0;
  const int64_t tokens = std::min(total, kMostRows / maps_per_cell(d));
  const int64_t tiles = std::min(tiles_at_most(d, batch, tokens), most_tiles(d));
  const MaskedWs w = carve_masked(d, batch, tiles, nullptr);
  // the largest batch that is cut has fewer than kAtOnce workgroups
  const int per = per_tile(d);
  return w.most ? w.bytes : carve_masked(d, batch, tiles, nullptr, (kAtOnce - 1) / per + kAtOnce / per + 1).bytes;
}

int launch_masked(const Dims &d, const MaskedArgs &m, void *ws, hipStream_t st) {
  const MaskedWs w = carve_masked(d, m.batch, tiles_at_most(d, m.batch, m.total), ws);
  RowsArgs a{};
  a.q = m.q; a.k = m.k; a.c = m.c; a.qs = m.q_stride; a.ks = m.k_stride; a.cs = m.c_stride; a.L = m.l_out;
  a.cu = m.cu; a.per_seq = (int)(m.total / m.batch); a.batch = m.batch;
  a.nq = d.nq; a.mpc = maps_per_cell(d); a.cells = d.nq / a.mpc; a.kdiv = d.qpk / a.mpc; a.cdiv = d.qpc / a.mpc; a.dl = d.dl;
  a.slices = d.dl / columns(d);
  a.rules = m.rules;
  a.list = w.list; a.count = w.count; a.tiles = (int)w.capacity; a.pacc = w.pacc; a.pml = w.pml;
  const int bq = tile_rows(d);
  // Where the chip holds every (tile, sequence) up to the longest at once and no chain of keys is long, tiles need no list and no cut.
  // With and without: one prompt of the paper's layer of 128 tokens 15.8 / 9.2 us, 500 24.6 / 15.5, 1000 35.8 / 24.3, 2000 45.1 / 41.4; of the
  // 1B shape 19.4 / 12.2, 30.7 / 20.5, 44.2 / 31.6, 51.1 / 53.5; fp32 paper's layer 19.0 / 11.9, 28.7 / 23.4, 46.9 / 38.3, 83.5 / 82.7.
  const int64_t levels = ((int64_t)std::min<int64_t>(m.max_len, m.total) * a.mpc + bq - 1) / bq;
  if (m.max_len <= kShort && levels * m.batch * a.cells * a.slices <= 2 * kAtOnce) {
    a.list = nullptr;
    a.tiles = (int)(levels * m.batch);
    if (d.dtype == GTA_BF16) launch_masked_bf16(d, a, st);
    else launch_rows_f32(d, a, false, st);
    return check_launch();
  }
  plan_kernel<<<1, kPlanThreads, 0, st>>>(PlanArgs{m.cu, a.per_seq, m.batch, a.mpc, bq, (int)w.capacity, m.max_len, m.rules.first, m.rules.last,
                                                  a.cells * a.slices, w.most, w.offsets, w.list, w.count, w.cut});
  if (d.dtype == GTA_BF16) launch_masked_bf16(d, a, st);
  else launch_rows_f32(d, a, false, st);
  if (w.most) {
    const dim3 grid((unsigned)(w.slots / 2 + 1), (unsigned)(bq / 4), (unsigned)a.cells);
    if (d.dtype == GTA_BF16) join_pieces_kernel<__bf16><<<grid, 256, 0, st>>>(a, w.cut, bq);
    else join_pieces_kernel<float><<<grid, 256, 0, st>>>(a, w.cut, bq);
  }
  return check_launch();
}

}  // namespace gta
