// Caches of 8-bit rows: blocks of 32 e4m3 elements with one power-of-two scale each.  A block with exponent e holds
// code * 2^e; its scale byte is e + 127.  Appended blocks have e in [kMxMinExp, kMxMaxExp], so that every value a block
// stands for is zero or a normal bf16 number: reading a row back in 16 bits, or feeding it to a matrix instruction, rounds
// nothing.
#pragma once
#include <algorithm>

#include "gta_internal.h"

namespace gta {

constexpr int kMxBlock = GTA_MX_BLOCK, kMxMinExp = -117, kMxMaxExp = 119;

struct MxView {
  uint8_t *k, *c, *ks, *cs;   // codes and scale bytes
  int32_t *seq_lens, *status;
  const int32_t *slots;
  int max_batch, max_seq;
  PageMap pm;
};

inline MxView mx_view_of(const gta_mx_cache &c, const int32_t *slots) {
  return MxView{(uint8_t *)c.k, (uint8_t *)c.c, c.k_scale, c.c_scale, c.seq_lens, c.status, slots, c.max_batch, c.max_seq,
                PageMap{c.block_table, c.page_size, c.pages_per_slot, c.num_pages}};
}

// Results of more bytes than the L2s hold (8 of 4 MiB) are stored past them (non-temporal) where a wave's stores fill whole lines,
// which is where a thread has one 16-byte word: nothing of the beginning would be left in the L2s when the next kernel asks for
// it, and the stores run faster (rows of 100 MB read back 42 -> 25 us, 44 MB of normed rows 22 -> 19).  Smaller ones stay for
// whoever reads them next, in the same time.  (Appended prompts have a rule of their own.)
inline bool stream_past_caches(int64_t bytes) { return bytes > (32 << 20); }

// 16 bytes
template <bool NT, typename V>
__device__ __forceinline__ void store16(V *p, const V &v) {
  static_assert(sizeof(V) == 16, "one word");
  if constexpr (NT) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// 2^e of a scale byte
__device__ __forceinline__ float mx_scale(unsigned byte) { return __uint_as_float(byte << 23); }

// Do heads and latents consist of whole blocks, and rows of no more elements than the kernels' divisions take?
inline bool mx_widths_ok(const Dims &d) { return d.dh % kMxBlock == 0 && d.dl % kMxBlock == 0 && d.wk_w + d.wc_w <= (1 << 18); }

int launch_mx_append(const Dims &d, const MxView &cv, const void *k_new, int64_t k_stride, const void *c_new, int64_t c_stride,
                     const int32_t *cu_new, int batch, int max_new, hipStream_t st);
int launch_mx_read(const Dims &d, const MxView &cv, const int32_t *first, const int32_t *cu_rows, int batch, int max_rows,
                   void *k_out, void *c_out, hipStream_t st);

// Attention of one token per sequence.
bool mx_decode_dims_ok(const Dims &d);
bool mx_decode_tuned(const Dims &d);   // taken by the matrix-instruction kernel, with pages of a power of two of at least 16 rows
size_t mx_decode_bytes(const Dims &d, int batch, int max_seq, int requested);
// GTA_ERR_WORKSPACE, with nothing launched, where the workspace is too small
int launch_mx_decode(const Dims &d, const void *q, const MxView &cv, int batch, int requested, void *ws, size_t ws_bytes, void *l_out,
                     hipStream_t st);

int launch_qk_norm_rope(const Dims &d, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *q_gain,
                        const void *k_gain, float eps, const int32_t *positions, int64_t total, void *q_out, void *k_out,
                        hipStream_t st);

}  // namespace gta
