// The paged cache of quantized keys and values, as its kernels see it: layout, look-up of a token's page, decoding to fp16.
//
// A page holds page_size tokens (a power of two from 16 to 256) of all heads, one block a head.  A block: keys [page_size][row], values [page_size][row],
// scales of the keys [page_size][groups], of the values [page_size][groups]; row = head_dim * bits / 8 bytes, groups = head_dim / 32.
// A scale is a byte s = k + 127 and stands for 2^k, with -14 <= k <= 7 (e4m3) or 13 (e2m1): with these limits every cached value, element
// times scale, is an exact fp16 (e4m3: multiples of 2^-23 up to 448 * 2^7 = 57344; e2m1: of 2^-15 up to 6 * 2^13 = 49152), so the tensor cores
// take what is decoded without a rounding.  Scales of 255 in a row mark a token of a head that held a NaN or an infinity.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "oq_internal.h"

namespace oq {
namespace cache {

constexpr int MAX_SEQS = 256;
constexpr int MIN_EXP = -14;
constexpr uint32_t BROKEN = 255u;                // scale byte of a token whose keys or values were not finite

struct View {
  uint8_t* pages;
  long long page_bytes;
  uint32_t block_bytes, off_v, off_ks, off_vs;   // parts of a block
  int n_pages, shift, kv_heads;                  // page_size = 1 << shift
  const int* table;
  long long ld_table;
  const int* lens;
  int n_seqs, max_len;                           // max_len: tokens that a row of the table can hold
};

template <int KIND, int D>
struct Format {
  static constexpr int BITS = KIND;                            // OQ_CACHE_FP8 = 8, OQ_CACHE_FP4 = 4
  static constexpr int ROW = D * BITS / 8, GROUPS = D / 32;
  static constexpr int MAX_EXP = BITS == 8 ? 7 : 13;
};

// The sequence that owns token `tok` of packed tokens (start[n + 1], ascending): by a whole warp, 31 boundaries a round.
__device__ __forceinline__ int find_seq(const int* start, int n, int tok) {
  int base = 0, count = n;
  const int lane = threadIdx.x & 31;
  while (count > 1) {
    const int step = (count + 31) / 32, at = lane * step;
    const bool at_or_after = lane > 0 && at < count && __ldg(start + base + at) <= tok;
    const int k = __popc(__ballot_sync(~0u, at_or_after));     // (ascending: the true ones come first)
    base += k * step;
    count = min(step, count - k * step);
  }
  return base;
}

// Tokens of sequence s, new ones included.
__device__ __forceinline__ int seq_len(const View& c, int s) { return min(max(__ldg(c.lens + s), 0), c.max_len); }
// The page of position `pos` (0 <= pos < max_len) of sequence s, or -1.
__device__ __forceinline__ int page_of(const View& c, int s, int pos) {
  const int page = __ldg(c.table + s * c.ld_table + (pos >> c.shift));
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}
__device__ __forceinline__ uint8_t* block_of(const View& c, int page, int head) {
  return c.pages + page * c.page_bytes + (long long)head * c.block_bytes;
}

// 2^k twice, in fp16, from the scale byte: fp16's exponent is k + 15 = s - 112.  (The mask keeps 255, whose low bits decode to 1, from
// reaching into the other half.)
__device__ __forceinline__ uint32_t scale_pair(uint32_t s0, uint32_t s1) { return (((s0 | s1 << 16) - 0x00700070u) << 10) & 0x7C007C00u; }

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// four e4m3 -> fp16
__device__ __forceinline__ void e4m3_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
}
// eight e2m1 -> fp16
__device__ __forceinline__ void e2m1_to_f16(uint32_t w, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  asm("{\n .reg .b8 p, q, r, s;\n mov.b32 {p, q, r, s}, %4;\n cvt.rn.f16x2.e2m1x2 %0, p;\n cvt.rn.f16x2.e2m1x2 %1, q;\n cvt.rn.f16x2.e2m1x2 %2, r;\n"
      " cvt.rn.f16x2.e2m1x2 %3, s;\n}"
      : "=r"(a), "=r"(b), "=r"(c), "=r"(d)
      : "r"(w));
}

// The part that `what` has in common: checks and fills the view (host).
int make_view(const oq_cache* c, const char* what, View* view);

// Rows of `width` elements, row (h, t) at h * ld_head + t * ld_token, each stride at least the width where it is used: whether one of them lies over a row of a second such set,
// which begins `apart` elements behind the first, or (apart == 0) over another one of its own (host).
bool rows_meet(long long apart, long long tokens, long long heads, long long ld_token, long long ld_head, int width);

}  // namespace cache
}  // namespace oq
