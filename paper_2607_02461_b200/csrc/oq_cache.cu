// Quantizing keys and values into the pages of a cache, and reading them back.
//
//   k = the smallest exponent with max |x| <= top * 2^k over 32 adjacent coordinates (top: 448 for e4m3, 6 for e2m1), kept in its limits
//   element = x * 2^-k rounded to the format, to nearest even;   value = element * 2^k
//
// 2^-k times a float is exact, so the one rounding is the element's, and an element is what any other exact form gives, bit for bit.  k comes
// from the bits of the maximum: top = 0.875 * 2^9 (0.75 * 2^3), so k is the maximum's exponent less 9 (3), one more where its fraction is larger.
// A power of two leaves up to a bit of the format's range unused, of which a floating-point element loses next to nothing; it makes
// decoding exact.
//
// Bound: memory, or the launch.  A lane owns 8 adjacent coordinates of a head (16 bytes of bf16, 8 or 4 bytes of the cache), a group is 4
// lanes, and a warp takes keys and values of some heads of one token, all requested before the first is used; the look-up of the token's
// page runs beside those loads.
//
// Measured (B200, device time of captured calls): reading 32760 tokens of 40 heads of 128 back from e4m3 to bf16, 1.0 GB: 166 us = 6.1 TB/s, 0.94 of the copy rate;
// writing 1560 tokens, 48 MB: 10.8 us, of which half is the launch and the chain start -> length -> page -> store; one token 2.6 us.
#include <string>

#include "oq_cache.cuh"

namespace oq {
namespace cache {

constexpr int WARPS = 8;

struct Rows {
  void* X;
  long long ld_token, ld_head;
};
struct CopyParams {
  View c;
  Rows k, v;                       // X may be NULL when reading
  const int* start;                // n_seqs + 1, or NULL: one sequence of all tokens
  int total, chunks;               // chunks of heads, a warp each
};

// 8 values as they were loaded (unpacked they take twice the registers, and a kernel that waits for its loads wants many warps).
template <typename T>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
};
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Page and place in it of token `tok` (of all new ones); page -1: it has none.
__device__ __forceinline__ int locate(const CopyParams& p, int tok, int& at) {
  int s = 0, end = p.total;
  bool owned = true;
  if (p.start) {
    s = find_seq(p.start, p.c.n_seqs, tok);
    end = min(max(__ldg(p.start + s + 1), 0), p.total);
    owned = tok >= __ldg(p.start + s) && tok < end;
  }
  const int pos = tok - end + seq_len(p.c, s);        // the new tokens are the sequence's last ones
  at = pos & ((1 << p.c.shift) - 1);
  if (!owned) return -2;
  return pos < 0 ? -1 : page_of(p.c, s, pos);
}

template <int KIND, int D, typename T>
__global__ void __launch_bounds__(32 * WARPS) write_kernel(const __grid_constant__ CopyParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  using F = Format<KIND, D>;
  constexpr int LANES = D / 8, HEADS = 32 / LANES, ITERS = 2;       // heads a warp takes at a time, and how many times
  const int lane = threadIdx.x & 31, sub = lane % LANES;
  const long long w = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
  const int tok = (int)(w / p.chunks), head0 = (int)(w % p.chunks) * HEADS * ITERS + lane / LANES;
  if (tok >= p.total) return;
  Raw<T> raw[2 * ITERS];
#pragma unroll
  for (int i = 0; i < 2 * ITERS; ++i) {
    const Rows& r = i & 1 ? p.v : p.k;
    const int head = head0 + HEADS * (i >> 1);
    if (head < p.c.kv_heads) raw[i].load(reinterpret_cast<const T*>(r.X) + tok * r.ld_token + head * r.ld_head + 8 * sub);
    else raw[i].clear();
  }
  int at;
  const int page = locate(p, tok, at);
  if (page < 0) return;
#pragma unroll
  for (int j = 0; j < ITERS; ++j) {
    uint32_t top[2];
    float x[2][8];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      raw[2 * j + i].get(x[i]);
      top[i] = 0u;                                     // magnitudes compare as whole numbers, NaN above all others
#pragma unroll
      for (int e = 0; e < 8; ++e) top[i] = max(top[i], __float_as_uint(x[i][e]) & 0x7FFFFFFFu);
      top[i] = max(top[i], __shfl_xor_sync(~0u, top[i], 1));
      top[i] = max(top[i], __shfl_xor_sync(~0u, top[i], 2));
      odd |= top[i] >= 0x7F800000u;
    }
    const uint32_t mine = (LANES == 32 ? ~0u : ((1u << LANES) - 1u)) << (lane & ~(LANES - 1));
    const bool broken = (__ballot_sync(~0u, odd) & mine) != 0u;
    const int head = head0 + HEADS * j;
    uint8_t* const block = block_of(p.c, page, head);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int biased = (int)(top[i] >> 23), more = (top[i] & 0x7FFFFFu) > (KIND == 8 ? 0x600000u : 0x400000u);
      const int k = min(max(biased - 126 - (KIND == 8 ? 9 : 3) + more, MIN_EXP), F::MAX_EXP);
      const float inv = __uint_as_float((uint32_t)(127 - k) << 23);
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = broken ? 0.f : x[i][e] * inv;
      uint32_t scale = (broken ? BROKEN : (uint32_t)(k + 127)) << (8 * (sub >> 2));
#pragma unroll
      for (int d = 4; d < LANES; d <<= 1) scale |= __shfl_xor_sync(~0u, scale, d);      // the row's scales in one word
      if (head >= p.c.kv_heads) continue;
      uint8_t* const row = block + (i ? p.c.off_v : 0u) + at * F::ROW + sub * KIND;
      if (KIND == 8) {
        uint32_t u[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          asm("{\n .reg .b16 a, b;\n cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n mov.b32 %0, {a, b};\n}"
              : "=r"(u[e]) : "f"(y[4 * e]), "f"(y[4 * e + 1]), "f"(y[4 * e + 2]), "f"(y[4 * e + 3]));
        *reinterpret_cast<uint2*>(row) = make_uint2(u[0], u[1]);
      } else {
        uint32_t u;
        asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
            " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
            : "=r"(u) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
        *reinterpret_cast<uint32_t*>(row) = u;
      }
      if (sub == 0) {
        uint8_t* const to = block + (i ? p.c.off_vs : p.c.off_ks) + at * F::GROUPS;
        if (F::GROUPS == 4) *reinterpret_cast<uint32_t*>(to) = scale;
        else *reinterpret_cast<uint16_t*>(to) = (uint16_t)scale;
      }
    }
  }
}

template <int KIND, int D, typename T>
__global__ void __launch_bounds__(32 * WARPS) read_kernel(const __grid_constant__ CopyParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  using F = Format<KIND, D>;
  constexpr int LANES = D / 8, HEADS = 32 / LANES, ITERS = 2;
  const int lane = threadIdx.x & 31, sub = lane % LANES;
  const long long w = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
  const int tok = (int)(w / p.chunks), head0 = (int)(w % p.chunks) * HEADS * ITERS + lane / LANES;
  if (tok >= p.total) return;
  int at;
  const int page = locate(p, tok, at);
  if (page == -2) return;                              // no sequence owns the token: its row stays as it was
  uint32_t data[2 * ITERS][2], scale[2 * ITERS];
#pragma unroll
  for (int i = 0; i < 2 * ITERS; ++i) {
    const int head = head0 + HEADS * (i >> 1);
    data[i][0] = data[i][1] = 0u;
    scale[i] = 127u;
    if (page >= 0 && head < p.c.kv_heads && (i & 1 ? p.v.X : p.k.X)) {
      const uint8_t* const block = block_of(p.c, page, head);
      const uint8_t* const row = block + (i & 1 ? p.c.off_v : 0u) + at * F::ROW + sub * KIND;
      data[i][0] = *reinterpret_cast<const uint32_t*>(row);
      if (KIND == 8) {
        const uint2 both = *reinterpret_cast<const uint2*>(row);
        data[i][0] = both.x;
        data[i][1] = both.y;
      }
      scale[i] = block[(i & 1 ? p.c.off_vs : p.c.off_ks) + at * F::GROUPS + (sub >> 2)];
    }
  }
#pragma unroll
  for (int i = 0; i < 2 * ITERS; ++i) {
    const Rows& r = i & 1 ? p.v : p.k;
    const int head = head0 + HEADS * (i >> 1);
    if (head >= p.c.kv_heads || !r.X) continue;
    uint32_t h[4];
    if (KIND == 8) {
      e4m3_to_f16(data[i][0], h[0], h[1]);
      e4m3_to_f16(data[i][1], h[2], h[3]);
    } else {
      e2m1_to_f16(data[i][0], h[0], h[1], h[2], h[3]);
    }
    const float s = scale[i] == BROKEN ? __uint_as_float(0x7FC00000u) : __uint_as_float(scale[i] << 23);
    float x[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float lo, hi;
      asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}" : "=f"(lo), "=f"(hi) : "r"(h[e]));
      x[2 * e] = lo * s;
      x[2 * e + 1] = hi * s;
    }
    store8(reinterpret_cast<T*>(r.X) + tok * r.ld_token + head * r.ld_head + 8 * sub, x);
  }
}

bool rows_meet(long long apart, long long tokens, long long heads, long long ld_token, long long ld_head, int width) {
  using wide = __int128;
  if (tokens < 2) ld_token = 0;
  if (heads < 2) ld_head = 0;
  const wide all_heads = (wide)(heads - 1) * ld_head + width, all_tokens = (wide)(tokens - 1) * ld_token + width;
  if (apart == 0) {                                  // the two usual orders of one set
    if (tokens < 2 || heads < 2 || ld_token >= all_heads || ld_head >= all_tokens) return false;
  } else {                                           // two sets, one behind the other
    const wide reach = all_heads + all_tokens - width;
    if (apart >= reach || -(wide)apart >= reach) return false;
    // beside each other in the rows of one tensor, and dealt out between each other's heads
    auto between = [&](long long ld, wide need) {
      const long long at = (apart % ld + ld) % ld;
      return at >= need && ld - at >= need;
    };
    if (ld_token && between(ld_token, all_heads)) return false;
    if (ld_head && ld_token % ld_head == 0 && between(ld_head, width)) return false;
  }
  // else: rows dh heads and dt tokens from each other are apart + dh ld_head + dt ld_token apart; of the dt only those beside the quotient can be close
  for (long long dh = 1 - heads; dh < heads; ++dh) {
    const wide at = (wide)apart + (wide)dh * ld_head;
    const long long near = ld_token ? (long long)(-at / ld_token) : 0;
    for (long long dt = near - 1; dt <= near + 1; ++dt) {
      const wide d = at + (wide)dt * ld_token;
      if (dt > -tokens && dt < tokens && (apart || dh || dt) && d > -width && d < width) return true;
    }
  }
  return false;
}

int make_view(const oq_cache* c, const char* what, View* view) {
  const std::string w(what);
  if (!c) return fail(OQ_ERR_INVALID_ARG, w + ": NULL cache");
  size_t block = 0;
  const int rc = oq_cache_block_bytes(c->kind, c->page_size, c->head_dim, &block);
  if (rc != OQ_OK) return rc;
  if (c->n_pages < 0 || c->n_kv_heads <= 0 || c->n_seqs < 1 || c->max_pages < 0) return fail(OQ_ERR_INVALID_ARG, w + ": bad sizes of the cache");
  if (c->n_kv_heads > 65535) return fail(OQ_ERR_UNSUPPORTED, w + ": more than 65535 heads");
  if (c->n_seqs > MAX_SEQS) return fail(OQ_ERR_UNSUPPORTED, w + ": more than 256 sequences");
  if ((long long)c->max_pages * c->page_size > (1 << 30)) return fail(OQ_ERR_UNSUPPORTED, w + ": more than 2^30 positions in a row of the table");
  if ((c->n_pages > 0 && !c->pages) || (c->max_pages > 0 && !c->table) || !c->lens) return fail(OQ_ERR_INVALID_ARG, w + ": NULL pages, table or lens");
  if (c->n_seqs > 1 && c->ld_table < c->max_pages) return fail(OQ_ERR_INVALID_ARG, w + ": rows of the table lie over each other");
  if (!aligned16(c->pages)) return fail(OQ_ERR_ALIGNMENT, w + ": pages must be 16-byte aligned");
  View& v = *view;
  v.pages = reinterpret_cast<uint8_t*>(c->pages);
  v.block_bytes = (uint32_t)block;
  v.page_bytes = (long long)block * c->n_kv_heads;
  const uint32_t row = (uint32_t)(c->head_dim * c->kind / 8), groups = (uint32_t)(c->head_dim / 32);
  v.off_v = row * c->page_size;
  v.off_ks = 2 * v.off_v;
  v.off_vs = v.off_ks + groups * c->page_size;
  v.n_pages = c->n_pages;
  v.shift = 0;
  while ((1 << v.shift) < c->page_size) ++v.shift;
  v.kv_heads = c->n_kv_heads;
  v.table = c->table;
  v.ld_table = c->n_seqs > 1 ? c->ld_table : 0;
  v.lens = c->lens;
  v.n_seqs = c->n_seqs;
  v.max_len = c->max_pages * c->page_size;
  return OQ_OK;
}

template <bool WRITE>
static int copy(const char* what, const oq_cache* c, const oq_cache_rows* k, const oq_cache_rows* v, int dtype, const int* start, int total, void* stream) {
  const std::string w(what);
  CopyParams p = {};
  int rc = make_view(c, what, &p.c);
  if (rc != OQ_OK) return rc;
  if (total < 0) return fail(OQ_ERR_INVALID_ARG, w + ": negative number of tokens");
  if (total > (1 << 30)) return fail(OQ_ERR_UNSUPPORTED, w + ": more than 2^30 tokens");
  if (dtype != OQ_BF16 && dtype != OQ_F32) return fail(OQ_ERR_INVALID_ARG, w + ": bad element type");
  if (c->n_seqs > 1 && !start) return fail(OQ_ERR_INVALID_ARG, w + ": several sequences need start");
  if (WRITE ? (!k || !v) : (!k && !v)) return fail(OQ_ERR_INVALID_ARG, w + ": NULL keys or values");
  const int unit = dtype == OQ_BF16 ? 8 : 4;
  const oq_cache_rows* both[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    if (!both[i]) continue;
    const oq_cache_rows& r = *both[i];
    if (total > 0 && !r.X) return fail(OQ_ERR_INVALID_ARG, w + ": NULL keys or values");
    if (!aligned16(r.X) || r.ld_token % unit || r.ld_head % unit) return fail(OQ_ERR_ALIGNMENT, w + ": pointers and strides must be multiples of 16 bytes");
    const long long least = WRITE ? 0 : c->head_dim;          // rows that are read may lie over each other
    if ((total > 1 && r.ld_token < least) || (c->n_kv_heads > 1 && r.ld_head < least)) return fail(OQ_ERR_INVALID_ARG, w + ": bad strides");
    (i ? p.v : p.k) = Rows{r.X, total > 1 ? r.ld_token : 0, c->n_kv_heads > 1 ? r.ld_head : 0};
    if (!WRITE && total > 0 && rows_meet(0, total, c->n_kv_heads, r.ld_token, r.ld_head, c->head_dim))
      return fail(OQ_ERR_INVALID_ARG, w + ": rows of the output lie over each other");
  }
  if (!WRITE && total > 0 && k && v) {
    // (rows of different strides are only seen to meet where both begin)
    const long long apart = (reinterpret_cast<intptr_t>(v->X) - reinterpret_cast<intptr_t>(k->X)) / (16 / unit);
    const bool alike = p.k.ld_token == p.v.ld_token && p.k.ld_head == p.v.ld_head;
    if (apart == 0 || (alike && rows_meet(apart, total, c->n_kv_heads, p.k.ld_token, p.k.ld_head, c->head_dim)))
      return fail(OQ_ERR_INVALID_ARG, w + ": keys and values lie over each other");
  }
  if (total == 0) return OQ_OK;
  p.start = start;
  p.total = total;
  const int heads = 2 * 256 / c->head_dim;                     // of a warp
  p.chunks = (c->n_kv_heads + heads - 1) / heads;
  const long long grid = ((long long)total * p.chunks + WARPS - 1) / WARPS;
  if (grid > 0x7FFFFFFFll) return fail(OQ_ERR_UNSUPPORTED, w + ": too many rows for one launch");
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto wk, auto rk) { return launch_dependent(WRITE ? wk : rk, (int)grid, 32 * WARPS, 0, st, p); };
  cudaError_t e;
  if (c->kind == OQ_CACHE_FP8) {
    if (c->head_dim == 128) e = dtype == OQ_BF16 ? go(write_kernel<8, 128, __nv_bfloat16>, read_kernel<8, 128, __nv_bfloat16>) : go(write_kernel<8, 128, float>, read_kernel<8, 128, float>);
    else e = dtype == OQ_BF16 ? go(write_kernel<8, 64, __nv_bfloat16>, read_kernel<8, 64, __nv_bfloat16>) : go(write_kernel<8, 64, float>, read_kernel<8, 64, float>);
  } else {
    if (c->head_dim == 128) e = dtype == OQ_BF16 ? go(write_kernel<4, 128, __nv_bfloat16>, read_kernel<4, 128, __nv_bfloat16>) : go(write_kernel<4, 128, float>, read_kernel<4, 128, float>);
    else e = dtype == OQ_BF16 ? go(write_kernel<4, 64, __nv_bfloat16>, read_kernel<4, 64, __nv_bfloat16>) : go(write_kernel<4, 64, float>, read_kernel<4, 64, float>);
  }
  return e == cudaSuccess ? OQ_OK : cuda_fail(e, what);
}

}  // namespace cache
}  // namespace oq

using namespace oq;

extern "C" {

int oq_cache_block_bytes(int kind, int page_size, int head_dim, size_t* bytes) {
  if (!bytes) return fail(OQ_ERR_INVALID_ARG, "oq_cache_block_bytes: bytes is NULL");
  *bytes = 0;
  if (kind != OQ_CACHE_FP8 && kind != OQ_CACHE_FP4) return fail(OQ_ERR_INVALID_ARG, "cache: kind must be OQ_CACHE_FP8 or OQ_CACHE_FP4");
  if (head_dim != 64 && head_dim != 128) return fail(OQ_ERR_UNSUPPORTED, "cache: head_dim must be 64 or 128");
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1))) return fail(OQ_ERR_UNSUPPORTED, "cache: page_size must be a power of two from 16 to 256");
  *bytes = 2 * (size_t)page_size * (size_t)(head_dim * kind / 8 + head_dim / 32);
  return OQ_OK;
}

int oq_cache_write(const oq_cache* c, const oq_cache_rows* K, const oq_cache_rows* V, int x_dtype, const int* start, int total, void* stream) {
  return cache::copy<true>("oq_cache_write", c, K, V, x_dtype, start, total, stream);
}

int oq_cache_read(const oq_cache* c, const oq_cache_rows* K, const oq_cache_rows* V, int y_dtype, const int* start, int total, void* stream) {
  return cache::copy<false>("oq_cache_read", c, K, V, y_dtype, start, total, stream);
}

}  // extern "C"
