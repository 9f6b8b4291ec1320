// Norms of queries and keys and their rotation by position, in one pass (between the QKV projection and attention).
//
//   n = x * rsqrt(mean(x^2) + eps) * w              the mean over one head, or over all heads of the token
//   angle(a, i) = pos[a] * theta^(-2 i / d_a)       axis a (time, height, width, ...) owns d_a coordinates of a head
//   (u, v) -> (u cos - v sin, u sin + v cos)        for the pair (u, v) that belongs to (a, i)
//
// Bound: memory.  Every value is read once and written once, and there are about 8 operations per value.  A lane owns
// 8 adjacent coordinates of a head (one 16-byte access in bf16), a warp 256 / head_dim heads at a time and ITERS such
// rows together.  Warps (with a norm over all heads: CTAs) stay and walk over the tokens, and request the next rows, the
// table entries of the next token and the positions of the one after it before they work on the present ones: three
// dependent latencies (position, table, rows) overlap with the arithmetic, and 2 KB a warp are always in flight.
// The table (fp64 on the host, rounded once) replaces the sine and cosine of an angle that fp32 could not hold: at
// position 32760 half a unit in the last place is already 1e-3.
//
// Measured (B200, head_dim 128, two sides, 3 axes; device time and share of the copy rate of 6.46 TB/s):
//   norm per head, 4608 tokens x (24 + 24) heads: bf16 pairs 21.4 us, 5.3 TB/s, 0.82; bf16 halves 31.2, 0.56; fp32 pairs 42.6, 0.82;
//     fp32 halves 55.8, 0.63; head_dim 64, (48 + 48) heads: bf16 pairs 25.9, 0.68; halves 34.2, 0.51
//   norm over the row, (40 + 40) heads: 32760 tokens bf16 pairs 243 us, 5.5 TB/s, 0.85; halves 440, 0.47; 16380 tokens fp32 pairs 273, 0.76;
//     halves 322, 0.65; (80 + 80) heads (WIDE_ROW): 16380 tokens bf16 pairs 372, 0.56; 8192 tokens fp32 pairs 521, 0.40; halves 734, 0.28
// bf16 pairs is what the two models here use and what was tuned: what is left there is instruction issue, about 140 instructions for
// 256 values, of which the pairwise arithmetic is half.  The other forms hold twice the table entries (halves) or rows (fp32) and
// spill: 8 to 24 bytes a thread for bf16 halves per head, 188 over the row, 52 to 336 for fp32, 450 to 940 for WIDE_ROW.
#include <cuda_bf16.h>
#include <math.h>

#include <mutex>
#include <new>
#include <string>
#include <vector>

#include "oq_internal.h"

struct oq_rope {
  int n_axes = 0, dim = 0, layout = 0;
  std::vector<int> axis_dim, max_pos;
  std::vector<float> table;          // (cos, sin) pairs: [axis][pos][d_a / 2]
  std::vector<int> base;             // first (cos, sin) pair of an axis in the table
  mutable std::mutex mutex;
  mutable float2* d_table = nullptr; // device copy, created on first GPU use
  mutable int device = -1;
};

namespace oq {
namespace qk {

constexpr int ITERS = 4;            // rows of 256 coordinates one warp holds at a time
constexpr int WARPS = 4;            // warps of a CTA when the norm stays inside a head
constexpr int ROW_WARPS = 8;        // and at most when it runs over a row that fits their registers
constexpr int MAX_AXES = 4;
constexpr int MAX_ROW_WARPS = 32;

struct Side {
  const void* X;
  void* Y;
  const __nv_bfloat16* w;
  long long ld_token, ld_head, ldy_token, ldy_head;
  float inv_count;                  // 1 / values of a row
  int heads, chunks;                // chunks of ITERS * (256 / head_dim) heads
};
struct Params {
  Side side[2];
  int tokens, lanes_per_head, head_dim, rot_dim, n_axes, norm;
  float eps, inv_dim;
  const int* pos;
  long long ldpos;
  const float2* table;
  int axis_end[MAX_AXES];           // in coordinates of the head
  int max_pos[MAX_AXES];
  int base[MAX_AXES];               // first table entry of an axis
};

__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}

// Two fp32 values in one instruction (the kernel is bound by instruction issue wherever it is not bound by memory).  A lane's
// 8 coordinates are held as 4 pairs, so that a value and its partner in the turn are the same half of two pairs:
// PAIRS layout (0 2) (4 6) (1 3) (5 7), HALVES layout (0 1) (2 3) (4 5) (6 7).
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n fma.rn.f32x2 x, x, y, z;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
template <bool HALVES>
__device__ __forceinline__ void to_pairs(const float (&x)[8], float2 (&p)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    p[i] = HALVES ? make_float2(x[2 * i], x[2 * i + 1]) : make_float2(x[4 * (i & 1) + (i >> 1)], x[4 * (i & 1) + 2 + (i >> 1)]);
}
template <bool HALVES>
__device__ __forceinline__ void from_pairs(const float2 (&p)[4], float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[HALVES ? 2 * i : 4 * (i & 1) + (i >> 1)] = p[i].x;
    x[HALVES ? 2 * i + 1 : 4 * (i & 1) + 2 + (i >> 1)] = p[i].y;
  }
}

template <typename T>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = load16(p); }
  __device__ __forceinline__ void get(float (&x)[8]) const { unpack8(a, x); }
};
template <>
struct Raw<float> {
  uint4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = load16(p);
    b = load16(p + 4);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
    x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint4 v;
  __nv_bfloat162 h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
  v.x = *reinterpret_cast<uint32_t*>(&h[0]); v.y = *reinterpret_cast<uint32_t*>(&h[1]);
  v.z = *reinterpret_cast<uint32_t*>(&h[2]); v.w = *reinterpret_cast<uint32_t*>(&h[3]);
  *reinterpret_cast<uint4*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

enum { HEAD = 0, ROW = 1, WIDE_ROW = 2 };      // WIDE_ROW: more than ROW_WARPS warps for a row, half the registers each (40 heads
                                               // of 128 would take 355 us in this form, 243 in the other)

// ROW: the norm runs over all heads of a token; a CTA is one (token, side), its warps meet once in shared memory.
// HEAD: a warp is one (token, side, chunk of heads) and the norm closes inside the lanes of a head.
// HALVES: the partner of a coordinate lies d_a / 2 further on (in another lane), otherwise right beside it.
// LANES: lanes of a head, 0: read from the parameters (head_dim 128, the one of the image and video models, with a norm per head has
// its own: 21.3 us where the general form takes 27.0; the other head_dims share the general form).
// A turned coordinate is y = x * A + partner * B; where the weights are the same for every head (HEAD) they are part of
// A and B, which are made once for a token and serve all of the warp's heads.  That, and reductions of fixed length,
// keep the kernel at ~140 instructions for 256 values; at 270 (weights and side read again for every head, loops of run-time
// length) it took twice the time.
template <typename In, typename Out, int MODE, bool HALVES, int LANES>
__global__ void __launch_bounds__(MODE == WIDE_ROW ? MAX_ROW_WARPS * 32 : (MODE == ROW ? ROW_WARPS : WARPS) * 32, MODE == WIDE_ROW ? 1 : (MODE == ROW ? 2 : 4))
qk_norm_rope_kernel(const __grid_constant__ Params p) {
  constexpr int NP = HALVES ? 8 : 4;           // pairs a lane has a part in
  __shared__ __align__(16) float red[2][MAX_ROW_WARPS];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int L = LANES ? LANES : p.lanes_per_head, sub = lane & (L - 1), c0 = 8 * sub, per_iter = 32 / L;

  // which table entries the lane's pairs have, apart from the position; top < 0: not turned
  int axis[NP], half[NP], entry[NP], top[NP];
  int partner = lane;
  bool upper = false;
#pragma unroll
  for (int e = 0; e < NP; ++e) {
    const int c = HALVES ? c0 + e : c0 + 2 * e;
    axis[e] = half[e] = entry[e] = 0;
    top[e] = -1;
    if (c < p.rot_dim) {
      int a = 0, begin = 0;
      while (a + 1 < p.n_axes && c >= p.axis_end[a]) begin = p.axis_end[a++];
      axis[e] = a;
      half[e] = (p.axis_end[a] - begin) >> 1;
      top[e] = p.max_pos[a];
      int f = HALVES ? c - begin : (c - begin) >> 1;
      if (HALVES) {                            // (the same for the lane's 8 coordinates: an axis' half is a multiple of 8)
        upper = f >= half[e];
        if (upper) f -= half[e];
        partner = upper ? lane - half[e] / 8 : lane + half[e] / 8;
      }
      entry[e] = p.base[a] + f;
    }
  }
  const bool all_turned = p.rot_dim == 8 * L;

  const int sides = (p.side[0].heads > 0) + (p.side[1].heads > 0);
  const int per_token = MODE == HEAD ? p.side[0].chunks + p.side[1].chunks : sides;
  const unsigned unit = MODE == HEAD ? blockIdx.x * WARPS + warp : blockIdx.x;
  const unsigned units = MODE == HEAD ? gridDim.x * WARPS : gridDim.x;
  const int step_token = (int)(units / per_token), step_r = (int)(units % per_token);
  struct Place {
    int token, r;
  };
  auto next = [&](Place a) {
    a.token += step_token;
    a.r += step_r;
    if (a.r >= per_token) {
      a.r -= per_token;
      ++a.token;
    }
    return a;
  };
  auto side_of = [&](const Place& a) { return MODE == HEAD ? (int)(a.r >= p.side[0].chunks) : (sides == 2 ? a.r : (int)(p.side[0].heads == 0)); };
  // rows of this lane that exist: row i is head first + i * per_iter
  auto first_head = [&](const Place& a, int s) { return (MODE == HEAD ? a.r - (s ? p.side[0].chunks : 0) : warp) * ITERS * per_iter + lane / L; };
  auto load_rows = [&](const Place& a, Raw<In> (&raw)[ITERS]) {
    if (a.token >= p.tokens) return;
    const int s = side_of(a);
    const Side& sd = p.side[s];
    const int h0 = first_head(a, s);
    const In* src = reinterpret_cast<const In*>(sd.X) + a.token * sd.ld_token + h0 * sd.ld_head + c0;
    const long long step = per_iter * sd.ld_head;
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
      if (h0 + i * per_iter < sd.heads) raw[i].load(src);
      src += step;
    }
  };
  auto load_pos = [&](const Place& a, int (&pos)[NP]) {
    if (p.rot_dim == 0 || a.token >= p.tokens) return;
    const int* row = p.pos + a.token * p.ldpos;
#pragma unroll
    for (int e = 0; e < NP; ++e) pos[e] = (HALVES && e) ? pos[0] : __ldg(row + axis[e]);
  };
  auto load_table = [&](const int (&pos)[NP], float2 (&t)[NP]) {
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      t[e] = top[e] < 0 ? make_float2(1.f, 0.f)                                          // not turned
                        : make_float2(__int_as_float(0x7FFFFFFF), __int_as_float(0x7FFFFFFF));   // a position outside the table shows as NaN
      if (pos[e] >= 0 && pos[e] < top[e]) t[e] = __ldg(p.table + entry[e] + pos[e] * half[e]);
    }
  };

  if (MODE == ROW) {
    if (threadIdx.x < 2 * ROW_WARPS) red[threadIdx.x / ROW_WARPS][threadIdx.x % ROW_WARPS] = 0.f;
    __syncthreads();
  }
  // A CTA of a row norm stays on one side (the grid is even where there are two), and a warp on its heads: their weights
  // are loaded once.
  uint4 row_weights[MODE == HEAD ? 1 : ITERS];
  if (MODE != HEAD) {
    const Place first{0, (int)(unit % per_token)};
    const int s = side_of(first), h0 = first_head(first, s);
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
      row_weights[MODE == HEAD ? 0 : i] = make_uint4(0u, 0u, 0u, 0u);
      if (p.side[s].w && h0 + i * per_iter < p.side[s].heads)
        row_weights[MODE == HEAD ? 0 : i] = __ldg(reinterpret_cast<const uint4*>(p.side[s].w + (long long)(h0 + i * per_iter) * p.head_dim + c0));
    }
  }
  Place here{(int)(unit / per_token), (int)(unit % per_token)}, there = next(here);
  Raw<In> raw[ITERS], raw_next[ITERS];
  float2 turn[NP], turn_next[NP];
  int pos[NP];
#pragma unroll
  for (int e = 0; e < NP; ++e) pos[e] = 0;
  load_rows(here, raw);
  load_pos(here, pos);
  load_table(pos, turn);
  load_pos(there, pos);
  for (int n = 0; here.token < p.tokens; ++n) {
    load_rows(there, raw_next);
    load_table(pos, turn_next);
    const Place after = next(there);
    load_pos(after, pos);

    const int s = side_of(here);
    const Side& sd = p.side[s];
    const int heads = sd.heads, head0 = first_head(here, s);
    const __nv_bfloat16* const weights = sd.w;
    // y = x * A + partner * B
    float2 A[4], Bc[4];
    {
      float c[8], d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c[e] = turn[HALVES ? e : e / 2].x;
        d[e] = HALVES ? (upper ? turn[HALVES ? e : 0].y : -turn[HALVES ? e : 0].y) : ((e & 1) ? turn[e / 2].y : -turn[e / 2].y);
      }
      if (MODE == HEAD && weights) {
        float w[8], wp[8];
        unpack8(__ldg(reinterpret_cast<const uint4*>(weights + c0)), w);
        if (HALVES) unpack8(__ldg(reinterpret_cast<const uint4*>(weights + 8 * (partner & (L - 1)))), wp);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c[e] *= w[e];
          d[e] *= HALVES ? wp[e] : w[e ^ 1];
        }
      }
      to_pairs<HALVES>(c, A);
      to_pairs<HALVES>(d, Bc);
    }
    float inv = 1.f;
    if (MODE != HEAD) {
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < ITERS; ++i) {
        if (head0 + i * per_iter >= heads) continue;
        float x[8];
        float2 v[4];
        raw[i].get(x);
        to_pairs<HALVES>(x, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = fma2(v[e], v[e], sum);
      }
      float all = sum.x + sum.y;
#pragma unroll
      for (int o = 16; o; o >>= 1) all += __shfl_xor_sync(~0u, all, o);
      if (lane == 0) red[n & 1][warp] = all;          // (two buffers: one barrier a token is enough)
      __syncthreads();
      float total;
      if (MODE == ROW) {                              // (places of warps that do not exist hold zero)
        const float4 a = *reinterpret_cast<const float4*>(&red[n & 1][0]), b = *reinterpret_cast<const float4*>(&red[n & 1][4]);
        total = ((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w));
      } else {
        total = lane < (int)(blockDim.x >> 5) ? red[n & 1][lane] : 0.f;
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
      }
      inv = rsqrtf(fmaf(total, sd.inv_count, p.eps));
    }
    Out* dst = reinterpret_cast<Out*>(sd.Y) + here.token * sd.ldy_token + head0 * sd.ldy_head + c0;
    const long long step = per_iter * sd.ldy_head;
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
      const bool have = head0 + i * per_iter < heads;      // lanes of another head may still need this lane's shuffles
      float x[8];
      float2 v[4], y[4];
      raw[i].get(x);                                 // (of a row that is not there: never stored, and its lanes meet only their own)
      to_pairs<HALVES>(x, v);
      if (MODE == HEAD && p.norm) {
        float2 sq = mul2(v[0], v[0]);
#pragma unroll
        for (int e = 1; e < 4; ++e) sq = fma2(v[e], v[e], sq);
        float sum = sq.x + sq.y;
        if (LANES) {
#pragma unroll
          for (int o = LANES >> 1; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        } else {
          for (int o = L >> 1; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        }
        inv = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
      }
      if (MODE != HEAD && weights) {
        float w[8];
        float2 wv[4];
        unpack8(row_weights[MODE == HEAD ? 0 : i], w);
        to_pairs<HALVES>(w, wv);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mul2(v[e], mul2(wv[e], make_float2(inv, inv)));
      } else if (MODE != HEAD || p.norm) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mul2(v[e], make_float2(inv, inv));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 other = HALVES ? make_float2(__shfl_sync(~0u, v[e].x, partner), __shfl_sync(~0u, v[e].y, partner)) : v[e ^ 2];
        y[e] = fma2(other, Bc[e], mul2(v[e], A[e]));
      }
      if (!all_turned) {                             // no part of a partner in what is not turned (an infinity stays one)
        float z[8], u[8], a[8];
        from_pairs<HALVES>(y, z);
        from_pairs<HALVES>(v, u);
        from_pairs<HALVES>(A, a);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (top[HALVES ? e : e / 2] < 0) z[e] = u[e] * a[e];
        to_pairs<HALVES>(z, y);
      }
      from_pairs<HALVES>(y, x);
      if (have) store8(dst, x);
      dst += step;
    }
    here = there;
    there = after;
#pragma unroll
    for (int i = 0; i < ITERS; ++i) raw[i] = raw_next[i];
#pragma unroll
    for (int e = 0; e < NP; ++e) turn[e] = turn_next[e];
  }
}

template <typename In, typename Out>
cudaError_t launch(const Params& p, int mode, bool halves, long long most_ctas, int threads, cudaStream_t st) {
  void (*kernel)(Params);
  if (mode == HEAD) {
    if (p.head_dim == 128) kernel = halves ? qk_norm_rope_kernel<In, Out, HEAD, true, 16> : qk_norm_rope_kernel<In, Out, HEAD, false, 16>;
    else kernel = halves ? qk_norm_rope_kernel<In, Out, HEAD, true, 0> : qk_norm_rope_kernel<In, Out, HEAD, false, 0>;
  } else if (mode == ROW) {
    kernel = halves ? qk_norm_rope_kernel<In, Out, ROW, true, 0> : qk_norm_rope_kernel<In, Out, ROW, false, 0>;
  } else {
    kernel = halves ? qk_norm_rope_kernel<In, Out, WIDE_ROW, true, 0> : qk_norm_rope_kernel<In, Out, WIDE_ROW, false, 0>;
  }
  // what fits beside each other is asked only where there are more CTAs than one an SM
  long long slots = 2;
  if (most_ctas > slots) {
    int dev = 0, sms = 0, per_sm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    slots = sms & ~1;
    if (e == cudaSuccess && most_ctas > slots) {
      e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, 0);
      slots = ((long long)sms * (per_sm < 1 ? 1 : per_sm)) & ~1ll;      // (even: a CTA of a row norm keeps its side)
    }
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(kernel, (int)(most_ctas < slots ? most_ctas : slots), threads, 0, st, p);
}

int ensure_table(const oq_rope* r) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  std::lock_guard<std::mutex> lock(r->mutex);
  if (r->d_table && r->device == dev) return OQ_OK;
  if (r->d_table) return fail(OQ_ERR_INVALID_ARG, "rope handle was first used on another device");
  FirstUse first;
  float2* d = nullptr;
  e = cudaMalloc(&d, r->table.size() * sizeof(float));
  if (e != cudaSuccess) return cuda_fail(e, "cudaMalloc(rope table)");
  e = upload(d, r->table.data(), r->table.size() * sizeof(float));
  if (e != cudaSuccess) {
    cudaFree(d);
    return cuda_fail(e, "cudaMemcpy(rope table)");
  }
  r->device = dev;
  r->d_table = d;
  return OQ_OK;
}

}  // namespace qk
}  // namespace oq

using namespace oq;

extern "C" {

int oq_make_rope(int n_axes, const int* axis_dims, const int* max_pos, double theta, int layout, oq_rope** out) {
  if (!out) return fail(OQ_ERR_INVALID_ARG, "oq_make_rope: out is NULL");
  *out = nullptr;
  if (!axis_dims || !max_pos) return fail(OQ_ERR_INVALID_ARG, "oq_make_rope: NULL axis_dims or max_pos");
  if (n_axes < 1 || n_axes > qk::MAX_AXES) return fail(OQ_ERR_UNSUPPORTED, "oq_make_rope: 1 to 4 axes");
  if (layout != OQ_ROPE_PAIRS && layout != OQ_ROPE_HALVES) return fail(OQ_ERR_INVALID_ARG, "oq_make_rope: unknown layout");
  if (!(theta > 0.0) || !std::isfinite(theta)) return fail(OQ_ERR_INVALID_ARG, "oq_make_rope: theta must be positive and finite");
  long long total = 0, dim = 0;
  for (int a = 0; a < n_axes; ++a) {
    const int d = axis_dims[a];
    if (d <= 0 || max_pos[a] <= 0) return fail(OQ_ERR_INVALID_ARG, "oq_make_rope: axis " + std::to_string(a) + ": dims and positions must be positive");
    if (d % (layout == OQ_ROPE_HALVES ? 16 : 2))
      return fail(OQ_ERR_UNSUPPORTED, "oq_make_rope: axis " + std::to_string(a) + ": dims must be even (halves layout: a multiple of 16)");
    dim += d;
    total += (long long)max_pos[a] * (d / 2);
  }
  if (dim > 256) return fail(OQ_ERR_UNSUPPORTED, "oq_make_rope: more than 256 coordinates");
  if (total > (1ll << 27)) return fail(OQ_ERR_UNSUPPORTED, "oq_make_rope: table above 1 GB");
  try {
    oq_rope* r = new oq_rope;
    try {
      r->n_axes = n_axes;
      r->dim = (int)dim;
      r->layout = layout;
      r->axis_dim.assign(axis_dims, axis_dims + n_axes);
      r->max_pos.assign(max_pos, max_pos + n_axes);
      r->table.resize((size_t)total * 2);
      size_t at = 0;
      for (int a = 0; a < n_axes; ++a) {
        const int half = axis_dims[a] / 2;
        r->base.push_back((int)(at / 2));
        std::vector<double> freq(half);
        for (int i = 0; i < half; ++i) freq[i] = pow(theta, -2.0 * i / axis_dims[a]);
        for (int q = 0; q < max_pos[a]; ++q)
          for (int i = 0; i < half; ++i) {
            const double angle = q * freq[i];
            r->table[at++] = (float)cos(angle);
            r->table[at++] = (float)sin(angle);
          }
      }
    } catch (...) {
      delete r;
      throw;
    }
    *out = r;
  } catch (const std::bad_alloc&) {
    return fail(OQ_ERR_NOMEM, "oq_make_rope: out of host memory");
  }
  return OQ_OK;
}

int oq_rope_dim(const oq_rope* rope) { return rope ? rope->dim : 0; }

void oq_rope_destroy(oq_rope* rope) {
  if (!rope) return;
  if (rope->d_table) cudaFree(rope->d_table);
  delete rope;
}

int oq_qk_norm_rope(const oq_qk_side* q, const oq_qk_side* k, int n_tokens, int head_dim, const oq_rope* rope, const int* pos,
                    int ldpos, int norm, float eps, int x_dtype, int y_dtype, void* stream) {
  if (n_tokens < 0) return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: n_tokens is negative");
  if (n_tokens >= 0x7FFFFFFF - (1 << 16)) return fail(OQ_ERR_UNSUPPORTED, "oq_qk_norm_rope: too many tokens for one launch");   // (the walk looks two strides ahead)
  if (!q && !k) return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: neither queries nor keys");
  if ((x_dtype != OQ_BF16 && x_dtype != OQ_F32) || (y_dtype != OQ_BF16 && y_dtype != OQ_F32))
    return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: unknown element type");
  if (norm != OQ_NORM_NONE && norm != OQ_NORM_HEAD && norm != OQ_NORM_ROW) return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: unknown norm");
  if (!(eps >= 0.f)) return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: eps must not be negative");
  if (head_dim != 32 && head_dim != 64 && head_dim != 128 && head_dim != 256)
    return fail(OQ_ERR_UNSUPPORTED, "oq_qk_norm_rope: head_dim must be 32, 64, 128 or 256");
  qk::Params p = {};
  if (rope) {
    if (rope->dim > head_dim) return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: the rotation has more coordinates than a head");
    if (n_tokens > 0 && !pos) return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: a rotation without positions");
    if (ldpos < rope->n_axes) return fail(OQ_ERR_INVALID_ARG, "oq_qk_norm_rope: ldpos is smaller than the number of axes");
  }
  const int per_chunk = qk::ITERS * 256 / head_dim;
  const oq_qk_side* in[2] = {q, k};
  const int xa = x_dtype == OQ_F32 ? 4 : 8, ya = y_dtype == OQ_F32 ? 4 : 8;       // elements of 16 bytes
  for (int s = 0; s < 2; ++s) {
    if (!in[s]) continue;
    const std::string who = std::string("oq_qk_norm_rope: ") + (s ? "keys: " : "queries: ");
    if (in[s]->n_heads <= 0) return fail(OQ_ERR_INVALID_ARG, who + "n_heads must be positive");
    if (norm == OQ_NORM_ROW && in[s]->n_heads > per_chunk * qk::MAX_ROW_WARPS) return fail(OQ_ERR_UNSUPPORTED, who + "a row above 32768 values");
    if (n_tokens == 0) continue;
    if (!in[s]->X || !in[s]->Y) return fail(OQ_ERR_INVALID_ARG, who + "NULL buffer");
    if (in[s]->w_bf16 && norm == OQ_NORM_NONE) return fail(OQ_ERR_INVALID_ARG, who + "weights without a norm");
    if (!aligned16(in[s]->X) || !aligned16(in[s]->Y) || !aligned16(in[s]->w_bf16) || in[s]->ld_token % xa || in[s]->ld_head % xa ||
        in[s]->ldy_token % ya || in[s]->ldy_head % ya)
      return fail(OQ_ERR_ALIGNMENT, who + "pointers must be 16-byte aligned and strides multiples of 16 bytes");
    // (rows of the output that lie over each other would overwrite each other; strides of one token or one head are not used)
    const bool tokens = n_tokens > 1, heads = in[s]->n_heads > 1;
    if ((tokens && in[s]->ldy_token < head_dim) || (heads && in[s]->ldy_head < head_dim))
      return fail(OQ_ERR_INVALID_ARG, who + "output strides must be at least head_dim");
    if (in[s]->Y == in[s]->X && (x_dtype != y_dtype || (tokens && in[s]->ldy_token != in[s]->ld_token) || (heads && in[s]->ldy_head != in[s]->ld_head)))
      return fail(OQ_ERR_INVALID_ARG, who + "Y is X with other strides or another type");
    qk::Side& d = p.side[s];
    d.X = in[s]->X;
    d.Y = in[s]->Y;
    d.w = reinterpret_cast<const __nv_bfloat16*>(in[s]->w_bf16);
    d.ld_token = in[s]->ld_token; d.ld_head = in[s]->ld_head;
    d.ldy_token = in[s]->ldy_token; d.ldy_head = in[s]->ldy_head;
    d.heads = in[s]->n_heads;
    d.inv_count = 1.f / ((float)d.heads * (float)head_dim);
    d.chunks = (d.heads + per_chunk - 1) / per_chunk;
  }
  if (n_tokens == 0) return OQ_OK;
  p.tokens = n_tokens;
  p.head_dim = head_dim;
  p.lanes_per_head = head_dim / 8;
  p.norm = norm;
  p.eps = eps;
  p.inv_dim = 1.f / (float)head_dim;      // (a power of two)
  bool halves = false;
  if (rope) {
    const int rc = qk::ensure_table(rope);
    if (rc != OQ_OK) return rc;
    p.pos = pos;
    p.ldpos = ldpos;
    p.table = rope->d_table;
    p.n_axes = rope->n_axes;
    p.rot_dim = rope->dim;
    halves = rope->layout == OQ_ROPE_HALVES;
    int end = 0;
    for (int a = 0; a < rope->n_axes; ++a) {
      p.axis_end[a] = (end += rope->axis_dim[a]);
      p.max_pos[a] = rope->max_pos[a];
      p.base[a] = rope->base[a];
    }
  }
  // Rows of up to ROW_WARPS warps keep two sets of rows in registers; longer ones run with half the registers.
  int mode = qk::HEAD, threads = 32 * qk::WARPS;
  long long ctas = ((long long)n_tokens * (p.side[0].chunks + p.side[1].chunks) + qk::WARPS - 1) / qk::WARPS;
  if (norm == OQ_NORM_ROW) {
    const int chunks = p.side[0].chunks > p.side[1].chunks ? p.side[0].chunks : p.side[1].chunks;
    mode = chunks <= qk::ROW_WARPS ? qk::ROW : qk::WIDE_ROW;
    ctas = (long long)n_tokens * ((p.side[0].heads > 0) + (p.side[1].heads > 0));
    threads = 32 * chunks;
  }
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e =
      x_dtype == OQ_BF16 ? (y_dtype == OQ_BF16 ? qk::launch<__nv_bfloat16, __nv_bfloat16>(p, mode, halves, ctas, threads, st)
                                               : qk::launch<__nv_bfloat16, float>(p, mode, halves, ctas, threads, st))
                         : (y_dtype == OQ_BF16 ? qk::launch<float, __nv_bfloat16>(p, mode, halves, ctas, threads, st)
                                               : qk::launch<float, float>(p, mode, halves, ctas, threads, st));
  if (e != cudaSuccess) return cuda_fail(e, "oq_qk_norm_rope");
  return OQ_OK;
}

}  // extern "C"
