// Low-rank adapters of several requests beside a shared projection (whose quantized weights cannot take the update):
//
//   Y[t] = base[t] + scale_a B_a (A_a x[t]),   a = the adapter of the segment of tokens that t belongs to (none: base)
//
// Bound: memory.  base is read and Y written once (4 or 8 bytes an element) and X read once; the two products are
// 2 r (d + m) operations a token, far below what the tensor cores do in that time.  Two kernels:
//
//   shrink   u = A x by tcgen05 for tiles of 128 tokens of one segment.  The k-blocks (64 columns of d) of all tiles, one after the
//            other, are one line of steps and every SM takes an equal stretch of it; a stretch leaves its sum of a tile, fp32,
//            in the workspace (a few per cent of the traffic)
//   expand   Y = base + u B^T, the column tiles of all token tiles again one line in equal stretches.  At a token tile's
//            start the parts of u are added in the order of the stretches (bit-reproducible), scaled and cut into pieces of bf16
//            as an MMA operand: 2 pieces (16 bits) for bf16 outputs, 3 (24 bits) for fp32, each a product of its own, so that
//            the update is as exact as the output's type can show (from 64 bits: bf16 1.66e-3, the output's own rounding; fp32 6e-8 to 1e-7).  base tiles come by TMA, are added to in shared memory and
//            leave by TMA
//
// (One kernel for both, a cluster of CTAs per token tile that exchanges u through distributed shared memory, needs no
// workspace, but clusters fill whole groups of SMs only: 38 tiles took 64 to 77 us where equal stretches take half.)
//
// Segments of a few tokens (serving one token each) run in a third kernel on the ordinary cores, see few_tokens.
//
// Measured (B200): 32760 tokens, 5120 -> 15360, rank 64, bf16: 427 us for 2.35 GB = 5.5 TB/s, 0.85 of the copy rate (shrink 62 us,
// expand 361); 4608 tokens, 3072 -> 9216, rank 32: 47 us where 200 MB take 31 (the two launches and their first loads are 10 of
// it); eight single tokens, 3072 -> 18432, rank 16, fp32: 7.2 us.
#include <cuda_bf16.h>

#include <string>

#include "oq_internal.h"
#include "oq_sm100.cuh"

namespace oq {
namespace adapter {

constexpr int BM = 128, KB = 64;           // tokens of a tile, columns of d in a shrink step
constexpr uint32_t ATOM = BM * 128;        // 128 rows of 128 bytes
constexpr int EPI = 8;                     // epilogue warps of the expand kernel: two groups that take turns at column tiles
constexpr int EXPAND_THREADS = (EPI + 2) * 32, SHRINK_THREADS = 6 * 32;
constexpr int FEW = 8;                     // tokens the few-token kernel holds at a time
constexpr int FEW_THREADS = 256, FEW_RANKS = 8;      // and its cluster
enum { W_FULL = 60, W_FREE = 61, W_U = 62, W_UFREE = 63, W_ACC = 64, W_ACCFREE = 65 };

struct Params {
  const __nv_bfloat16 *X, *A, *B;
  const void* base;
  long long ldx, ldb;
  const float* scale;
  const int *seg_start, *seg_adapter;
  int n_segs, n_tokens, n_adapters, rank, rank16, d, m;
  void* Y;
  long long ldy;
  int copy;                                // Y is not base: rows without an adapter are copied
  float* part;                             // [tiles][parts][128][rank16]
  int max_tiles;                           // places for tiles: as many as segments that share no token can make
  int parts;                               // places for them, the most stretches a tile can meet
  int ctas;                                // stretches of the shrink line, at most
  int chunk;                               // k-blocks added up in tensor memory at a time
  int* status;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 load_remote(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tma_store_2d(const void* map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
               ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// What a piece leaves of a value; an infinite piece leaves nothing (inf - inf is NaN).
__device__ __forceinline__ float rest_of(float w, uint32_t piece) {
  const float rest = w - __uint_as_float(piece);
  return fabsf(rest) < INFINITY ? rest : 0.f;
}

// Up to SIZE tokens of one segment.  Tiles are counted segment by segment.
struct Tile {
  int tok0, rows, id;                      // id: the adapter, or -1
};
// By a whole warp: tile `want`; rows = 0 and tok0 = the number of tiles when there are no more than `want`.
template <int SIZE>
__device__ __forceinline__ Tile find_tile(const Params& p, int want) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int s0 = 0; s0 < p.n_segs; s0 += 32) {
    const int s = s0 + lane;
    int b = 0, n = 0, id = -1;
    if (s < p.n_segs) {
      b = min(max(__ldg(p.seg_start + s), 0), p.n_tokens);
      n = min(max(__ldg(p.seg_start + s + 1), b), p.n_tokens) - b;
      id = __ldg(p.seg_adapter + s);
      if (id < 0 || id >= p.n_adapters) id = -1;
    }
    const int tiles = (n + SIZE - 1) / SIZE;
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(~0u, sum, d);
      if (lane >= d) sum += o;
    }
    const int at = want - (before + sum - tiles);
    const uint32_t mine = __ballot_sync(~0u, at >= 0 && at < tiles);
    if (mine) {
      const int l = __ffs(mine) - 1;
      Tile t;
      t.tok0 = __shfl_sync(~0u, b + at * SIZE, l);
      t.rows = __shfl_sync(~0u, min(SIZE, n - at * SIZE), l);
      t.id = __shfl_sync(~0u, id, l);
      return t;
    }
    before = min(before + __shfl_sync(~0u, sum, 31), 1 << 30);     // (more than any call has, even of a table that is not ascending)
  }
  return Tile{before, 0, -1};
}
// Tiles that the two kernels work on.  A table that is not ascending names tokens more than once and makes more tiles than the
// workspace has places for: those are left out.
__device__ __forceinline__ int count_tiles(const Params& p) { return min(find_tile<BM>(p, 0x7FFFFFFF).tok0, p.max_tiles); }
// Steps of a stretch of the shrink line: an equal share, but so many that the kbs steps of a tile never meet more than
// p.parts stretches, however few tiles the segments turn out to make: ceil((kbs - 1) / len) + 1 <= parts.
__device__ __forceinline__ long long shrink_stretch(const Params& p, long long total, int kbs) {
  return max((total + p.ctas - 1) / p.ctas, (long long)(p.parts > 1 ? (kbs + p.parts - 2) / (p.parts - 1) : 1));
}

// Up to FEW rows of a segment: a 128-row MMA would multiply padding, and what bounds this case is reading the weights once.
// CTA k of the cluster takes columns d0 .. d1 - 1 of the first product (a warp for each rank, lanes along d) and
// columns m0 .. m1 - 1 of the second (a thread for each column); the shares of u meet in distributed shared memory.
template <bool F32, int ROWS>
__device__ __forceinline__ void few_rows(const Params& p, unsigned char* smem, int tok0, int rows, int id, int d0, int d1, int m0, int m1) {
  float* const part = reinterpret_cast<float*>(smem);            // [FEW][128] this CTA's share of A x
  float* const u = part + FEW * 128;                             // [FEW][128] scale * A x
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  const __nv_bfloat16* const Bw = p.B + (long long)(id >= 0 ? id : 0) * p.m * p.rank;
  if (id >= 0) {
    // the second product's weights travel to L2 while the first one runs
    for (long long i = (long long)m0 * p.rank * 2 + 128 * threadIdx.x; i < (long long)m1 * p.rank * 2; i += 128 * FEW_THREADS)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char*>(Bw) + i));
    const __nv_bfloat16* const A = p.A + (long long)id * p.rank * p.d;
    for (int r = warp; r < p.rank; r += FEW_THREADS / 32) {
      float sum[ROWS];
#pragma unroll
      for (int t = 0; t < ROWS; ++t) sum[t] = 0.f;
#pragma unroll 2
      for (int k = d0 + 8 * lane; k < d1; k += 256) {            // (d is a multiple of 8)
        float w[8];
        unpack8(__ldg(reinterpret_cast<const uint4*>(A + (long long)r * p.d + k)), w);
#pragma unroll
        for (int t = 0; t < ROWS; ++t)
          if (t < rows) {
            float x[8];
            unpack8(__ldg(reinterpret_cast<const uint4*>(p.X + (long long)(tok0 + t) * p.ldx + k)), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[t] = fmaf(w[e], x[e], sum[t]);
          }
      }
#pragma unroll
      for (int t = 0; t < ROWS; ++t)
        if (t < rows) {
#pragma unroll
          for (int o = 16; o; o >>= 1) sum[t] += __shfl_xor_sync(~0u, sum[t], o);
          if (lane == 0) part[t * 128 + r] = sum[t];
        }
    }
    cluster_sync();
    const float sc = __ldg(p.scale + id);
    for (int i = (int)threadIdx.x; i < rows * (p.rank / 4); i += FEW_THREADS) {
      const int t = i / (p.rank / 4), r = 4 * (i % (p.rank / 4));
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float4 o[FEW_RANKS];
#pragma unroll
      for (uint32_t k = 0; k < FEW_RANKS; ++k) o[k] = load_remote(map_rank(smem_u32(part + t * 128 + r), k));
#pragma unroll
      for (uint32_t k = 0; k < FEW_RANKS; ++k) {
        v.x += o[k].x; v.y += o[k].y; v.z += o[k].z; v.w += o[k].w;
      }
      *reinterpret_cast<float4*>(u + t * 128 + r) = make_float4(v.x * sc, v.y * sc, v.z * sc, v.w * sc);
    }
    cluster_sync();                                              // (nobody leaves while its share is being read)
  }
  constexpr int COLS = ROWS == 1 ? 4 : 1;                        // columns a thread has in flight
#pragma unroll COLS
  for (int col = m0 + (int)threadIdx.x; col < m1; col += FEW_THREADS) {
    float y[ROWS];
#pragma unroll
    for (int t = 0; t < ROWS; ++t) {
      y[t] = 0.f;
      if (t < rows) {
        const long long at = (long long)(tok0 + t) * p.ldb + col;
        y[t] = F32 ? reinterpret_cast<const float*>(p.base)[at] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.base)[at]);
      }
    }
    if (id >= 0) {
      float add[ROWS];
#pragma unroll
      for (int t = 0; t < ROWS; ++t) add[t] = 0.f;
#pragma unroll 2
      for (int r = 0; r < p.rank; r += 8) {
        float w[8];
        unpack8(__ldg(reinterpret_cast<const uint4*>(Bw + (long long)col * p.rank + r)), w);
#pragma unroll
        for (int t = 0; t < ROWS; ++t)
          if (t < rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) add[t] = fmaf(w[e], u[t * 128 + r + e], add[t]);
          }
      }
#pragma unroll
      for (int t = 0; t < ROWS; ++t) y[t] += add[t];
    }
#pragma unroll
    for (int t = 0; t < ROWS; ++t)
      if (t < rows) {
        const long long at = (long long)(tok0 + t) * p.ldy + col;
        if (F32) reinterpret_cast<float*>(p.Y)[at] = y[t];
        else reinterpret_cast<__nv_bfloat16*>(p.Y)[at] = __float2bfloat16_rn(y[t]);
      }
  }
}

template <bool F32>
__global__ void __launch_bounds__(FEW_THREADS) few_kernel(const __grid_constant__ Params p) {
  __shared__ __align__(16) unsigned char smem[2 * FEW * 128 * 4];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t rank = cluster_rank();
  const Tile t = find_tile<FEW>(p, (int)blockIdx.x / FEW_RANKS);   // (the same in every CTA of the cluster)
  if (t.rows == 0 || (t.id < 0 && !p.copy)) return;
  const int kb = (p.d + 63) / 64, nb = (p.m + 63) / 64;
  const int d0 = 64 * (kb * (int)rank / FEW_RANKS), d1 = min(64 * (kb * ((int)rank + 1) / FEW_RANKS), p.d);
  const int m0 = 64 * (nb * (int)rank / FEW_RANKS), m1 = min(64 * (nb * ((int)rank + 1) / FEW_RANKS), p.m);
  if (t.rows == 1) few_rows<F32, 1>(p, smem, t.tok0, 1, t.id, d0, d1, m0, m1);
  else few_rows<F32, FEW>(p, smem, t.tok0, t.rows, t.id, d0, d1, m0, m1);
}

// ------------------------------------------------- shrink -------------------------------------------------
template <int RB>
struct Shrink {
  static constexpr uint32_t STAGE = ATOM + RB * 8192;           // 128 tokens and up to 64 RB ranks, 64 columns of d each
  static constexpr int STAGES = RB == 1 ? 9 : 6;
  static constexpr uint32_t SMEM = 1024 + STAGES * STAGE;
};
template <int RB>
__global__ void __launch_bounds__(SHRINK_THREADS, 1) shrink_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a,
                                                                   const __grid_constant__ Params p) {
  using S = Shrink<RB>;
  constexpr int STAGES = S::STAGES, LOAD_WARP = 4, MMA_WARP = 5;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[2 * STAGES + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u, b0 = smem_u32(bars);
  auto full = [&](uint32_t s) { return b0 + 8u * s; };
  auto freed = [&](uint32_t s) { return b0 + 8u * (STAGES + s); };
  auto u_full = [&](uint32_t a) { return b0 + 8u * (2 * STAGES + a); };
  auto u_free = [&](uint32_t a) { return b0 + 8u * (2 * STAGES + 2 + a); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full(s), 1);
      mbar_init(freed(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(u_full(a), 1);
      mbar_init(u_free(a), 4);
    }
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(256) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // (the second kernel may start once every CTA of this one has passed its wait: what was written before this kernel is then
  // complete, and the second kernel reads its base tiles without waiting for this kernel's end: on SMs whose CTA of this one
  // is done, as the two do not fit beside each other, 217 and 225 KB of shared memory)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int kbs = (p.d + KB - 1) / KB;
  const long long total = (long long)count_tiles(p) * kbs;
  const long long len = shrink_stretch(p, total, kbs);
  const int c = (int)blockIdx.x;
  long long pos = c * len;
  const long long end = min(pos + len, total);
  // runs: the k-blocks k .. k + count - 1 of one token tile, at most p.chunk; first: of the tile in this stretch
  Tile t;
  int tile = 0, k = 0, count = 0;
  bool first = true;
  auto next_run = [&]() {
    while (pos < end) {
      tile = (int)(pos / kbs);
      k = (int)(pos % kbs);
      count = min((int)min((long long)(kbs - k), end - pos), p.chunk);
      first = k == 0 || pos == c * len;
      pos += count;
      t = find_tile<BM>(p, tile);
      if (t.id >= 0) return true;
    }
    return false;
  };
  uint32_t st = 0, ph = 0, runs = 0;
  auto advance = [&]() {
    if (++st == (uint32_t)STAGES) {
      st = 0;
      ph ^= 1u;
    }
  };
  if (warp == LOAD_WARP) {
    while (next_run()) {
      if (lane == 0)
        for (int i = 0; i < count && !abort_flag; ++i) {
          mbar_spin(freed(st), ph ^ 1u, &abort_flag, p.status, W_FREE);
          const uint32_t at = smem + st * S::STAGE;
          mbar_expect_tx(full(st), ATOM + (uint32_t)p.rank16 * 128u);
          tma_load_2d(at, &map_x, (k + i) * KB, t.tok0, full(st));
          tma_load_3d(at + ATOM, &map_a, (k + i) * KB, 0, t.id, full(st));
          advance();
        }
      __syncwarp();
    }
    // copies still in flight end before the CTA does (after an abort nobody else waits for them)
    if (lane == 0 && abort_flag)
      for (uint32_t s = 0; s < (uint32_t)STAGES; ++s)
        for (int i = 0; i < (1 << 16) && !mbar_try(full(s), (s < st ? ph : ph ^ 1u)); ++i) {}
  } else if (warp == MMA_WARP) {
    const uint32_t leader = elect_leader();
    const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BM >> 4) << 24) | ((uint32_t)(p.rank16 >> 3) << 17);
    for (; next_run(); ++runs) {
      const uint32_t a = runs & 1u;
      if (runs >= 2) mbar_spin(u_free(a), ((runs >> 1) - 1u) & 1u, &abort_flag, p.status, W_UFREE);
      for (int i = 0; i < count && !abort_flag; ++i) {
        mbar_spin(full(st), ph, &abort_flag, p.status, W_FULL);
        tc_fence_after();
        const uint64_t da = smem_desc(smem + st * S::STAGE), db = smem_desc(smem + st * S::STAGE + ATOM);
#pragma unroll
        for (uint32_t q = 0; q < KB / 16; ++q) mma_ss(tmem + 128u * a, da + 2 * q, db + 2 * q, idesc, i > 0 || q > 0, leader);
        mma_commit(freed(st), leader);
        advance();
      }
      mma_commit(u_full(a), leader);
    }
  } else {
    float sum[64 * RB];                                          // of the tile's runs so far
    for (; next_run(); ++runs) {
      const uint32_t a = runs & 1u;
      mbar_spin(u_full(a), (runs >> 1) & 1u, &abort_flag, p.status, W_U);
      __syncwarp();
      tc_fence_after();
      const int row = warp * 32 + lane, place = c - (int)((long long)tile * kbs / len);
      float4* const dst = reinterpret_cast<float4*>(p.part + (((long long)tile * p.parts + place) * BM + row) * p.rank16);
      const bool last = k + count == kbs || pos == end;          // of the tile in this stretch
#pragma unroll
      for (int q = 0; q < 4 * RB; ++q)
        if (16 * q < p.rank16) {
          uint32_t r[16];
          tmem_load16_at(tmem + ((uint32_t)(warp * 32) << 16) + 128u * a + 16u * (uint32_t)q, r);
          tmem_use16(r);
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[16 * q + i] = first ? __uint_as_float(r[i]) : sum[16 * q + i] + __uint_as_float(r[i]);
          if (last && row < t.rows)
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[4 * q + i] = make_float4(sum[16 * q + 4 * i], sum[16 * q + 4 * i + 1], sum[16 * q + 4 * i + 2], sum[16 * q + 4 * i + 3]);
        }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(u_free(a));
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(256) : "memory");
}

// ------------------------------------------------- expand -------------------------------------------------
template <bool F32, int RB>
struct Expand {
  static constexpr int BN = F32 ? 32 : 64;                       // columns of a tile: 128 bytes
  static constexpr int PIECES = F32 ? 3 : 2;
  static constexpr uint32_t U_BYTES = PIECES * RB * ATOM;
  static constexpr uint32_t B_ATOM = BN * 128, STAGE = ATOM + RB * B_ATOM;      // a base tile and the rows of B for its columns
  static constexpr int STAGES = (int)((226 * 1024 - U_BYTES) / STAGE) < 8 ? (int)((226 * 1024 - U_BYTES) / STAGE) : 8;
  static constexpr uint32_t SMEM = 1024 + U_BYTES + STAGES * STAGE;
};
template <bool F32, int RB>
__global__ void __launch_bounds__(EXPAND_THREADS, 1) expand_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_base,
                                                                   const __grid_constant__ CUtensorMap map_y, const __grid_constant__ Params p) {
  using S = Expand<F32, RB>;
  constexpr int STAGES = S::STAGES, BN = S::BN, LOAD_WARP = EPI, MMA_WARP = EPI + 1;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[2 * STAGES + 5];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned char* const smem_p = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  const uint32_t smem_u = smem_u32(smem_p), smem_st = smem_u + S::U_BYTES, b0 = smem_u32(bars);
  auto full = [&](uint32_t s) { return b0 + 8u * s; };
  auto freed = [&](uint32_t s) { return b0 + 8u * (STAGES + s); };
  auto acc_full = [&](uint32_t a) { return b0 + 8u * (2 * STAGES + a); };
  auto acc_free = [&](uint32_t a) { return b0 + 8u * (2 * STAGES + 2 + a); };
  const uint32_t u_ready = b0 + 8u * (2 * STAGES + 4);
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full(s), 1);
      mbar_init(freed(s), 1 + 4);           // the mma warp's commit, and the four warps whose tile it is
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full(a), 1);
      mbar_init(acc_free(a), 4);
    }
    mbar_init(u_ready, EPI);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(128) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int nbs = (p.m + BN - 1) / BN, kbs = (p.d + KB - 1) / KB, steps = p.rank16 / 16;
  const int tiles = count_tiles(p);
  const long long total = (long long)tiles * nbs, len = shrink_stretch(p, (long long)tiles * kbs, kbs);
  long long pos = total * blockIdx.x / gridDim.x;
  const long long end = total * (blockIdx.x + 1) / gridDim.x;
  // runs: the column tiles k .. k + count - 1 of one token tile
  Tile t;
  int tile = 0, k = 0, count = 0;
  auto next_run = [&]() {
    while (pos < end) {
      tile = (int)(pos / nbs);
      k = (int)(pos % nbs);
      count = (int)min((long long)(nbs - k), end - pos);
      pos += count;
      t = find_tile<BM>(p, tile);
      if (t.id >= 0 || p.copy) return true;
    }
    return false;
  };
  uint32_t st = 0, ph = 0, i = 0, updates = 0;                   // stage ring; column tiles so far; runs with an adapter so far
  auto advance = [&]() {
    ++i;
    if (++st == (uint32_t)STAGES) {
      st = 0;
      ph ^= 1u;
    }
  };
  if (warp == LOAD_WARP) {
    while (next_run()) {
      if (lane == 0)
        for (int q = 0; q < count && !abort_flag; ++q) {
          mbar_spin(freed(st), ph ^ 1u, &abort_flag, p.status, W_FREE);
          const uint32_t at = smem_st + st * S::STAGE;
          mbar_expect_tx(full(st), ATOM + (t.id >= 0 ? RB * S::B_ATOM : 0u));
          tma_load_2d(at, &map_base, (k + q) * BN, t.tok0, full(st));
          if (t.id >= 0)
            for (uint32_t r = 0; r < RB; ++r) tma_load_3d(at + ATOM + r * S::B_ATOM, &map_b, 64 * (int)r, (k + q) * BN, t.id, full(st));
          advance();
        }
      __syncwarp();
    }
    if (lane == 0 && abort_flag)
      for (uint32_t s = 0; s < (uint32_t)STAGES; ++s)
        for (int q = 0; q < (1 << 16) && !mbar_try(full(s), (s < st ? ph : ph ^ 1u)); ++q) {}
  } else if (warp == MMA_WARP) {
    const uint32_t leader = elect_leader();
    constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BM >> 4) << 24) | ((uint32_t)(BN >> 3) << 17);
    while (next_run()) {
      if (t.id >= 0) mbar_spin(u_ready, updates++ & 1u, &abort_flag, p.status, W_U);
      for (int x = 0; x < count && !abort_flag; ++x) {
        const uint32_t a = i & 1u;
        mbar_spin(full(st), ph, &abort_flag, p.status, W_FULL);
        if (i >= 2) mbar_spin(acc_free(a), ((i >> 1) - 1u) & 1u, &abort_flag, p.status, W_ACCFREE);
        tc_fence_after();
        if (t.id >= 0) {
          const uint32_t bt = smem_st + st * S::STAGE + ATOM;
          for (int q = S::PIECES - 1; q >= 0; --q)                // (the small pieces first)
            for (int s = 0; s < steps; ++s) {
              const uint64_t da = smem_desc(smem_u + (uint32_t)(q * RB + (s >> 2)) * ATOM) + 2u * (uint32_t)(s & 3);
              const uint64_t db = smem_desc(bt + (uint32_t)(s >> 2) * S::B_ATOM) + 2u * (uint32_t)(s & 3);
              mma_ss(tmem + 64u * a, da, db, IDESC, q < S::PIECES - 1 || s > 0, leader);
            }
        }
        mma_commit(acc_full(a), leader);
        mma_commit(freed(st), leader);
        advance();
      }
    }
  } else {
    asm volatile("griddepcontrol.wait;" ::: "memory");           // u's parts are complete; and nothing of Y is written before
    const int group = warp >> 2, row = (warp & 3) * 32 + lane;
    uint32_t held = 0;                                           // the stage whose tile is still being stored, + 1
    while (next_run()) {                    // (the groups meet at barriers: no warp leaves early, not even when a wait has given up)
      if (t.id >= 0) {
        // u of this token tile as an MMA operand.  (All MMAs that read the last one are done: both groups have had their results.)
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const int parts = (int)(((long long)(tile + 1) * kbs - 1) / len - (long long)tile * kbs / len) + 1;
        const float sc = __ldg(p.scale + t.id);
        const int quads = p.rank16 / 4;
        for (int x0 = (int)threadIdx.x; x0 < BM * quads; x0 += 4 * 32 * EPI) {       // 4 values a thread, their parts requested together
          float4 u[4];
          const float4* src[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int x = x0 + e * 32 * EPI, r = x / quads;
            u[e] = make_float4(0.f, 0.f, 0.f, 0.f);
            src[e] = r < t.rows ? reinterpret_cast<const float4*>(p.part + ((long long)tile * p.parts * BM + r) * p.rank16 + 4 * (x % quads)) : nullptr;
          }
#pragma unroll 4
          for (int q = 0; q < parts; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (src[e]) {
                const float4 v = __ldcg(src[e] + (long long)q * BM * quads);
                u[e].x += v.x; u[e].y += v.y; u[e].z += v.z; u[e].w += v.w;
              }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int x = x0 + e * 32 * EPI, r = x / quads, col = 4 * (x % quads);
            if (r >= BM) break;
            // (the ranks that fill up the last 16 have no adapter, but 0 * inf in A x where X holds an infinity)
            float w[4] = {u[e].x * sc, u[e].y * sc, u[e].z * sc, u[e].w * sc};
            if (col >= p.rank) w[0] = w[1] = w[2] = w[3] = 0.f;
            unsigned char* dst = smem_p + (col >> 6) * (int)ATOM + r * 128 + ((((col & 63) >> 3) ^ (r & 7)) << 4) + (col & 4) * 2;
#pragma unroll
            for (int q = 0; q < S::PIECES; ++q) {
              const uint32_t lo = pack2(w[0], w[1]), hi = pack2(w[2], w[3]);
              *reinterpret_cast<uint2*>(dst + q * RB * (int)ATOM) = make_uint2(lo, hi);
              w[0] = rest_of(w[0], lo << 16);
              w[1] = rest_of(w[1], lo & 0xFFFF0000u);
              w[2] = rest_of(w[2], hi << 16);
              w[3] = rest_of(w[3], hi & 0xFFFF0000u);
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(u_ready);
      }
      for (int x = 0; x < count && !abort_flag; ++x) {
        if ((int)(i & 1u) != group) {                            // the other group's tile
          advance();
          continue;
        }
        const uint32_t a = i & 1u;
        mbar_spin(full(st), ph, &abort_flag, p.status, W_FULL);
        mbar_spin(acc_full(a), (i >> 1) & 1u, &abort_flag, p.status, W_ACC);
        __syncwarp();
        tc_fence_after();
        unsigned char* const box = smem_p + S::U_BYTES + st * S::STAGE;
        if (t.id >= 0) {
          uint32_t acc[BN];
#pragma unroll
          for (int q = 0; q < BN / 32; ++q) tmem_load32_nowait(tmem + ((uint32_t)((warp & 3) * 32) << 16) + 64u * a + 32u * q, acc + 32 * q);
#pragma unroll
          for (int q = 0; q < BN / 32; ++q) tmem_use32(acc + 32 * q);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(acc_free(a));
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            uint4* const at = reinterpret_cast<uint4*>(box + row * 128 + ((e ^ (row & 7)) << 4));
            const uint4 v = *at;
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (F32) w[q] = __float_as_uint(__uint_as_float(w[q]) + __uint_as_float(acc[(4 * e + q) % BN]));
              else w[q] = pack2(__uint_as_float(w[q] << 16) + __uint_as_float(acc[(8 * e + 2 * q) % BN]),
                                __uint_as_float(w[q] & 0xFFFF0000u) + __uint_as_float(acc[(8 * e + 2 * q + 1) % BN]));
            }
            *at = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else if (lane == 0) {
          mbar_arrive(acc_free(a));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        const int col = (k + x) * BN, r0 = (warp & 3) * 32;
        if (r0 + 32 <= t.rows) {
          if (lane == 0) {
            tma_store_2d(&map_y, col, t.tok0 + r0, smem_st + st * S::STAGE + (uint32_t)r0 * 128u);
            // the stage before this one has been read by its store
            asm volatile("cp.async.bulk.commit_group;\n cp.async.bulk.wait_group.read 1;" ::: "memory");
            if (held) mbar_arrive(freed(held - 1));
            held = st + 1;
          }
        } else {                                                 // the segment ends inside the warp's rows
          constexpr int EL = F32 ? 4 : 8;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int r = r0 + 4 * e + lane / 8, ch = lane % 8;
            const uint4 v = *reinterpret_cast<const uint4*>(box + r * 128 + ((ch ^ (r & 7)) << 4));
            if (r < t.rows && col + ch * EL < p.m)
              *reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(p.Y) + ((long long)(t.tok0 + r) * p.ldy + col + ch * EL) * (F32 ? 4 : 2)) = v;
          }
          __syncwarp();
          if (lane == 0) {
            if (held) {
              asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
              mbar_arrive(freed(held - 1));
              held = 0;
            }
            mbar_arrive(freed(st));
          }
        }
        advance();
      }
    }
    if (lane == 0) {
      asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      if (held) mbar_arrive(freed(held - 1));
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(128) : "memory");
}

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
  return sms;
}
// The few-token kernel's time grows with tokens and rank, that of the other two hardly does.  (8 segments of a 3072 x 9216 layer,
// bf16, rank 16: 1 token each 6.5 us against 19, 4 tokens 15 against 18, 8 tokens 20 against 18; rank 64: 1 token 16 against
// 23, 2 tokens 30 against 23.)  The segments' lengths are on the device, so the rule goes by their average; where one has nearly all tokens,
// each 8 of them have a cluster: 256 tokens in one of 64 places 28 us (in one cluster of 8 tokens after the other 281).
bool few_tokens(int n_tokens, int n_segs, int rank) { return (long long)n_tokens * rank <= 64ll * n_segs; }
int most_tiles(int n_tokens, int n_segs, int size) {
  const long long most = (n_tokens + size - 1) / size + (long long)n_segs;
  return (int)(most < n_tokens ? most : n_tokens);
}
// Stretches that a tile's k-blocks meet when the segments cover all tokens without gaps (shrink_stretch keeps the stretches
// long enough for this number in every other case).
int most_parts(int n_tokens, int kbs, int sms) {
  const long long total = (long long)((n_tokens + BM - 1) / BM) * kbs, len = (total + sms - 1) / sms;
  const long long parts = (kbs - 1 + len - 1) / len + 1;
  return (int)(parts < kbs ? parts : kbs);
}

template <bool F32>
cudaError_t launch_few(const Params& p, int tiles, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)tiles * FEW_RANKS);
  cfg.blockDim = dim3(FEW_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = FEW_RANKS;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, few_kernel<F32>, p);
}
template <bool F32, int RB>
cudaError_t launch(const Params& p, const CUtensorMap& mx, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mbase, const CUtensorMap& my,
                   int sms, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(shrink_kernel<RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shrink<RB>::SMEM);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(expand_kernel<F32, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Expand<F32, RB>::SMEM);
  if (e == cudaSuccess) e = launch_dependent(shrink_kernel<RB>, p.ctas, SHRINK_THREADS, Shrink<RB>::SMEM, st, mx, ma, p);
  if (e == cudaSuccess) e = launch_dependent(expand_kernel<F32, RB>, sms, EXPAND_THREADS, Expand<F32, RB>::SMEM, st, mb, mbase, my, p);
  return e;
}

}  // namespace adapter
}  // namespace oq

using namespace oq;

extern "C" {

int oq_adapter_workspace_bytes(int n_tokens, int n_segs, int dim, int rank, size_t* bytes) {
  if (!bytes) return fail(OQ_ERR_INVALID_ARG, "oq_adapter_workspace_bytes: bytes is NULL");
  *bytes = 0;
  if (n_tokens < 0 || n_segs < 0 || dim <= 0 || rank <= 0) return fail(OQ_ERR_INVALID_ARG, "oq_adapter_workspace_bytes: bad sizes");
  if (n_tokens == 0 || n_segs == 0 || adapter::few_tokens(n_tokens, n_segs, rank)) return OQ_OK;
  const int kbs = (dim + adapter::KB - 1) / adapter::KB;
  *bytes = (size_t)adapter::most_tiles(n_tokens, n_segs, adapter::BM) * adapter::most_parts(n_tokens, kbs, adapter::sm_count()) * adapter::BM *
           (size_t)((rank + 15) / 16 * 16) * sizeof(float);
  return OQ_OK;
}

int oq_adapter_add(const void* X_bf16, int n_tokens, int ldx, int dim, const void* A_bf16, const void* B_bf16, int n_adapters,
                              int rank, const float* scale, const int* seg_start, const int* seg_adapter, int n_segs, const void* base,
                              int ldb, void* Y, int ldy, int m, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (n_tokens < 0 || n_segs < 0) return fail(OQ_ERR_INVALID_ARG, "oq_adapter_add: negative count");
  if (dim <= 0 || m <= 0 || rank <= 0 || n_adapters <= 0) return fail(OQ_ERR_INVALID_ARG, "oq_adapter_add: sizes must be positive");
  if (dtype != OQ_BF16 && dtype != OQ_F32) return fail(OQ_ERR_INVALID_ARG, "oq_adapter_add: unknown dtype");
  if (rank % 8 || rank > 128) return fail(OQ_ERR_UNSUPPORTED, "oq_adapter_add: rank must be a multiple of 8, at most 128");
  if (dim % 8 || m % 8) return fail(OQ_ERR_UNSUPPORTED, "oq_adapter_add: dim and m must be multiples of 8");
  if (n_tokens > (1 << 24) || n_segs > (1 << 16)) return fail(OQ_ERR_UNSUPPORTED, "oq_adapter_add: more than 2^24 tokens or 2^16 segments");
  if (n_tokens == 0 || n_segs == 0) return OQ_OK;
  if (!X_bf16 || !A_bf16 || !B_bf16 || !scale || !seg_start || !seg_adapter || !base || !Y)
    return fail(OQ_ERR_INVALID_ARG, "oq_adapter_add: NULL buffer");
  if (ldx < dim || ldb < m || ldy < m) return fail(OQ_ERR_INVALID_ARG, "oq_adapter_add: leading dimension too small");
  const int el = dtype == OQ_F32 ? 4 : 8;
  if (ldx % 8 || ldb % el || ldy % el || !aligned16(X_bf16) || !aligned16(A_bf16) || !aligned16(B_bf16) || !aligned16(base) || !aligned16(Y))
    return fail(OQ_ERR_ALIGNMENT, "oq_adapter_add: pointers must be 16-byte aligned and leading dimensions multiples of 16 bytes");
  if (Y == base && ldy != ldb) return fail(OQ_ERR_INVALID_ARG, "oq_adapter_add: Y is base with another leading dimension");
  adapter::Params p = {};
  p.X = reinterpret_cast<const __nv_bfloat16*>(X_bf16);
  p.A = reinterpret_cast<const __nv_bfloat16*>(A_bf16);
  p.B = reinterpret_cast<const __nv_bfloat16*>(B_bf16);
  p.base = base;
  p.ldx = ldx;
  p.ldb = ldb;
  p.scale = scale;
  p.seg_start = seg_start;
  p.seg_adapter = seg_adapter;
  p.n_segs = n_segs; p.n_tokens = n_tokens; p.n_adapters = n_adapters;
  p.rank = rank;
  p.rank16 = (rank + 15) / 16 * 16;
  p.d = dim; p.m = m;
  p.Y = Y;
  p.ldy = ldy;
  p.copy = Y != base;
  p.status = device_status_word();
  if (!p.status) return fail(OQ_ERR_CUDA, "oq_adapter_add: cannot allocate the device status word");
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (adapter::few_tokens(n_tokens, n_segs, rank)) {
    const int tiles = adapter::most_tiles(n_tokens, n_segs, adapter::FEW);
    e = dtype == OQ_F32 ? adapter::launch_few<true>(p, tiles, st) : adapter::launch_few<false>(p, tiles, st);
    if (e != cudaSuccess) return cuda_fail(e, "oq_adapter_add");
    return OQ_OK;
  }
  size_t need = 0;
  const int rc = oq_adapter_workspace_bytes(n_tokens, n_segs, dim, rank, &need);
  if (rc != OQ_OK) return rc;
  if (need > workspace_bytes || !workspace || !aligned16(workspace))
    return fail(OQ_ERR_NOMEM, "oq_adapter_add: workspace of " + std::to_string(need) + " bytes (16-byte aligned) needed");
  const int sms = adapter::sm_count();
  p.part = reinterpret_cast<float*>(workspace);
  p.ctas = sms;
  p.max_tiles = adapter::most_tiles(n_tokens, n_segs, adapter::BM);
  // The tensor cores do not round their running sums to nearest, so an error of the sum's last bits grows with its length: for
  // fp32 outputs 256 columns are added up at a time (relative error of the result at d = 8192: 1.7e-6 without this).
  p.chunk = dtype == OQ_F32 ? 4 : 1 << 30;
  p.parts = adapter::most_parts(n_tokens, (dim + adapter::KB - 1) / adapter::KB, sms);
  CUtensorMap mx, ma, mb, mbase, my;
  const uint64_t size = dtype == OQ_F32 ? 4 : 2;
  {
    const uint64_t dims[2] = {(uint64_t)dim, (uint64_t)n_tokens}, strides[1] = {(uint64_t)ldx * 2};
    const uint32_t box[2] = {64, 128};
    e = encode_tensor_map_sw128(&mx, X_bf16, false, 2, dims, strides, box);
  }
  if (e == cudaSuccess) {
    const uint64_t dims[3] = {(uint64_t)dim, (uint64_t)rank, (uint64_t)n_adapters}, strides[2] = {(uint64_t)dim * 2, (uint64_t)dim * rank * 2};
    const uint32_t box[3] = {64, (uint32_t)p.rank16, 1};
    e = encode_tensor_map_sw128(&ma, A_bf16, false, 3, dims, strides, box);
  }
  if (e == cudaSuccess) {
    const uint64_t dims[3] = {(uint64_t)rank, (uint64_t)m, (uint64_t)n_adapters}, strides[2] = {(uint64_t)rank * 2, (uint64_t)m * rank * 2};
    const uint32_t box[3] = {64, dtype == OQ_F32 ? 32u : 64u, 1};
    e = encode_tensor_map_sw128(&mb, B_bf16, false, 3, dims, strides, box);
  }
  const uint64_t dims[2] = {(uint64_t)m, (uint64_t)n_tokens};
  if (e == cudaSuccess) {
    const uint64_t strides[1] = {(uint64_t)ldb * size};
    const uint32_t box[2] = {(uint32_t)(128 / size), 128};
    e = encode_tensor_map_sw128(&mbase, base, dtype == OQ_F32, 2, dims, strides, box);
  }
  if (e == cudaSuccess) {
    const uint64_t strides[1] = {(uint64_t)ldy * size};
    const uint32_t box[2] = {(uint32_t)(128 / size), 32};
    e = encode_tensor_map_sw128(&my, Y, dtype == OQ_F32, 2, dims, strides, box);
  }
  if (e != cudaSuccess) return cuda_fail(e, "oq_adapter_add (tensor map)");
  const bool wide = rank > 64;
  if (dtype == OQ_F32) e = wide ? adapter::launch<true, 2>(p, mx, ma, mb, mbase, my, sms, st) : adapter::launch<true, 1>(p, mx, ma, mb, mbase, my, sms, st);
  else e = wide ? adapter::launch<false, 2>(p, mx, ma, mb, mbase, my, sms, st) : adapter::launch<false, 1>(p, mx, ma, mb, mbase, my, sms, st);
  if (e != cudaSuccess) return cuda_fail(e, "oq_adapter_add");
  return OQ_OK;
}

}  // extern "C"
