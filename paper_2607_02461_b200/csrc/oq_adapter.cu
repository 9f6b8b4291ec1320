// Low-rank adapters of several requests beside a shared projection (whose quantized weights cannot take the update):
//
//   Y[t] = base[t] + scale_a B_a (A_a x[t]),   a = the adapter of the segment of tokens that t belongs to (none: base)
//
// Bound: memory.  base is read and Y written once (4 or 8 bytes an element) and X read once; the two products are
// 2 r (d + m) multiply-adds a token, far below what the tensor cores do in that time.  So everything travels by TMA
// and one kernel does both products: a cluster of up to 8 CTAs takes 128 tokens of one segment,
//
//   shrink   CTA k multiplies its share of the d columns:  U_k = X A^T  (tcgen05, fp32 in tensor memory);
//            the shares are added over the cluster's shared memory in CTA order (bit-reproducible), each CTA a part of
//            the rows, which it scales, cuts into bf16 pieces and hands to all CTAs of the cluster as an MMA operand
//   expand   CTA k multiplies its share of the m columns, 64 at a time: acc = U B^T, and adds the base's tile
//
// The cluster's size only divides the columns: no byte is read twice for it, and no workspace or second launch is
// needed.  U is cut into 2 pieces of bf16 for bf16 outputs (16 bits) and 3 for fp32 (24 bits), each a product of its own, so that
// the update is as exact as the output's type can show.
#include <cuda_bf16.h>

#include <string>

#include "oq_internal.h"
#include "oq_sm100.cuh"

namespace oq {
namespace adapter {

#ifndef OQ_AD
#define OQ_AD 592
#endif
constexpr int EPI = 8;                     // epilogue warps: two for each 32 rows, 32 columns of an expand tile each
constexpr int THREADS = (EPI + 2) * 32;
constexpr int LOAD_WARP = EPI, MMA_WARP = EPI + 1;
constexpr int FEW = 8;                     // rows up to which a tile runs on the ordinary cores
constexpr int BM = 128, KB = 64, BN = 64;  // tokens, columns of d in a shrink step, columns of m in an expand step
constexpr int TMEM_COLS = 256;             // U: 128 columns at most, two accumulators of 64
constexpr uint32_t COL_U = 0, COL_ACC = 128;
constexpr uint32_t ATOM = BM * 128;        // 128 rows of 128 bytes
enum { W_FULL = 60, W_FREE = 61, W_U = 62, W_ACC = 63, W_ACCFREE = 64 };

// RB: blocks of 64 ranks; a stage holds an X tile and an A tile while shrinking, a base tile and a B tile while expanding
template <bool F32, int RB>
struct Shape {
  static constexpr int PIECES = F32 ? 3 : 2;
  static constexpr uint32_t U_BYTES = PIECES * RB * ATOM;
  static constexpr uint32_t BASE = F32 ? 2 * ATOM : ATOM;
  static constexpr uint32_t WEIGHTS = RB * 64 * 128;                     // 64 x RB blocks (A), or RB atoms of 64 rows (B)
  static constexpr uint32_t STAGE = BASE + WEIGHTS;
  static constexpr int STAGES = F32 && RB == 2 ? 2 : 3;              // (what fits in 227 KB beside U)
  static constexpr uint32_t PART = BM * (RB * 64 * 4 + 16);              // one CTA's share of U, fp32; lies over the stages
  static constexpr uint32_t SMEM = 1024 + U_BYTES + (STAGES * STAGE > PART ? STAGES * STAGE : PART);
};

struct Params {
  const __nv_bfloat16 *X, *A, *B;          // (the tensor maps read them; these serve tiles of few rows)
  const void* base;
  long long ldx, ldb;
  const float* scale;
  const int *seg_start, *seg_adapter;
  int n_segs, n_tokens, n_adapters, rank, rank16, d, m;
  void* Y;
  long long ldy;
  int copy;                                // Y is not base: rows without an adapter are copied
  int* status;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
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
__device__ __forceinline__ void store_remote(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1,%2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y) : "memory");
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

// A tile of up to FEW rows: a 128-row MMA would multiply padding, and its pipeline of tiles would cost more time than reading
// the weights once, which is what bounds this case.  CTA k of the cluster takes columns d0 .. d1 - 1 of the first
// product (a warp for each rank, lanes along d) and columns m0 .. m1 - 1 of the second (a thread for each column).
template <bool F32>
__device__ __noinline__ void few_rows(const Params& p, unsigned char* smem, int tok0, int rows, int id, uint32_t rank, uint32_t ranks, int d0, int d1,
                                      int m0, int m1) {
  float* const part = reinterpret_cast<float*>(smem);            // [FEW][128] this CTA's share of A x
  float* const u = part + FEW * 128;                             // [FEW][128] scale * A x
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  if (id >= 0) {
    const __nv_bfloat16* const A = p.A + (long long)id * p.rank * p.d;
    for (int r = warp; r < p.rank; r += THREADS / 32) {
      float sum[FEW];
#pragma unroll
      for (int t = 0; t < FEW; ++t) sum[t] = 0.f;
#pragma unroll 2
      for (int k = d0 + 8 * lane; k < d1; k += 256) {            // (d is a multiple of 8)
        float w[8];
        unpack8(__ldg(reinterpret_cast<const uint4*>(A + (long long)r * p.d + k)), w);
#pragma unroll
        for (int t = 0; t < FEW; ++t)
          if (t < rows) {
            float x[8];
            unpack8(__ldg(reinterpret_cast<const uint4*>(p.X + (long long)(tok0 + t) * p.ldx + k)), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[t] = fmaf(w[e], x[e], sum[t]);
          }
      }
#pragma unroll
      for (int t = 0; t < FEW; ++t)
        if (t < rows) {
#pragma unroll
          for (int o = 16; o; o >>= 1) sum[t] += __shfl_xor_sync(~0u, sum[t], o);
          if (lane == 0) part[t * 128 + r] = sum[t];
        }
    }
    cluster_sync();
    const float sc = __ldg(p.scale + id);
    for (int i = (int)threadIdx.x; i < rows * (p.rank / 4); i += THREADS) {
      const int t = i / (p.rank / 4), r = 4 * (i % (p.rank / 4));
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (uint32_t k = 0; k < ranks; ++k) {
        const float4 o = load_remote(map_rank(smem_u32(part + t * 128 + r), k));
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
      }
      *reinterpret_cast<float4*>(u + t * 128 + r) = make_float4(v.x * sc, v.y * sc, v.z * sc, v.w * sc);
    }
    cluster_sync();                                              // (nobody leaves while its share is being read)
  }
  const __nv_bfloat16* const Bw = p.B + (long long)(id >= 0 ? id : 0) * p.m * p.rank;
#pragma unroll 2
  for (int col = m0 + (int)threadIdx.x; col < m1; col += THREADS) {
    float y[FEW];
#pragma unroll
    for (int t = 0; t < FEW; ++t) {
      y[t] = 0.f;
      if (t < rows) {
        const long long at = (long long)(tok0 + t) * p.ldb + col;
        y[t] = F32 ? reinterpret_cast<const float*>(p.base)[at] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.base)[at]);
      }
    }
    if (id >= 0) {
      float add[FEW];
#pragma unroll
      for (int t = 0; t < FEW; ++t) add[t] = 0.f;
#pragma unroll 2
      for (int r = 0; r < p.rank; r += 8) {
        float w[8];
        unpack8(__ldg(reinterpret_cast<const uint4*>(Bw + (long long)col * p.rank + r)), w);
#pragma unroll
        for (int t = 0; t < FEW; ++t)
          if (t < rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) add[t] = fmaf(w[e], u[t * 128 + r + e], add[t]);
          }
      }
#pragma unroll
      for (int t = 0; t < FEW; ++t) y[t] += add[t];
    }
#pragma unroll
    for (int t = 0; t < FEW; ++t)
      if (t < rows) {
        const long long at = (long long)(tok0 + t) * p.ldy + col;
        if (F32) reinterpret_cast<float*>(p.Y)[at] = y[t];
        else reinterpret_cast<__nv_bfloat16*>(p.Y)[at] = __float2bfloat16_rn(y[t]);
      }
  }
}

template <bool F32, int RB>
__global__ void __launch_bounds__(THREADS, F32 || RB == 2 ? 1 : 2) adapter_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a,
                                                          const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_base,
                                                          const __grid_constant__ Params p) {
  using S = Shape<F32, RB>;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 5];
  __shared__ int tile_info[3];              // first token, tokens, adapter
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned char* const smem_p = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  const uint32_t smem_u = smem_u32(smem_p), smem_st = smem_u + S::U_BYTES;
  const uint32_t b0 = smem_u32(bars);
  auto full = [&](int s) { return b0 + 8u * (uint32_t)s; };
  auto freed = [&](int s) { return b0 + 8u * (uint32_t)(S::STAGES + s); };
  const uint32_t u_full = b0 + 8u * (2 * S::STAGES);
  auto acc_full = [&](int a) { return b0 + 8u * (uint32_t)(2 * S::STAGES + 1 + a); };
  auto acc_free = [&](int a) { return b0 + 8u * (uint32_t)(2 * S::STAGES + 3 + a); };
  const uint32_t rank = cluster_rank(), ranks = cluster_size();

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::STAGES; ++s) {
      mbar_init(full(s), 1);
      mbar_init(freed(s), 1 + EPI);         // the mma warp's commit, and the epilogue warps (expanding only)
    }
    mbar_init(u_full, 1);
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full(a), 1);
      mbar_init(acc_free(a), EPI);
    }
    abort_flag = 0;
    tile_info[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  if (warp == 0) {
    // which 128 tokens: tiles are counted segment by segment
    const int want = (int)(blockIdx.x / ranks);
    int before = 0;
    for (int s0 = 0; s0 < p.n_segs && before <= want; s0 += 32) {
      const int s = s0 + lane;
      int b = 0, n = 0;
      if (s < p.n_segs) {
        b = min(max(__ldg(p.seg_start + s), 0), p.n_tokens);
        n = min(max(__ldg(p.seg_start + s + 1), b), p.n_tokens) - b;
      }
      const int tiles = (n + BM - 1) / BM;
      int sum = tiles;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, sum, d);
        if (lane >= d) sum += o;
      }
      const int at = want - (before + sum - tiles);
      if (at >= 0 && at < tiles) {
        tile_info[0] = b + at * BM;
        tile_info[1] = min(BM, n - at * BM);
        const int a = __ldg(p.seg_adapter + s);
        tile_info[2] = a >= 0 && a < p.n_adapters ? a : -1;
      }
      before += __shfl_sync(~0u, sum, 31);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int tok0 = tile_info[0], rows = tile_info[1], id = tile_info[2];
  const bool few = rows <= FEW;                                  // (all of these are the same in every CTA of the cluster)
  const bool update = rows > 0 && id >= 0 && !few;
  const int kb_all = (p.d + KB - 1) / KB, nb_all = (p.m + BN - 1) / BN;
  const int kb0 = (int)((long long)kb_all * rank / ranks), kb1 = (int)((long long)kb_all * (rank + 1) / ranks);
  const int nb0 = (int)((long long)nb_all * rank / ranks), nb1 = (int)((long long)nb_all * (rank + 1) / ranks);
  const int steps = p.rank16 / 16;
  const uint32_t leader = elect_leader();
  uint32_t st = 0, ph = 0;                                       // stage ring position of the load and mma threads
  auto advance = [&]() {
    if (++st == (uint32_t)S::STAGES) {
      st = 0;
      ph ^= 1u;
    }
  };

  // ------------------------------------------------- shrink -------------------------------------------------
  if (update) {
    if (warp == LOAD_WARP && lane == 0) {
      for (int k = kb0; k < kb1 && !abort_flag; ++k) {
        mbar_spin(freed(st), ph ^ 1u, &abort_flag, p.status, W_FREE);
        const uint32_t at = smem_st + st * S::STAGE;
        mbar_expect_tx(full(st), ATOM + (uint32_t)p.rank16 * 128u);
        tma_load_2d(at, &map_x, k * KB, tok0, full(st));
        tma_load_3d(at + S::BASE, &map_a, k * KB, 0, id, full(st));
        advance();
      }
    } else if (warp == MMA_WARP) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BM >> 4) << 24) | ((uint32_t)(p.rank16 >> 3) << 17);
      for (int k = kb0; k < kb1 && !abort_flag; ++k) {
        mbar_spin(full(st), ph, &abort_flag, p.status, W_FULL);
        tc_fence_after();
        const uint64_t a = smem_desc(smem_st + st * S::STAGE), b = smem_desc(smem_st + st * S::STAGE + S::BASE);
#pragma unroll
        for (uint32_t i = 0; i < KB / 16; ++i)
          mma_ss(tmem + COL_U, a + 2 * i, b + 2 * i, idesc, k > kb0 || i > 0, leader);
        mma_commit(freed(st), leader);
        if (lane < EPI) mbar_arrive(freed(st));      // no epilogue warp uses a stage while shrinking
        advance();
      }
      if (kb1 > kb0) mma_commit(u_full, leader);
    } else if (warp < 4) {                   // (one warp for each 32 rows is enough here)
      const int row = warp * 32 + lane;
      unsigned char* dst = smem_p + S::U_BYTES + (uint32_t)row * (uint32_t)(p.rank16 * 4 + 16);
      if (kb1 > kb0) {
        mbar_spin(u_full, 0, &abort_flag, p.status, W_U);
        __syncwarp();
        tc_fence_after();
      }
      // (every stage has been read: the MMAs that this barrier follows were the last to read one)
      for (int c = 0; c < p.rank16; c += 16) {
        uint32_t r[16];
        if (kb1 > kb0) {
          tmem_load16_nowait(tmem + ((uint32_t)(warp * 32) << 16) + COL_U + (uint32_t)c, r);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) r[i] = 0u;
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(dst + 4 * (c + i)) = make_uint4(r[i], r[i + 1], r[i + 2], r[i + 3]);
      }
    }
    __syncwarp();
    cluster_sync();
    if (warp < EPI) {
      const int part = (BM + (int)ranks - 1) / (int)ranks, r0 = (int)rank * part, quads = p.rank16 / 4;
      const float sc = __ldg(p.scale + id);
      for (int i = (int)threadIdx.x; i < part * quads; i += 32 * EPI) {
        const int row = r0 + i / quads, c = 4 * (i % quads);
        if (row >= BM) break;
        const uint32_t src = smem_st + (uint32_t)row * (uint32_t)(p.rank16 * 4 + 16) + 4u * (uint32_t)c;
        float4 u = load_remote(map_rank(src, 0));
        for (uint32_t k = 1; k < ranks; ++k) {
          const float4 v = load_remote(map_rank(src, k));
          u.x += v.x; u.y += v.y; u.z += v.z; u.w += v.w;
        }
        float x[4] = {u.x * sc, u.y * sc, u.z * sc, u.w * sc};
        const uint32_t dst = smem_u + (uint32_t)(c >> 6) * ATOM + (uint32_t)row * 128u + (uint32_t)((((c & 63) >> 3) ^ (row & 7)) << 4) + (uint32_t)(c & 4) * 2u;
#pragma unroll
        for (int q = 0; q < S::PIECES; ++q) {
          const uint32_t lo = pack2(x[0], x[1]), hi = pack2(x[2], x[3]);
          for (uint32_t k = 0; k < ranks; ++k) store_remote(map_rank(dst + (uint32_t)q * RB * ATOM, k), lo, hi);
          x[0] -= __uint_as_float(lo << 16);
          x[1] -= __uint_as_float(lo & 0xFFFF0000u);
          x[2] -= __uint_as_float(hi << 16);
          x[3] -= __uint_as_float(hi & 0xFFFF0000u);
        }
      }
      asm volatile("fence.proxy.async;" ::: "memory");
    }
    tc_fence_before();
    __syncwarp();
    cluster_sync();
    tc_fence_after();
    asm volatile("fence.proxy.async;" ::: "memory");
    if (warp < EPI) {                        // where the other roles' ring stands now
      st = (uint32_t)(kb1 - kb0) % S::STAGES;
      ph = ((uint32_t)(kb1 - kb0) / S::STAGES) & 1u;
    }
  }

  // ------------------------------------------------- expand -------------------------------------------------
  if (update || (rows > 0 && id < 0 && p.copy)) {
    if (warp == LOAD_WARP && lane == 0) {
      for (int n = nb0; n < nb1 && !abort_flag; ++n) {
        mbar_spin(freed(st), ph ^ 1u, &abort_flag, p.status, W_FREE);
        const uint32_t at = smem_st + st * S::STAGE;
        mbar_expect_tx(full(st), S::BASE + (update ? S::WEIGHTS : 0u));
        tma_load_2d(at, &map_base, n * BN, tok0, full(st));
        if (F32) tma_load_2d(at + ATOM, &map_base, n * BN + 32, tok0, full(st));
        if (update)
          for (int r = 0; r < RB; ++r) tma_load_3d(at + S::BASE + (uint32_t)r * 8192u, &map_b, 64 * r, n * BN, id, full(st));
        advance();
      }
      // copies still in flight end before the CTA does (after an abort nobody else waits for them)
      for (int s = 0; s < S::STAGES; ++s)
        for (int n = 0; abort_flag && n < (1 << 16); ++n) mbar_try(full(s), ph);
    } else if (warp == MMA_WARP) {
      constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BM >> 4) << 24) | ((uint32_t)(BN >> 3) << 17);
      for (int n = nb0; n < nb1 && !abort_flag; ++n) {
        const uint32_t i = (uint32_t)(n - nb0), a = i & 1u;
        mbar_spin(full(st), ph, &abort_flag, p.status, W_FULL);
        if (i >= 2) mbar_spin(acc_free((int)a), ((i >> 1) - 1u) & 1u, &abort_flag, p.status, W_ACCFREE);
        tc_fence_after();
        if (update) {
          const uint32_t bt = smem_st + st * S::STAGE + S::BASE;
          for (int q = 0; q < S::PIECES; ++q)
            for (int s = 0; s < steps; ++s) {
              const uint64_t da = smem_desc(smem_u + (uint32_t)(q * RB + (s >> 2)) * ATOM) + 2u * (uint32_t)(s & 3);
              const uint64_t db = smem_desc(bt + (uint32_t)(s >> 2) * 8192u) + 2u * (uint32_t)(s & 3);
              mma_ss(tmem + COL_ACC + 64u * a, da, db, IDESC, q > 0 || s > 0, leader);
            }
        }
        mma_commit(acc_full((int)a), leader);
        mma_commit(freed(st), leader);
        advance();
      }
    } else if (warp < EPI) {
      // this warp: 32 rows, half of the tile's columns (CH chunks of 16 bytes from chunk C0 on)
      constexpr int CH = F32 ? 8 : 4, EL = F32 ? 4 : 8;
      const int row = (warp & 3) * 32 + lane, half = warp >> 2;
      for (int n = nb0; n < nb1 && !abort_flag; ++n) {
        const uint32_t i = (uint32_t)(n - nb0), a = i & 1u;
        mbar_spin(full(st), ph, &abort_flag, p.status, W_FULL);
        mbar_spin(acc_full((int)a), (i >> 1) & 1u, &abort_flag, p.status, W_ACC);
        __syncwarp();
        tc_fence_after();
        // (fp32: a half is a box of its own; bf16: chunks 0-3 or 4-7 of the one box)
        unsigned char* const box = smem_p + S::U_BYTES + st * S::STAGE + (F32 ? half * (int)ATOM : 0);
        const int chunk0 = F32 ? 0 : 4 * half;
        uint32_t acc[32];
        if (update) {
          tmem_load32_nowait(tmem + ((uint32_t)((warp & 3) * 32) << 16) + COL_ACC + 64u * a + 32u * (uint32_t)half, acc);
          tmem_use32(acc);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acc_free((int)a));
        if (update) {
#pragma unroll
          for (int c = 0; c < CH; ++c) {
            uint4* const at = reinterpret_cast<uint4*>(box + row * 128 + (((chunk0 + c) ^ (row & 7)) << 4));
            uint4 v = *at;
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (F32) w[e] = __float_as_uint(__uint_as_float(w[e]) + __uint_as_float(acc[(EL * c + e) & 31]));
              else w[e] = pack2(__uint_as_float(w[e] << 16) + __uint_as_float(acc[(EL * c + 2 * e) & 31]),
                                __uint_as_float(w[e] & 0xFFFF0000u) + __uint_as_float(acc[(EL * c + 2 * e + 1) & 31]));
            }
            *at = make_uint4(w[0], w[1], w[2], w[3]);
          }
          __syncwarp();
        }
        // the warp's 32 rows leave as whole 64-byte (bf16) or 128-byte (fp32) pieces
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const int r = (warp & 3) * 32 + k * (32 / CH) + lane / CH, c = chunk0 + lane % CH, col = n * BN + (F32 ? 32 * half : 0) + c * EL;
          const uint4 v = *reinterpret_cast<const uint4*>(box + r * 128 + ((c ^ (r & 7)) << 4));
          if (r < rows && col < p.m)
            *reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(p.Y) + ((long long)(tok0 + r) * p.ldy + col) * (F32 ? 4 : 2)) = v;
        }
        // (the next TMA load into this stage is ordered after these reads and writes by the barrier and a proxy fence)
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(freed(st));
        advance();
      }
    }
  }
  if (few && rows > 0 && (id >= 0 || p.copy)) few_rows<F32>(p, smem_p, tok0, rows, id, rank, ranks, kb0 * KB, min(kb1 * KB, p.d), nb0 * BN, min(nb1 * BN, p.m));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TMEM_COLS) : "memory");
}

template <bool F32, int RB>
cudaError_t launch(const Params& p, const CUtensorMap& mx, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mbase, int tiles,
                   int ranks, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(adapter_kernel<F32, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<F32, RB>::SMEM);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * ranks));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = Shape<F32, RB>::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ranks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, adapter_kernel<F32, RB>, mx, ma, mb, mbase, p);
}

}  // namespace adapter
}  // namespace oq

using namespace oq;

extern "C" int oq_adapter_add(const void* X_bf16, int n_tokens, int ldx, int dim, const void* A_bf16, const void* B_bf16, int n_adapters,
                              int rank, const float* scale, const int* seg_start, const int* seg_adapter, int n_segs, const void* base,
                              int ldb, void* Y, int ldy, int m, int dtype, void* stream) {
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
  CUtensorMap mx, ma, mb, mbase;
  const uint64_t size = dtype == OQ_F32 ? 4 : 2;
  cudaError_t e;
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
    const uint32_t box[3] = {64, 64, 1};
    e = encode_tensor_map_sw128(&mb, B_bf16, false, 3, dims, strides, box);
  }
  if (e == cudaSuccess) {
    const uint64_t dims[2] = {(uint64_t)m, (uint64_t)n_tokens}, strides[1] = {(uint64_t)ldb * size};
    const uint32_t box[2] = {(uint32_t)(128 / size), 128};
    e = encode_tensor_map_sw128(&mbase, base, dtype == OQ_F32, 2, dims, strides, box);
  }
  if (e != cudaSuccess) return cuda_fail(e, "oq_adapter_add (tensor map)");
  // Tiles of 128 tokens, counted segment by segment (the segments' ends are on the device: an upper bound).  The cluster
  // grows until there are two rounds of CTAs for every SM, two at a time.
  const long long most = (n_tokens + adapter::BM - 1) / adapter::BM + (long long)n_segs;
  const int tiles = (int)(most < n_tokens ? most : n_tokens);
  int ranks = 1;
  while (ranks < 8 && (long long)tiles * ranks < OQ_AD) ranks *= 2;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool wide = rank > 64;
  if (dtype == OQ_F32) e = wide ? adapter::launch<true, 2>(p, mx, ma, mb, mbase, tiles, ranks, st) : adapter::launch<true, 1>(p, mx, ma, mb, mbase, tiles, ranks, st);
  else e = wide ? adapter::launch<false, 2>(p, mx, ma, mb, mbase, tiles, ranks, st) : adapter::launch<false, 1>(p, mx, ma, mb, mbase, tiles, ranks, st);
  if (e != cudaSuccess) return cuda_fail(e, "oq_adapter_add");
  return OQ_OK;
}
