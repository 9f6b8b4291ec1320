// Attention of chunks of new tokens over a paged cache: many rows (tokens times the heads of a group) for a key and value head.
//
// One pass over the keys with a running reference m and a running sum: with a row's factor c the kernel holds l = sum_j 2^(c (s_j - m)) and
// O = sum_j 2^(c (s_j - m)) v_j for any m that keeps the powers in range, so m follows the running maximum only when that has moved by more
// than 2^SLACK; then O and l are multiplied by 2^(c (m - m')).  The sums are fp32; the powers are rounded once, to fp16, as the tensor cores'
// operand (l sums the unrounded ones).  That is 2^-11 where the output's own rounding to bf16 is 2^-9: results differ from those of unrounded
// powers by less than a tenth of what that rounding does.
//
// Bound: the tensor cores and the exponentials alike, as without a cache (256 rows x 128 keys x 128 coordinates: 2048 cycles of products, 2048 of
// exponentials).  What the cache adds, decoding 2 x 128 x 128 elements for the 256 rows, is done by four warps of their own beside them: 16 bytes
// a load, one conversion and one multiplication a pair, 16 bytes a store into the swizzled tile from which the tensor cores read.  (In fp16, since
// an element times its scale is exact there, and since the hardware converts the cache's formats to fp16.)
//
//   2 x 4 warps              softmax, one thread per row: the item's queries to shared memory in fp16; then S from tensor memory, mask, maximum,
//                            powers, P (fp16) over S
//   4 warps                  convert: K and V tiles of 128 keys from the pages to a ring of shared-memory slots, loads one tile ahead
//   2 mma warps              one per 128 rows: S_t = Q_t K^T into tensor memory, O_t += P_t V with P_t from tensor memory
//
// Of a tile's 256 columns of tensor memory S has 128, over which P lies, and O the rest.  The mma warp issues P_t V of a key tile before the next
// S_t, so "S_t is there" also says that O_t holds the tiles before it, and that all of an item's products with Q before it are done.
#include <string>

#include "oq_cache_attention.cuh"
#include "oq_sm100.cuh"

namespace oq {
namespace cache {
namespace chunk {

constexpr int THREADS = 512;
// Registers: 512 threads start with 128 each.  A group of four warps each: softmax 200, 200, convert 72, mma 40.
constexpr int CONVERT_WARP = 8, MMA_WARP = 12;
constexpr int BM = 128;                            // rows of a query tile, of which a CTA has two
constexpr int SLOTS = 4;
constexpr uint32_t COL_S = 0, COL_P = 0, COL_O = BN;
constexpr float SLACK = 8.f;
enum { W_Q = 50, W_KV = 51, W_KVFREE = 52, W_S = 53, W_P = 54, W_O = 55 };
static_assert(CHUNK_ROWS == 2 * BM, "two query tiles an item");

template <int D>
struct Shape {
  static constexpr uint32_t ATOMS = D / 64;
  static constexpr uint32_t Q_ATOM = BM * 128, KV_ATOM = BN * 128;      // 64 coordinates of all rows, 128 bytes each
  static constexpr uint32_t Q_TILE = ATOMS * Q_ATOM, KV_TILE = ATOMS * KV_ATOM;
  static constexpr uint32_t SMEM = 1024 + 2 * Q_TILE + SLOTS * KV_TILE;
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// two fp32 lanes in one instruction
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b, float c) {
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %4};\n mov.b64 c, {%5, %5};\n fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b), "f"(c));
}
__device__ __forceinline__ void add2(float& d0, float& d1, float a0, float a1) {
  asm("{\n .reg .b64 a, d;\n mov.b64 a, {%2, %3};\n mov.b64 d, {%0, %1};\n add.rn.f32x2 d, d, a;\n mov.b64 {%0, %1}, d;\n}"
      : "+f"(d0), "+f"(d1) : "f"(a0), "f"(a1));
}
// bits 0 .. n-1 of a word, n clamped to 0 .. 32
__device__ __forceinline__ uint32_t ones_below(int n) { return n >= 32 ? ~0u : (n <= 0 ? 0u : (1u << n) - 1u); }

__device__ __forceinline__ void store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A convert warp's share of a tile: 32 keys, 16 bytes of a row a lane.  The lanes are dealt so that the 8 of them whose stores go together hit 8
// different 16-byte units of the 128-byte swizzle (unit ^ row % 8): pieces of 2 units (e4m3) of two rows, of 4 units (e2m1) of four.
template <int KIND, int D>
struct Share {
  using F = Format<KIND, D>;
  static constexpr int LPR = F::ROW / 16, RPI = 32 / LPR, ITERS = LPR;         // lanes a row, rows at a time, times
  static constexpr int UNITS = 16 / KIND;                                     // 16-byte units of fp16 that a lane's 16 bytes become
  __device__ static __forceinline__ int piece(int lane) {
    if (KIND == 8) return D == 128 ? (lane & 3) + 4 * ((lane >> 3) & 1) : lane & 3;
    return D == 128 ? (lane & 1) + 2 * ((lane >> 3) & 1) : lane & 1;
  }
  __device__ static __forceinline__ int row(int lane) {
    if (KIND == 8) return D == 128 ? ((lane >> 2) & 1) + 2 * (lane >> 4) : lane >> 2;
    return D == 128 ? ((lane >> 1) & 3) + 4 * (lane >> 4) : lane >> 1;
  }
};

template <int KIND, int D>
__global__ void __launch_bounds__(THREADS, 1) chunk_kernel(const __grid_constant__ AttnParams p) {
  using S = Shape<D>;
  using F = Format<KIND, D>;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[10 + 2 * SLOTS];
  __shared__ PlanMemory pm;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const uint32_t smem_q = smem, smem_kv = smem + 2 * S::Q_TILE;
  const uint32_t b0 = smem_u32(bars);
  auto q_full = [&](int t) { return b0 + 8u * (uint32_t)t; };
  auto s_full = [&](int t) { return b0 + 8u * (uint32_t)(2 + t); };
  auto p_part = [&](int t) { return b0 + 8u * (uint32_t)(4 + t); };     // P of the first 96 keys is there (and O rescaled, and read at an item's end)
  auto p_full = [&](int t) { return b0 + 8u * (uint32_t)(6 + t); };     // all of P is there
  auto o_done = [&](int t) { return b0 + 8u * (uint32_t)(8 + t); };     // the item's last P V has been added: O may be read
  auto kv_full = [&](int s) { return b0 + 8u * (uint32_t)(10 + s); };
  auto kv_free = [&](int s) { return b0 + 8u * (uint32_t)(10 + SLOTS + s); };

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full(t), 4);
      mbar_init(s_full(t), 1);
      mbar_init(p_part(t), 4);
      mbar_init(p_full(t), 4);
      mbar_init(o_done(t), 1);
    }
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(kv_full(s), 4);
      mbar_init(kv_free(s), 2);           // both mma warps, also when one of them does not use the slot
    }
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  Stretch st = plan<CHUNK_ROWS, THREADS>(p, pm);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  // All roles walk over the same steps: the key tiles of this CTA's items (of the parts of them in its stretch), one after the other.
  auto run_of = [&](const Item& it) { return (int)min((long long)(it.tiles - st.off), st.count); };
  auto next_item = [&](int n) {
    st.count -= n;
    st.off = 0;
    if (++st.block == st.blocks) {
      st.block = 0;
      ++st.head;
    }
  };

  if (warp < CONVERT_WARP) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ------------------------------------------------ softmax ------------------------------------------------
    const int t = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t columns = tmem + ((uint32_t)(quarter * 32) << 16) + 256u * (uint32_t)t;
    const uint32_t col_s = columns + COL_S, col_p = columns + COL_P, col_o = columns + COL_O;
    uint32_t steps = 0, items = 0;              // of this tile so far
    auto warp_wait = [&](uint32_t bar, uint32_t parity, int code) {
      mbar_spin(bar, parity, &abort_flag, p.status, code);
      __syncwarp();
    };
    // Warp w of tile 0 and of tile 1 sit on the same scheduler and take turns at the exponentials.  (The turns are counted, so no warp leaves
    // its loops early, not even when a wait has given up.)
    auto turn_wait = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + 2 * quarter + t) : "memory"); };
    auto turn_pass = [&]() { asm volatile("bar.arrive %0, 64;" ::"r"(2 + 2 * quarter - t) : "memory"); };
    while (st.count > 0) {
      int rows, first, hi, lo, full_hi, full_lo, tiles, n_sink, skipped, seq, nk;
      bool turns;
      float c;
      {
        const Item it = make_item<CHUNK_ROWS>(p, pm.prefix, st.head, st.block);
        rows = min(max(it.rows - t * BM, 0), BM);
        const int r0 = it.r0 + t * BM, last = r0 + max(rows, 1) - 1;
        const int mine = min(r0 + row, last);             // (rows that do not exist stand in for the last one)
        hi = row_hi(p, it.s, mine / p.group);
        lo = row_lo(p, it.s, mine / p.group);
        full_hi = row_hi(p, it.s, r0 / p.group);          // what every row of the tile sees
        full_lo = row_lo(p, it.s, last / p.group);
        first = st.off;
        tiles = run_of(it);
        n_sink = it.n_sink - first;                       // step j: key tile first + j, with a gap after the sinks
        skipped = it.win0 - it.n_sink;
        turns = it.rows - BM > quarter * 32;              // both warps have rows (tile 0 is full where tile 1 has any)
        seq = it.seq;
        nk = it.s.nk;
        if (rows > 0) {
          // the row's queries to fp16 (the products with the last item's are done: its last S has been waited for)
          const __nv_bfloat16* src = p.Q + (long long)(it.s.q_base + mine / p.group) * p.ldq + (long long)(it.head * p.group + mine % p.group) * p.hdq;
          uint32_t largest = 0;
#pragma unroll
          for (int x = 0; x < D / 8; ++x) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(src) + x);
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) largest = max(largest, max((u[e] << 16) & 0x7FFFFFFFu, u[e] & 0x7FFF0000u));
          }
          const RowScale rs = row_scale(largest, p.scale_log2);
          c = rs.c;
          const uint32_t to = smem_q + (uint32_t)t * S::Q_TILE + 128u * (uint32_t)row;
#pragma unroll 4
          for (int x = 0; x < D / 8; ++x) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(src) + x);
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = pack_f16(__uint_as_float(u[e] << 16) * rs.mul, __uint_as_float(u[e] & 0xFFFF0000u) * rs.mul);
            store16(to + (uint32_t)(x >> 3) * S::Q_ATOM + (uint32_t)((x ^ row) & 7) * 16u, h[0], h[1], h[2], h[3]);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(q_full(t));
        }
      }
      if (rows == 0) {
        next_item(tiles);
        continue;
      }
      const bool idle = quarter * 32 >= rows;              // none of the warp's rows exists
      // pages of the tile's 16-key pieces that are there: lane x looks up piece x, a step ahead
      auto piece_page = [&](int j) {
        const int pos = BN * (first + j + (j < n_sink ? 0 : skipped)) + 16 * lane;
        return lane < 8 && j < tiles && pos < nk ? page_of(p.c, seq, pos) : 0;
      };
      int page = piece_page(0);
      float m = -INFINITY, l = 0.f, shift = 0.f;
      for (int j = 0; j < tiles; ++j, ++steps) {
        const int k0 = BN * (first + j + (j < n_sink ? 0 : skipped));
        const uint32_t there = __ballot_sync(~0u, page >= 0);
        page = piece_page(j + 1);
        warp_wait(s_full(t), steps & 1, W_S);
        if (idle) {                             // (O's rows are never read: whatever P holds there may stay)
          if (lane == 0) {
            mbar_arrive(p_part(t));
            mbar_arrive(p_full(t));
          }
          continue;
        }
        tc_fence_after();
        uint32_t sr[BN];
#pragma unroll
        for (int q = 0; q < BN / 32; ++q) tmem_load32_nowait(col_s + 32u * q, sr + 32 * q);
#pragma unroll
        for (int q = 0; q < BN / 32; ++q) tmem_use32(sr + 32 * q);
        if (!(k0 + BN - 1 <= full_hi && (k0 >= full_lo || k0 + BN <= p.sinks)) || there != ~0u) {
          uint32_t some = 0;
#pragma unroll
          for (int q = 0; q < BN / 32; ++q) {
            const int b = k0 + 32 * q;
            uint32_t keep = ones_below(hi + 1 - b) & (~ones_below(lo - b) | ones_below(p.sinks - b));
            if (!((there >> (2 * q)) & 1u)) keep &= 0xFFFF0000u;
            if (!((there >> (2 * q + 1)) & 1u)) keep &= 0x0000FFFFu;
            some |= keep;
            if (__all_sync(~0u, keep == ~0u)) continue;          // (an edge of the mask crosses one or two of the four)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!((keep >> e) & 1u)) sr[32 * q + e] = 0xFF800000u;
          }
          if (!__any_sync(~0u, some)) {         // the warp's rows see nothing of this tile: weights of zero, m and l stay
            uint32_t zero[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) zero[e] = 0u;
#pragma unroll
            for (int q = 0; q < BN / 32; ++q) tmem_store16(col_p + 16u * q, zero);
            tmem_wait_st();
            if (turns && (t == 1 || j > 0)) turn_wait();
            if (turns && (t == 0 || j + 1 < tiles)) turn_pass();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(p_part(t));
              mbar_arrive(p_full(t));
            }
            continue;
          }
        }
        float mx[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          mx[q] = fmaxf(__uint_as_float(sr[q]), __uint_as_float(sr[4 + q]));
#pragma unroll
          for (int e = 2; e < BN / 4; e += 2) mx[q] = max3(mx[q], __uint_as_float(sr[4 * e + q]), __uint_as_float(sr[4 * e + 4 + q]));
        }
        const float mn = max3(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]), m);
        if (j == 0) {
          m = mn;
          c = tame(c, m);
          shift = m == -INFINITY ? 0.f : -m * c;
        } else if (__any_sync(~0u, (mn - m) * c > SLACK)) {
          // (S_t of this key tile is there, so O_t holds the tiles before it and nothing is writing it)
          c = tame(c, mn);
          const float a = m == mn ? 1.f : exp2_fast((m - mn) * c);
          m = mn;
          l *= a;
          shift = m == -INFINITY ? 0.f : -m * c;
#pragma unroll 1
          for (int x = 0; x < D / 16; ++x) {
            uint32_t o[16];
            tmem_load16_at(col_o + 16u * x, o);
            tmem_use16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
            tmem_store16(col_o + 16u * x, o);
          }
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        // one warp of the two that share a scheduler exponentiates while the other does all else
        if (turns && (t == 1 || j > 0)) turn_wait();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x, y;
            fma2(x, y, __uint_as_float(sr[32 * q + 2 * e]), __uint_as_float(sr[32 * q + 2 * e + 1]), c, shift);
            x = exp2_fast(x);
            y = exp2_fast(y);
            add2(sum[2 * (e & 1)], sum[2 * (e & 1) + 1], x, y);
            pk[e] = pack_f16(x, y);
          }
          if (q == 3 && turns && (t == 0 || j + 1 < tiles)) turn_pass();
          tmem_store16(col_p + 16u * q, pk);
          if (q >= 2) {                                   // the first 96 keys, then the rest
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(q == 2 ? p_part(t) : p_full(t));
          }
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      // ------------------------------------------- the item's result -------------------------------------------
      warp_wait(o_done(t), items++ & 1, W_O);
      if (!idle) {
        const Item it = make_item<CHUNK_ROWS>(p, pm.prefix, st.head, st.block);
        tc_fence_after();
        const bool mine = row < rows, whole = first == 0 && tiles == it.tiles;
        const int r = it.r0 + t * BM + row, i = it.s.q_base + r / p.group, head = it.head * p.group + r % p.group;
        const long long slot_row = (2 * (long long)blockIdx.x + (first == 0 ? 1 : 0)) * CHUNK_ROWS + t * BM + row;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat16* const dst = p.out + (long long)i * p.ldo + head * p.hdo;
#pragma unroll 1
        for (int q = 0; q < D / 32; ++q) {
          uint32_t o[32];
          tmem_load32_nowait(col_o + 32u * q, o);
          tmem_use32(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(l != 0.f ? __uint_as_float(o[e]) * inv : 0.f);
          if (!mine) continue;
          if (!whole) {
            uint4* const to = reinterpret_cast<uint4*>(p.part_o + slot_row * D + 32 * q);
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          } else {
            uint32_t v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = pack_bf16(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
#pragma unroll
            for (int e = 0; e < 4; ++e) reinterpret_cast<uint4*>(dst + 32 * q)[e] = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          }
        }
        if (mine) {
          // the powers had m c rounded in them, which shows in the sum (not in the weights' ratios)
          if (l != 0.f && m > -INFINITY) l *= exp2_fast(-fmaf(m, c, shift));
          if (!whole) p.part_ml[slot_row] = make_float4(m, l, c, 0.f);
          else if (p.lse) p.lse[(long long)head * p.total_q + i] = natural_lse(m, l, c);
        }
        tc_fence_before();                        // (the next item's first P, which lets O be overwritten, comes after this)
      }
      next_item(tiles);
    }
  } else if (warp < MMA_WARP) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    // ------------------------------------------------ convert ------------------------------------------------
    using H = Share<KIND, D>;
    const int part = warp - CONVERT_WARP, piece = H::piece(lane), my_row = H::row(lane);
    const int group = piece * (128 / KIND) / 32;
    uint32_t slot = 0, round = 0;
    uint32_t raw[H::ITERS][4];
    uint32_t scale[H::ITERS];
    // addresses of the present tile's two pieces of 16 keys, and how many keys of this warp's 32 exist
    const uint8_t *at0 = nullptr, *at1 = nullptr;
    int exist = 0;
    const int in_page = (1 << p.c.shift) - 1;
    auto look_up = [&](int seq, int head, int pos, int nk) {
      exist = min(max(nk - pos, 0), 32);
      const int a = exist > 0 ? page_of(p.c, seq, pos) : -1, b = exist > 16 ? page_of(p.c, seq, pos + 16) : -1;
      at0 = a < 0 ? nullptr : block_of(p.c, a, head);
      at1 = b < 0 ? nullptr : block_of(p.c, b, head);
    };
    auto load = [&](int i, int pos, bool values) {
      const int r = i * H::RPI + my_row;
      const uint8_t* const block = r < 16 ? at0 : at1;
      raw[i][0] = raw[i][1] = raw[i][2] = raw[i][3] = 0u;
      scale[i] = 127u;
      if (block && r < exist) {
        const int at = (pos + r) & in_page;
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(block + (values ? p.c.off_v : 0u) + at * F::ROW + 16 * piece));
        raw[i][0] = v.x; raw[i][1] = v.y; raw[i][2] = v.z; raw[i][3] = v.w;
        scale[i] = __ldg(block + (values ? p.c.off_vs : p.c.off_ks) + at * F::GROUPS + group);
      }
    };
    auto convert = [&](int i, bool values) {
      const int r = i * H::RPI + my_row, e0 = piece * (128 / KIND);
      const uint32_t f = !values && scale[i] == BROKEN ? 0x7FFF7FFFu : scale_pair(scale[i], scale[i]);
      const uint32_t to = smem_kv + slot * S::KV_TILE + (uint32_t)(e0 / 64) * S::KV_ATOM + 128u * (uint32_t)(32 * part + r);
#pragma unroll
      for (int u = 0; u < H::UNITS; ++u) {
        uint32_t h[4];
        if constexpr (KIND == 8) {
          e4m3_to_f16(raw[i][2 * u], h[0], h[1]);
          e4m3_to_f16(raw[i][2 * u + 1], h[2], h[3]);
        } else {
          e2m1_to_f16(raw[i][u], h[0], h[1], h[2], h[3]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = mul_f16x2(h[e], f);
        store16(to + (uint32_t)(((e0 / 8 + u) ^ r) & 7) * 16u, h[0], h[1], h[2], h[3]);
      }
    };
    auto take_slot = [&]() {
      if (round > 0) mbar_spin(kv_free(slot), (round - 1) & 1, &abort_flag, p.status, W_KVFREE);
      __syncwarp();
    };
    auto give_slot = [&]() {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(kv_full(slot));
      if (++slot == SLOTS) {
        slot = 0;
        ++round;
      }
    };
    bool begun = false;
    Item it;
    int n = 0, j = 0, pos = 0;
    auto enter = [&]() {
      it = make_item<CHUNK_ROWS>(p, pm.prefix, st.head, st.block);
      n = run_of(it);
      j = 0;
    };
    if (st.count > 0) {
      enter();
      begun = true;
      pos = it.key0(st.off) + 32 * part;
      look_up(it.seq, it.head, pos, it.s.nk);
#pragma unroll
      for (int i = 0; i < H::ITERS; ++i) load(i, pos, false);
    }
    while (begun) {
      take_slot();
#pragma unroll
      for (int i = 0; i < H::ITERS; ++i) {
        convert(i, false);
        load(i, pos, true);
      }
      give_slot();
      // the next step
      if (++j == n) {
        next_item(n);
        if (st.count > 0) enter(); else begun = false;
      }
      if (begun) {
        pos = it.key0(st.off + j) + 32 * part;
        look_up(it.seq, it.head, pos, it.s.nk);
      }
      take_slot();
#pragma unroll
      for (int i = 0; i < H::ITERS; ++i) {
        convert(i, true);
        if (begun) load(i, pos, false);
      }
      give_slot();
      if (abort_flag) break;
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp < MMA_WARP + 2) {
      const int t = warp - MMA_WARP;
      const uint32_t leader = elect_leader();       // (the whole warp runs this, one lane issues)
      constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)(BM >> 4) << 24);                  // fp16 operands, fp32 result
      constexpr uint32_t IDESC_S = IDESC | ((uint32_t)(BN >> 3) << 17);
      constexpr uint32_t IDESC_O = IDESC | ((uint32_t)(D >> 3) << 17) | (1u << 16);        // V is N-major
      const uint32_t columns = tmem + 256u * (uint32_t)t;
      uint32_t slot = 0, round = 0, q_use = 0, p_use = 0;
      auto advance = [&]() {
        if (++slot == SLOTS) {
          slot = 0;
          ++round;
        }
      };
      // (Both warps see every slot filled and free it, whether they use it or not: a wait tells phases apart by their parity alone, so no warp
      // may get a whole round ahead of a slot or behind it.)
      auto do_s = [&](bool active, bool first) {
        mbar_spin(kv_full(slot), round & 1, &abort_flag, p.status, W_KV);
        if (!active) {
          if (leader) mbar_arrive(kv_free(slot));
        } else {
          if (first) mbar_spin(q_full(t), q_use++ & 1, &abort_flag, p.status, W_Q);
          tc_fence_after();
          const uint64_t a = smem_desc(smem_q + (uint32_t)t * S::Q_TILE), b = smem_desc(smem_kv + slot * S::KV_TILE);
#pragma unroll
          for (uint32_t k = 0; k < D / 16; ++k)
            mma_ss(columns + COL_S, a + (uint64_t)((k >> 2) * (S::Q_ATOM >> 4) + 2 * (k & 3)), b + (uint64_t)((k >> 2) * (S::KV_ATOM >> 4) + 2 * (k & 3)),
                   IDESC_S, k > 0, leader);
          mma_commit(s_full(t), leader);
          mma_commit(kv_free(slot), leader);
        }
        advance();
      };
      auto do_o = [&](bool active, bool first, bool last) {
        mbar_spin(kv_full(slot), round & 1, &abort_flag, p.status, W_KV);
        if (!active) {
          if (leader) mbar_arrive(kv_free(slot));
        } else {
          mbar_spin(p_part(t), p_use & 1, &abort_flag, p.status, W_P);
          tc_fence_after();
          const uint64_t b = smem_desc_mn(smem_kv + slot * S::KV_TILE, S::KV_ATOM, 1024);
#pragma unroll
          for (uint32_t k = 0; k < BN / 16; ++k) {
            if (k == 6) {
              mbar_spin(p_full(t), p_use++ & 1, &abort_flag, p.status, W_P);
              tc_fence_after();
            }
            mma_ts(columns + COL_O, columns + COL_P + 8 * k, b + (uint64_t)(k * (2048 >> 4)), IDESC_O, !first || k > 0, leader);
          }
          if (last) mma_commit(o_done(t), leader);
          mma_commit(kv_free(slot), leader);
        }
        advance();
      };
      int n = 0, j = 0;
      bool active = false, have = st.count > 0;
      auto enter = [&]() {
        const Item it = make_item<CHUNK_ROWS>(p, pm.prefix, st.head, st.block);
        n = run_of(it);
        j = 0;
        active = it.rows > t * BM;
      };
      if (have) {
        enter();
        do_s(active, true);
      }
      while (have && !abort_flag) {
        do_o(active, j == 0, j + 1 == n);
        if (++j == n) {
          next_item(n);
          have = st.count > 0;
          if (have) enter();
        }
        if (have) do_s(active, j == 0);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

template <int KIND, int D>
cudaError_t go(const AttnParams& p, cudaStream_t st) {
  // (the attribute belongs to the device that is current, so it is set every time)
  const cudaError_t e = cudaFuncSetAttribute(chunk_kernel<KIND, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<D>::SMEM);
  if (e != cudaSuccess) return e;
  return launch_dependent(chunk_kernel<KIND, D>, p.ctas, THREADS, Shape<D>::SMEM, st, p);
}

}  // namespace chunk

cudaError_t launch_chunk(const AttnParams& p, int kind, int head_dim, cudaStream_t st) {
  if (kind == OQ_CACHE_FP8) return head_dim == 128 ? chunk::go<8, 128>(p, st) : chunk::go<8, 64>(p, st);
  return head_dim == 128 ? chunk::go<4, 128>(p, st) : chunk::go<4, 64>(p, st);
}

}  // namespace cache
}  // namespace oq
