// Attention of chunks of new tokens over a paged cache: many rows (tokens times the heads of a group) for a key and value head.
//
// One pass over the keys with a running reference m and a running sum: with a row's factor c the kernel holds l = sum_j 2^(c (s_j - m)) and
// O = sum_j 2^(c (s_j - m)) v_j for any m that keeps the powers in range, so m follows the running maximum only when that has moved by more
// than 2^SLACK; then O and l are multiplied by 2^(c (m - m')).  The sums are fp32; the powers are rounded once, to fp16, as the tensor cores'
// operand (l sums the unrounded ones), after a multiplication that keeps them in fp16's range (see HEAD): 2^-11 of a weight, or 2^-36 of the
// largest where that is more.  The output's own rounding to bf16 is 2^-8 of a value.
//
// Bound: the tensor cores and the exponentials alike, as without a cache (256 rows x 128 keys x 128 coordinates: 2048 cycles of products, 2048 of
// exponentials).  What the cache adds, decoding 2 x 128 x 128 elements for the 256 rows, is done by four warps of their own beside them: 16 bytes
// a load, one conversion and one multiplication a pair, 16 bytes a store into the swizzled tile from which the tensor cores read.  (In fp16, since
// an element times its scale is exact there, and since the hardware converts the cache's formats to fp16.)
//
//   2 x 4 warps              softmax, one thread per row: the item's queries to shared memory in fp16; then S from tensor memory, mask, maximum,
//                            powers, P (fp16) over S
//   load warp                finds the pages and requests their parts of a tile as they are, by bulk copies into a ring of stages
//   4 warps                  convert: from a stage, 128 keys of K or V, to a slot of a second ring, fp16 in the tensor cores' order
//   2 mma warps              one per 128 rows: S_t = Q_t K^T into tensor memory, O_t += P_t V with P_t from tensor memory
//
// Measured (B200, head_dim 128; device time of captured calls): 2048 tokens over 16385, 24 heads on 8, causal, e2m1 381 us = 1.01 PFLOP/s; a streamed frame of
// 1560 tokens over 15600 of 32760, 40 heads, e4m3 544 us = 0.87; 4608 over 4608, 24 heads, e4m3 299 us = 0.87 (oq_attention on bf16 keys and values on the same GPU: 376, 470 and
// 221 us, without a cache to keep, read back or move; head_dim 64 is bound by the exponentials, 0.61 PFLOP/s).  A step of 256 rows x 128 keys takes 3850 cycles, an
// item's begin and end as much as four of them.  What decoding costs: a copy of this kernel that stored nothing in the slots took 6 to 12 % less, one whose mma
// warps did not wait for slots at all 25 % (the softmax and the products alone).  Other arrangements that were measured, beside the 512 us of the first form of the
// 381: K and V loaded into the convert warps' registers 504; stages of half a tile, a slot more 476 beside 458; S read from tensor memory twice, 32 columns at a
// time, for fewer registers 560 beside 458; the next turn at the exponentials given away a quarter earlier 462 beside 462, a half earlier 470; one copy of each
// MMA sequence instead of two 422 beside 387; a row of queries loaded by 16 lanes instead of one 414 beside 390.
//
// Of a tile's 256 columns of tensor memory S has 128, over which P lies, and O the rest.  The mma warp issues P_t V of a key tile before the next
// S_t, so "S_t is there" also says that O_t holds the tiles before it, and that all of an item's products with Q before it are done.
#include <string>

#include "oq_cache_attention.cuh"

namespace oq {
namespace cache {
namespace chunk {

constexpr int THREADS = 512;
// Registers: 512 threads start with 128 each.  What a group of four warps takes more than that, others have to give up first: the shares' sum is bounded.
constexpr int SOFTMAX_REGS = 208, CONVERT_REGS = 48, MMA_REGS = 48;
static_assert(2 * SOFTMAX_REGS + CONVERT_REGS + MMA_REGS <= 4 * 128, "setmaxnreg.inc would wait for ever");
constexpr int CONVERT_WARP = 8, MMA_WARP = 12, LOAD_WARP = 14;
constexpr int BM = 128;                            // rows of a query tile, of which a CTA has two
constexpr int PIECE = 16, PIECES = BN / PIECE;     // keys that lie in one page whatever its size
constexpr uint32_t COL_S = 0, COL_P = 0, COL_O = BN;
// A power is 2^(c s + shift) with shift = HEAD - c m rounded, so all of a row's are off by one factor, which cancels, as long as it stays small: it is 2^0.06 at most while
// |c m| < 2^20.  The warps that have a row beyond that take s - m first.
constexpr float FAR = 1048576.f;
enum { W_Q = 50, W_KV = 51, W_KVFREE = 52, W_S = 53, W_P = 54, W_O = 55, W_RAW = 56, W_RAWFREE = 57 };
static_assert(CHUNK_ROWS == 2 * BM, "two query tiles an item");

template <int KIND, int D>
struct Shape {
  using F = Format<KIND, D>;
  static constexpr uint32_t ATOMS = D / 64;
  static constexpr uint32_t Q_ATOM = BM * 128, KV_ATOM = BN * 128;      // 64 coordinates of all rows, 128 bytes each
  static constexpr uint32_t Q_TILE = ATOMS * Q_ATOM, KV_TILE = ATOMS * KV_ATOM;
  static constexpr int STAGES = 3, SLOTS = F::ROW == 128 ? 3 : 4;        // (a fourth slot where it fits)
  static constexpr uint32_t RAW_SCALES = BN * F::ROW, RAW = RAW_SCALES + BN * F::GROUPS;      // a stage: rows, then their scales
  static constexpr uint32_t SMEM = 1024 + 2 * Q_TILE + SLOTS * KV_TILE + STAGES * RAW;
};

// two fp32 lanes in one instruction
__device__ __forceinline__ uint64_t twice(float x) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %1};" : "=l"(d) : "f"(x));
  return d;
}
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, uint64_t b, uint64_t c) {
  asm("{\n .reg .b64 a, d;\n mov.b64 a, {%2, %3};\n fma.rn.f32x2 d, a, %4, %5;\n mov.b64 {%0, %1}, d;\n}" : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "l"(b), "l"(c));
}

__device__ __forceinline__ void store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ uint4 load_row16(const __nv_bfloat16* p) {        // (volatile: requested together)
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void store32(void* p, const uint32_t* v) {         // 32 bytes: a whole sector
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void load_shared16(uint32_t at, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t load_shared1(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// A convert warp's share of a tile: 32 keys, 16 bytes of a row a lane.  The lanes are dealt so that 8 of them, whose accesses go together, read 128
// bytes that lie in different banks and hit 8 different 16-byte units of the 128-byte swizzle (unit ^ row % 8) when they store: pieces of 2 units
// (e4m3) of two rows, of 4 units (e2m1) of four.
template <int KIND, int D>
struct Share {
  using F = Format<KIND, D>;
  static constexpr int LPR = F::ROW / 16, RPI = 32 / LPR, ITERS = LPR;         // lanes a row, rows at a time, times
  static constexpr int UNITS = 16 / KIND;                                     // 16-byte units of fp16 that a lane's 16 bytes become
  __device__ static __forceinline__ int piece(int lane) {
    if (KIND == 8) return D == 128 ? lane & 7 : lane & 3;                      // (rows of 128 bytes: the halves of two rows, see row)
    return D == 128 ? (lane & 1) + 2 * ((lane >> 2) & 1) : lane & 1;           // (rows of 64: halves of four)
  }
  __device__ static __forceinline__ int row(int lane) {
    if (KIND == 8) return D == 128 ? 2 * (lane >> 4) + (((lane >> 2) ^ (lane >> 3)) & 1) : lane >> 2;
    return D == 128 ? 4 * (lane >> 4) + (((lane >> 1) & 1) | (((lane >> 2) ^ (lane >> 3)) & 1) << 1) : lane >> 1;
  }
};

// A thread's row of the item's query tile t to shared memory in fp16; returns its factor c.  (A function, as two places want it: straight-line
// code that runs once an item comes from far away each time.)
template <int D>
__device__ __noinline__ float prepare_row(const AttnParams& p, const Item& it, int t, int row, uint32_t to, uint32_t atom) {
  const int r = min(it.r0 + t * BM + row, it.r0 + it.rows - 1), i = token_of(p, r);      // (rows that do not exist stand in for the last one)
  const __nv_bfloat16* src = p.Q + (long long)(it.s.q_base + i) * p.ldq + (long long)(it.head * p.group + r - i * p.group) * p.hdq;
  uint4 v[D / 8];
#pragma unroll
  for (int x = 0; x < D / 8; ++x) v[x] = load_row16(src + 8 * x);
  uint32_t largest = 0;
#pragma unroll
  for (int x = 0; x < D / 8; ++x) {
    const uint32_t u[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) largest = max(largest, max((u[e] << 16) & 0x7FFFFFFFu, u[e] & 0x7FFF0000u));
  }
  const RowScale rs = row_scale(largest, p.scale_log2);
  to += 128u * (uint32_t)row;
#pragma unroll
  for (int x = 0; x < D / 8; ++x) {
    const uint32_t u[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
    uint32_t h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = pack_f16(__uint_as_float(u[e] << 16) * rs.mul, __uint_as_float(u[e] & 0xFFFF0000u) * rs.mul);
    store16(to + (uint32_t)(x >> 3) * atom + (uint32_t)((x ^ row) & 7) * 16u, h[0], h[1], h[2], h[3]);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  return rs.c;
}

template <int KIND, int D, bool WHOLE>
__global__ void __launch_bounds__(THREADS, 1) chunk_kernel(const __grid_constant__ AttnParams p) {
  using S = Shape<KIND, D>;
  using F = Format<KIND, D>;
  constexpr int SLOTS = S::SLOTS, STAGES = S::STAGES;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[10 + 2 * SLOTS + 2 * STAGES];
  __shared__ Plan pm;
  // what a stage holds: number of keys that exist; the pieces of 16 whose page is missing in bits 8 .. 15; from bit 16 and from bit 24 on, the first
  // key between the sinks and the first window of the item, which no row sees, and the first one behind these
  __shared__ uint32_t raw_keys[STAGES];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const uint32_t smem_q = smem, smem_kv = smem + 2 * S::Q_TILE, smem_raw = smem_kv + SLOTS * S::KV_TILE;
  const uint32_t b0 = smem_u32(bars);
  auto q_full = [&](int t) { return b0 + 8u * (uint32_t)t; };
  auto s_full = [&](int t) { return b0 + 8u * (uint32_t)(2 + t); };
  auto p_part = [&](int t) { return b0 + 8u * (uint32_t)(4 + t); };     // P of the first 96 keys is there (and O rescaled, and read at an item's end)
  auto p_full = [&](int t) { return b0 + 8u * (uint32_t)(6 + t); };     // all of P is there
  auto o_done = [&](int t) { return b0 + 8u * (uint32_t)(8 + t); };     // the item's last P V has been added: O may be read
  auto kv_full = [&](int s) { return b0 + 8u * (uint32_t)(10 + s); };
  auto kv_free = [&](int s) { return b0 + 8u * (uint32_t)(10 + SLOTS + s); };
  auto raw_full = [&](int s) { return b0 + 8u * (uint32_t)(10 + 2 * SLOTS + s); };
  auto raw_free = [&](int s) { return b0 + 8u * (uint32_t)(10 + 2 * SLOTS + STAGES + s); };

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
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(raw_full(s), 1);
      mbar_init(raw_free(s), 4);
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
  Stretch st = plan<CHUNK_ROWS, THREADS, CHUNK_OVERHEAD, WHOLE>(p, pm);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  // All roles walk over the same steps: the key tiles of this CTA's items (of the parts of them in its stretch), one after the other.
  auto run_of = [&](const Item& it) { return (int)min((long long)(it.tiles - st.off), st.count); };
  if (warp < CONVERT_WARP) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
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
    // The queries of an item are prepared while the tensor cores are at the end of the one before it: its products with Q are done once its
    // last S has been waited for.
    auto prepare = [&](const Stretch& at) {
      const Item it = make_item<CHUNK_ROWS>(p, pm, at.head, at.block);
      if (it.rows <= t * BM) return 0.f;
      const float c = prepare_row<D>(p, it, t, row, smem_q + (uint32_t)t * S::Q_TILE, S::Q_ATOM);
      if (lane == 0) mbar_arrive(q_full(t));
      return c;
    };
    float c_next = st.count > 0 ? prepare(st) : 0.f;
    while (st.count > 0) {
      int rows, first, hi, lo, full_hi, full_lo, tiles, n_sink, skipped, seq, nk;
      bool turns;
      const float c = c_next;
      {
        const Item it = make_item<CHUNK_ROWS>(p, pm, st.head, st.block);
        rows = min(max(it.rows - t * BM, 0), BM);
        const int r0 = it.r0 + t * BM, last = r0 + max(rows, 1) - 1;
        const int mine = min(r0 + row, last);             // (rows that do not exist stand in for the last one)
        hi = row_hi(p, it.s, token_of(p, mine));
        lo = row_lo(p, it.s, token_of(p, mine));
        full_hi = row_hi(p, it.s, token_of(p, r0));       // what every row of the tile sees
        full_lo = row_lo(p, it.s, token_of(p, last));
        first = st.off;
        tiles = run_of(it);
        n_sink = it.n_sink - first;                       // step j: key tile first + j, with a gap after the sinks
        skipped = it.win0 - it.n_sink;
        turns = it.rows - BM > quarter * 32;              // both warps have rows (tile 0 is full where tile 1 has any)
        seq = it.seq;
        nk = it.s.nk;
      }
      Stretch next = st;
      next_item(next, tiles);
      if (rows == 0) {
        if (next.count > 0) c_next = prepare(next);
        st = next;
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
      float minus = 0.f;                                   // -m where a row of the warp is far, else 0: the powers are 2^(c (s + minus) + shift)
      // Brings the reference to mn.  Returns what sums and O have to be multiplied by: the change of the power at the old reference, as the roundings of both references
      // have it.
      auto move_to = [&](float mn) {
        const float old = m, from = fmaf(old + minus, c, shift);
        m = mn;
        const bool far = __any_sync(~0u, fabsf(m) * c > FAR && m > -INFINITY);
        minus = far && m > -INFINITY ? -m : 0.f;
        shift = far || m == -INFINITY ? HEAD : fmaf(-m, c, HEAD);
        return old > -INFINITY ? exp2_fast(fmaf(old + minus, c, shift) - from) : 1.f;
      };
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
        if (__any_sync(~0u, (mn - m) * c > SLACK)) {
          // (S_t of this key tile is there, so O_t holds the tiles before it, none at j == 0, and nothing is writing it)
          const float a = move_to(mn);
          l *= a;
#pragma unroll 1
          for (int x = j == 0 ? D / 16 : 0; x < D / 16; ++x) {
            uint32_t o[16];
            tmem_load16_at(col_o + 16u * x, o);
            tmem_use16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
            tmem_store16(col_o + 16u * x, o);
          }
        }
        if (__any_sync(~0u, minus != 0.f)) {
#pragma unroll
          for (int e = 0; e < BN; e += 2) {
            float x = __uint_as_float(sr[e]), y = __uint_as_float(sr[e + 1]);
            add2(x, y, minus, minus);
            sr[e] = __float_as_uint(x);
            sr[e + 1] = __float_as_uint(y);
          }
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        const uint64_t c2 = twice(c), shift2 = twice(shift);
        // one warp of the two that share a scheduler exponentiates while the other does all else
        if (turns && (t == 1 || j > 0)) turn_wait();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x, y;
            fma2(x, y, __uint_as_float(sr[32 * q + 2 * e]), __uint_as_float(sr[32 * q + 2 * e + 1]), c2, shift2);
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
      if (next.count > 0) c_next = prepare(next);
      // ------------------------------------------- the item's result -------------------------------------------
      warp_wait(o_done(t), items++ & 1, W_O);
      if (!idle) {
        const Item it = make_item<CHUNK_ROWS>(p, pm, st.head, st.block);
        tc_fence_after();
        const bool mine = row < rows, whole = first == 0 && tiles == it.tiles;
        const int r = it.r0 + t * BM + row, tok = token_of(p, r), i = it.s.q_base + tok, head = it.head * p.group + r - tok * p.group;
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
#pragma unroll
            for (int e = 0; e < 4; ++e) store32(p.part_o + slot_row * D + 32 * q + 8 * e, o + 8 * e);
          } else {
            uint32_t v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = pack_bf16(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
            if (p.wide_out) {
#pragma unroll
              for (int e = 0; e < 2; ++e) store32(dst + 32 * q + 16 * e, v + 8 * e);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) reinterpret_cast<uint4*>(dst + 32 * q)[e] = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
            }
          }
        }
        if (mine) {
          // the powers had HEAD and m c, rounded, in them, which shows in the sum (not in the weights' ratios)
          if (l != 0.f && m > -INFINITY) l *= exp2_fast(-fmaf(m + minus, c, shift));
          if (!whole) p.part_ml[slot_row] = make_float4(m, l, c, 0.f);
          else if (p.lse) p.lse[(long long)head * p.total_q + i] = natural_lse(m, l, c);
        }
        tc_fence_before();                        // (the next item's first P, which lets O be overwritten, comes after this)
      }
      st = next;
    }
  } else if (warp < MMA_WARP) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(CONVERT_REGS));
    // ------------------------------------------------ convert ------------------------------------------------
    using H = Share<KIND, D>;
    const int part = warp - CONVERT_WARP, piece = H::piece(lane), my_row = 32 * part + H::row(lane);
    const int e0 = piece * (128 / KIND);                       // first coordinate
    const uint32_t from = smem_raw + (uint32_t)(my_row * F::ROW + 16 * piece), from_scale = smem_raw + S::RAW_SCALES + (uint32_t)(my_row * F::GROUPS + e0 / 32);
    const uint32_t to = smem_kv + (uint32_t)(e0 / 64) * S::KV_ATOM + 128u * (uint32_t)my_row;
    uint32_t slot = 0, round = 0, stage = 0, raw_round = 0;
    // One short loop for keys and values: the code of all roles together has to stay near the schedulers (unrolled over a whole tile, and once for
    // each of the two, a scheduler's warps waited for instructions an eighth of the time, and 2048 tokens over 16385 took 439 us for 387).
    constexpr int BATCH = H::ITERS < 2 ? H::ITERS : 2;
    for (long long n = 2 * st.count; n > 0 && !abort_flag; --n) {
      const uint32_t broken = n & 1 ? 256u : BROKEN;           // (a broken token's keys become NaN, its values stay zeros)
      if (round > 0) mbar_spin(kv_free(slot), (round - 1) & 1, &abort_flag, p.status, W_KVFREE);
      mbar_spin(raw_full(stage), raw_round & 1, &abort_flag, p.status, W_RAW);
      __syncwarp();
      const uint32_t keys = raw_keys[stage];
      uint32_t src = from + stage * S::RAW, src_scale = from_scale + stage * S::RAW, dst = to + slot * S::KV_TILE;
      int r = my_row;
#pragma unroll 1
      for (int i0 = 0; i0 < H::ITERS; i0 += BATCH) {
        uint32_t raws[BATCH][4], scales[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          load_shared16(src + (uint32_t)(i * H::RPI * F::ROW), raws[i]);
          scales[i] = load_shared1(src_scale + (uint32_t)(i * H::RPI * F::GROUPS));
        }
        if (keys != BN) {                            // some keys do not exist, or nobody sees them: zeros, whatever lies in their places
#pragma unroll
          for (int i = 0; i < BATCH; ++i) {
            const uint32_t row = (uint32_t)(r + i * H::RPI);
            if (row >= (keys & 255u) || ((keys >> (8 + row / PIECE)) & 1u) || (row >= ((keys >> 16) & 255u) && row < keys >> 24)) {
              raws[i][0] = raws[i][1] = raws[i][2] = raws[i][3] = 0u;
              scales[i] = 127u;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const uint32_t f = scales[i] == broken ? 0x7FFF7FFFu : scale_pair(scales[i], scales[i]);
#pragma unroll
          for (int u = 0; u < H::UNITS; ++u) {
            uint32_t h[4];
            if constexpr (KIND == 8) {
              e4m3_to_f16(raws[i][2 * u], h[0], h[1]);
              e4m3_to_f16(raws[i][2 * u + 1], h[2], h[3]);
            } else {
              e2m1_to_f16(raws[i][u], h[0], h[1], h[2], h[3]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = mul_f16x2(h[e], f);
            store16(dst + (uint32_t)(i * H::RPI * 128) + (uint32_t)(((e0 / 8 + u) ^ (r + i * H::RPI)) & 7) * 16u, h[0], h[1], h[2], h[3]);
          }
        }
        src += BATCH * H::RPI * F::ROW;
        src_scale += BATCH * H::RPI * F::GROUPS;
        dst += BATCH * H::RPI * 128;
        r += BATCH * H::RPI;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(raw_free(stage));
        mbar_arrive(kv_full(slot));
      }
      if (++slot == SLOTS) {
        slot = 0;
        ++round;
      }
      if (++stage == STAGES) {
        stage = 0;
        ++raw_round;
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(MMA_REGS));
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
        const Item it = make_item<CHUNK_ROWS>(p, pm, st.head, st.block);
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
          next_item(st, n);
          have = st.count > 0;
          if (have) enter();
        }
        if (have) do_s(active, j == 0);
      }
    } else if (warp == LOAD_WARP) {
      // lanes 0 .. 7: a piece of 16 keys each; the first piece of a page's part of the tile requests all of it
      const int run = min(PIECES, 1 << (p.c.shift - 4));       // pieces of the tile that lie in one page
      uint32_t stage = 0, round = 0;
      Item it;
      int n = 0, j = 0, pos = 0, page = -1;
      auto look_up = [&]() {
        pos = it.key0(st.off + j) + PIECE * lane;
        page = lane < PIECES && pos < it.s.nk ? page_of(p.c, it.seq, pos) : -1;
      };
      if (lane == 0 && p.cuts) p.cuts[blockIdx.x] = Cut{};
      auto enter = [&]() {
        it = make_item<CHUNK_ROWS>(p, pm, st.head, st.block);
        n = run_of(it);
        j = 0;
        if (lane == 0 && st.off == 0 && n < it.tiles) p.cuts[blockIdx.x] = cut_here<CHUNK_OVERHEAD>(st, it);
      };
      bool have = st.count > 0;
      if (have) {
        enter();
        look_up();
      }
      while (have && !abort_flag) {
        const uint32_t there = __ballot_sync(~0u, page >= 0);
        const int k0 = it.key0(st.off + j), exist = min(it.s.nk - k0, BN), at = pos & ((1 << p.c.shift) - 1);
        const int unseen = min(max(p.sinks - k0, 0), BN), seen = min(it.lo - k0, BN);
        const uint32_t what = (uint32_t)exist | (~there & 255u) << 8 | (seen > unseen ? (uint32_t)unseen << 16 | (uint32_t)seen << 24 : 0u);
        const bool mine = page >= 0 && lane % run == 0;
        const uint32_t keys = (uint32_t)(min(PIECES - lane, run) * PIECE);
        const uint8_t* const block = mine ? block_of(p.c, page, it.head) : nullptr;
        // pieces of a page that lie behind the sequence's end come along: the page has room for them
        const uint32_t pieces = (uint32_t)__reduce_add_sync(~0u, mine ? keys : 0u);
        const int first_piece = lane;
        // the next step's pages, while the copies are waited for
        if (++j == n) {
          next_item<CHUNK_OVERHEAD>(st, it, n);
          have = st.count > 0;
          if (have) enter();
        }
        if (have) look_up();
#pragma unroll 1
        for (int v = 0; v < 2; ++v) {
          if (round > 0) mbar_wait(raw_free(stage), (round - 1) & 1, &abort_flag, p.status, W_RAWFREE);
          __syncwarp();
          if (lane == 0) {
            raw_keys[stage] = what;
            mbar_expect_tx(raw_full(stage), pieces * (F::ROW + F::GROUPS));
          }
          __syncwarp();
          if (mine) {
            const uint32_t dst = smem_raw + stage * S::RAW;
            bulk_load(dst + (uint32_t)(first_piece * PIECE * F::ROW), block + (v ? p.c.off_v : 0u) + at * F::ROW, keys * F::ROW, raw_full(stage));
            bulk_load(dst + S::RAW_SCALES + (uint32_t)(first_piece * PIECE * F::GROUPS), block + (v ? p.c.off_vs : p.c.off_ks) + at * F::GROUPS, keys * F::GROUPS,
                      raw_full(stage));
          }
          if (++stage == STAGES) {
            stage = 0;
            ++round;
          }
        }
      }
      // copies still in flight end before the CTA does (after an abort nobody else waits for them)
      for (uint32_t s = 0; s < STAGES; ++s) {
        const uint32_t fills = round + (s < stage ? 1u : 0u);
        for (int k = 0; fills > 0 && k < (1 << 20) && !mbar_try(raw_full((int)s), (fills - 1) & 1); ++k) {}
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

template <int KIND, int D, bool WHOLE>
cudaError_t go_as(const AttnParams& p, int ctas, cudaStream_t st) {
  // (the attribute belongs to the device that is current, so it is set every time)
  const cudaError_t e = cudaFuncSetAttribute(chunk_kernel<KIND, D, WHOLE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<KIND, D>::SMEM);
  if (e != cudaSuccess) return e;
  return launch_dependent(chunk_kernel<KIND, D, WHOLE>, ctas, THREADS, Shape<KIND, D>::SMEM, st, p);
}
template <int KIND, int D>
cudaError_t go(const AttnParams& p, int ctas, cudaStream_t st) {
  return p.whole ? go_as<KIND, D, true>(p, ctas, st) : go_as<KIND, D, false>(p, ctas, st);
}

}  // namespace chunk

cudaError_t launch_chunk(const AttnParams& p, int kind, int head_dim, int ctas, cudaStream_t st) {
  if (kind == OQ_CACHE_FP8) return head_dim == 128 ? chunk::go<8, 128>(p, ctas, st) : chunk::go<8, 64>(p, ctas, st);
  return head_dim == 128 ? chunk::go<4, 128>(p, ctas, st) : chunk::go<4, 64>(p, ctas, st);
}

}  // namespace cache
}  // namespace oq
