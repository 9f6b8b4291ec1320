// Softmax attention with a sliding window and first keys that stay visible, over packed sequences.
//
//   query i of a sequence (nq queries, nk keys) stands at place p = i + nk - nq among the keys;
//   it sees key j iff  j <= p + right (right < 0: no limit)  and  (j >= p - left (left < 0: no limit) or j < sinks)
//   z_j = scale * q . k_j,   lse = log sum_j exp(z_j),   out = sum_j exp(z_j - lse) v_j     (sees nothing: 0, -inf)
//
// One pass over the keys with a running reference m and a running sum: with c = scale * log2(e) the kernel holds
//   l = sum_j 2^(c (s_j - m)),   O = sum_j 2^(c (s_j - m)) v_j
// for ANY m that keeps the powers in range, so m follows the running maximum only when that has moved by more than
// 2^SLACK; then O and l are multiplied by 2^(c (m - m')).  The sums are fp32; the powers are rounded once, to bf16, as
// the tensor cores' operand for the product with V (l sums the unrounded ones): an MMA takes both operands in one type, and V is
// bf16.  That is a choice: the result is 2.3e-3 from 64 bits (relative, over a tensor of normal values) where the output's own
// rounding is 1.66e-3; with the powers in two bf16 pieces, each multiplied with V, it was 1.66e-3, and the calls below took 377 us for 256
// (joint), 789 for 542 (streamed frame), 89 for 65 (packed requests) and 162 for 132 (one query).
//
// Bound: the tensor cores and the exponentials alike.  128 queries x 128 keys take 128^3 multiply-adds for each of the
// two products at head_dim 128 and 16384 exponentials: both about 1000 cycles of an SM.  So a CTA carries two query
// tiles: while the tensor cores multiply for one, the threads of the other exponentiate.
//
//   load warp   (1 thread)   TMA: Q tiles, then K and V tiles of 128 keys through one ring of shared-memory slots
//   2 mma warps              one per query tile: S_t = Q_t K^T into tensor memory, O_t += P_t V with P_t from tensor memory
//   2 x 4 warps              one thread per query row: S from tensor memory, mask, maximum, powers, P (bf16) over S
//
// Of a tile's 256 columns of tensor memory S has 128, over which P lies, and O the rest.  The mma warp issues P_t V of a
// key tile before the next S_t, so "S_t is there" also says that O_t holds the tiles before it.
//
// Measured (B200, head_dim 128), 4608 queries x 4608 keys x 24 heads: 222 us in bursts of 10 ms = 1.18 PFLOP/s, 0.70 of the measured
// burst rate of a library product; the power cap then holds the clock at 1.7 GHz: 239 us in 0.15 s, 252 in 2 s, 255 a call through the Python
// entry point.  A step of 2 x 128 queries x 128 keys takes ~3200 cycles, 1200 of them P V, S and their latency,
// 600 the load and the maximum, 1400 the powers, in two chains that run against each other.  Other arrangements that were measured (beside 216 us):
// S beside P and tiles of 80 keys (nothing waits for P V, but what a step costs besides is paid more often) 247 us;
// four softmax threads of which two share a row 239 us; a third of the powers as polynomials of degree 4 on the fused
// multiply-add pipe 255 us (that pipe takes as long for them); no turns at the exponentials 246 us; the maximum taken while the
// powers are made with the old reference 227 us.
//
// NaN and infinities in keys and values that a row does not see must not reach it, but 0 * NaN is NaN: a row whose
// result is not finite (checked once, at the end) is made again over what it sees, unless what it sees explains it (redo_rows).
#include <cuda_bf16.h>

#include <string>

#include "oq_internal.h"
#include "oq_sm100.cuh"

namespace oq {
namespace attn {

constexpr int THREADS = 384;              // 8 softmax warps; the load warp, two mma warps and one that only fills their group
// Registers: 384 threads start with 168 each (64512).  The softmax threads hold a row of S and grow to 216; the last
// group shrinks to 72: 256 * 216 + 128 * 72 = 64512.
constexpr int LOAD_WARP = 8, MMA_WARP = 9;
constexpr int BM = 128, BN = 128;         // query rows and keys of a tile
constexpr int MAX_SEQS = 256;
constexpr int MAX_PARTS = 32;
constexpr uint32_t COL_S = 0, COL_P = 0, COL_O = BN;           // columns of a query tile's 256: P lies over S
constexpr float SLACK = 8.f;              // powers stay below 2^8
constexpr float FAR = 65536.f;            // rows whose reference passes this (as an exponent) are made again, see below
// While a warp makes rows again the others wait for it: the limit of the waits has this for each key, nearly three times what 32 rows take.
constexpr long long REDO_CYCLES = 16384;
enum { W_Q = 40, W_QFREE = 41, W_KV = 42, W_KVFREE = 43, W_S = 44, W_P = 45, W_O = 46 };

template <int D>
struct Shape {
  static constexpr uint32_t ATOMS = D / 64;
  static constexpr uint32_t Q_ATOM = BM * 128, KV_ATOM = BN * 128;      // 64 coordinates of all rows, 128 bytes each
  static constexpr uint32_t Q_TILE = ATOMS * Q_ATOM, KV_TILE = ATOMS * KV_ATOM;
  static constexpr int SLOTS = D == 128 ? 5 : 8;
  static constexpr uint32_t SMEM = 1024 + 2 * Q_TILE + SLOTS * KV_TILE;
};

struct Params {
  const __nv_bfloat16 *Q, *K, *V;         // (the tensor maps read them; these serve the rows that are computed again)
  long long ldq, hdq, ldk, hdk, ldv, hdv;
  __nv_bfloat16* out;
  long long ldo, hdo;
  int wide_out;                           // rows of out begin on 32 bytes: whole sectors a store (packed ragged requests 63 us, in 16 bytes 68)
  float* lse;                             // [heads][total_q] or NULL
  float* part_o;                          // [parts][heads][total_q][D]: sums scaled to weights that add up to one
  float2* part_ml;                        // [parts][heads][total_q]: reference m and sum l of a part's powers
  const int *q_start, *k_start;           // n_seqs + 1, or NULL: one sequence
  int total_q, total_k, n_seqs, heads, group;
  int q_step, k_step, v_step;             // of the head coordinate in the tensor maps: 1, or 0 where one head serves all (stride 0)
  int splits;                             // runs that an item's key tiles are cut into
  int dual;                               // see below
  int parts;                              // results of a row to be joined: splits, twice as many when dual
  int left, right, sinks;
  float scale, scale_log2;
  long long max_wait;                     // cycles, see REDO_CYCLES
  int* status;
};

// What one CTA works on at a time: a block of queries of one head and a run of their key tiles.  A block is 256 queries, one
// tile of 128 after the other.  With few queries (dual) it is 128, both query tiles hold the same ones, and each takes
// every other key tile: two chains S -> softmax -> P V run where one would leave everything waiting for the other stages.
struct Item {
  int q_base, k_base;      // first query and key of the sequence
  int nq, nk;
  int q0;                  // first query of the item inside the sequence
  int rows0, rows1;        // queries of the two tiles
  int head, split;
  int tiles, n_sink, win0; // key tiles: j < n_sink -> j, else win0 + j - n_sink
  int first;               // first tile of this run
  __device__ __forceinline__ int key0(int j) const {
    j += first;
    return BN * (j < n_sink ? j : win0 + (j - n_sink));
  }
};

__device__ __forceinline__ int row_hi(const Params& p, const Item& it, int qi) {       // last visible key
  return p.right < 0 ? it.nk - 1 : min(it.nk - 1, qi + it.nk - it.nq + p.right);
}
__device__ __forceinline__ int row_lo(const Params& p, const Item& it, int qi) {       // first key of the window
  return p.left < 0 ? 0 : max(0, qi + it.nk - it.nq - p.left);
}

__device__ __forceinline__ int block_rows(const Params& p) { return p.dual ? BM : 2 * BM; }
// whether query tile t takes step j of an item that it has rows of
__device__ __forceinline__ bool takes(const Params& p, int t, int j) { return !p.dual || (j & 1) == t; }
// prefix[s]: blocks of queries before sequence s
__device__ __forceinline__ Item make_item(const Params& p, const int* prefix, int index) {
  Item it;
  it.split = 0;
  if (p.splits > 1) {
    it.split = index % p.splits;
    index /= p.splits;
  }
  const int blocks = prefix[p.n_seqs];
  it.head = index / blocks;
  int b = blocks - 1 - index % blocks;         // the last queries see the most keys under a causal mask: first
  int s = 0, e = p.n_seqs;
  while (e - s > 1) {
    const int m = (s + e) >> 1;
    if (prefix[m] <= b) s = m; else e = m;
  }
  b -= prefix[s];
  if (p.q_start) {
    it.q_base = min(max(__ldg(p.q_start + s), 0), p.total_q);
    it.nq = min(max(__ldg(p.q_start + s + 1), it.q_base), p.total_q) - it.q_base;
    it.k_base = min(max(__ldg(p.k_start + s), 0), p.total_k);
    it.nk = min(max(__ldg(p.k_start + s + 1), it.k_base), p.total_k) - it.k_base;
  } else {
    it.q_base = it.k_base = 0;
    it.nq = p.total_q;
    it.nk = p.total_k;
  }
  it.q0 = block_rows(p) * b;
  const int rows = min(block_rows(p), it.nq - it.q0);
  it.rows0 = min(rows, BM);
  it.rows1 = p.dual ? rows : rows - it.rows0;
  const int hi = row_hi(p, it, it.q0 + rows - 1), lo = row_lo(p, it, it.q0);
  it.tiles = it.n_sink = it.win0 = 0;
  if (hi >= 0) {
    it.win0 = lo / BN;
    it.n_sink = min((min(p.sinks, hi + 1) + BN - 1) / BN, it.win0);
    it.tiles = it.n_sink + hi / BN - it.win0 + 1;
  }
  it.first = 0;
  if (p.splits > 1) {
    it.first = (int)((long long)it.tiles * it.split / p.splits);
    it.tiles = (int)((long long)it.tiles * (it.split + 1) / p.splits) - it.first;
  }
  return it;
}

// two fp32 lanes in one instruction
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b, float c) {
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %4};\n mov.b64 c, {%5, %5};\n fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b), "f"(c));
}

__device__ __forceinline__ float natural_lse(const Params& p, float m, float l) {
  return l == 0.f ? -INFINITY : fmaf(m, p.scale_log2, log2f(l)) * 0.69314718055994531f;
}

// Rows `again` of a warp's 32 (row r: query qi0 + r) once more, over the keys that they see and no others.  Four rows and 8 keys at a
// time: a quarter of a key per lane for the scores, then D / 32 coordinates per lane for the values.  What bounds it are the latencies of its
// loads, which the rows share: 190 cycles for a row and a key with all 8 warps at it (two rows at a time 230, one 490).
// (Kept below the 168 registers that the kernel is launched with, without spills: a form that held 32 keys and the sums of 32 rows wanted
// twice that, with 1120 bytes of stack, and its first call ended as an illegal instruction.)
template <int D>
__device__ __noinline__ void exact_rows(const Params& p, const Item& it, int qi0, int t, uint32_t again) {
  constexpr int N = D / 32, ROWS = 4;
  const int lane = threadIdx.x & 31, hk = it.head / p.group, quarter = lane >> 3;
  const float c = p.scale_log2;
  const int nk = it.nk, tiles = it.tiles, sinks = p.sinks;
  const long long ldk = p.ldk, ldv = p.ldv;
  const __nv_bfloat16* const Q = p.Q + (long long)(it.q_base + qi0) * p.ldq + it.head * p.hdq + lane * N;
  const __nv_bfloat16 *const K = p.K + it.k_base * p.ldk + hk * p.hdk + quarter * (D / 4), *const V = p.V + it.k_base * p.ldv + hk * p.hdv + lane * N;
  while (again) {
    int row[ROWS], hi[ROWS], lo[ROWS];
    uint32_t q[ROWS][N / 2];
    float m[ROWS], l[ROWS], o[ROWS][N];            // o: the mean of the values so far (their sum may leave the range)
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      row[r] = again ? __ffs(again) - 1 : -1;
      again &= again - 1;
      hi[r] = row[r] < 0 ? -1 : row_hi(p, it, qi0 + row[r]);
      lo[r] = row_lo(p, it, qi0 + max(row[r], 0));
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) q[r][i] = __ldg(reinterpret_cast<const uint32_t*>(Q + max(row[r], 0) * p.ldq) + i);
#pragma unroll
      for (int i = 0; i < N; ++i) o[r][i] = 0.f;
    }
    for (int j = 0; j < tiles; ++j) {
      if (!takes(p, t, j)) continue;
      for (int k0 = it.key0(j), end = min(k0 + BN, nk); k0 < end; k0 += 8) {
        const int key = k0 + (lane & 7);
        uint4 k[D / 32];
        uint32_t v[8][N / 2];
        // (keys past the end are seen by no row: the last one stands in for them)
        const uint4* const kp = reinterpret_cast<const uint4*>(K + min(key, nk - 1) * ldk);
#pragma unroll
        for (int x = 0; x < D / 32; ++x) k[x] = __ldg(kp + x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const __nv_bfloat16* const vp = V + min(k0 + e, nk - 1) * ldv;
          if (N == 4) {
            const uint2 two = __ldg(reinterpret_cast<const uint2*>(vp));
            v[e][0] = two.x;
            v[e][N / 2 - 1] = two.y;
          } else {
            v[e][0] = __ldg(reinterpret_cast<const uint32_t*>(vp));
          }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          const bool see = key <= hi[r] && (key >= lo[r] || key < sinks);
          const uint32_t seen = __ballot_sync(~0u, see);
          if (!seen) continue;
          float s = 0.f;
#pragma unroll
          for (int x = 0; x < D / 32; ++x) {
            const uint32_t w[4] = {k[x].x, k[x].y, k[x].z, k[x].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {          // the quarter's pair 4 x + e of the query is in lane 8 quarter + (4 x + e) / (N / 2)
              const uint32_t u = __shfl_sync(~0u, q[r][(4 * x + e) % (N / 2)], 8 * quarter + (4 * x + e) / (N / 2));
              s = fmaf(__uint_as_float(u << 16), __uint_as_float(w[e] << 16), s);
              s = fmaf(__uint_as_float(u & 0xFFFF0000u), __uint_as_float(w[e] & 0xFFFF0000u), s);
            }
          }
          s += __shfl_xor_sync(~0u, s, 16);
          s += __shfl_xor_sync(~0u, s, 8);
          if (!see) s = -INFINITY;
          float mn = s;
#pragma unroll
          for (int d = 4; d; d >>= 1) mn = fmaxf(mn, __shfl_xor_sync(~0u, mn, d));
          mn = fmaxf(mn, m[r]);
          float w = s == -INFINITY ? 0.f : exp2f((s - mn) * c), sum = w;
#pragma unroll
          for (int d = 4; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
          const float before = l[r] * (m[r] == mn ? 1.f : exp2f((m[r] - mn) * c)), inv = before + sum == 0.f ? 0.f : 1.f / (before + sum);
          m[r] = mn;
          l[r] = before + sum;
          w *= inv;
#pragma unroll
          for (int i = 0; i < N; ++i) o[r][i] *= before * inv;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float we = __shfl_sync(~0u, w, e);
            if ((seen >> e) & 1u)
#pragma unroll
              for (int i = 0; i < N; ++i) o[r][i] = fmaf(we, __uint_as_float(i & 1 ? v[e][i / 2] & 0xFFFF0000u : v[e][i / 2] << 16), o[r][i]);
          }
        }
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (row[r] < 0) continue;
      const int qi = qi0 + row[r];
      const long long at = (long long)it.head * p.total_q + it.q_base + qi;
      if (p.parts > 1) {
        const long long part = (long long)(p.dual ? 2 * it.split + t : it.split) * p.heads * p.total_q + at;
#pragma unroll
        for (int i = 0; i < N; ++i) p.part_o[part * D + lane * N + i] = o[r][i];
        if (lane == 0) p.part_ml[part] = make_float2(m[r], l[r]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p.out[(long long)(it.q_base + qi) * p.ldo + it.head * p.hdo + lane * N + i] = __float2bfloat16_rn(o[r][i]);
        if (lane == 0 && p.lse) p.lse[at] = natural_lse(p, m[r], l[r]);
      }
    }
  }
}

// Rows `odd` of a warp's 32 (row r: query qi0 + r) have finite weights and a result that is not finite.  In most cases that is the result: a
// value that the row sees is not finite.  It is not where the only such values in a column are ones that the row does not see (0 * NaN), or
// where the sums left the range on their way.  So the values of the item's tiles are looked through (only until all is
// explained), and the rows with a column that what they see does not explain are returned: of one NaN in the values those are at most
// the rows of the blocks at the mask's edges, whatever the number of rows that see it.  (8192 x 8192 x 4 heads, causal: 0.16 ms, with one NaN
// seen by all but 300 rows 0.90 ms; with every such row made again 144 ms.)
template <int D>
__device__ uint32_t unexplained_rows(const Params& p, const Item& it, int qi0, int t, uint32_t odd) {
  constexpr int N = D / 32, AHEAD = 8;
  const int lane = threadIdx.x & 31, hk = it.head / p.group;
  // bit r of a lane's words: row r, in the lane's N columns
  uint32_t bad[N], nan_seen[N], inf_seen[N], hidden[N];
#pragma unroll
  for (int i = 0; i < N; ++i) bad[i] = nan_seen[i] = inf_seen[i] = hidden[i] = 0u;
  for (uint32_t rest = odd; rest; rest &= rest - 1) {
    const int r = __ffs(rest) - 1;
    const long long row = (long long)it.head * p.total_q + it.q_base + qi0 + r;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float v = p.parts > 1 ? p.part_o[((long long)(p.dual ? 2 * it.split + t : it.split) * p.heads * p.total_q + row) * D + lane * N + i]
                                  : __bfloat162float(p.out[(long long)(it.q_base + qi0 + r) * p.ldo + it.head * p.hdo + lane * N + i]);
      if (!(fabsf(v) < INFINITY)) bad[i] |= 1u << r;
    }
  }
  const int hi = row_hi(p, it, qi0 + lane), lo = row_lo(p, it, qi0 + lane);
  const __nv_bfloat16* const V = p.V + it.k_base * p.ldv + hk * p.hdv + lane * N;
  for (int j = 0; j < it.tiles; ++j) {
    if (!takes(p, t, j)) continue;
    const int k0 = it.key0(j), end = min(k0 + BN, it.nk);
    for (int k = k0; k < end; k += AHEAD) {
      uint32_t v[AHEAD][N / 2], some = 0;
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[e][i] = k + e < end ? *reinterpret_cast<const uint32_t*>(V + (k + e) * p.ldv + 2 * i) : 0u;
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
#pragma unroll
        for (int i = 0; i < N / 2; ++i) some |= (v[e][i] & 0x7F80u) == 0x7F80u || (v[e][i] & 0x7F800000u) == 0x7F800000u;
      if (!__any_sync(~0u, some)) continue;
      bool explained = true;
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) {
        const uint32_t sees = __ballot_sync(~0u, k + e <= hi && (k + e >= lo || k + e < p.sinks));
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t x = (i & 1 ? v[e][i / 2] >> 16 : v[e][i / 2]) & 0x7FFFu;
          if (x < 0x7F80u) continue;
          if (x > 0x7F80u) nan_seen[i] |= sees; else inf_seen[i] |= sees;
          hidden[i] |= ~sees;
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) explained &= !(bad[i] & ~nan_seen[i]);
      if (__all_sync(~0u, explained)) return 0u;
    }
  }
  uint32_t again = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) again |= bad[i] & ~nan_seen[i] & ~(inf_seen[i] & ~hidden[i]);
  return __reduce_or_sync(~0u, again);
}

// By a whole warp: rows `odd` where what they see does not explain them, and rows `sure` in any case.
template <int D>
__device__ __noinline__ void redo_rows(const Params& p, const Item& it, int qi0, int t, uint32_t odd, uint32_t sure) {
  __syncwarp();                                  // (each row was written by a lane of its own)
  const uint32_t again = sure | (odd ? unexplained_rows<D>(p, it, qi0, t, odd) : 0u);
  if (again) exact_rows<D>(p, it, qi0, t, again);
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                               const __grid_constant__ CUtensorMap map_v, const __grid_constant__ Params p) {
  using S = Shape<D>;
  constexpr int SLOTS = S::SLOTS;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[12 + 2 * SLOTS];
  __shared__ int prefix[MAX_SEQS + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const uint32_t smem_q = smem, smem_kv = smem + 2 * S::Q_TILE;
  const uint32_t b0 = smem_u32(bars);
  auto q_full = [&](int t) { return b0 + 8u * (uint32_t)t; };
  auto q_free = [&](int t) { return b0 + 8u * (uint32_t)(2 + t); };
  auto s_full = [&](int t) { return b0 + 8u * (uint32_t)(4 + t); };
  auto p_part = [&](int t) { return b0 + 8u * (uint32_t)(6 + t); };     // P of the first 96 keys is there (and O rescaled, and read at an item's end)
  auto p_full = [&](int t) { return b0 + 8u * (uint32_t)(8 + t); };     // all of P is there
  auto o_done = [&](int t) { return b0 + 8u * (uint32_t)(10 + t); };    // the item's last P V has been added: O may be read
  auto kv_full = [&](int s) { return b0 + 8u * (uint32_t)(12 + s); };
  auto kv_free = [&](int s) { return b0 + 8u * (uint32_t)(12 + SLOTS + s); };

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full(t), 1);
      mbar_init(q_free(t), 1);
      mbar_init(s_full(t), 1);
      mbar_init(p_part(t), 4);
      mbar_init(p_full(t), 4);
      mbar_init(o_done(t), 1);
    }
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(kv_full(s), 1);
      mbar_init(kv_free(s), 2);           // both mma warps, also when one of them does not use the slot (see below)
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
  if (warp == 0) {
    // blocks of queries before each sequence
    int before = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += 32) {
      const int s = s0 + lane;
      int n = 0;
      if (s < p.n_seqs) {
        n = p.total_q;
        if (p.q_start) {
          const int b = min(max(__ldg(p.q_start + s), 0), p.total_q);
          n = min(max(__ldg(p.q_start + s + 1), b), p.total_q) - b;
        }
        n = (n + block_rows(p) - 1) / block_rows(p);
      }
      int sum = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, sum, d);
        if (lane >= d) sum += o;
      }
      if (s < p.n_seqs) prefix[s] = before + sum - n;
      before += __shfl_sync(~0u, sum, 31);
    }
    if (lane == 0) prefix[p.n_seqs] = before;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int n_items = prefix[p.n_seqs] * p.heads * p.splits;
  // All roles walk over the same steps: the key tiles of this CTA's items, one after the other.
  struct Step {
    Item it;
    int index, j;          // the item's number; the key tile inside it
  };
  auto first_from = [&](Step& s, int index) {        // the first step of the first item from `index` on that has a key tile
    for (; index < n_items; index += gridDim.x) {
      s.it = make_item(p, prefix, index);
      if (s.it.tiles > 0) {
        s.index = index;
        s.j = 0;
        return true;
      }
    }
    return false;
  };
  auto next_step = [&](Step& s) {
    if (++s.j < s.it.tiles) return true;
    return first_from(s, s.index + (int)gridDim.x);
  };

  if (warp < LOAD_WARP) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ------------------------------------------------ softmax ------------------------------------------------
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t columns = tmem + ((uint32_t)((warp & 3) * 32) << 16) + 256u * (uint32_t)t;
    const uint32_t col_s = columns + COL_S, col_p = columns + COL_P, col_o = columns + COL_O;
    const float c = p.scale_log2;
    uint32_t steps = 0, items = 0;              // of this tile so far
    auto warp_wait = [&](uint32_t bar, uint32_t parity, int code) {
      mbar_spin(bar, parity, &abort_flag, p.status, code, p.max_wait);
      __syncwarp();
    };
    // Warp w of tile 0 and of tile 1 sit on the same scheduler.  They take turns: left alone they run in step, fight for the
    // exponential unit and then leave it idle together.  (The turns are counted, so no warp leaves its loops early, not
    // even when a wait has given up.)
    const int quarter = warp & 3;
    auto is_far = [&](float m) { return fabsf(m) * c > FAR && fabsf(m) < INFINITY; };
    auto turn_wait = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + 2 * quarter + t) : "memory"); };
    auto turn_pass = [&]() { asm volatile("bar.arrive %0, 64;" ::"r"(2 + 2 * quarter - t) : "memory"); };
    for (int i = blockIdx.x; i < n_items; i += gridDim.x) {
      // (What only the item's beginning and end need is not kept through the loop, whose registers hold a row of scores: the
      // end works the item out again.)
      int rows, first, hi, lo, full_hi, full_lo, tiles, n_sink, skipped;
      bool turns;
      {
        const Item it = make_item(p, prefix, i);
        rows = t ? it.rows1 : it.rows0;
        const int r0 = it.q0 + (p.dual ? 0 : t * BM);
        hi = row_hi(p, it, r0 + row);
        lo = row_lo(p, it, r0 + row);
        full_hi = row_hi(p, it, r0);                     // what every row of the tile sees
        full_lo = row_lo(p, it, r0 + rows - 1);
        tiles = it.tiles;
        n_sink = it.n_sink - it.first;                   // step j: key tile first + j, with a gap after the sinks
        skipped = it.win0 - it.n_sink;
        turns = !p.dual && it.rows1 > quarter * 32;      // both warps have rows (tile 0 is full where tile 1 has any)
        first = it.first;
      }
      if (rows == 0) continue;
      const bool idle = quarter * 32 >= rows;            // none of the warp's rows exists
      float m = -INFINITY, l = 0.f;
      // The powers are 2^(s c - m c) with m c rounded: the maximum's own power, which has to be 1, is off by half a unit of m c in the
      // exponent.  Up to FAR that is at most 2^-9, as s c itself is; beyond 2^31 it lost the power altogether.  Rows that have passed
      // FAR are made again with s - m before the scaling.  (Subtracting first here, in a branch that is never taken, cost 2 us an item.)
      bool far = false;
      const int j0 = p.dual ? t : 0, jd = p.dual ? 2 : 1;
      for (int j = j0; j < tiles; j += jd, ++steps) {
        const int k0 = BN * (first + j + (j < n_sink ? 0 : skipped));
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
        if (!(k0 + BN - 1 <= full_hi && (k0 >= full_lo || k0 + BN <= p.sinks))) {
          uint32_t some = 0;
#pragma unroll
          for (int q = 0; q < BN / 32; ++q) {
            const int b = k0 + 32 * q;
            const uint32_t keep = ones_below(hi + 1 - b) & (~ones_below(lo - b) | ones_below(p.sinks - b));
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
        if (j == j0) {
          m = mn;
          far = is_far(m);
        } else if (__any_sync(~0u, (mn - m) * c > SLACK)) {
          // (S_t of this key tile is there, so O_t holds the tiles before it and nothing is writing it)
          const float a = m == mn ? 1.f : exp2_fast((m - mn) * c);
          m = mn;
          far = far || is_far(m);
          l *= a;
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
        const float shift = m == -INFINITY ? 0.f : -m * c;
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
            pk[e] = pack_bf16(x, y);
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
      int again_i = i;
      asm volatile("" : "+r"(again_i));
      const Item it = make_item(p, prefix, again_i);
      const int qi = it.q0 + (p.dual ? 0 : t * BM) + row;
      const bool any = tiles > j0, mine = row < rows;
      if (any) warp_wait(o_done(t), items++ & 1, W_O);
      if (idle) continue;
      // (32 columns at a time in a loop that is not unrolled: straight-line code for all of them ran once an item and came from
      // far away each time, 6000 cycles for a block where this takes 2000.)
      tc_fence_after();
      const float inv = l == 0.f ? 0.f : 1.f / l;
      float probe[4] = {0.f, 0.f, 0.f, 0.f};
      const float lse = natural_lse(p, m, l);
      const long long out_row = (long long)it.head * p.total_q + it.q_base + qi;
      const long long part_row = (long long)(p.dual ? 2 * it.split + t : it.split) * p.heads * p.total_q + out_row;
      __nv_bfloat16* const dst = p.out + (long long)(it.q_base + qi) * p.ldo + it.head * p.hdo;
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        if (any) {
          tmem_load32_nowait(col_o + 32u * q, o);
          tmem_use32(o);
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const float v = l != 0.f ? __uint_as_float(o[e]) * inv : 0.f;
          probe[e & 3] = fmaf(v, 0.f, probe[e & 3]);               // stays zero while everything is finite
          o[e] = __float_as_uint(v);
        }
        if (!mine) continue;
        if (p.parts > 1) {
          uint4* const to = reinterpret_cast<uint4*>(p.part_o + part_row * D + 32 * q);
#pragma unroll
          for (int e = 0; e < 8; ++e) to[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        } else {
          uint32_t v[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = pack_bf16(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
          if (p.wide_out) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
              asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst + 32 * q + 16 * e), "r"(v[8 * e]), "r"(v[8 * e + 1]),
                           "r"(v[8 * e + 2]), "r"(v[8 * e + 3]), "r"(v[8 * e + 4]), "r"(v[8 * e + 5]), "r"(v[8 * e + 6]), "r"(v[8 * e + 7])
                           : "memory");
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) reinterpret_cast<uint4*>(dst + 32 * q)[e] = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          }
        }
      }
      if (mine) {
        if (p.parts > 1) p.part_ml[part_row] = make_float2(m, l);
        else if (p.lse) p.lse[out_row] = lse;
      }
      tc_fence_before();                        // (the next item's first P, which lets O be overwritten, comes after this)
      // (Where l is not finite, the row sees a score that is not, and has its result.)
      const uint32_t sure = __ballot_sync(~0u, mine && far);
      const uint32_t odd = __ballot_sync(~0u, mine && fabsf(l) < INFINITY && !((probe[0] + probe[1]) + (probe[2] + probe[3]) == 0.f));
      if (sure | odd) redo_rows<D>(p, it, qi - lane, t, odd & ~sure, sure);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    uint32_t slot = 0, round = 0;               // position in the ring, the same sequence in all three warps
    auto advance = [&]() {
      if (++slot == SLOTS) {
        slot = 0;
        ++round;
      }
    };
    if (warp == LOAD_WARP) {
      if (lane == 0) {
        uint32_t q_use[2] = {0, 0};
        auto load_kv = [&](const Step& s, const CUtensorMap* map, int head_step) {
          if (round > 0) mbar_wait(kv_free(slot), (round - 1) & 1, &abort_flag, p.status, W_KVFREE, p.max_wait);
          mbar_expect_tx(kv_full(slot), S::KV_TILE);
          for (uint32_t a = 0; a < S::ATOMS; ++a)
            tma_load_3d(smem_kv + slot * S::KV_TILE + a * S::KV_ATOM, map, 64 * (int)a, s.it.head / p.group * head_step, s.it.k_base + s.it.key0(s.j), kv_full(slot));
          advance();
        };
        auto load_k = [&](const Step& s) {
          if (s.j == 0) {
            for (int t = 0; t < 2; ++t) {
              if (t == 1 && (s.it.rows1 == 0 || (p.dual && s.it.tiles == 1))) continue;      // no step of this tile
              if (q_use[t] > 0) mbar_wait(q_free(t), (q_use[t] - 1) & 1, &abort_flag, p.status, W_QFREE, p.max_wait);
              ++q_use[t];
              mbar_expect_tx(q_full(t), S::Q_TILE);
              for (uint32_t a = 0; a < S::ATOMS; ++a)
                tma_load_3d(smem_q + (uint32_t)t * S::Q_TILE + a * S::Q_ATOM, &map_q, 64 * (int)a, s.it.head * p.q_step, s.it.q_base + s.it.q0 + (p.dual ? 0 : t * BM), q_full(t));
            }
          }
          load_kv(s, &map_k, p.k_step);
        };
        Step now, ahead;
        bool have = first_from(now, blockIdx.x);
        if (have) load_k(now);
        while (have && !abort_flag) {
          ahead = now;
          have = next_step(ahead);
          load_kv(now, &map_v, p.v_step);
          if (have) load_k(ahead);
          now = ahead;
        }
        // copies still in flight end before the CTA does (after an abort nobody else waits for them)
        for (uint32_t s = 0; s < SLOTS; ++s) {
          const uint32_t fills = round + (s < slot ? 1u : 0u);
          for (int n = 0; fills > 0 && n < (1 << 20) && !mbar_try(kv_full((int)s), (fills - 1) & 1); ++n) {}
        }
        for (int t = 0; t < 2; ++t)
          for (int n = 0; q_use[t] > 0 && n < (1 << 20) && !mbar_try(q_full(t), (q_use[t] - 1) & 1); ++n) {}
      }
    } else if (warp < MMA_WARP + 2) {
      const int t = warp - MMA_WARP;
      const uint32_t leader = elect_leader();       // (the whole warp runs this, one lane issues)
      constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BM >> 4) << 24);
      constexpr uint32_t IDESC_S = IDESC | ((uint32_t)(BN >> 3) << 17);
      constexpr uint32_t IDESC_O = IDESC | ((uint32_t)(D >> 3) << 17) | (1u << 16);      // V is N-major
      const uint32_t columns = tmem + 256u * (uint32_t)t;
      uint32_t q_use = 0, p_use = 0;
      auto active = [&](const Step& s) { return (t == 0 || s.it.rows1 > 0) && takes(p, t, s.j); };
      const int jd = p.dual ? 2 : 1, j0 = p.dual ? t : 0;        // this tile's steps of an item
      auto do_s = [&](const Step& s) {
        // (Both warps see every slot filled and free it, whether they use it or not: a wait tells phases apart by their
        // parity alone, so no warp may get a whole round ahead of a slot or behind it.)
        mbar_spin(kv_full(slot), round & 1, &abort_flag, p.status, W_KV, p.max_wait);
        if (!active(s)) {
          if (leader) mbar_arrive(kv_free(slot));
        } else {
          if (s.j == j0) mbar_spin(q_full(t), q_use++ & 1, &abort_flag, p.status, W_Q, p.max_wait);
          tc_fence_after();
          const uint64_t a = smem_desc(smem_q + (uint32_t)t * S::Q_TILE), b = smem_desc(smem_kv + slot * S::KV_TILE);
#pragma unroll
          for (uint32_t k = 0; k < D / 16; ++k)
            mma_ss(columns + COL_S, a + (uint64_t)((k >> 2) * (S::Q_ATOM >> 4) + 2 * (k & 3)), b + (uint64_t)((k >> 2) * (S::KV_ATOM >> 4) + 2 * (k & 3)),
                   IDESC_S, k > 0, leader);
          mma_commit(s_full(t), leader);
          mma_commit(kv_free(slot), leader);
          if (s.j + jd >= s.it.tiles) mma_commit(q_free(t), leader);       // the query tile's last S
        }
        advance();
      };
      auto do_o = [&](const Step& s) {
        mbar_spin(kv_full(slot), round & 1, &abort_flag, p.status, W_KV, p.max_wait);
        if (!active(s)) {
          if (leader) mbar_arrive(kv_free(slot));
        } else {
          // Rows of V past the end of the sequence (another one's, or a buffer's that nothing has been written to) have weights of zero, but
          // may be NaN: they are cleared, which takes less time than the weights do.  (Both mma warps write the same zeros.)
          const int valid = s.it.nk - s.it.key0(s.j);
          if (valid < BN && s.it.k_base + s.it.nk < p.total_k) {
            for (uint32_t a = 0; a < S::ATOMS; ++a)
              for (int x = valid * 8 + lane; x < BN * 8; x += 32)
                asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(smem_kv + slot * S::KV_TILE + a * S::KV_ATOM + 16u * (uint32_t)x), "r"(0u) : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
          mbar_spin(p_part(t), p_use & 1, &abort_flag, p.status, W_P, p.max_wait);
          tc_fence_after();
          const uint64_t b = smem_desc_mn(smem_kv + slot * S::KV_TILE, S::KV_ATOM, 1024);
#pragma unroll
          for (uint32_t k = 0; k < BN / 16; ++k) {
            if (k == 6) {
              mbar_spin(p_full(t), p_use++ & 1, &abort_flag, p.status, W_P, p.max_wait);
              tc_fence_after();
            }
            mma_ts(columns + COL_O, columns + COL_P + 8 * k, b + (uint64_t)(k * (2048 >> 4)), IDESC_O, s.j > j0 || k > 0, leader);
          }
          if (s.j + jd >= s.it.tiles) mma_commit(o_done(t), leader);
          mma_commit(kv_free(slot), leader);
        }
        advance();
      };
      Step now, ahead;
      bool have = first_from(now, blockIdx.x);
      if (have) do_s(now);
      while (have && !abort_flag) {
        ahead = now;
        have = next_step(ahead);
        do_o(now);
        if (have) do_s(ahead);
        now = ahead;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// Joins the parts of a row: weights l_i 2^(c (m_i - max m)) over their sum.  (Not from the parts' log sums: with scores of 1e9 those hold no
// more than m.)  One warp per (token, head).
template <int D>
__global__ void __launch_bounds__(256) attention_join_kernel(const __grid_constant__ Params p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31;
  const long long rows = (long long)p.heads * p.total_q;
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int head = (int)(row / p.total_q), tok = (int)(row % p.total_q);
  if (p.q_start && (tok < __ldg(p.q_start) || tok >= __ldg(p.q_start + p.n_seqs))) return;      // no sequence owns it: no part was written
  constexpr int AHEAD = 8;                         // parts requested together (the first ones before their weights are known)
  float v[AHEAD][N];
  auto load = [&](int s0) {
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
#pragma unroll
      for (int i = 0; i < N; ++i) v[s][i] = s0 + s < p.parts ? p.part_o[((s0 + s) * rows + row) * D + lane * N + i] : 0.f;
  };
  const float2 mine = lane < p.parts ? p.part_ml[lane * rows + row] : make_float2(-INFINITY, 0.f);
  load(0);
  float top = mine.x;
#pragma unroll
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  const float w = mine.y == 0.f ? 0.f : mine.y * exp2f((mine.x - top) * p.scale_log2);
  float total = w;
#pragma unroll
  for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(~0u, total, d);
  const float share = total == 0.f ? 0.f : w / total;      // (shares first: a sum of weights times values may leave the range)
  float o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = 0.f;
  for (int s0 = 0; s0 < p.parts; s0 += AHEAD) {
    if (s0 > 0) load(s0);
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const float ws = __shfl_sync(~0u, share, s0 + s);
      if (ws == 0.f) continue;                     // an empty split, or one whose share is below 2^-126
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = fmaf(ws, v[s][i], o[i]);
    }
  }
  __nv_bfloat16* dst = p.out + (long long)tok * p.ldo + head * p.hdo + lane * N;
#pragma unroll
  for (int i = 0; i < N; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = pack_bf16(o[i], o[i + 1]);
  if (lane == 0 && p.lse) p.lse[row] = natural_lse(p, top, total);
}

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
  return sms;
}

// Items (blocks of queries times heads) that do not fill the SMs, or fill them unevenly, are cut along their keys.  The time of a cut is
// estimated as (rounds of items over the SMs) x (steps of an item + what it costs besides, in steps); a step of a dual item is
// half as long as one of two query tiles.  (One query against 32760 keys of 40 heads: 3 runs each, one round, 114 us; 5, two rounds,
// 145 us; 7 121 us; 11 128 us.  The floor is 104 us.)
// Where the sequences have at most 128 queries on average, the better cut with dual items is set against the better one without, now
// with what the queries and the parts cost (a part is written and read for every row).  (8, 24 and 40 heads of 128; 3 to 256 key tiles; 1 to
// 32 sequences of 1 to 128 queries, 192 calls measured both ways: 0.6 % above the better one on average and 9 % at worst; dual from 16 key
// tiles on 2.7 and 30 %.  One query, 40 heads, 256 tiles: 113 us dual, 140 not; 16 queries, 8 heads, 64 tiles: 26 and 21; 32 sequences of 128
// queries, 24 heads, 20 tiles: 293 and 226.)
struct Plan {
  int splits, dual, parts;
};
Plan make_plan(long long total_q, long long total_k, int n_seqs, int heads, int left, int right, int sinks, int sms) {
  if (total_q == 0 || total_k == 0) return Plan{1, 0, 1};
  long long keys = total_k / n_seqs;
  if (left >= 0 && right >= 0) {
    const long long window = (long long)left + right + 2 * BM + sinks;
    if (window < keys) keys = window;
  }
  const long long tiles = (keys + 127) / 128;
  Plan best{1, 0, 1};
  double best_total = 1e30;
  for (int dual = 0; dual < (total_q <= (long long)BM * n_seqs ? 2 : 1); ++dual) {
    const long long rows = dual ? BM : 2 * BM, blocks = (total_q + rows / 2 * n_seqs + rows / 2 - 1) / rows;
    const long long items = (blocks < n_seqs ? n_seqs : blocks) * heads;
    double best_cost = 1e30, total = 0.0;
    int splits = 1;
    for (int n = 1; n <= MAX_PARTS / (dual ? 2 : 1) && (n == 1 || n * 4 <= tiles) && (n == 1 || items < 2LL * sms); ++n) {
      const double rounds = (double)((items * n + sms - 1) / sms), steps = (double)((tiles + n - 1) / n) * (dual ? 0.5 : 1.0);
      const double cost = rounds * (steps + (dual ? 6.0 : 3.0)) + (n > 1 ? 3.0 : 0.0);
      if (cost < best_cost * 0.97) {
        const int parts = dual ? 2 * n : n;
        best_cost = cost;
        splits = n;
        total = rounds * (steps + (dual ? 4.0 + (double)total_q / ((double)n_seqs * BM) : 3.0));
        if (parts > 1) total += 3.0 + parts * (0.2 + 2.0 * (double)total_q * heads / ((double)sms * BM));
      }
    }
    if (total < best_total) {
      best_total = total;
      best = Plan{splits, dual, dual ? 2 * splits : splits};
    }
  }
  return best;
}

template <int D>
cudaError_t launch(const Params& p, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, int sms, cudaStream_t st) {
  // (the attribute belongs to the device that is current, so it is set every time)
  cudaError_t e = cudaFuncSetAttribute(attention_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<D>::SMEM);
  if (e != cudaSuccess) return e;
  const int rows = p.dual ? BM : 2 * BM;
  const long long most = ((long long)(p.total_q + rows - 1) / rows + p.n_seqs) * p.heads * p.splits;
  e = launch_dependent(attention_kernel<D>, (int)(most < sms ? most : sms), THREADS, Shape<D>::SMEM, st, mq, mk, mv, p);
  if (e != cudaSuccess || p.parts == 1) return e;
  return launch_dependent(attention_join_kernel<D>, (int)(((long long)p.heads * p.total_q + 7) / 8), 256, 0, st, p);
}

}  // namespace attn
}  // namespace oq

using namespace oq;

static int attention_check(const oq_attention_args* a) {
  if (!a) return fail(OQ_ERR_INVALID_ARG, "oq_attention: NULL arguments");
  if (a->total_q < 0 || a->total_k < 0 || a->n_seqs < 1) return fail(OQ_ERR_INVALID_ARG, "oq_attention: bad sizes");
  if (a->total_q > (1 << 30) || a->total_k > (1 << 30)) return fail(OQ_ERR_UNSUPPORTED, "oq_attention: more than 2^30 tokens");
  if (a->n_seqs > attn::MAX_SEQS) return fail(OQ_ERR_UNSUPPORTED, "oq_attention: more than 256 sequences");
  if (a->n_heads <= 0 || a->n_kv_heads <= 0 || a->n_heads % a->n_kv_heads)
    return fail(OQ_ERR_INVALID_ARG, "oq_attention: n_heads must be a positive multiple of n_kv_heads");
  if (a->head_dim != 64 && a->head_dim != 128) return fail(OQ_ERR_UNSUPPORTED, "oq_attention: head_dim must be 64 or 128");
  if ((!a->q_start) != (!a->k_start)) return fail(OQ_ERR_INVALID_ARG, "oq_attention: q_start and k_start go together");
  if (a->n_seqs > 1 && !a->q_start) return fail(OQ_ERR_INVALID_ARG, "oq_attention: several sequences need q_start and k_start");
  if (a->sinks < 0) return fail(OQ_ERR_INVALID_ARG, "oq_attention: sinks must not be negative");
  if (!(a->scale >= 0.f) || !(a->scale < 1e30f)) return fail(OQ_ERR_INVALID_ARG, "oq_attention: scale must be positive, or 0 for 1 / sqrt(head_dim)");
  if ((long long)a->total_q * a->n_heads > (1ll << 33)) return fail(OQ_ERR_UNSUPPORTED, "oq_attention: too many rows for one launch");
  return OQ_OK;
}

// A stride is used where there is more than one token or head.  Inputs may have a head stride of 0 (one head serves all); any other stride
// that is used must reach past a head's coordinates: the tensor maps have no rows that lie over each other, and rows of the
// output that do would overwrite each other.
static bool strides_ok(long long ld, long long hd, int tokens, int heads, int head_dim, bool input) {
  return ld >= 0 && hd >= 0 && (tokens <= 1 || ld >= head_dim) && (heads <= 1 || hd >= head_dim || (input && hd == 0));
}

static attn::Plan attention_plan(const oq_attention_args* a) {
  return attn::make_plan(a->total_q, a->total_k, a->n_seqs, a->n_heads, a->left, a->right, a->sinks, attn::sm_count());
}

extern "C" {

int oq_attention_workspace_bytes(const oq_attention_args* a, size_t* bytes) {
  if (!bytes) return fail(OQ_ERR_INVALID_ARG, "oq_attention_workspace_bytes: bytes is NULL");
  *bytes = 0;
  const int rc = attention_check(a);
  if (rc != OQ_OK) return rc;
  const int n = attention_plan(a).parts;
  if (n > 1) *bytes = (size_t)n * a->n_heads * (size_t)a->total_q * (size_t)(a->head_dim + 4) * sizeof(float);
  return OQ_OK;
}

int oq_attention(const oq_attention_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = attention_check(a);
  if (rc != OQ_OK) return rc;
  if (a->total_q == 0) return OQ_OK;
  if (!a->Q || !a->out || (a->total_k > 0 && (!a->K || !a->V))) return fail(OQ_ERR_INVALID_ARG, "oq_attention: NULL buffer");
  if (!aligned16(a->Q) || !aligned16(a->K) || !aligned16(a->V) || !aligned16(a->out) || a->ldq_token % 8 || a->ldq_head % 8 ||
      a->ldk_token % 8 || a->ldk_head % 8 || a->ldv_token % 8 || a->ldv_head % 8 || a->ldo_token % 8 || a->ldo_head % 8)
    return fail(OQ_ERR_ALIGNMENT, "oq_attention: pointers must be 16-byte aligned and strides multiples of 8");
  if (!strides_ok(a->ldq_token, a->ldq_head, a->total_q, a->n_heads, a->head_dim, true) ||
      !strides_ok(a->ldk_token, a->ldk_head, a->total_k, a->n_kv_heads, a->head_dim, true) ||
      !strides_ok(a->ldv_token, a->ldv_head, a->total_k, a->n_kv_heads, a->head_dim, true) ||
      !strides_ok(a->ldo_token, a->ldo_head, a->total_q, a->n_heads, a->head_dim, false))
    return fail(OQ_ERR_INVALID_ARG, "oq_attention: strides must be at least head_dim (head strides of the inputs: or 0, one head for all)");
  attn::Params p = {};
  const attn::Plan plan = attention_plan(a);
  p.splits = plan.splits;
  p.dual = plan.dual;
  p.parts = plan.parts;
  size_t need = 0;
  rc = oq_attention_workspace_bytes(a, &need);
  if (rc != OQ_OK) return rc;
  if (need > workspace_bytes || (need && (!workspace || !aligned16(workspace))))
    return fail(OQ_ERR_NOMEM, "oq_attention: workspace of " + std::to_string(need) + " bytes (16-byte aligned) needed");
  p.Q = reinterpret_cast<const __nv_bfloat16*>(a->Q);
  p.K = reinterpret_cast<const __nv_bfloat16*>(a->K);
  p.V = reinterpret_cast<const __nv_bfloat16*>(a->V);
  p.ldq = a->ldq_token; p.hdq = a->ldq_head;
  p.ldk = a->ldk_token; p.hdk = a->ldk_head;
  p.ldv = a->ldv_token; p.hdv = a->ldv_head;
  p.out = reinterpret_cast<__nv_bfloat16*>(a->out);
  p.ldo = a->ldo_token; p.hdo = a->ldo_head;
  p.wide_out = reinterpret_cast<uintptr_t>(a->out) % 32 == 0 && a->ldo_token % 16 == 0 && a->ldo_head % 16 == 0;
  p.lse = a->lse;
  p.part_o = reinterpret_cast<float*>(workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)p.parts * a->n_heads * (size_t)a->total_q * (size_t)a->head_dim);
  p.q_start = a->q_start; p.k_start = a->k_start;
  p.total_q = a->total_q; p.total_k = a->total_k;
  p.n_seqs = a->n_seqs; p.heads = a->n_heads; p.group = a->n_heads / a->n_kv_heads;
  const int far = 1 << 30;                         // no sequence is longer
  p.left = a->left < 0 ? -1 : (a->left > far ? far : a->left);
  p.right = a->right < 0 ? -1 : (a->right > far ? far : a->right);
  p.sinks = a->sinks > far ? far : a->sinks;
  p.scale = a->scale > 0.f ? a->scale : (a->head_dim == 128 ? 0.08838834764831845f : 0.125f);
  p.scale_log2 = p.scale * 1.4426950408889634f;
  p.max_wait = WAIT_CYCLES + attn::REDO_CYCLES * a->total_k;
  p.status = device_status_word();
  if (!p.status) return fail(OQ_ERR_CUDA, "oq_attention: cannot allocate the device status word");
  CUtensorMap mq, mk, mv;
  p.q_step = a->ldq_head > 0;
  p.k_step = a->ldk_head > 0;
  p.v_step = a->ldv_head > 0;
  auto make_map = [&](CUtensorMap* map, const void* base, int heads, long long tokens, long long ld, long long hd, int rows) {
    if (hd == 0) heads = 1;                        // (one head, or one for all: the coordinate stays 0)
    const uint64_t dims[3] = {(uint64_t)a->head_dim, (uint64_t)heads, (uint64_t)tokens};
    // a stride that is not used (one head, one token) still has to be one that the encoder takes
    const uint64_t strides[2] = {(uint64_t)(heads > 1 ? hd : a->head_dim) * 2, (uint64_t)(tokens > 1 ? ld : (long long)a->head_dim * heads) * 2};
    const uint32_t box[3] = {64, 1, (uint32_t)rows};
    return encode_tensor_map_sw128(map, base, false, 3, dims, strides, box);
  };
  cudaError_t e = make_map(&mq, a->Q, a->n_heads, a->total_q, a->ldq_token, a->ldq_head, attn::BM);
  if (e == cudaSuccess && a->total_k > 0) e = make_map(&mk, a->K, a->n_kv_heads, a->total_k, a->ldk_token, a->ldk_head, attn::BN);
  if (e == cudaSuccess && a->total_k > 0) e = make_map(&mv, a->V, a->n_kv_heads, a->total_k, a->ldv_token, a->ldv_head, attn::BN);
  if (e != cudaSuccess) return cuda_fail(e, "oq_attention (tensor map)");
  if (a->total_k == 0) mk = mv = mq;               // no key tile is ever loaded
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  e = a->head_dim == 128 ? attn::launch<128>(p, mq, mk, mv, attn::sm_count(), st) : attn::launch<64>(p, mq, mk, mv, attn::sm_count(), st);
  if (e != cudaSuccess) return cuda_fail(e, "oq_attention");
  return OQ_OK;
}

}  // extern "C"
