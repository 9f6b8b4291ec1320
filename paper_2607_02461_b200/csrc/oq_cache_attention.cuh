// What the kernels of attention over a paged cache share: arguments, items of work and their division among the CTAs.
//
//   query i of a sequence (nq new tokens, nk cached ones, the new ones included) stands at place p = i + nk - nq among the keys;
//   it sees key j iff  j <= p + right (right < 0: no limit)  and  (j >= p - left (left < 0: no limit) or j < sinks)  and j's page is there
//   out = sum_j softmax_j(scale * q . k_j) v_j,   lse = log sum_j exp(scale * q . k_j)
//
// The queries of all heads that share a key and value head are rows of one matrix: row r of a sequence is query r / group, head r % group of the group.
// An item is a block of BM rows of one sequence and key and value head, with the tiles of 128 keys that some row of it sees (one, if
// there are none).  All items' tiles, one after the other, are a line that is cut into as many equal stretches as there are CTAs, so the lengths may
// be of any kind: they are on the device only, and every CTA finds its own stretch from them.  An item that lies in one stretch is
// finished there; of others each CTA writes its part, and a second kernel joins them.  A CTA has at most two such parts: of the item that its stretch begins
// inside of, and of the one that it ends inside of.
#pragma once
#include "oq_cache.cuh"

namespace oq {
namespace cache {

constexpr int BN = 128;                    // keys of a tile

struct AttnParams {
  View c;
  const __nv_bfloat16* Q;
  long long ldq, hdq;
  __nv_bfloat16* out;
  long long ldo, hdo;
  float* lse;                              // [heads][total_q] or NULL
  float* part_o;                           // [2 * CTAs][BM][D]: weights that add up to one
  float4* part_ml;                         // [2 * CTAs][BM]: reference m, sum l of the powers 2^(c (s - m)), c
  const int* q_start;                      // n_seqs + 1, or NULL: one sequence
  int total_q, group, ctas;
  int row_min, row_max;                    // this kernel takes the sequences with row_min < rows <= row_max
  int left, right, sinks;
  float scale, scale_log2;
  int* status;
};

struct Seq {
  int q_base, nq, nk;
};
__device__ __forceinline__ Seq get_seq(const AttnParams& p, int s) {
  Seq q;
  q.q_base = 0;
  q.nq = p.total_q;
  if (p.q_start) {
    q.q_base = min(max(__ldg(p.q_start + s), 0), p.total_q);
    q.nq = min(max(__ldg(p.q_start + s + 1), q.q_base), p.total_q) - q.q_base;
  }
  q.nk = seq_len(p.c, s);
  return q;
}

struct Item {
  Seq s;
  int seq, head;                           // key and value head
  int r0, rows;                            // first row, rows of the block (1 .. BM)
  int hi, lo;                              // last and first key of the window that some row sees
  int tiles, n_sink, win0;                 // key tiles: j < n_sink -> j, else win0 + j - n_sink
  __device__ __forceinline__ int key0(int j) const { return BN * (j < n_sink ? j : win0 + (j - n_sink)); }
};
__device__ __forceinline__ int row_hi(const AttnParams& p, const Seq& s, int i) {
  return p.right < 0 ? s.nk - 1 : min(s.nk - 1, i + s.nk - s.nq + p.right);
}
__device__ __forceinline__ int row_lo(const AttnParams& p, const Seq& s, int i) { return p.left < 0 ? 0 : max(0, i + s.nk - s.nq - p.left); }

// prefix[s]: blocks before sequence s
template <int BM>
__device__ __forceinline__ Item make_item(const AttnParams& p, const int* prefix, int head, int block) {
  Item it;
  it.head = head;
  int s = 0, e = p.c.n_seqs;
  while (e - s > 1) {
    const int m = (s + e) >> 1;
    if (prefix[m] <= block) s = m; else e = m;
  }
  it.seq = s;
  it.s = get_seq(p, s);
  it.r0 = BM * (block - prefix[s]);
  it.rows = min(BM, it.s.nq * p.group - it.r0);
  it.hi = row_hi(p, it.s, (it.r0 + it.rows - 1) / p.group);
  it.lo = row_lo(p, it.s, it.r0 / p.group);
  it.n_sink = it.win0 = 0;
  it.tiles = 1;
  if (it.hi >= 0) {
    it.win0 = min(it.lo, it.hi) / BN;
    it.n_sink = min((min(p.sinks, it.hi + 1) + BN - 1) / BN, it.win0);
    it.tiles = it.n_sink + it.hi / BN - it.win0 + 1;
  }
  return it;
}

struct PlanMemory {
  int prefix[MAX_SEQS + 1];
  long long sums[32];
  int block, off;
};
// A position on the line of all tiles (heads, then sequences, then blocks, then tiles) and the tiles from there to the stretch's end.
struct Stretch {
  int head, block, off;
  long long count;
  int blocks;                              // of one head
};

// Sum over the CTA; `before`: the sum over the threads before this one.
template <int THREADS>
__device__ __forceinline__ long long block_scan(long long v, long long* sums, long long& before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long o = __shfl_up_sync(~0u, x, d);
    if (lane >= d) x += o;
  }
  __syncthreads();
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  long long total = 0;
  before = x - v;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += sums[w];
    total += sums[w];
  }
  return total;
}

// Position `at` of the line (its tiles numbered through) as head, block and tile; by the whole CTA.
template <int BM, int THREADS>
__device__ __forceinline__ void find_place(const AttnParams& p, PlanMemory& m, long long per_head, long long at, int& head, int& block, int& off) {
  const int blocks = m.prefix[p.c.n_seqs];
  head = (int)(at / per_head);
  const long long r = at - head * per_head;
  long long done = 0;
  for (int b0 = 0; b0 < blocks && done <= r; b0 += THREADS) {
    const int b = b0 + threadIdx.x;
    const long long n = b < blocks ? make_item<BM>(p, m.prefix, 0, b).tiles : 0;
    long long before;
    const long long total = block_scan<THREADS>(n, m.sums, before);
    before += done;
    if (n > 0 && before <= r && r < before + n) {
      m.block = b;
      m.off = (int)(r - before);
    }
    done += total;
  }
  __syncthreads();
  block = m.block;
  off = m.off;
}

// Blocks before each sequence, and the tiles of one head; by the whole CTA.
template <int BM, int THREADS>
__device__ __forceinline__ long long measure_line(const AttnParams& p, PlanMemory& m) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int before = 0;
    for (int s0 = 0; s0 < p.c.n_seqs; s0 += 32) {
      const int s = s0 + lane;
      int n = 0;
      if (s < p.c.n_seqs) {
        const int rows = get_seq(p, s).nq * p.group;
        if (rows > p.row_min && rows <= p.row_max) n = (rows + BM - 1) / BM;
      }
      int sum = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, sum, d);
        if (lane >= d) sum += o;
      }
      if (s < p.c.n_seqs) m.prefix[s] = before + sum - n;
      before += __shfl_sync(~0u, sum, 31);
    }
    if (lane == 0) m.prefix[p.c.n_seqs] = before;
  }
  __syncthreads();
  const int blocks = m.prefix[p.c.n_seqs];
  long long n = 0, unused;
  for (int b = threadIdx.x; b < blocks; b += THREADS) n += make_item<BM>(p, m.prefix, 0, b).tiles;
  return block_scan<THREADS>(n, m.sums, unused);
}

__device__ __forceinline__ long long stretch_begin(const AttnParams& p, long long all, int cta) { return all * cta / p.ctas; }

template <int BM, int THREADS>
__device__ __forceinline__ Stretch plan(const AttnParams& p, PlanMemory& m) {
  Stretch st;
  const long long per_head = measure_line<BM, THREADS>(p, m), all = per_head * p.c.kv_heads;
  st.blocks = m.prefix[p.c.n_seqs];
  const long long at = stretch_begin(p, all, blockIdx.x);
  st.count = stretch_begin(p, all, blockIdx.x + 1) - at;
  st.head = st.block = st.off = 0;
  if (st.count > 0) find_place<BM, THREADS>(p, m, per_head, at, st.head, st.block, st.off);
  return st;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// The queries are bf16 and the tensor cores' operand is fp16, of more digits and a smaller range: a row is multiplied by the power of two
// that brings its largest magnitude into [2^14, 2^15), and the row's factor c takes it back.  What lies 2^-29 below that or lower is rounded, at 2^-39
// of the largest at most.  (The largest as its bits without the sign; rows with NaN or infinity stay what they are: NaN in all products.)
struct RowScale {
  float mul, c;
};
__device__ __forceinline__ RowScale row_scale(uint32_t largest, float scale_log2) {
  const int e = max((int)(largest >> 23) - 127, -100);
  RowScale r;
  r.mul = largest >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)(127 + 14 - e) << 23);
  r.c = scale_log2 * __uint_as_float((uint32_t)(127 - 14 + min(e, 127)) << 23);
  return r;
}
// Scores of 2^26 and more in the exponent: there a product c s of 24 digits is off by more than the powers bear.  With a smaller c the largest
// score still has all the weight (others differ from it by 2^-24 of it at least, and still fall short by units), and nothing overflows.
constexpr float FAR = 67108864.f;
__device__ __forceinline__ float tame(float c, float m) { return fabsf(m) * c > FAR && fabsf(m) < INFINITY ? FAR / fabsf(m) : c; }

__device__ __forceinline__ float natural_lse(float m, float l, float c) {
  return l == 0.f ? -INFINITY : fmaf(m, c, log2f(l)) * 0.69314718055994531f;
}

// kernels (a file each)
cudaError_t launch_few(const AttnParams& p, int kind, int head_dim, cudaStream_t st);
cudaError_t launch_chunk(const AttnParams& p, int kind, int head_dim, cudaStream_t st);
constexpr int FEW_ROWS = 16, CHUNK_ROWS = 256;      // rows of their items
constexpr int FEW_CTAS = 2;                         // of an SM
constexpr int FEW_LIMIT = 32;                       // rows up to which a sequence goes to the kernel for few

}  // namespace cache
}  // namespace oq
