// What the kernels of attention over a paged cache share: arguments, items of work and their division among the CTAs.
//
//   query i of a sequence (nq new tokens, nk cached ones, the new ones included) stands at place p = i + nk - nq among the keys;
//   it sees key j iff  j <= p + right (right < 0: no limit)  and  (j >= p - left (left < 0: no limit) or j < sinks)  and j's page is there
//   out = sum_j softmax_j(scale * q . k_j) v_j,   lse = log sum_j exp(scale * q . k_j)
//
// The queries of all heads that share a key and value head are rows of one matrix: row r of a sequence is query r / group, head r % group of the group.
// An item is a block of BM rows of one sequence and key and value head, with the tiles of 128 keys that some row of it sees (one, if
// there are none).  All items, one after the other, are a line that is cut into as many equal stretches as there are CTAs, so the lengths may
// be of any kind: they are on the device only, and every CTA finds its own stretch from them.  The line's units are tiles, and beside an item's tiles
// as many units, in front of them, as it takes time to begin and end it (requests of a few tiles beside long ones: 113 us without them, 88 with, 85 with the present join).  Where a cut
// falls among these the item begins in the stretch behind it.  An item that lies in one stretch is
// finished there; of others each CTA writes its part.  A CTA has at most two such parts: part 0 of the item that its stretch begins inside of, and part 1 of
// the one that begins in it and goes on behind it.  Of an item of few rows who writes the last part joins them (in the order of the keys, whoever it is, so
// results do not depend on it): that saves a launch, 2 us of the 20 of four requests of five tokens.  The parts of an item of 256 rows are too long to be joined by what wrote
// one of them (2048 tokens over 16385: 416 us) and have a kernel of their own (381).
#pragma once
#include "oq_cache.cuh"
#include "oq_sm100.cuh"

namespace oq {
namespace cache {

constexpr int BN = 128;                    // keys of a tile

struct AttnParams {
  View c;
  const __nv_bfloat16* Q;
  long long ldq, hdq;
  __nv_bfloat16* out;
  long long ldo, hdo;
  int wide_out;                            // rows of out begin on 32 bytes
  float* lse;                              // [heads][total_q] or NULL
  unsigned long long* arrivals;            // few rows: [CTAs], see arrive
  unsigned long long tag;                  // of this call
  struct Cut* cuts;                        // many rows: [CTAs]: the item that the CTA's stretch ends inside of and begins at or before
  float4* part_ml;                         // [2 * CTAs][BM]: reference m, sum l of the powers 2^(c (s - m)), c
  float* part_o;                           // [2 * CTAs][BM][D]: weights that add up to one
  const int* q_start;                      // n_seqs + 1, or NULL: one sequence
  int total_q, group;
  uint32_t group_mul, group_shift;         // row / group = (mulhi(row, group_mul) + row) >> group_shift, for rows below 2^31
  int row_min, row_max;                    // this kernel takes the sequences with row_min < rows <= row_max
  int whole;                               // items are not cut
  int left, right, sinks;
  float scale_log2;                        // scale / ln 2
  int* status;
};

// An item in parts: the first is part 1 of this CTA, the others part 0 of the CTAs after it.  rows == 0: none.
struct __align__(16) Cut {
  int q_base, r0, rows, head, parts, unused[3];
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

__device__ __forceinline__ int token_of(const AttnParams& p, int row) { return (int)((__umulhi((uint32_t)row, p.group_mul) + (uint32_t)row) >> p.group_shift); }

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

// What a CTA finds out first: the sequences, the blocks before each of them, and where its stretch begins and ends.
struct Plan {
  int prefix[MAX_SEQS + 1];
  Seq seq[MAX_SEQS];
  long long sums[32];
  long long found[2], units[2];        // first unit of the block, its units
  int block[2];
};

template <int BM>
__device__ __forceinline__ Item make_item(const AttnParams& p, const Plan& m, int head, int block) {
  Item it;
  it.head = head;
  int s = 0, e = p.c.n_seqs;
  while (e - s > 1) {
    const int mid = (s + e) >> 1;
    if (m.prefix[mid] <= block) s = mid; else e = mid;
  }
  it.seq = s;
  it.s = m.seq[s];
  it.r0 = BM * (block - m.prefix[s]);
  it.rows = min(BM, it.s.nq * p.group - it.r0);
  it.hi = row_hi(p, it.s, token_of(p, it.r0 + it.rows - 1));
  it.lo = row_lo(p, it.s, token_of(p, it.r0));
  it.n_sink = it.win0 = 0;
  it.tiles = 1;
  if (it.hi >= 0) {
    it.win0 = min(it.lo, it.hi) / BN;
    it.n_sink = min((min(p.sinks, it.hi + 1) + BN - 1) / BN, it.win0);
    it.tiles = it.n_sink + it.hi / BN - it.win0 + 1;
  }
  return it;
}

// Where a CTA stands: tile `off` of an item, the first unit of that item on the line, and the tiles from there to the stretch's end.
struct Stretch {
  int head, block, off;
  int blocks;                              // of one head
  long long unit, count;
  long long all;                           // units of the line
  int ctas;                                // that share it: no more than there are units
};
__device__ __forceinline__ long long divide(long long a, long long b) {       // (the short form where it serves)
  return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

template <typename T>
__device__ __forceinline__ T warp_scan(T v) {      // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const T o = __shfl_up_sync(~0u, v, d);
    if (lane >= d) v += o;
  }
  return v;
}
// Sum over the CTA; `before`: the sum over the threads before this one.
template <int THREADS>
__device__ __forceinline__ long long block_scan(long long v, long long* sums, long long& before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long x = warp_scan(v);
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

// By the whole CTA.  OVERHEAD: units of an item beside its tiles.  WHOLE: items are not cut, a stretch begins with the first item that begins in it (a
// parameter of the kernels, as its few lines in all of them took 1.6% of 2048 tokens over 16385).  Up to 32 sequences and 32 blocks (a step of single tokens, one long chunk) every warp
// works out for itself: what is waited for is the length of a call's shortest part.
template <int BM, int THREADS, int OVERHEAD, bool WHOLE>
__device__ __forceinline__ Stretch plan(const AttnParams& p, Plan& m) {
  static_assert(THREADS >= MAX_SEQS, "a thread for each sequence");
  Stretch st = {};
  long long before, n = 0;
  const int lane = threadIdx.x & 31;
  auto blocks_of = [&](const Seq& s) {
    const int rows = s.nq * p.group;
    return rows > p.row_min && rows <= p.row_max ? (rows + BM - 1) / BM : 0;
  };
  auto units_of = [&](int b) { return b < st.blocks ? make_item<BM>(p, m, 0, b).tiles + OVERHEAD : 0; };
  if (p.c.n_seqs <= 32) {
    int mine = 0;
    if (lane < p.c.n_seqs) {
      const Seq s = get_seq(p, lane);
      mine = blocks_of(s);
      if (threadIdx.x < 32) m.seq[lane] = s;
    }
    const int sum = warp_scan(mine);
    st.blocks = __shfl_sync(~0u, sum, 31);
    if (threadIdx.x < 32) {
      m.prefix[lane] = sum - mine;
      if (lane == 0) m.prefix[p.c.n_seqs] = m.prefix[32] = st.blocks;
    }
  } else {
    if ((int)threadIdx.x < p.c.n_seqs) {
      const Seq s = get_seq(p, threadIdx.x);
      m.seq[threadIdx.x] = s;
      n = blocks_of(s);
    }
    st.blocks = (int)block_scan<THREADS>(n, m.sums, before);
    if ((int)threadIdx.x < p.c.n_seqs) m.prefix[threadIdx.x] = (int)before;
    if (threadIdx.x == 0) m.prefix[p.c.n_seqs] = st.blocks;
  }
  __syncthreads();
  if (st.blocks == 0) return st;
  // units of one head; the first round's sums are kept, as there is one round mostly
  const bool short_line = st.blocks <= 32;
  long long first, per_head, unused;
  if (short_line) {
    n = units_of(lane);
    before = warp_scan(n);
    first = per_head = __shfl_sync(~0u, before, 31);
    before -= n;
  } else {
    n = units_of(threadIdx.x);
    first = per_head = block_scan<THREADS>(n, m.sums, before);
    for (int b0 = THREADS; b0 < st.blocks; b0 += THREADS) per_head += block_scan<THREADS>(units_of(b0 + threadIdx.x), m.sums, unused);
  }
  st.all = per_head * p.c.kv_heads;
  st.ctas = (int)min((long long)gridDim.x, st.all);
  if ((int)blockIdx.x >= st.ctas) return st;
  long long at[2], head[2], found[2], units[2];
  int block[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {                    // where the stretch begins, and where the next one does
    at[i] = divide(st.all * (blockIdx.x + i), st.ctas);
    head[i] = divide(at[i], per_head);
    at[i] -= head[i] * per_head;
  }
  if (short_line) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      block[i] = __popc(__ballot_sync(~0u, before + n <= at[i] && lane < st.blocks));
      found[i] = __shfl_sync(~0u, before, block[i]);
      if (WHOLE) units[i] = __shfl_sync(~0u, n, block[i]);
    }
  } else {
    long long done = 0, total = first;
    for (int b0 = 0;;) {
      before += done;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (before <= at[i] && at[i] < before + n) {
          m.block[i] = b0 + threadIdx.x;
          m.found[i] = before;
          if (WHOLE) m.units[i] = n;
        }
      done += total;
      b0 += THREADS;
      if (b0 >= st.blocks) break;
      n = units_of(b0 + threadIdx.x);
      total = block_scan<THREADS>(n, m.sums, before);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      block[i] = m.block[i];
      found[i] = m.found[i];
      if (WHOLE) units[i] = m.units[i];
    }
  }
  // tiles before a place: units before its block less what is no tile of them, and what is behind the block's own OVERHEAD
  const long long tiles = per_head - (long long)OVERHEAD * st.blocks;
  long long number[2];
  int off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (WHOLE && at[i] > found[i]) {                 // the item is the stretch's before
      at[i] = found[i] += units[i];
      if (++block[i] == st.blocks) {
        block[i] = 0;
        ++head[i];
        at[i] = found[i] = 0;
      }
    }
    off[i] = max((int)(at[i] - found[i]) - OVERHEAD, 0);
    number[i] = head[i] * tiles + found[i] - (long long)OVERHEAD * block[i] + off[i];
  }
  st.head = (int)head[0];
  st.block = block[0];
  st.off = off[0];
  st.unit = head[0] * per_head + found[0];
  st.count = number[1] - number[0];
  return st;
}

// Which CTAs have parts of the item that the stretch stands at: parts CTAs from `first` on.  (Stretch c begins at all * c / ctas rounded down, so unit x
// is in stretch ((x + 1) * ctas - 1) / all rounded down.)
struct Parts {
  int first, parts;
};
template <int OVERHEAD>
__device__ __forceinline__ Parts parts_of(const Stretch& st, int tiles) {
  Parts q;
  q.first = (int)divide((st.unit + OVERHEAD + 1) * st.ctas - 1, st.all);
  q.parts = (int)divide((st.unit + OVERHEAD + tiles) * st.ctas - 1, st.all) - q.first + 1;
  return q;
}
// By one thread, when what it and those that it has waited for wrote of a part is written: true for the last part.  The counter needs no preparation: it
// counts only while its upper 48 bits are the call's tag, which no other call has, and anything else is replaced by no arrival.  The last one
// clears it, so that a captured call, whose tag comes again, finds it so.  (No arrival waits for another: a compare-and-swap a count took 30 us for 37.)
__device__ __forceinline__ bool arrive(unsigned long long* counter, unsigned long long tag, int parts) {
  __threadfence();
  const unsigned long long seen = *reinterpret_cast<volatile unsigned long long*>(counter);
  if (seen >> 16 != tag) atomicCAS(counter, seen, tag << 16);          // (who comes too late finds the tag there)
  const bool last = (int)(atomicAdd(counter, 1ull) & 0xFFFFu) + 1 == parts;
  if (last) {
    *reinterpret_cast<volatile unsigned long long*>(counter) = 0ull;
    __threadfence();
  }
  return last;
}
// The item that the stretch stands at begins here and goes on behind the stretch: its parts.
template <int OVERHEAD>
__device__ __forceinline__ Cut cut_here(const Stretch& st, const Item& it) {
  Cut c = {};
  c.q_base = it.s.q_base;
  c.r0 = it.r0;
  c.rows = it.rows;
  c.head = it.head;
  c.parts = (int)divide((st.unit + OVERHEAD + it.tiles) * st.ctas - 1, st.all) - (int)blockIdx.x + 1;
  return c;
}
// Behind the n tiles of an item that are in the stretch (all that are left of the item, or of the stretch).  Who asks for cuts keeps the unit too.
__device__ __forceinline__ void next_item(Stretch& st, int n) {
  st.count -= n;
  st.off = 0;
  if (++st.block == st.blocks) {
    st.block = 0;
    ++st.head;
  }
}
template <int OVERHEAD>
__device__ __forceinline__ void next_item(Stretch& st, const Item& it, int n) {
  st.unit += it.tiles + OVERHEAD;
  next_item(st, n);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
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
  // (kept above 0, since minus infinity in a place that is not seen times 0 is NaN, and below infinity, which times a score of 0 is NaN: scores beyond these ends are
  // alike, or differ by more than the powers bear, with any factor of the kind)
  r.c = fminf(fmaxf(scale_log2 * __uint_as_float((uint32_t)(127 - 14 + min(e, 127)) << 23), 0x1p-126f), 0x1.fffffep127f);
  return r;
}
// The powers of two that become the second product's fp16 operand, 2^(c (s - m)), are held times 2^HEAD: the reference m follows the maximum when that is 2^SLACK above it, so
// they stay below 2^15 (fp16 ends at 2^16), and are whole fp16 down to 2^-25 of the reference's own; what is less is rounded to 2^-36 of that.  Without HEAD, a first key that
// has 2^26 times the weight of each of 32760 others, and no value of its own, left up to 0.8 of the result out (the sum of the powers is fp32 and had all of them).  A smaller SLACK moves the
// reference more often: with 4 chunks take 0.5 to 1.4% longer than with 6 and a HEAD of 9, which has two bits less.
constexpr float SLACK = 4.f, HEAD = 11.f, UNHEAD = 1.f / 2048.f;

__device__ __forceinline__ float natural_lse(float m, float l, float c) {
  return l == 0.f ? -INFINITY : fmaf(m, c, log2f(l)) * 0.69314718055994531f;
}

// Row `row` of an item (one from `rows` on stands in for the last) from the parts of CTAs q.first .. : by a warp, its parts share, share + step, ... of them; lane l has
// coordinates N l .. of the result, and the row's reference and sum are returned.  Parts are weighed by l 2^(c (m - max m)); the first ones are requested before their
// weights are known.
template <int BM, int D>
__device__ __forceinline__ void join_row(const AttnParams& p, const Parts& q, int row, int rows, int share, int step, float (&acc)[D / 32], float& top, float& total,
                                         float& factor) {
  constexpr int N = D / 32, AHEAD = 4;
  const int lane = threadIdx.x & 31;
  auto slot = [&](int i) { return (2ll * (q.first + i) + (i == 0 ? 1 : 0)) * BM + min(row, rows - 1); };
  float v[AHEAD][N];
  auto load = [&](int i0) {
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int i = i0 + s * step;
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float2 x = i < q.parts ? __ldcg(reinterpret_cast<const float2*>(p.part_o + slot(i) * D + N * lane + e)) : make_float2(0.f, 0.f);
        v[s][e] = x.x;
        v[s][e + 1] = x.y;
      }
    }
  };
  load(share);
  const float4 ml = __ldcg(p.part_ml + slot(min(lane, q.parts - 1)));
  top = ml.x;
  factor = ml.z;
  for (int i = lane + 32; i < q.parts; i += 32) top = fmaxf(top, __ldcg(p.part_ml + slot(i)).x);
#pragma unroll
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  auto weight = [&](const float4& x) { return x.y == 0.f ? 0.f : x.y * (x.x == top ? 1.f : exp2_fast((x.x - top) * factor)); };
  const float w = lane < q.parts ? weight(ml) : 0.f;
  total = w;
  for (int i = lane + 32; i < q.parts; i += 32) total += weight(__ldcg(p.part_ml + slot(i)));
#pragma unroll
  for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(~0u, total, d);
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  for (int i0 = share; i0 < q.parts; i0 += AHEAD * step) {
    if (i0 != share) load(i0);
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int i = i0 + s * step;
      if (i >= q.parts) continue;
      const float x = (i < 32 ? __shfl_sync(~0u, w, i) : weight(__ldcg(p.part_ml + slot(i)))) * inv;
      if (x == 0.f) continue;
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] = fmaf(x, v[s][e], acc[e]);
    }
  }
}
// Row r of a sequence whose queries begin at q_base, for a key and value head: its result, by a warp.
template <int D>
__device__ __forceinline__ void write_row(const AttnParams& p, int q_base, int kv_head, int r, const float (&acc)[D / 32], float top, float total, float factor) {
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31, tok = token_of(p, r), i = q_base + tok, head = kv_head * p.group + r - tok * p.group;
  __nv_bfloat16* dst = p.out + (long long)i * p.ldo + head * p.hdo + N * lane;
#pragma unroll
  for (int e = 0; e < N; e += 2) *reinterpret_cast<uint32_t*>(dst + e) = pack_bf16(acc[e], acc[e + 1]);
  if (lane == 0 && p.lse) p.lse[(long long)head * p.total_q + i] = natural_lse(top, total, factor);
}

// kernels (a file each)
cudaError_t launch_few(const AttnParams& p, int kind, int head_dim, int ctas, cudaStream_t st);
cudaError_t launch_chunk(const AttnParams& p, int kind, int head_dim, int ctas, cudaStream_t st);
constexpr int FEW_ROWS = 8, CHUNK_ROWS = 256;      // rows of their items
constexpr int FEW_OVERHEAD = 2, CHUNK_OVERHEAD = 4;       // what an item takes beside its tiles, in tiles
constexpr int FEW_CTAS = 2;                         // of an SM
// Rows up to which a sequence goes to the kernel for few, which reads the cache once for 8 of them where the other reads it once for 256 but takes
// longer to begin.  us, kernel for few / for chunks, e4m3: 16384 keys x 40 heads, 8 rows 40 / 85, 16 rows 67 / 85, 24 rows 92 / 86, 32 rows 121 / 86;
// 4096 keys x 8 heads, 24 rows 15 / 19, 40 rows 17 / 19, 64 rows 21 / 20; 16384 keys x 8 heads, 24 rows 28 / 31, 40 rows 37 / 31, 64 rows 51 / 33.
constexpr int FEW_LIMIT = 24;

}  // namespace cache
}  // namespace oq
