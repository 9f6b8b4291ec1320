// Attention of a few rows (new tokens times the heads of a group) over a paged cache.
//
// With up to 8 rows for a key and value head the cache is read once and every byte is used a few times, so the memory is the bound: 346 MB for one
// token over 32760 tokens of 40 heads in 8 bits, 53 us at the copy rate.  Decoding is what the SM does most of: 24 elements a cycle for the
// bytes that arrive (48 in 4 bits), an instruction a pair each for conversion and scale.  So nothing passes through shared memory: a lane reads the cache in 16
// bytes a time, decodes them in registers, and what it has is its fragment of the operand,
//   S^T [16 keys x 8 rows] = K [16 x D] Q^T,      O^T [D x 8 rows] += V^T [D x 16 keys] P^T,
// with the keys (the coordinates) as the 16 rows of an instruction and the queries as its 8 columns.  Which coordinate goes where in the
// contraction over D is free as long as Q goes the same way, and so is the order of V's coordinates in the result.  S^T has the queries in the columns and
// so has O^T: a query's maximum and factors stay in the lanes that need them, and P^T comes from S^T by one transposition of 8 x 8 numbers.
// The tensor cores' older instruction serves here: they are idle most of the time.
//
// 8 warps each take 16 keys of a tile of 128 and keep their own maximum, sum and O; they are put together at the end of an item.  A warp's
// next keys are requested as soon as the present ones are decoded, its next values likewise; two CTAs an SM have 66 KB on their way.
//
// Measured (B200, device time of captured calls): one token over 32760 of 40 heads of 128 in e4m3 65.6 us = 5.3 TB/s, 0.81 of the copy rate (the loop alone runs at 0.95 of it;
// 5 us go by before the first keys arrive, as much at the end); in e2m1 57 us = 3.1 TB/s, bound by issue and latency: 410 instructions for 16 keys x 128 a warp, 145 of
// them at half rate; 16 requests of one token, 17 to 16384 cached, 24 heads on 8, e2m1 37 us; four of five tokens 14.7 us.  With 16 rows a block (twice the sums and fragments,
// spilled) the first took 270 us; loads that the compiler could move to their use 2 us more; one CTA an SM 87 us; three, with spills, 65 (e2m1); two sums of S in
// turn, to halve its chain of products, no less.
#include <string>

#include "oq_cache_attention.cuh"

namespace oq {
namespace cache {

namespace few {

constexpr int WARPS = 8, THREADS = 32 * WARPS;

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if (N == 1) {
    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
  } else if (N == 2) {
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[N > 1 ? 1 : 0]) : "l"(p));
  } else {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(w[0]), "=r"(w[N > 1 ? 1 : 0]), "=r"(w[N > 2 ? 2 : 0]), "=r"(w[N > 3 ? 3 : 0]) : "l"(p));
  }
}

template <int N>
__device__ __forceinline__ uint32_t load_scales(const uint8_t* p) {      // (volatile, as all these: left to itself the compiler moves loads to their use)
  uint32_t x;
  if (N == 4) asm volatile("ld.global.u32 %0, [%1];" : "=r"(x) : "l"(p));
  else if (N == 2) asm volatile("ld.global.u16 %0, [%1];" : "=r"(x) : "l"(p));
  else asm volatile("ld.global.u8 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}

__device__ __forceinline__ int load_entry(const int* p) {
  int x;
  asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}

template <int KIND, int D>
struct Lane {
  using F = Format<KIND, D>;
  static constexpr int LOADS = F::ROW >= 128 ? 2 : 1;          // of a key row by one of its 4 lanes
  static constexpr int KW = F::ROW / 16 / LOADS;               // words of each
  static constexpr int VW = F::ROW / 32;                       // words of a value row by one of its 8 lanes
  // first coordinate of load x by lane t of a row: e4m3 in pieces of 16, e2m1 in one of D / 4
  __device__ static __forceinline__ int coord(int x, int t) { return KIND == 8 ? 64 * x + 16 * t : D / 4 * t; }
  static constexpr int PER_WORD = 32 / KIND;                   // coordinates of a word
};

// The loads of one step (16 keys) by a lane: rows g and g + 8 of the keys, keys 2t, 2t+1, 2t+8, 2t+9 of the values.
template <int KIND, int D>
struct Keys {
  using L = Lane<KIND, D>;
  uint32_t w[2][L::LOADS][L::KW];
  uint32_t scale[2];
};
template <int KIND, int D>
struct Values {
  uint32_t w[4][Lane<KIND, D>::VW];
  uint32_t scale[4];
};

template <int KIND, int D, bool WHOLE>
__global__ void __launch_bounds__(THREADS, FEW_CTAS) few_kernel(const __grid_constant__ AttnParams p) {
  using F = Format<KIND, D>;
  using L = Lane<KIND, D>;
  constexpr int BM = FEW_ROWS, QP = D + 8;
  static_assert(BM == 8, "the columns of an instruction");
  extern __shared__ __align__(16) unsigned char smem[];
  float* const part = reinterpret_cast<float*>(smem);                     // [WARPS][BM][D]
  __shared__ __align__(16) uint16_t q_s[BM * QP];
  __shared__ float c_s[BM], m_s[WARPS][BM], l_s[WARPS][BM];
  __shared__ Plan pm;
  __shared__ int last_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  Stretch st = plan<BM, THREADS, FEW_OVERHEAD, WHOLE>(p, pm);

  while (st.count > 0) {
    const Item it = make_item<BM>(p, pm, st.head, st.block);
    const int first = st.off, end = (int)min((long long)it.tiles, st.off + st.count);
    // The warp's steps: 16 keys of each tile, where some row may see one of them and their page is there.  The 16 lie in one page, so all of
    // a step's loads have one address and constants beside it; keys behind the sequence's end and in front of the window are in the page too, and are read (K's scores are
    // replaced and V's rows cleared).
    const int in_page = (1 << p.c.shift) - 1;
    int j = first;
    const int* const table = p.c.table + it.seq * p.c.ld_table;
    auto next_pos = [&]() {
      while (j < end) {
        const int pos = it.key0(j++) + 16 * warp;
        if (pos <= it.hi && (pos + 15 >= it.lo || pos < p.sinks)) return pos;
      }
      return -1;
    };
    auto look_up = [&](int pos) { return pos < 0 ? 0 : load_entry(table + (pos >> p.c.shift)); };
    Keys<KIND, D> k;
    Values<KIND, D> v;
    const uint32_t k_lane = (uint32_t)(g * F::ROW + L::coord(0, t) * KIND / 8), v_lane = p.c.off_v + (uint32_t)(2 * t * F::ROW + g * (F::ROW / 8));
    const uint32_t ks_lane = p.c.off_ks + (uint32_t)(g * F::GROUPS), vs_lane = p.c.off_vs + (uint32_t)(2 * t * F::GROUPS + g * F::GROUPS / 8);
    auto load_keys = [&](const uint8_t* block, int at) {
      const uint8_t *rows = block + (k_lane + (uint32_t)(at * F::ROW)), *scales = block + (ks_lane + (uint32_t)(at * F::GROUPS));
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int x = 0; x < L::LOADS; ++x) load_words(rows + 8 * r * F::ROW + (L::coord(x, 0) - L::coord(0, 0)) * KIND / 8, k.w[r][x]);
        k.scale[r] = load_scales<F::GROUPS>(scales + 8 * r * F::GROUPS);
      }
    };
    auto load_values = [&](const uint8_t* block, int at) {
      const uint8_t *rows = block + (v_lane + (uint32_t)(at * F::ROW)), *scales = block + (vs_lane + (uint32_t)(at * F::GROUPS));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = (e & 1) + 8 * (e >> 1);
        load_words(rows + key * F::ROW, v.w[e]);
        v.scale[e] = load_scales<1>(scales + key * F::GROUPS);
      }
    };
    // the next step whose page is there, looked up a step before its loads (again where it is not)
    auto settle = [&](int& pos, int page) -> const uint8_t* {
      while (pos >= 0 && (unsigned)page >= (unsigned)p.c.n_pages) {
        pos = next_pos();
        page = look_up(pos);
      }
      return pos < 0 ? nullptr : block_of(p.c, page, it.head);
    };
    int pos = next_pos();
    const int page_0 = look_up(pos);
    // ------------------------------------------------ queries ------------------------------------------------
    for (int r = warp; r < BM; r += WARPS) {
      constexpr int N = D / 32;
      float x[N];
      uint32_t largest = 0;
      const int row = it.r0 + r;
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = 0.f;
      if (r < it.rows) {
        const int i = token_of(p, row);
        const __nv_bfloat16* src = p.Q + (long long)(it.s.q_base + i) * p.ldq + (long long)(it.head * p.group + row - i * p.group) * p.hdq + N * lane;
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const uint32_t u = __ldg(reinterpret_cast<const uint32_t*>(src + e));
          x[e] = __uint_as_float(u << 16);
          x[e + 1] = __uint_as_float(u & 0xFFFF0000u);
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) largest = max(largest, __float_as_uint(x[e]) & 0x7FFFFFFFu);
      largest = __reduce_max_sync(~0u, largest);
      const RowScale rs = row_scale(largest, p.scale_log2);
#pragma unroll
      for (int e = 0; e < N; e += 2) *reinterpret_cast<uint32_t*>(q_s + r * QP + N * lane + e) = pack_f16(x[e] * rs.mul, x[e + 1] * rs.mul);
      if (lane == 0) c_s[r] = rs.c;
    }
    const uint8_t* block = settle(pos, page_0);
    if (pos >= 0) {
      load_keys(block, pos & in_page);
      load_values(block, pos & in_page);
    }
    int pos_n = next_pos(), page_n = look_up(pos_n);
    __syncthreads();
    // columns of this lane: queries 2 t and the next
    float c[2], m[2], l[2];
    int hi[2], lo[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 2 * t + e, i = token_of(p, it.r0 + r);
      c[e] = c_s[r];
      m[e] = -INFINITY;
      l[e] = 0.f;
      hi[e] = r < it.rows ? row_hi(p, it.s, i) : -1;
      lo[e] = row_lo(p, it.s, i);
    }
    const int full_hi = row_hi(p, it.s, token_of(p, it.r0)), full_lo = row_lo(p, it.s, token_of(p, it.r0 + it.rows - 1));     // what every row sees
    float o[D / 16][4];
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][e] = 0.f;

    while (pos >= 0) {
      // ---------------------------------------------- S^T = K Q^T ----------------------------------------------
      float s[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = 0.f;
#pragma unroll
      for (int x = 0; x < L::LOADS; ++x) {
        uint32_t f[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t b = (k.scale[r] >> (8 * (L::coord(x, t) / 32))) & 255u;
          f[r] = b == BROKEN ? 0x7FFF7FFFu : scale_pair(b, b);
        }
#pragma unroll
        for (int w = 0; w < L::KW; ++w) {
          uint32_t a[2][L::PER_WORD / 2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            if constexpr (KIND == 8) e4m3_to_f16(k.w[r][x][w], a[r][0], a[r][1]);
            else e2m1_to_f16(k.w[r][x][w], a[r][0], a[r][1], a[r][2], a[r][3]);
#pragma unroll
            for (int e = 0; e < L::PER_WORD / 2; ++e) a[r][e] = mul_f16x2(a[r][e], f[r]);
          }
#pragma unroll
          for (int h = 0; h < L::PER_WORD / 4; ++h) {            // (Q^T's fragment in the order in which the lanes hold the keys' coordinates)
            const uint2 b = *reinterpret_cast<const uint2*>(q_s + g * QP + L::coord(x, t) + L::PER_WORD * w + 4 * h);
            mma(s, a[0][2 * h], a[1][2 * h], a[0][2 * h + 1], a[1][2 * h + 1], b.x, b.y);
          }
        }
      }
      const uint8_t* const block_n = settle(pos_n, page_n);
      if (pos_n >= 0) load_keys(block_n, pos_n & in_page);
      // ------------------------------------------------ softmax ------------------------------------------------
      if (!(pos + 15 <= full_hi && (pos >= full_lo || pos + 16 <= p.sinks))) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = pos + g + 8 * (e >> 1);
          if (key > hi[e & 1] || (key < lo[e & 1] && key >= p.sinks)) s[e] = -INFINITY;
        }
      }
      bool over = false;
#pragma unroll
      for (int e = 0; e < 2; ++e) over |= (fmaxf(s[e], s[e + 2]) - m[e]) * c[e] > SLACK;
      if (__any_sync(~0u, over)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = fmaxf(m[e], fmaxf(s[e], s[e + 2]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
          const float a = x == m[e] ? 1.f : exp2_fast((m[e] - x) * c[e]);
          m[e] = x;
          l[e] *= a;
#pragma unroll
          for (int y = 0; y < D / 16; ++y) {
            o[y][e] *= a;
            o[y][e + 2] *= a;
          }
        }
      }
      uint32_t b[2];
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float ref = m[e & 1] == -INFINITY ? 0.f : m[e & 1];
        w[e] = exp2_fast(fmaf(s[e] - ref, c[e & 1], HEAD));
        l[e & 1] += w[e];
      }
      b[0] = transpose8(pack_f16(w[0], w[1]));
      b[1] = transpose8(pack_f16(w[2], w[3]));
      // --------------------------------------------- O^T += V^T P^T ---------------------------------------------
      if (pos + 16 > it.s.nk || (pos < it.lo && pos + 16 > p.sinks)) {       // what lies behind the end, or in front of all windows, may be anything
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = pos + 2 * t + (e & 1) + 8 * (e >> 1);
          if (key >= it.s.nk || (key < it.lo && key >= p.sinks)) {
            v.scale[e] = 127u;
#pragma unroll
            for (int w = 0; w < L::VW; ++w) v.w[e][w] = 0u;
          }
        }
      }
      const uint32_t f0 = scale_pair(v.scale[0], v.scale[1]), f1 = scale_pair(v.scale[2], v.scale[3]);
#pragma unroll
      for (int w = 0; w < L::VW; ++w) {
        // pairs of keys for each coordinate of the word: keys 2t, 2t+1 and 2t+8, 2t+9
        uint32_t a[2][L::PER_WORD];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x = v.w[2 * h][w], y = v.w[2 * h + 1][w];
          if constexpr (KIND == 8) {
            uint32_t p01, p23;
            asm("prmt.b32 %0, %1, %2, 0x5140;" : "=r"(p01) : "r"(x), "r"(y));
            asm("prmt.b32 %0, %1, %2, 0x7362;" : "=r"(p23) : "r"(x), "r"(y));
            e4m3_to_f16(p01, a[h][0], a[h][1]);
            e4m3_to_f16(p23, a[h][2], a[h][3]);
          } else {
            const uint32_t even = (x & 0x0F0F0F0Fu) | ((y << 4) & 0xF0F0F0F0u), odd = ((x >> 4) & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u);
            e2m1_to_f16(even, a[h][0], a[h][2], a[h][4], a[h][6]);
            e2m1_to_f16(odd, a[h][1], a[h][3], a[h][5], a[h][7]);
          }
#pragma unroll
          for (int e = 0; e < L::PER_WORD; ++e) a[h][e] = mul_f16x2(a[h][e], h ? f1 : f0);
        }
#pragma unroll
        for (int e = 0; e < L::PER_WORD / 2; ++e)
          mma(o[w * (L::PER_WORD / 2) + e], a[0][2 * e], a[0][2 * e + 1], a[1][2 * e], a[1][2 * e + 1], b[0], b[1]);
      }
      if (pos_n >= 0) load_values(block_n, pos_n & in_page);
      pos = pos_n;
      pos_n = next_pos();
      page_n = look_up(pos_n);
    }
    // ----------------------------------------------- the item's result -----------------------------------------------
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[e] += __shfl_xor_sync(~0u, l[e], d);
        const int r = 2 * t + e;
        if (g == 0) {
          m_s[warp][r] = m[e];
          l_s[warp][r] = l[e];
        }
        float* to = part + (warp * BM + r) * D + g * (D / 8);
#pragma unroll
        for (int y = 0; y < D / 16; ++y) *reinterpret_cast<float2*>(to + 2 * y) = make_float2(o[y][e], o[y][e + 2]);
      }
    __syncthreads();
    const bool whole = first == 0 && end == it.tiles;
    const long long slot = 2 * (long long)blockIdx.x + (first == 0 ? 1 : 0);
    constexpr int N = D / 32;
    for (int r = warp; r < it.rows; r += WARPS) {
      float top = -INFINITY, total = 0.f, acc[N];
#pragma unroll
      for (int w = 0; w < WARPS; ++w) top = fmaxf(top, m_s[w][r]);
      const float cr = c_s[r];
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float lw = l_s[w][r], a = m_s[w][r] == top ? 1.f : exp2_fast((m_s[w][r] - top) * cr);
        if (lw == 0.f) continue;                        // (saw nothing; NaN goes on)
        total = fmaf(lw, a, total);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = fmaf(part[(w * BM + r) * D + N * lane + e], a, acc[e]);
      }
      const float inv = total == 0.f ? 0.f : 1.f / total;
      total *= UNHEAD;
      if (whole) {
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] *= inv;
        write_row<D>(p, it.s.q_base, it.head, it.r0 + r, acc, top, total, c_s[r]);
      } else {
        float* dst = p.part_o + (slot * BM + r) * D + N * lane;
#pragma unroll
        for (int e = 0; e < N; ++e) dst[e] = acc[e] * inv;
        if (lane == 0) p.part_ml[slot * BM + r] = make_float4(top, total, c_s[r], 0.f);
      }
    }
    __syncthreads();
    if (!whole) {
      const Parts q = parts_of<FEW_OVERHEAD>(st, it.tiles);
      if (threadIdx.x == 0) last_s = arrive(p.arrivals + q.first, p.tag, q.parts);
      __syncthreads();
      if (last_s) {
        // as many warps a row as there are, each with every so many of its parts
        int per_row = WARPS;
        while (per_row > 1 && per_row * it.rows > WARPS) per_row >>= 1;
        const int r = warp / per_row, share = warp % per_row;
        float acc[N], top, total, factor;
        join_row<BM, D>(p, q, r, it.rows, share, per_row, acc, top, total, factor);
#pragma unroll
        for (int e = 0; e < N; ++e) part[warp * D + N * lane + e] = acc[e];
        __syncthreads();
        if (r < it.rows && share == 0) {
          for (int w = 1; w < per_row; ++w)
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += part[(warp + w) * D + N * lane + e];
          write_row<D>(p, it.s.q_base, it.head, it.r0 + r, acc, top, total, factor);
        }
        __syncthreads();
      }
    }
    next_item<FEW_OVERHEAD>(st, it, end - first);
  }
}

template <int KIND, int D>
cudaError_t go(const AttnParams& p, int ctas, cudaStream_t st) {
  const size_t smem = (size_t)WARPS * FEW_ROWS * D * sizeof(float);
  static_assert(WARPS * FEW_ROWS * D * sizeof(float) + FEW_ROWS * (2 * (D + 8) + 4 + 8 * WARPS) + sizeof(Plan) + 256 <= 48 * 1024, "what every launch may have");
  return p.whole ? launch_dependent(few_kernel<KIND, D, true>, ctas, THREADS, smem, st, p) : launch_dependent(few_kernel<KIND, D, false>, ctas, THREADS, smem, st, p);
}

}  // namespace few

cudaError_t launch_few(const AttnParams& p, int kind, int head_dim, int ctas, cudaStream_t st) {
  if (kind == OQ_CACHE_FP8) return head_dim == 128 ? few::go<8, 128>(p, ctas, st) : few::go<8, 64>(p, ctas, st);
  return head_dim == 128 ? few::go<4, 128>(p, ctas, st) : few::go<4, 64>(p, ctas, st);
}

}  // namespace cache
}  // namespace oq
