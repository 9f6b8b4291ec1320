// Attention of new tokens over a paged cache: the entry point, the choice of kernels, and the kernel that joins the parts of items which
// were cut along their keys.
#include <atomic>
#include <chrono>
#include <string>

#include "oq_cache_attention.cuh"

namespace oq {
namespace cache {

constexpr int JOIN_WARPS = 8, JOIN_ROWS = JOIN_WARPS;

// CTA (c, y): rows 8 y .. 8 y + 7 of the item that CTA c of the kernel before began and did not finish, if there is one.  The warps that a row has beside the others' take
// every so many parts each.  (Four rows a warp, for more bytes on their way or fewer instructions: the same time with two parts a row, 2 to 8 us more with eighteen.)
template <int D>
__global__ void __launch_bounds__(32 * JOIN_WARPS) cache_join_kernel(const __grid_constant__ AttnParams p) {
  constexpr int N = D / 32;
  __shared__ float sums[JOIN_WARPS][D];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Cut cut = p.cuts[blockIdx.x];
  const int row0 = JOIN_ROWS * blockIdx.y, rows = min(JOIN_ROWS, cut.rows - row0);
  if (rows <= 0) return;
  int per_row = JOIN_WARPS;
  while (per_row > 1 && per_row * rows > JOIN_WARPS) per_row >>= 1;
  const int r = warp / per_row, share = warp % per_row;
  float acc[N], top, total, factor;
  join_row<CHUNK_ROWS, D>(p, Parts{(int)blockIdx.x, cut.parts}, row0 + r, cut.rows, share, per_row, acc, top, total, factor);
  if (per_row > 1) {
#pragma unroll
    for (int e = 0; e < N; ++e) sums[warp][N * lane + e] = acc[e];
    __syncthreads();
  }
  if (r >= rows || share) return;
  for (int w = 1; w < per_row; ++w)
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] += sums[warp + w][N * lane + e];
  write_row<D>(p, cut.q_base, cut.head, cut.r0 + row0 + r, acc, top, total, factor);
}

static cudaError_t launch_join(const AttnParams& p, int head_dim, int ctas, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas, (unsigned)(CHUNK_ROWS / JOIN_ROWS));
  cfg.blockDim = dim3(32 * JOIN_WARPS);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return head_dim == 128 ? cudaLaunchKernelEx(&cfg, cache_join_kernel<128>, p) : cudaLaunchKernelEx(&cfg, cache_join_kernel<64>, p);
}

static int sm_count() {
  static std::atomic<int> known[64];               // of each device (asked twice a call otherwise)
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if ((sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
  known[dev].store(sms, std::memory_order_relaxed);
  return sms;
}

// 48 bits that are another call's, or what lies in a workspace by chance, once in 2^48 times.
static unsigned long long next_tag() {
  static std::atomic<unsigned long long> calls{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull};
  return calls.fetch_add(0x9E3779B97F4A7C15ull, std::memory_order_relaxed) >> 16;
}

// Items of up to so many tiles are not cut along their keys: joining the parts takes longer than the tiles do.  Measured at 1, 3, 20, 80 and 300 rows, 4 and 24 heads, one
// sequence and eight: whole items are better in all of 20 at 256 keys, in 19 at 384, in 18 at 512, in 6 at 1024.  us, cut / whole: one token, 4 heads, 256 keys 8.4 / 6.2,
// 512 keys 8.4 / 8.1, 1024 keys 8.6 / 11.9; eight sequences of 20 rows, 24 heads, 512 keys 28.1 / 20.7; 300 rows, 24 heads, 512 keys 30.2 / 24.5; those that lose, 4 heads:
// 80 rows, 384 keys 13.5 / 14.9, 512 keys 13.8 / 16.8, 300 rows, 512 keys 21.0 / 23.1.  (At 1024 keys whole ones win where there are many items, eight sequences of 300 rows,
// 24 heads 100 / 90, if their lengths are alike, which is not known here.)
constexpr long long WHOLE_TILES = 4;

// Which kernels run, with how many CTAs, and what their parts take.  Nothing is known here of the sequences but their number, the tokens of all
// together and what a row of the table can hold: these bound the items and their tiles.
struct Choice {
  bool few, chunk, whole;
  int few_ctas, chunk_ctas;
  int row_cut;                   // sequences of at most so many rows go to the kernel for few
  size_t few_bytes, chunk_bytes, bytes;
};
static Choice choose(const oq_cache_attention_args* a, const View& v) {
  Choice c = {};
  const int sms = sm_count(), group = a->n_heads / v.kv_heads;
  const long long most = (long long)(a->max_q > 0 && a->max_q < a->total_q ? a->max_q : a->total_q) * group;
  c.few = most <= FEW_LIMIT || v.n_seqs > 1;
  c.chunk = most > FEW_LIMIT;
  c.row_cut = FEW_LIMIT;
  const long long tiles = v.max_len > 0 ? (v.max_len + BN - 1) / BN : 1;
  c.whole = tiles <= WHOLE_TILES;
  auto ctas = [&](int bm, int all) {
    const long long items = (((long long)a->total_q * group + bm - 1) / bm + v.n_seqs) * v.kv_heads;
    const long long most = c.whole ? items : items * tiles;
    return (int)(items >= all || most >= all ? all : most);
  };
  auto part_bytes = [&](int bm, int n) { return !c.whole && n > 1 ? n * (sizeof(Cut) + (size_t)2 * bm * ((size_t)a->cache.head_dim * sizeof(float) + sizeof(float4))) : (size_t)0; };
  if (c.few) {
    c.few_ctas = ctas(FEW_ROWS, FEW_CTAS * sms);
    c.few_bytes = part_bytes(FEW_ROWS, c.few_ctas);
  }
  c.bytes = c.few_bytes;
  if (c.chunk) {
    c.chunk_ctas = ctas(CHUNK_ROWS, sms);
    c.chunk_bytes = part_bytes(CHUNK_ROWS, c.chunk_ctas);
    c.bytes += c.chunk_bytes;
  }
  if (c.bytes) c.bytes += 32;                          // the parts begin on 32 bytes, the workspace on 16
  return c;
}

static int check(const oq_cache_attention_args* a, View* v) {
  if (!a) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: NULL arguments");
  const int rc = make_view(&a->cache, "oq_cache_attention", v);
  if (rc != OQ_OK) return rc;
  if (a->total_q < 0 || a->max_q < 0) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: bad sizes");
  if (a->n_heads <= 0 || a->n_heads % a->cache.n_kv_heads)
    return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: n_heads must be a positive multiple of the cache's heads");
  if ((long long)a->total_q * (a->n_heads / a->cache.n_kv_heads) > (1 << 30)) return fail(OQ_ERR_UNSUPPORTED, "oq_cache_attention: more than 2^30 rows");
  if (a->cache.n_seqs > 1 && !a->q_start) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: several sequences need q_start");
  if (a->sinks < 0) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: sinks must not be negative");
  if (!(a->scale >= 0.f) || !(a->scale < 1e30f)) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: scale must be positive, or 0 for 1 / sqrt(head_dim)");
  return OQ_OK;
}

}  // namespace cache
}  // namespace oq

using namespace oq;

extern "C" {

int oq_cache_attention_workspace_bytes(const oq_cache_attention_args* a, size_t* bytes) {
  if (!bytes) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention_workspace_bytes: bytes is NULL");
  *bytes = 0;
  cache::View v;
  const int rc = cache::check(a, &v);
  if (rc != OQ_OK) return rc;
  if (a->total_q > 0) *bytes = cache::choose(a, v).bytes;
  return OQ_OK;
}

int oq_cache_attention(const oq_cache_attention_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace cache;
  AttnParams p = {};
  const int rc = check(a, &p.c);
  if (rc != OQ_OK) return rc;
  if (a->total_q == 0) return OQ_OK;
  const int d = a->cache.head_dim;
  if (!a->Q || !a->out) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: NULL buffer");
  if (!aligned16(a->Q) || !aligned16(a->out) || a->ldq_token % 8 || a->ldq_head % 8 || a->ldo_token % 8 || a->ldo_head % 8)
    return fail(OQ_ERR_ALIGNMENT, "oq_cache_attention: pointers must be 16-byte aligned and strides multiples of 8");
  if (a->ldq_token < 0 || a->ldq_head < 0 || (a->total_q > 1 && a->ldo_token < d) || (a->n_heads > 1 && a->ldo_head < d))
    return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: strides of Q must not be negative, those of out at least head_dim");
  const Choice ch = choose(a, p.c);
  if (ch.bytes > workspace_bytes || (ch.bytes && (!workspace || !aligned16(workspace))))
    return fail(OQ_ERR_NOMEM, "oq_cache_attention: workspace of " + std::to_string(ch.bytes) + " bytes (16-byte aligned) needed");
  p.Q = reinterpret_cast<const __nv_bfloat16*>(a->Q);
  p.ldq = a->total_q > 1 ? a->ldq_token : 0;
  p.hdq = a->n_heads > 1 ? a->ldq_head : 0;
  p.out = reinterpret_cast<__nv_bfloat16*>(a->out);
  p.ldo = a->total_q > 1 ? a->ldo_token : 0;
  p.hdo = a->n_heads > 1 ? a->ldo_head : 0;
  if (rows_meet(0, a->total_q, a->n_heads, p.ldo, p.hdo, d)) return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: rows of out lie over each other");
  // (Q and out of different strides are only seen to meet where both begin)
  const long long apart = (reinterpret_cast<intptr_t>(a->out) - reinterpret_cast<intptr_t>(a->Q)) / 2;
  if (apart == 0 || (p.ldq == p.ldo && p.hdq == p.hdo && rows_meet(apart, a->total_q, a->n_heads, p.ldo, p.hdo, d)))
    return fail(OQ_ERR_INVALID_ARG, "oq_cache_attention: out lies over Q");
  p.wide_out = reinterpret_cast<uintptr_t>(a->out) % 32 == 0 && p.ldo % 16 == 0 && p.hdo % 16 == 0;
  p.lse = a->lse;
  p.q_start = a->q_start;
  p.total_q = a->total_q;
  p.group = a->n_heads / a->cache.n_kv_heads;
  while ((1ll << p.group_shift) < p.group) ++p.group_shift;
  p.group_mul = (uint32_t)(((1ull << 32) * ((1ull << p.group_shift) - (uint64_t)p.group)) / (uint64_t)p.group + 1);
  const int far = 1 << 30;                         // no sequence is longer
  p.left = a->left < 0 ? -1 : (a->left > far ? far : a->left);
  p.right = a->right < 0 ? -1 : (a->right > far ? far : a->right);
  p.sinks = a->sinks > far ? far : a->sinks;
  p.scale_log2 = (a->scale > 0.f ? a->scale : (d == 128 ? 0.08838834764831845f : 0.125f)) * 1.4426950408889634f;
  p.status = device_status_word();
  if (!p.status) return fail(OQ_ERR_CUDA, "oq_cache_attention: cannot allocate the device status word");
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  p.tag = next_tag();
  p.whole = ch.whole;
  auto run = [&](auto launch, int ctas, int rows, size_t at, size_t bytes) {
    if (bytes) {
      p.cuts = reinterpret_cast<Cut*>(((reinterpret_cast<uintptr_t>(workspace) + 31) & ~(uintptr_t)31) + at);
      p.arrivals = reinterpret_cast<unsigned long long*>(p.cuts);      // (the one or the other)
      p.part_ml = reinterpret_cast<float4*>(p.cuts + ctas);
      p.part_o = reinterpret_cast<float*>(p.part_ml + (size_t)2 * ctas * rows);
    } else {
      p.cuts = nullptr;                              // nothing is cut
    }
    cudaError_t err = launch(p, a->cache.kind, d, ctas, st);
    if (err == cudaSuccess && bytes && rows == CHUNK_ROWS) err = launch_join(p, d, ctas, st);
    return err;
  };
  if (ch.chunk) {
    p.row_min = ch.few ? ch.row_cut : 0;
    p.row_max = 1 << 30;
    e = run(launch_chunk, ch.chunk_ctas, CHUNK_ROWS, ch.few_bytes, ch.chunk_bytes);
  }
  if (ch.few && e == cudaSuccess) {
    p.row_min = 0;
    p.row_max = ch.chunk ? ch.row_cut : 1 << 30;
    e = run(launch_few, ch.few_ctas, FEW_ROWS, 0, ch.few_bytes);
  }
  if (e != cudaSuccess) return cuda_fail(e, "oq_cache_attention");
  return OQ_OK;
}

}  // extern "C"
