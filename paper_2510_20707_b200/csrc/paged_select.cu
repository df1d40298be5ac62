// Which pages of the paged cache a query attends to (score and order: include/mixkv.h).
//
// Score.  Lane l holds dimensions 4 l .. 4 l + 3 of the pages' bounds; of q max(q, 0) and min(q, 0) lie in shared memory.  Of a term's
// two products with them one is zero, the other exact (11 + 6 bits), so that two neighbouring terms and their sum are one product and
// three multiply-adds, rounded once; dimensions 0, 1 and 2, 3 of a lane go in the halves of one instruction.  The next sum is
// inside the lane, five are across lanes; these are done for 32 (page, query row)
// pairs at a time, every exchange halving the number of sums a lane still holds (31 exchanges for 32 sums, not 160).
//
// A cluster has one (sequence, KV head): its warps score runs of pages, four at a time, the scores go as order-preserving
// words into the first CTA's shared memory, and that CTA lists the `top` largest.
//
// What bounds it: the longest head.  32 heads of 16001 to 65536 rows in pages of 32 (40 800 pages, seven query heads) take 21 us: 5 to
// start, 14 to score the longest with four CTAs (512 pages a head 3.7 us, 3600 clocks a step of sixteen warps, instructions issued in
// 70 % of them), 2 to find the threshold; the multiprocessors work for half of that time.  8 heads of 131072 rows in pages
// of 64, four query heads: 11.  Equal runs of pages of all heads in a kernel of their own, through memory, took as long, and 1 us
// more where there are few pages; clusters of eight CTAs with 256 threads 24, of 128 threads 33, of 512, more than fit at once, 27.
// Lanes that choose between their sums instead of taking the rows in their own order, and one dimension to an instruction: 22.5.
// Query rows in registers, bounds asked for further ahead, q without its parts (fewer reads of shared memory, more instructions):
// level or slower.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace mixkv {
namespace {

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr int kSelBins = 2 * kSelThreads;
// Query rows at a time, and pages of a warp at a time: 32 sums.
__host__ __device__ constexpr int rows_at_once(const int R) { return R <= 4 ? 4 : 8; }
__host__ __device__ constexpr int padded_rows(const int R) { return (R + rows_at_once(R) - 1) / rows_at_once(R) * rows_at_once(R); }
constexpr uint32_t kKeyForced = 0xffffffffu, kKeyNan = 0xfffffffeu;   // (no number has either)

struct SelArgs {
  PagePool p;
  const void* q;
  long long q_batch, q_token;
  int T, G, R;
  Divider by_group;
  int max_rows, pages;     // most pages of a head: room for its keys
  int top, first, last;
  int *list, *counts;
};

__device__ __forceinline__ uint32_t key_of(float x) {   // larger scores have larger words; NaN above all numbers
  if (x != x) return kKeyNan;
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0 and 0 are one score)
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Sums of v[i] over all lanes, neighbouring lanes first; v[kPages * r + i] holds a term of page i and query row r ^ row_of(lane).
// Every halving of the query rows keeps the lower half: what a lane gives there is its neighbour's.  Afterwards v[0] is that of
// row_of(lane) and of the page whose bits are the lane's upper ones, reversed.
template <int RP>
__device__ __forceinline__ float sum_each(float (&v)[32], const int lane) {
#pragma unroll
  for (int o = 1, n = 16; o < 32; o <<= 1, n >>= 1) {
    if (o < RP) {
#pragma unroll
      for (int i = 0; i < n; ++i) v[i] = v[i] + __shfl_xor_sync(0xffffffffu, v[i + n], o);
    } else {
      const bool odd = lane & o;
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float give = odd ? v[i] : v[i + n], keep = odd ? v[i + n] : v[i];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
  }
  return v[0];
}
template <int RP>
__device__ __forceinline__ int row_of(const int lane) { return (int)(__brev(lane) >> 27) / (32 / RP); }

// Sum of x over the CTA's threads before this one (exclusive); *total: of all.  sums: a word per warp.
__device__ __forceinline__ uint32_t block_before(const uint32_t x, uint32_t* sums, uint32_t* total, const int lane, const int warp) {
  uint32_t upto = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  const uint32_t other = lane < kSelWarps ? sums[lane] : 0u;
  uint32_t before = lane < warp ? other : 0u, all = other;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, o);
    all += __shfl_xor_sync(0xffffffffu, all, o);
  }
  *total = all;
  return before + upto - x;
}

// Words of pages begin .. end - 1 of a unit that has `pages`, by one warp; the next pages' bounds are on their way meanwhile.
template <int RP>
__device__ __forceinline__ void score_run(const SelArgs& a, const int* table, const int pages, const int begin, const int end,
                                          const float4* qs, uint32_t* keys) {
  constexpr int kPages = 32 / RP;
  const int lane = threadIdx.x & 31, mine = row_of<RP>(lane);
  // Bounds as they lie in memory, dimensions 4 lane .. + 3.  Of four pages at a time there is room for the next ones; eight are
  // asked for again where they were.
  constexpr int kSets = RP == 8 ? 2 : 1;
  uint2 lo[kSets][kPages], hi[kSets][kPages];
  int ids = begin + lane < end ? fresh(table + begin + lane) : -1;     // of 32 pages from the last multiple of 32
  auto fetch = [&](const int p0, uint2 (&to_lo)[kPages], uint2 (&to_hi)[kPages]) {
#pragma unroll
    for (int i = 0; i < kPages; ++i) {
      const int id = __shfl_sync(0xffffffffu, ids, (p0 - begin + i) & 31);
      to_lo[i] = to_hi[i] = make_uint2(0, 0);    // (a page outside the pool scores zero)
      if (p0 + i < end && id >= 0 && id < a.p.num_pages) {
        const __half* src = a.p.bounds + (long long)id * 2 * kHeadDim + 4 * lane;
        to_lo[i] = fresh(reinterpret_cast<const uint2*>(src)), to_hi[i] = fresh(reinterpret_cast<const uint2*>(src + kHeadDim));
      }
    }
  };
  fetch(begin, lo[kSets - 1], hi[kSets - 1]);
  float4 up4[4], dn4[4];
  if constexpr (RP == 4) {
#pragma unroll
    for (int r = 0; r < 4; ++r) up4[r] = qs[(r ^ mine) * 64 + lane], dn4[r] = qs[(r ^ mine) * 64 + 32 + lane];
  }
  for (int p0 = begin; p0 < end; p0 += kPages) {
    uint32_t best = 0;
    const bool more = p0 + kPages < end;
    if (more && (p0 + kPages - begin) % 32 == 0) ids = p0 + kPages + lane < end ? fresh(table + p0 + kPages + lane) : -1;
    if constexpr (kSets == 2) {
#pragma unroll
      for (int i = 0; i < kPages; ++i) lo[0][i] = lo[1][i], hi[0][i] = hi[1][i];
      if (more) fetch(p0 + kPages, lo[1], hi[1]);
    }
#pragma unroll 1
    for (int r0 = 0; r0 < padded_rows(a.R); r0 += RP) {
      float v[32];
      // neighbouring terms of dimensions 0 and 2, then 1 and 3
      auto term = [&](const float4& up, const float4& dn, const f32x2 (&l)[2], const f32x2 (&g)[2]) {
        f32x2 x = fma2(pack2(up.x, up.y), g[0], mul2(pack2(dn.x, dn.y), l[0]));
        x = fma2(pack2(up.z, up.w), g[1], fma2(pack2(dn.z, dn.w), l[1], x));
        float a, b;
        unpack2(x, a, b);
        return __fadd_rn(a, b);
      };
      auto widen = [&](const uint2& w, f32x2 (&x)[2]) {
        const float2 p = widen2<__half>(w.x), q = widen2<__half>(w.y);
        x[0] = pack2(p.x, q.x), x[1] = pack2(p.y, q.y);
      };
      if constexpr (RP == 4) {     // the query rows stay in registers, a page is widened at a time
#pragma unroll
        for (int i = 0; i < kPages; ++i) {
          f32x2 l[2], g[2];
          widen(lo[0][i], l), widen(hi[0][i], g);
#pragma unroll
          for (int r = 0; r < RP; ++r) v[kPages * r + i] = term(up4[r], dn4[r], l, g);
        }
      } else {     // four pages stay widened, a query row is read at a time (read again for every page they were 256 of 450 clocks)
        f32x2 l[kPages][2], g[kPages][2];
#pragma unroll
        for (int i = 0; i < kPages; ++i) widen(lo[0][i], l[i]), widen(hi[0][i], g[i]);
#pragma unroll
        for (int r = 0; r < RP; ++r) {
          const float4 up = qs[(r0 + (r ^ mine)) * 64 + lane], dn = qs[(r0 + (r ^ mine)) * 64 + 32 + lane];
#pragma unroll
          for (int i = 0; i < kPages; ++i) v[kPages * r + i] = term(up, dn, l[i], g[i]);
        }
      }
      if (kSets == 1 && more) fetch(p0 + kPages, lo[0], hi[0]);      // (RP == 4: there is one round of query rows)
      uint32_t k = key_of(sum_each<RP>(v, lane));
#pragma unroll
      for (int o = 1; o < RP; o <<= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
      best = max(best, k);
    }
    const int p = p0 + (int)(__brev(lane) >> 27) % kPages;
    if (lane % RP == 0 && p < end) keys[p] = p < a.first || p >= pages - a.last ? kKeyForced : best;
  }
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads, 1) k_paged_select(const SelArgs a) {
  extern __shared__ __align__(16) unsigned char sm[];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), crank = (int)cluster.block_rank(), u = cluster_id();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = a.p.by_heads.div(u), h = u - b * a.p.H;
  float4* qs = reinterpret_cast<float4*>(sm);                    // [R padded][2][32]: max(q, 0), min(q, 0), dimensions 0, 2, 1, 3 of a lane
  uint32_t* keys = reinterpret_cast<uint32_t*>(qs + padded_rows(a.R) * 64);   // [pages], the first CTA's
  __shared__ uint32_t hist[kSelBins];
  __shared__ uint32_t sums[2][kSelWarps];
  __shared__ uint32_t found[2];
  pdl_wait();
  for (int e = tid; e < padded_rows(a.R) * 32; e += kSelThreads) {
    const int r = min(e >> 5, a.R - 1);      // (the rows of the padding repeat the last: a maximum does not mind)
    const int token = a.by_group.div(r);
    const T* src = static_cast<const T*>(a.q) + b * a.q_batch + token * a.q_token +
                   (long long)(h * a.G + r - token * a.G) * kHeadDim + 4 * (e & 31);
    const uint2 w = fresh(reinterpret_cast<const uint2*>(src));
    float2 x = widen2<T>(w.x), y = widen2<T>(w.y);
    // (a NaN stays one in both parts; an infinity becomes one, whatever the bounds that it would meet)
    auto known = [](float z) { return fabsf(z) < INFINITY ? z : NAN; };
    x.x = known(x.x), x.y = known(x.y), y.x = known(y.x), y.y = known(y.y);
    auto up = [](float z) { return z < 0.f ? 0.f : z; };
    auto down = [](float z) { return z > 0.f ? 0.f : z; };
    qs[(e >> 5) * 64 + (e & 31)] = make_float4(up(x.x), up(y.x), up(x.y), up(y.y));
    qs[(e >> 5) * 64 + 32 + (e & 31)] = make_float4(down(x.x), down(y.x), down(x.y), down(y.y));
  }
  int n = min(a.p.rows[u], a.max_rows);
  n = (int)min((long long)n, (long long)a.p.max_pages * a.p.page_rows);
  const int pages = n <= 0 ? 0 : min(a.p.by_rows.div(n + a.p.page_rows - 1), a.pages);
  const int* table = a.p.table + (long long)u * a.p.max_pages;
  const int at_once = 32 / rows_at_once(a.R), share = (pages + S * kSelWarps - 1) / (S * kSelWarps);
  const int run = (share + at_once - 1) / at_once * at_once, begin = (crank * kSelWarps + warp) * run;
  uint32_t* keys0 = cluster.map_shared_rank(keys, 0);
  if (S > 1) cluster.sync();     // the first CTA runs
  else __syncthreads();
  if (begin < pages) {
    if (a.R <= 4) score_run<4>(a, table, pages, begin, min(begin + run, pages), qs, keys0);
    else score_run<8>(a, table, pages, begin, min(begin + run, pages), qs, keys0);
  }
  if (S > 1) cluster.sync();
  else __syncthreads();
  // (the next kernel's CTAs come now, spread over the GPU: at the start they would have crowded the multiprocessors without a cluster)
  pdl_launch_dependents();
  if (crank) return;

  // The `top`-th largest word: keys between `low` and `high` are counted in bins, the bin that holds it is taken apart next, until
  // a bin's lower end separates as many as are wanted, or the bin is one word.  A thread has a run of pages.
  const int take = min(a.top, pages), each = (pages + kSelThreads - 1) / kSelThreads;
  const int p0 = min(tid * each, pages), p1 = min(p0 + each, pages);
  uint32_t low = 0xffffffffu, high = 0;       // of all keys
  for (int p = p0; p < p1; ++p) low = min(low, keys[p]), high = max(high, keys[p]);
  low = __reduce_min_sync(0xffffffffu, low), high = __reduce_max_sync(0xffffffffu, high);
  if (lane == 0) sums[0][warp] = low, sums[1][warp] = high;
  __syncthreads();
  low = __reduce_min_sync(0xffffffffu, lane < kSelWarps ? sums[0][lane] : 0xffffffffu);
  high = __reduce_max_sync(0xffffffffu, lane < kSelWarps ? sums[1][lane] : 0u);
  __syncthreads();     // sums is written again, at once where all words are one: a late warp would see other ends and search alone
  uint32_t want = take;     // of the words low .. high
  bool exact = take == pages;       // all words from `low` on are taken
  while (!exact && low < high) {
    const int shift = max(0, 32 - __clz((high - low) / kSelBins));   // ((high - low) >> shift < kSelBins)
    hist[tid] = hist[tid + kSelThreads] = 0;
    __syncthreads();
    for (int p = p0; p < p1; ++p) {
      const uint32_t k = keys[p];
      if (k >= low && k <= high) atomicAdd(&hist[(k - low) >> shift], 1u);
    }
    __syncthreads();
    // bins from the top: how many lie above a thread's two
    const int top_bin = kSelBins - 1 - 2 * tid;
    const uint32_t c1 = hist[top_bin], c0 = hist[top_bin - 1];
    uint32_t total;
    const uint32_t above = block_before(c1 + c0, sums[0], &total, lane, warp);
    if (above < want && above + c1 >= want) found[0] = top_bin, found[1] = above;
    else if (above + c1 < want && above + c1 + c0 >= want) found[0] = top_bin - 1, found[1] = above + c1;
    __syncthreads();
    const uint32_t bin = found[0], more = want - found[1];      // of the bin's
    exact = hist[bin] == more;
    low += bin << shift;
    high = low + min(high - low, (1u << shift) - 1u);
    if (!exact) want = more;
    __syncthreads();     // hist and found are written again
  }
  // listed: all words above `high`, and of those from low to high either all (exact) or, being one word, the first `want`
  uint32_t above = 0, equal = 0;
  for (int p = p0; p < p1; ++p) {
    const uint32_t k = keys[p];
    above += exact ? k >= low : k > low;
    equal += !exact && k == low;
  }
  uint32_t total, skip;
  uint32_t before_eq = block_before(equal, sums[0], &total, lane, warp);
  const uint32_t room = before_eq < want ? min(equal, want - before_eq) : 0u;      // of this thread's equal words
  uint32_t at = block_before(above + (exact ? 0u : room), sums[1], &skip, lane, warp);
  int* list = a.list + (long long)u * a.top;
  uint32_t left = room;
  for (int p = p0; p < p1; ++p) {
    const uint32_t k = keys[p];
    bool on = exact ? k >= low : k > low;
    if (!exact && k == low && left) on = true, --left;
    if (on) list[at++] = p;
  }
  for (int i = take + tid; i < a.top; i += kSelThreads) list[i] = -1;
  if (tid == 0) a.counts[u] = take;
}

size_t select_smem(const int R, const int pages) {
  return (size_t)padded_rows(R) * 1024 + (size_t)pages * 4;
}

}  // namespace
}  // namespace mixkv

using namespace mixkv;

extern "C" int mixkv_paged_select(const mixkv_pages* c, const void* q, int32_t type, int64_t q_batch_stride,
                                  int64_t q_token_stride, int32_t q_tokens, int32_t gqa_ratio, int32_t max_rows,
                                  int32_t top, int32_t keep_first, int32_t keep_last, int32_t* page_list,
                                  int32_t* counts, void* stream) {
  SelArgs a = {};
  int rc = check_pages(c, &a.p);
  if (rc != MIXKV_OK) return rc;
  if (!c->bounds_opt || !q || !page_list || !counts || (type != MIXKV_TYPE_BF16 && type != MIXKV_TYPE_FP16) ||
      q_tokens < 1 || gqa_ratio < 1 || max_rows < 1 || top < 1 || keep_first < 0 || keep_last < 0 || q_batch_stride < 0 ||
      q_token_stride < 0 || q_batch_stride % 8 || q_token_stride % 8 || !aligned(q, 16) || !aligned(page_list, 4) || !aligned(counts, 4))
    return MIXKV_ERR_INVALID_ARG;
  const long long R = (long long)q_tokens * gqa_ratio;
  const long long seen = max_rows < (long long)c->max_pages * c->page_rows ? max_rows : (long long)c->max_pages * c->page_rows;
  const long long pages = (seen + c->page_rows - 1) / c->page_rows;
  const long long units = (long long)c->batch * c->kv_heads;
  if (R > MIXKV_PAGED_MAX_QUERIES || pages > MIXKV_PAGES_MAX || top > kMostListed) return MIXKV_ERR_UNSUPPORTED;
  const size_t smem = select_smem((int)R, (int)pages), most = 227 * 1024 - 8192;
  if (smem > most) return MIXKV_ERR_UNSUPPORTED;
  if ((rc = device_check(nullptr)) != MIXKV_OK) return rc;
  a.q = q, a.q_batch = q_batch_stride, a.q_token = q_token_stride, a.T = q_tokens, a.G = gqa_ratio, a.R = (int)R;
  a.by_group = Divider(gqa_ratio);
  a.max_rows = max_rows, a.pages = (int)pages, a.top = top, a.first = keep_first, a.last = keep_last;
  a.list = page_list, a.counts = counts;
  const bool bf16 = type == MIXKV_TYPE_BF16;
  void (*kernel)(SelArgs) = bf16 ? k_paged_select<__nv_bfloat16> : k_paged_select<__half>;
  static std::atomic<bool> done[2][kMaxDevices];
  const int dev = device_slot();
  if (ensure_smem(kernel, most, done[bf16], dev) != cudaSuccess) return MIXKV_ERR_CUDA;
  // As many CTAs as keep four pages for every warp, while the clusters are all resident at once, a CTA to an SM (asked with the most
  // shared memory: what is remembered does not depend on the call).  65536 rows in pages of 32, seven query heads, us, with the largest
  // number that fits / with one CTA to every SM, of which some clusters wait: 16 heads 17.4 / 22.5, 24 19.6 / 29.3, 37 25.8 / 36.2,
  // 47 34.4 / 45.8.  Heads of lengths from a quarter to that make room for one another: 24 18.4 / 18.4, 37 25.3 / 28.6, 47 33.5 / 28.2.
  int S = (int)(device_sm_count() / units < kMaxCluster ? device_sm_count() / units : kMaxCluster);
  const long long rounds = (pages + kSelWarps * 4 - 1) / (kSelWarps * 4);
  if (S > rounds) S = (int)rounds;
  if (S < 1) S = 1;
  static ClusterFit fits[2];
  while (S > 1 && units > fits[bf16].ask(kernel, kSelThreads, most, S, dev)) --S;
  const cudaError_t e = launch_pdl(kernel, dim3((unsigned)(units * S)), dim3(kSelThreads), smem, (cudaStream_t)stream, S, a);
  return e == cudaSuccess ? MIXKV_OK : MIXKV_ERR_CUDA;
}
