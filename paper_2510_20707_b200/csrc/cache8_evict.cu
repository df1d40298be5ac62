// Eviction by accumulated attention weight (include/mixkv.h): which rows of a head are kept, and their copy into other pages.
//
// k_cache8_pick: a cluster has a head.  A row's mass becomes a 32-bit key in the order of the numbers; the key of the last row that is kept
// is found by its digits (11, 11 and 10 bits), each from one histogram of the keys that share the digits before it, summed over the
// cluster through distributed shared memory.  Keys stay in shared memory between the passes where they fit.  Then every warp has
// a run of rows: it counts what it keeps, learns where its run begins in the list, and writes it in order.  Equal keys are taken from the
// lowest row on, so the list does not depend on how the rows were dealt out.
//
// k_cache8_move: a warp has a tile of the new cache, and gathers its rows: lanes as in an append (cache8_rows.cu).
//
// What bounds it.  128 heads of 6001 to 16384 rows, cut to 2048: 21 us for the pick (issue slots 65 %: three passes over the keys, a list in
// order), 41 for the move.  That reads 130 MB for 67 MB of kept rows: a row's 128 bytes lie at any multiple of 16 and touch three pieces of 64
// bytes, its block's scales another; 4 TB/s of such pieces, whatever the number of warps (8, 10 and 12 CTAs an SM 41 to 45 us).  K and V in
// one warp 41 us, apart 50; values kept in registers between the search for the largest and the rounding 51, since they halve the warps.
// Eight rows of a thread on their way for the pick: 22 us for 35; sixteen: no more.
#include <cooperative_groups.h>

#include "cache8.cuh"

namespace cg = cooperative_groups;

namespace mixkv {
namespace {

constexpr int kPickThreads = 1024, kPickWarps = kPickThreads / 32;   // (as many warps as a warp has lanes)
constexpr int kBins = 2048;
constexpr int kPickKeys = 40960;       // keys that a CTA keeps in shared memory
constexpr int kPickRows = 2048;        // rows that a CTA of a cluster should have
constexpr int kMoveWarps = 4;

struct EvictArgs {
  CachePool p, into;
  int budget;
  const int* budgets;
  int first, last;
  int max_rows;
  int cached;              // keys that fit a CTA's shared memory
  int* idx;                // [units][budget]
  int* status;
  int slots;               // tiles of a budget
  Divider by_slots;
};

// The key of a row: the order of keys is that of masses, NaN above all and a row without a page below.
__device__ __forceinline__ uint32_t key_of(const CachePool& p, const int u, const int row) {
  const int page = p.by_rows.div(row);
  const int id = fresh(p.table + (long long)u * p.max_pages + page);
  if (id < 0 || id >= p.num_pages) return 0u;
  const float m = fresh(p.mass + (long long)id * p.page_rows + (row - page * p.page_rows)) + 0.f;      // (-0 is 0)
  const uint32_t b = __float_as_uint(m);
  return m != m ? 0xffffffffu : b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// Of the numbers that lanes have, one for each warp: the sum of those before warp `warp`'s.
__device__ __forceinline__ int sum_below(const int x, const int warp, const int lane) {
  return __reduce_add_sync(0xffffffffu, lane < warp ? x : 0);
}

__global__ void __launch_bounds__(kPickThreads) k_cache8_pick(const EvictArgs a) {
  extern __shared__ uint32_t keys[];
  __shared__ __align__(8) int hist[kBins];
  __shared__ int2 sums[kBins / 2];           // over the cluster, two bins each
  __shared__ int warp_sum[kPickWarps];
  __shared__ int2 warp_run[kPickWarps];      // of a warp's run: keys above the threshold, keys equal to it
  __shared__ int2 cta_run;
  __shared__ int found[3];                   // bin, what is left to take of it, keys in it
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), u = cluster_id();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  int n = min(fresh(a.p.rows + u), a.max_rows);
  n = max(0, (int)min((long long)n, (long long)a.p.max_pages * a.p.page_rows));
  const int budget = a.budgets ? min(max(fresh(a.budgets + u), a.first + a.last), a.budget) : a.budget;
  const int kept = min(n, budget);
  int* idx = a.idx + (long long)u * a.budget;
  if (rank == 0) {
    if (tid == 0) a.into.rows[u] = kept;
    for (int i = kept + tid; i < a.budget; i += kPickThreads) idx[i] = -1;
  }
  if (n <= budget) {       // (the whole cluster)
    for (int i = rank * kPickThreads + tid; i < n; i += S * kPickThreads) idx[i] = i;
    return;
  }
  // rows m0 .. m0 + m - 1 compete for k places
  const int m0 = a.first, m = n - a.first - a.last, k = budget - a.first - a.last;
  if (rank == 0) {
    for (int i = tid; i < a.first; i += kPickThreads) idx[i] = i;
    for (int i = tid; i < a.last; i += kPickThreads) idx[a.first + k + i] = n - a.last + i;
  }
  if (k == 0) return;
  const int each = (m + S - 1) / S, lo = min(rank * each, m), hi = min(lo + each, m), mine = hi - lo;
  const bool cached = mine <= a.cached;
  auto key = [&](const int i) { return cached ? keys[i] : key_of(a.p, u, m0 + lo + i); };
  for (int i = tid; i < kBins; i += kPickThreads) hist[i] = 0;
  __syncthreads();
  // the highest digit is counted as the keys come; eight rows of a thread on their way: a page, then its mass, are two trips to memory
  constexpr int kAtOnce = 8;
  for (int i = tid; i < mine; i += kAtOnce * kPickThreads) {
    uint32_t x[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) x[j] = key_of(a.p, u, m0 + lo + min(i + j * kPickThreads, mine - 1));
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (i + j * kPickThreads < mine) {
        if (cached) keys[i + j * kPickThreads] = x[j];
        atomicAdd(&hist[x[j] >> 21], 1);
      }
  }

  uint32_t prefix = 0;       // digits that are known, in place
  int left = k;
  bool exact = false;        // all that have them are taken
  int shift = 21;
#pragma unroll 1
  for (int pass = 0;;) {
    cluster.sync();
    // Every CTA sums its part of the bins over the cluster and hands it to all: 16 KB in and out where reading all histograms would be
    // 64 KB with eight CTAs (one head of 32768 rows to each of eight clusters: the call 27.7 us for 31.0).
    if (S > 1 && tid < kBins / 2 / S) {
      const int at = rank * (kBins / 2 / S) + tid;
      int2 sum = make_int2(0, 0);
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r)
        if (r < S) {
          const int2 x = *reinterpret_cast<const int2*>(cluster.map_shared_rank(&hist[2 * at], r));
          sum.x += x.x, sum.y += x.y;
        }
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r)
        if (r < S) *cluster.map_shared_rank(&sums[at], r) = sum;
    }
    if (S > 1) cluster.sync();          // (no CTA clears its histogram before all have read it)
    // thread t has bins 2047 - 2 t and the next lower one: the sum of what is above them
    const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
    const int2 two = S > 1 ? sums[b0 / 2] : *reinterpret_cast<const int2*>(&hist[b0]);
    const int n0 = two.x, n1 = two.y;
    int upto = n0 + n1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    const int before = upto - n0 - n1 + sum_below(warp_sum[lane], warp, lane);
    if (before < left && before + n1 >= left) found[0] = b1, found[1] = left - before, found[2] = n1;
    else if (before + n1 < left && before + n1 + n0 >= left) found[0] = b0, found[1] = left - before - n1, found[2] = n0;
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    left = found[1];
    exact = found[1] == found[2];
    if (exact || ++pass == 3) break;
    const uint32_t above = 0xffffffffu << shift;
    const int bits = pass == 2 ? 10 : 11;
    shift -= bits;
    for (int i = tid; i < kBins; i += kPickThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < mine; i += kPickThreads) {
      const uint32_t x = key(i);
      if ((x & above) == prefix) atomicAdd(&hist[(x >> shift) & ((1u << bits) - 1u)], 1);
    }
  }
  // kept: keys above `top`, and the first `left` of those equal to it
  const uint32_t top = exact ? prefix - 1u : prefix;     // (the lowest digits of a prefix are zero; key 0 alone is never all)
  if (exact) left = 0;

  const int run = (((mine + kPickWarps - 1) / kPickWarps) + 31) & ~31, from = min(warp * run, mine), to = min(from + run, mine);
  int above = 0, equal = 0;
#pragma unroll 4
  for (int i = from + lane; i - lane < to; i += 32) {
    const uint32_t x = i < to ? key(i) : 0u;
    above += i < to && x > top, equal += i < to && x == top;
  }
  above = __reduce_add_sync(0xffffffffu, above), equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) warp_run[warp] = make_int2(above, equal);
  __syncthreads();
  const int2 runs = warp_run[lane];
  if (warp == 0) {
    const int x = __reduce_add_sync(0xffffffffu, runs.x), y = __reduce_add_sync(0xffffffffu, runs.y);
    if (lane == 0) cta_run = make_int2(x, y);
  }
  cluster.sync();
  // of all rows before the warp's run
  above = sum_below(runs.x, warp, lane), equal = sum_below(runs.y, warp, lane);
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r)
    if (r < rank) {
      const int2 x = *cluster.map_shared_rank(&cta_run, r);
      above += x.x, equal += x.y;
    }
#pragma unroll 2
  for (int i = from; i < to; i += 32) {
    const bool in = i + lane < to;
    const uint32_t x = in ? key(i + lane) : 0u;
    const unsigned more = __ballot_sync(0xffffffffu, in && x > top), same = __ballot_sync(0xffffffffu, in && x == top);
    const unsigned below = (1u << lane) - 1u;
    const int g = above + __popc(more & below), e = equal + __popc(same & below);
    if (in && (x > top || (x == top && e < left))) idx[a.first + g + min(e, left)] = m0 + lo + i + lane;
    above += __popc(more), equal += __popc(same);
  }
  cluster.sync();            // a CTA's shared memory stays alive until its peers have read it
}

__device__ __forceinline__ float max_nan(const float x, const float y) {   // NaN if one is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
// The largest magnitude of sixteen codes.
template <bool E4M3>
__device__ __forceinline__ float largest_code(const uint4& c) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
  __half2 m = __float2half2_rn(0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo, hi;
    codes_to_half<E4M3>(w[i], lo, hi);
    m = __hmax2(m, __hmax2(__habs2(*reinterpret_cast<const __half2*>(&lo)), __habs2(*reinterpret_cast<const __half2*>(&hi))));
  }
  return fmaxf(__low2float(m), __high2float(m));
}

template <bool E4M3>
__global__ void __launch_bounds__(kMoveWarps * 32) k_cache8_move(const EvictArgs a, const int tasks) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane & 7, sub = lane >> 3;
  const int job = blockIdx.x * kMoveWarps + warp;
  pdl_wait();
  if (job >= tasks) return;
  const int u = a.by_slots.div(job), t = job - u * a.slots, begin = t * kBlockRows;
  // row `lane` of the tile (lanes 0 .. 15): its place in the old cache, -1: none.  (What is asked for does not wait for the number of rows.)
  const int kept = min(fresh(a.into.rows + u), a.budget);
  const int page = a.into.by_tiles.div(t), in = t - page * a.into.tiles;
  const int id = page < a.into.max_pages ? fresh(a.into.table + (long long)u * a.into.max_pages + page) : -1;
  int row = lane < kBlockRows && begin + lane < a.budget ? fresh(a.idx + (long long)u * a.budget + begin + lane) : -1;
  if (begin >= kept) return;
  if (id < 0 || id >= a.into.num_pages) {
    if (a.status && lane == 0) *a.status = MIXKV_ERR_INVALID_ARG;
    return;
  }
  int block = -1;
  if (row >= 0) {
    const int from = a.p.by_rows.div(row);
    const int old = from < a.p.max_pages ? fresh(a.p.table + (long long)u * a.p.max_pages + from) : -1;
    row -= from * a.p.page_rows;
    if (old >= 0 && old < a.p.num_pages) block = old * a.p.tiles + (row >> 4);
  }
  uint4 codes[2][4];
  float2 scale[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = __shfl_sync(0xffffffffu, block, 4 * i + sub), r = __shfl_sync(0xffffffffu, row, 4 * i + sub) & 15;
    codes[0][i] = codes[1][i] = make_uint4(0, 0, 0, 0), scale[i] = make_float2(0.f, 0.f);
    if (at >= 0) {
      const unsigned char* tile = a.p.pool + (long long)at * kBlockBytes;
      codes[0][i] = *reinterpret_cast<const uint4*>(tile + piece_at(r, g));
      codes[1][i] = *reinterpret_cast<const uint4*>(tile + kBlockV + piece_at(r, g));
      scale[i] = *reinterpret_cast<const float2*>(tile + kBlockScales);
    }
  }
  if (a.into.mass && lane < kBlockRows && begin + lane < kept)
    a.into.mass[(long long)id * a.into.page_rows + in * kBlockRows + lane] =
        block >= 0 ? fresh(a.p.mass + (long long)block * kBlockRows + (row & 15)) : 0.f;
  unsigned char* tile = block_ptr(a.into, id, in);
  float to[2];
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    // the largest magnitude: of a row's codes, times its scale (rounding keeps the order)
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max_nan(most, fabsf(__fmul_rn(largest_code<E4M3>(codes[v][i]), v ? scale[i].y : scale[i].x)));
    const uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(most) & 0x7fffffffu);
    to[v] = scale_of_largest<E4M3>(__uint_as_float(bits));
    const float by = by_scale(to[v]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x2 x[8];
      values16<E4M3>(codes[v][i], v ? scale[i].y : scale[i].x, x);
      *reinterpret_cast<uint4*>(tile + v * kBlockV + piece_at(4 * i + sub, g)) = encode16<E4M3>(x, by);
    }
  }
  if (lane == 0) *reinterpret_cast<float2*>(tile + kBlockScales) = make_float2(to[0], to[1]);
}

}  // namespace
}  // namespace mixkv

using namespace mixkv;

extern "C" int mixkv_cache_evict(const mixkv_cache8* c, const mixkv_cache8* into, int32_t budget, const int32_t* budgets_opt,
                                  int32_t keep_first, int32_t keep_last, int32_t max_rows, int32_t* idx,
                                  int32_t* status_dev, void* stream) {
  EvictArgs a = {};
  int rc = check_cache(c, &a.p);
  if (rc != MIXKV_OK || (rc = check_cache(into, &a.into)) != MIXKV_OK) return rc;
  if (!c->mass_opt || !idx || budget < 1 || keep_first < 0 || keep_last < 0 || (long long)keep_first + keep_last > budget ||
      max_rows < 1 || into->batch != c->batch || into->kv_heads != c->kv_heads || into->code != c->code || into->rows == c->rows ||
      !aligned(idx, 4) || !aligned(budgets_opt, 4) || !aligned(status_dev, 4))
    return MIXKV_ERR_INVALID_ARG;
  const long long units = (long long)c->batch * c->kv_heads, slots = ((long long)budget + kBlockRows - 1) / kBlockRows;
  if (budget > (1 << 30) || units * slots > 0x3fffff00ll) return MIXKV_ERR_UNSUPPORTED;
  if ((rc = device_check(nullptr)) != MIXKV_OK) return rc;
  a.budget = budget, a.budgets = budgets_opt, a.first = keep_first, a.last = keep_last, a.max_rows = max_rows;
  a.idx = idx, a.status = status_dev, a.slots = (int)slots, a.by_slots = Divider((uint32_t)slots);
  const long long room = (long long)c->max_pages * c->page_rows, rows = max_rows < room ? max_rows : room;
  constexpr size_t kMost = (size_t)kPickKeys * 4;
  static std::atomic<bool> done[kMaxDevices];
  const int dev = device_slot();
  if (ensure_smem(k_cache8_pick, kMost, done, dev) != cudaSuccess) return MIXKV_ERR_CUDA;
  // CTAs of a head: as many as its rows are worth, no more than one to an SM, and in clusters that are all resident at once (asked with
  // the most shared memory: what is remembered does not depend on the call).  65536 rows, an eighth kept, us a call, with clusters that fit /
  // with one CTA to every SM, of which some clusters wait: 16 heads 45.9 / 52.4, 18 47.8 / 55.6, 36 80.2 / 84.8.  A device that holds no
  // cluster of a size would refuse the launch.
  int S = 1;
  while (S < kMaxCluster && S * (long long)kPickRows < rows && units * S * 2 <= device_sm_count()) S *= 2;
  static ClusterFit fits;
  while (S > 1 && units > fits.ask(k_cache8_pick, kPickThreads, kMost, S, dev)) S /= 2;
  const long long each = (rows + S - 1) / S;
  a.cached = (int)(each < kPickKeys ? each : kPickKeys);
  const size_t smem = (size_t)a.cached * 4;
  const cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = launch_pdl(k_cache8_pick, dim3((unsigned)(units * S)), dim3(kPickThreads), smem, st, S, a);
  const int tasks = (int)(units * slots);
  if (e == cudaSuccess)
    e = launch_pdl(c->code == MIXKV_CODE_E4M3 ? k_cache8_move<true> : k_cache8_move<false>,
                   dim3((unsigned)((tasks + kMoveWarps - 1) / kMoveWarps)), dim3(kMoveWarps * 32), 0, st, 1, a, tasks);
  return e == cudaSuccess ? MIXKV_OK : MIXKV_ERR_CUDA;
}
