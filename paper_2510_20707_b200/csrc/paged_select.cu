// Which pages of the paged cache a query attends to (score and order: include/mixkv.h).
//
// A cluster has one (sequence, KV head): its warps score the pages four at a time, the scores go as order-preserving
// words into the first CTA's shared memory, and that CTA lists the `top` largest.
//
// Score.  Lane l holds dimensions 4 l .. 4 l + 3 of the pages' bounds; of q max(q, 0) and min(q, 0) lie in shared memory, so a
// term is fma(max(q, 0), hi, min(q, 0) * lo): one of the two products is zero, the other exact (11 + 6 bits).  The sum over
// neighbouring pairs is two additions inside the lane and five across lanes; these are done for 32 (page, query row)
// pairs at a time, every exchange halving the number of sums a lane still holds (31 exchanges for 32 sums, not 160).
#include <cooperative_groups.h>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace mixkv {
namespace {

constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32;
constexpr int kSelPages = 4, kSelRows = 8;   // pages of a warp at a time; query rows at a time
constexpr uint32_t kKeyForced = 0xffffffffu, kKeyNan = 0xfffffffeu;

struct SelArgs {
  PagePool p;
  const void* q;
  long long q_batch, q_token;
  int T, G, R;
  int max_rows, pages;     // most pages of a head: room for its keys
  int top, first, last;
  int *list, *counts;
};

__device__ __forceinline__ uint32_t key_of(float x) {   // larger scores have larger words; NaN above all numbers
  if (x != x) return kKeyNan;
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0 and 0 are one score)
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Sums of v[i] over all lanes, neighbouring lanes first; afterwards v[0] is that of i = lane's number with its bits reversed.
__device__ __forceinline__ float sum_each(float (&v)[32], const int lane) {
#pragma unroll
  for (int o = 1, n = 16; o < 32; o <<= 1, n >>= 1) {
    const bool odd = lane & o;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float give = odd ? v[i] : v[i + n], keep = odd ? v[i + n] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  return v[0];
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads) k_paged_select(const SelArgs a) {
  extern __shared__ __align__(16) unsigned char sm[];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), crank = (int)cluster.block_rank(), u = blockIdx.x / S;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = u / a.p.H, h = u % a.p.H, rows_pad = (a.R + kSelRows - 1) / kSelRows * kSelRows;
  float4* qs = reinterpret_cast<float4*>(sm);                    // [R padded][2][32]: max(q, 0), min(q, 0)
  uint32_t* keys = reinterpret_cast<uint32_t*>(qs + rows_pad * 64);   // [pages], the first CTA's
  __shared__ uint32_t hist[256];
  __shared__ uint32_t warp_sum_s[kSelWarps];
  __shared__ uint32_t found[2];
  pdl_launch_dependents();
  pdl_wait();
  int n = min(a.p.rows[u], a.max_rows);
  n = (int)min((long long)n, (long long)a.p.max_pages * a.p.page_rows);
  const int pages = n <= 0 ? 0 : min((n + a.p.page_rows - 1) / a.p.page_rows, a.pages);
  for (int e = tid; e < rows_pad * 32; e += kSelThreads) {
    const int r = min(e >> 5, a.R - 1);      // (the rows of the padding repeat the last: a maximum does not mind)
    const T* src = static_cast<const T*>(a.q) + b * a.q_batch + (r / a.G) * a.q_token +
                   (long long)(h * a.G + r % a.G) * kHeadDim + 4 * (e & 31);
    const uint2 w = __ldg(reinterpret_cast<const uint2*>(src));
    const float2 x = widen2<T>(w.x), y = widen2<T>(w.y);
    // (a NaN stays one in both parts)
    auto up = [](float z) { return z < 0.f ? 0.f : z; };
    auto down = [](float z) { return z > 0.f ? 0.f : z; };
    qs[(e >> 5) * 64 + (e & 31)] = make_float4(up(x.x), up(x.y), up(y.x), up(y.y));
    qs[(e >> 5) * 64 + 32 + (e & 31)] = make_float4(down(x.x), down(x.y), down(y.x), down(y.y));
  }
  __syncthreads();
  uint32_t* keys0 = cluster.map_shared_rank(keys, 0);
  const int* table = a.p.table + (long long)u * a.p.max_pages;
  if (S > 1) cluster.sync();     // the first CTA runs
  for (int p0 = (crank * kSelWarps + warp) * kSelPages; p0 < pages; p0 += S * kSelWarps * kSelPages) {
    float lo[kSelPages][4], hi[kSelPages][4];
#pragma unroll
    for (int i = 0; i < kSelPages; ++i) {
      const int p = min(p0 + i, pages - 1), id = __ldg(table + p);
      uint2 wl = make_uint2(0, 0), wh = wl;    // (a page outside the pool scores zero)
      if (id >= 0 && id < a.p.num_pages) {
        const __half* src = a.p.bounds + (long long)id * 2 * kHeadDim + 4 * lane;
        wl = __ldg(reinterpret_cast<const uint2*>(src)), wh = __ldg(reinterpret_cast<const uint2*>(src + kHeadDim));
      }
      const float2 l0 = widen2<__half>(wl.x), l1 = widen2<__half>(wl.y), h0 = widen2<__half>(wh.x), h1 = widen2<__half>(wh.y);
      lo[i][0] = l0.x, lo[i][1] = l0.y, lo[i][2] = l1.x, lo[i][3] = l1.y;
      hi[i][0] = h0.x, hi[i][1] = h0.y, hi[i][2] = h1.x, hi[i][3] = h1.y;
    }
    uint32_t best = 0;
    for (int r0 = 0; r0 < rows_pad; r0 += kSelRows) {
      float v[32];
#pragma unroll
      for (int r = 0; r < kSelRows; ++r) {
        const float4 up = qs[(r0 + r) * 64 + lane], dn = qs[(r0 + r) * 64 + 32 + lane];
#pragma unroll
        for (int i = 0; i < kSelPages; ++i) {
          const float x0 = fmaf(up.x, hi[i][0], __fmul_rn(dn.x, lo[i][0])), x1 = fmaf(up.y, hi[i][1], __fmul_rn(dn.y, lo[i][1]));
          const float x2 = fmaf(up.z, hi[i][2], __fmul_rn(dn.z, lo[i][2])), x3 = fmaf(up.w, hi[i][3], __fmul_rn(dn.w, lo[i][3]));
          v[kSelRows * i + r] = __fadd_rn(__fadd_rn(x0, x1), __fadd_rn(x2, x3));
        }
      }
      uint32_t k = key_of(sum_each(v, lane));
      // lane bits 0, 1 (the first halvings) are the page's, 2 .. 4 the query row's
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
      best = max(best, k);
    }
    const int p = p0 + (__brev(lane) >> 30);
    if (lane < 4 && p < pages) keys0[p] = p < a.first || p >= pages - a.last ? kKeyForced : best;
  }
  if (S > 1) cluster.sync();
  else __syncthreads();
  if (crank) return;

  // The `top`-th largest word, eight bits at a time; ties to the lower page
  const int take = min(a.top, pages);
  uint32_t prefix = 0, mask = 0;
  int want = take;       // among words with this prefix
  if (take < pages) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < pages; i += kSelThreads) {
        const uint32_t k = keys[i];
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
      }
      __syncthreads();
      // bin 255 - tid: how many lie in it and above
      uint32_t c = hist[255 - tid], s = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += x;
      }
      if (lane == 31) warp_sum_s[warp] = s;
      __syncthreads();
      for (int w = 0; w < warp; ++w) s += warp_sum_s[w];
      if (s >= (uint32_t)want && s - c < (uint32_t)want) found[0] = 255 - tid, found[1] = s - c;
      __syncthreads();
      prefix |= found[0] << shift, mask |= 255u << shift;
      want -= (int)found[1];
    }
  }
  // all above `prefix`, and the first `want` equal to it
  int *list = a.list + (long long)u * a.top;
  int listed = 0, equal = 0;
  for (int base = 0; base < pages; base += kSelThreads) {
    const int p = base + tid;
    const uint32_t k = p < pages ? keys[p] : 0u;
    const bool in = p < pages, all = take == pages, same = in && !all && k == prefix;
    const uint32_t eq = __ballot_sync(0xffffffffu, same);
    __syncthreads();
    if (lane == 0) warp_sum_s[warp] = __popc(eq);
    __syncthreads();
    int before = equal, total = 0;
    for (int w = 0; w < kSelWarps; ++w) {
      if (w < warp) before += warp_sum_s[w];
      total += warp_sum_s[w];
    }
    before += __popc(eq & ((1u << lane) - 1u));
    equal += total;
    const bool on = in && (all || k > prefix || (same && before < want));
    const uint32_t yes = __ballot_sync(0xffffffffu, on);
    __syncthreads();
    if (lane == 0) warp_sum_s[warp] = __popc(yes);
    __syncthreads();
    int at = listed;
    total = 0;
    for (int w = 0; w < kSelWarps; ++w) {
      if (w < warp) at += warp_sum_s[w];
      total += warp_sum_s[w];
    }
    at += __popc(yes & ((1u << lane) - 1u));
    listed += total;
    if (on) list[at] = p;
  }
  for (int i = take + tid; i < a.top; i += kSelThreads) list[i] = -1;
  if (tid == 0) a.counts[u] = take;
}

size_t select_smem(const int R, const int pages) {
  return (size_t)((R + kSelRows - 1) / kSelRows * kSelRows) * 1024 + (size_t)pages * 4;
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
      q_token_stride < 0 || q_batch_stride % 8 || q_token_stride % 8 || (reinterpret_cast<uintptr_t>(q) & 15u))
    return MIXKV_ERR_INVALID_ARG;
  const long long R = (long long)q_tokens * gqa_ratio;
  const long long seen = max_rows < (long long)c->max_pages * c->page_rows ? max_rows : (long long)c->max_pages * c->page_rows;
  const long long pages = (seen + c->page_rows - 1) / c->page_rows;
  const long long units = (long long)c->batch * c->kv_heads;
  if (R > MIXKV_PAGED_MAX_QUERIES || pages > MIXKV_PAGES_MAX) return MIXKV_ERR_UNSUPPORTED;
  const size_t smem = select_smem((int)R, (int)pages), most = 227 * 1024 - 2048;
  if (smem > most) return MIXKV_ERR_UNSUPPORTED;
  if ((rc = device_check(nullptr)) != MIXKV_OK) return rc;
  a.q = q, a.q_batch = q_batch_stride, a.q_token = q_token_stride, a.T = q_tokens, a.G = gqa_ratio, a.R = (int)R;
  a.max_rows = max_rows, a.pages = (int)pages, a.top = top, a.first = keep_first, a.last = keep_last;
  a.list = page_list, a.counts = counts;
  const bool bf16 = type == MIXKV_TYPE_BF16;
  void (*kernel)(SelArgs) = bf16 ? k_paged_select<__nv_bfloat16> : k_paged_select<__half>;
  static std::atomic<bool> done[2][kMaxDevices];
  if (ensure_smem(kernel, most, done[bf16]) != cudaSuccess) return MIXKV_ERR_CUDA;
  // as many CTAs as keep a round of pages for every warp, while they fit the GPU
  int S = (int)(2LL * device_sm_count() / units < kMaxCluster ? 2LL * device_sm_count() / units : kMaxCluster);
  const long long rounds = (pages + kSelWarps * kSelPages - 1) / (kSelWarps * kSelPages);
  if (S > rounds) S = (int)rounds;
  if (S < 1) S = 1;
  const cudaError_t e = launch_pdl(kernel, dim3((unsigned)(units * S)), dim3(kSelThreads), smem, (cudaStream_t)stream, S, a);
  return e == cudaSuccess ? MIXKV_OK : MIXKV_ERR_CUDA;
}
