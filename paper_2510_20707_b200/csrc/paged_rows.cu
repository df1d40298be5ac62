// Rows into the paged 4-bit cache and back (format and rounding: include/mixkv.h).
//
// Append.  One CTA has one page of one head, so a page's bounds have one owner and need no atomics.  Half of its warps
// take K, half V; a warp takes two rows at a time, sixteen lanes each, a lane eight dimensions (16 bytes in, one word of
// codes out): a block of 16 is two lanes, and the largest magnitude of a block one exchange.  The rotation's partner
// dimensions lie rot_dim / 2 on, in another lane's registers.
#include "paged.cuh"

namespace mixkv {
namespace {

constexpr int kRowThreads = 256;   // of a CTA that may get many rows of a page; one row per head: 64

struct RowArgs {
  PagePool p;
  const int* offsets;     // nullptr: token b
  int per_head, max_new, slots;
  long long num_tokens;
  long long k_row, k_head, v_row, v_head;   // strides, elements
  const float *cosv, *sinv;
  const int* positions;
  int table_len, rot;
  int* status;
};

// The new rows of a unit (head h of sequence b) that lie on the CTA's page.
struct PageSpan {
  int u, h, page;          // unit, its head, column of the page table
  int lo, hi;              // rows of the page, lo < hi
  long long token;         // token (or row of the input) of row `lo`
  int id;                  // page of the pool, -1: none
  bool bad;                // a new row that has no place
};
__device__ __forceinline__ PageSpan page_span(const RowArgs& a) {
  PageSpan s;
  s.u = blockIdx.x / a.slots;
  const int slot = blockIdx.x % a.slots, b = s.u / a.p.H;
  s.h = s.u % a.p.H;
  const int rows = a.p.rows[s.u];
  long long first = b, n = 1;
  if (a.offsets) {
    const int i = a.per_head ? s.u : b;
    first = a.offsets[i], n = a.offsets[i + 1] - first;
  }
  if (n > a.max_new) first += n - a.max_new, n = a.max_new;
  long long r0 = (long long)rows - n;      // row of the first new token
  s.bad = false;
  if (r0 < 0) first -= r0, n += r0, r0 = 0, s.bad = true;
  s.page = (int)(r0 / a.p.page_rows) + slot;
  const long long begin = (long long)s.page * a.p.page_rows;
  const long long lo = r0 > begin ? r0 : begin, end = begin + a.p.page_rows;
  const long long hi = (long long)rows < end ? rows : end;
  s.lo = (int)(lo - begin), s.hi = (int)(hi - begin), s.token = first + (lo - r0), s.id = -1;
  if (n <= 0 || s.lo >= s.hi) {
    s.lo = s.hi = 0;
  } else if (s.page >= a.p.max_pages) {
    s.bad = true;
  } else {
    const int id = a.p.table[(long long)s.u * a.p.max_pages + s.page];
    if (id >= 0 && id < a.p.num_pages) s.id = id;
    else s.bad = true;
  }
  return s;
}
// Rows of the page, among s.lo .. s.hi - 1, whose token is in the input.
struct PageRows {
  int lo, hi;
};
__device__ __forceinline__ PageRows rows_in(const RowArgs& a, const PageSpan& s) {
  const long long left = a.num_tokens - s.token;     // of the input, from row s.lo on
  PageRows r = {s.lo, s.hi};
  if (s.token < 0) r.lo = s.token < s.lo - s.hi ? s.hi : s.lo - (int)s.token;
  if (left < s.hi - s.lo) r.hi = left < 0 ? s.lo : s.lo + (int)left;
  return r;
}

__device__ __forceinline__ float max_nan(const float x, const float y) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
// Eight values of a lane (half a block; the other half is in the neighbouring lane) -> their codes; *scale: the block's.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], const float inv6, const float third, uint32_t* scale) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max_nan(m, fabsf(x[i]));
  m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, 1));
  unsigned short s;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(s) : "f"(0.f), "f"(__fmul_rn(m, inv6)));
  *scale = s & 0xffu;
  const uint32_t wide = scales_to_f16(*scale);
  const float d = __fmul_rn(__low2float(*reinterpret_cast<const __half2*>(&wide)), third);
  // x / d, rounded to nearest, by Markstein's correction of x times the rounded reciprocal: the remainder of the first
  // quotient is exact, and one step with it rounds correctly while nothing over- or underflows (8 divisions: 110 instructions
  // of 300).  Blocks of infinities and of extreme scales are divided.
  const float by = __frcp_rn(d);
  const bool plain = m < 1e30f && d > 1e-30f;     // (false for NaN, and for d == 0)
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float q[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float first = __fmul_rn(x[2 * i + e], by);
      q[e] = __fmaf_rn(__fmaf_rn(-first, d, x[2 * i + e]), by, first);
    }
    if (!plain) {
#pragma unroll
      for (int e = 0; e < 2; ++e) q[e] = d == 0.f ? 0.f : __fdiv_rn(x[2 * i + e], d);
    }
    uint32_t c;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(c) : "f"(q[1]), "f"(q[0]));
    w |= c << (8 * i);
  }
  return w;
}

// Where the codes of row r, dimensions 8 c .. 8 c + 7, and the scale of block g lie inside a tile.
__device__ __forceinline__ int k_code_at(const int r, const int c) {
  return 512 * ((r >> 1) & 1) + 64 * ((r >> 2) * 2 + (r & 1)) + 4 * c;
}
__device__ __forceinline__ int v_code_at(const int r, const int c) {
  return kTileV + 512 * ((r >> 1) & 1) + 64 * (c >> 1) + 16 * (r >> 2) + 8 * (r & 1) + 4 * (c & 1);
}
__device__ __forceinline__ int k_scale_at(const int r, const int g) {
  return kTileKs + 16 * ((r >> 2) * 2 + (r & 1)) + 4 * (g >> 1) + 2 * ((r >> 1) & 1) + (g & 1);
}
__device__ __forceinline__ int v_scale_at(const int r, const int g) { return kTileVs + 16 * g + r; }

template <typename T>
__device__ __forceinline__ void widen8(const uint4& raw, float (&x)[8]) {
  const float2 a = widen2<T>(raw.x), b = widen2<T>(raw.y), c = widen2<T>(raw.z), d = widen2<T>(raw.w);
  x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
}

// Rotation of a lane's eight dimensions 8 c ..; products and differences are rounded one by one.
// ROPE 1: pairs (i, i + rot / 2); 2: (2 i, 2 i + 1).  All lanes of the warp take part.
template <typename T, int ROPE>
__device__ __forceinline__ void rotate8(const uint4& raw, float (&x)[8], const int c, const int rot, const float* cosv,
                                        const float* sinv) {
  const int half = rot >> 1;
  const bool inside = 8 * c < rot;
  if constexpr (ROPE == 1) {
    const int away = half >> 3;
    const bool low = 8 * c < half;
    const int lane = threadIdx.x & 31;
    const int from = !inside ? lane : low ? lane + away : lane - away;
    uint4 other;
    other.x = __shfl_sync(0xffffffffu, raw.x, from), other.y = __shfl_sync(0xffffffffu, raw.y, from);
    other.z = __shfl_sync(0xffffffffu, raw.z, from), other.w = __shfl_sync(0xffffffffu, raw.w, from);
    if (!inside || !cosv) return;
    float y[8], cs[8], sn[8];
    widen8<T>(other, y);
    const int at = low ? 8 * c : 8 * c - half;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      *reinterpret_cast<float4*>(&cs[4 * i]) = __ldg(reinterpret_cast<const float4*>(cosv + at) + i);
      *reinterpret_cast<float4*>(&sn[4 * i]) = __ldg(reinterpret_cast<const float4*>(sinv + at) + i);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float own = __fmul_rn(x[i], cs[i]), cross = __fmul_rn(y[i], sn[i]);
      x[i] = low ? __fsub_rn(own, cross) : __fadd_rn(own, cross);
    }
  } else if (ROPE == 2 && inside && cosv) {
    const float4 cs = __ldg(reinterpret_cast<const float4*>(cosv + 4 * c)), sn = __ldg(reinterpret_cast<const float4*>(sinv + 4 * c));
    const float cc[4] = {cs.x, cs.y, cs.z, cs.w}, ss[4] = {sn.x, sn.y, sn.z, sn.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = __fsub_rn(__fmul_rn(a, cc[i]), __fmul_rn(b, ss[i]));
      x[2 * i + 1] = __fadd_rn(__fmul_rn(b, cc[i]), __fmul_rn(a, ss[i]));
    }
  }
}

template <typename T, int ROPE>
__global__ void __launch_bounds__(kRowThreads)
k_paged_append(const RowArgs a, const T* __restrict__ k, const T* __restrict__ v) {
  __shared__ __half2 part[kRowThreads / 64][16][8];   // K warps: minima and maxima of eight dimensions
  pdl_launch_dependents();
  pdl_wait();
  const PageSpan s = page_span(a);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = lane & 15, pair = lane >> 4;
  if (s.bad && tid == 0 && a.status) *a.status = MIXKV_ERR_INVALID_ARG;
  if (s.id < 0) return;
  const bool keys = (warp & 1) == 0;
  const int half_warps = blockDim.x >> 6;
  const T* src = keys ? k : v;
  const long long row_stride = keys ? a.k_row : a.v_row;
  const long long base = a.per_head ? 0 : s.h * (keys ? a.k_head : a.v_head);
  const float third = keys ? a.p.k_scale : a.p.v_scale;
  const float inv6 = (float)(1.0 / (6.0 * (double)third));
  __half2 lo[4], hi[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) lo[i] = __float2half2_rn(INFINITY), hi[i] = __float2half2_rn(-INFINITY);
  const T* rows = src + base + (s.token - s.lo) * row_stride + 8 * c;    // row r of the page at r * row_stride
  const int* positions = a.positions + (s.token - s.lo);
  const PageRows in = rows_in(a, s);
  for (int r0 = s.lo + 2 * (warp >> 1) + pair; r0 - pair < s.hi; r0 += 4 * half_warps) {
    // two pairs of rows on their way at a time
    uint4 raw[2];
    int pos[2];
    bool on[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = r0 + 2 * half_warps * j;
      on[j] = r >= in.lo && r < in.hi;
      pos[j] = ROPE && on[j] ? __ldg(positions + r) : 0;
      raw[j] = on[j] ? __ldg(reinterpret_cast<const uint4*>(rows + r * row_stride)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = r0 + 2 * half_warps * j;
      if (r - pair >= s.hi) break;     // (the whole warp)
      if (ROPE && (pos[j] < 0 || pos[j] >= a.table_len)) on[j] = false;   // (of V too: a token is written whole or not at all)
      if (r < s.hi && !on[j] && c == 0 && a.status) *a.status = MIXKV_ERR_INVALID_ARG;
      float x[8];
      widen8<T>(raw[j], x);
      if (ROPE && keys) {
        const long long at = (long long)pos[j] * (a.rot >> 1);
        rotate8<T, ROPE>(raw[j], x, c, a.rot, on[j] ? a.cosv + at : nullptr, a.sinv + at);
      }
      uint32_t scale;
      const uint32_t w = quantise8(x, inv6, third, &scale);
      if (!on[j]) continue;
      unsigned char* tile = tile_ptr(a.p, s.id, r / kPageTile);
      const int rt = r % kPageTile;
      *reinterpret_cast<uint32_t*>(tile + (keys ? k_code_at(rt, c) : v_code_at(rt, c))) = w;
      if ((c & 1) == 0) tile[keys ? k_scale_at(rt, c >> 1) : v_scale_at(rt, c >> 1)] = (unsigned char)scale;
      if (keys && a.p.bounds) {
        uint32_t f[4];
        codes_to_f16(w, f);
        const uint32_t ss = scales_to_f16(scale | scale << 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t y = mul_f16x2(f[i], ss);
          lo[i] = __hmin2_nan(lo[i], *reinterpret_cast<const __half2*>(&y));
          hi[i] = __hmax2_nan(hi[i], *reinterpret_cast<const __half2*>(&y));
        }
      }
    }
  }
  if (!a.p.bounds) return;
  if (keys) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = __hmin2_nan(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], 16));
      hi[i] = __hmax2_nan(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], 16));
      if (pair == 0) part[warp >> 1][c][i] = lo[i], part[warp >> 1][c][4 + i] = hi[i];
    }
  }
  __syncthreads();
  if (tid < 128) {   // a thread takes one pair of dimensions of one bound (64 threads: two)
    for (int e = tid; e < 128; e += blockDim.x) {
      const int cc = e >> 3, i = e & 7;   // (i < 4: minimum)
      __half2 x = part[0][cc][i];
      for (int w = 1; w < half_warps; ++w) x = i < 4 ? __hmin2_nan(x, part[w][cc][i]) : __hmax2_nan(x, part[w][cc][i]);
      __half2* out = reinterpret_cast<__half2*>(a.p.bounds + ((long long)s.id * 2 + (i >> 2)) * kHeadDim) + 4 * cc + (i & 3);
      if (s.lo > 0) x = i < 4 ? __hmin2_nan(x, *out) : __hmax2_nan(x, *out);
      *out = x;
    }
  }
}

// A lane has eight dimensions of a row, as above.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_paged_read(const RowArgs a, T* __restrict__ k, T* __restrict__ v) {
  pdl_launch_dependents();
  pdl_wait();
  const PageSpan s = page_span(a);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = lane & 15, pair = lane >> 4;
  if (s.id < 0) return;
  const bool keys = (warp & 1) == 0;
  T* dst = keys ? k : v;
  const float third = keys ? a.p.k_scale : a.p.v_scale;
  const PageRows in = rows_in(a, s);
  const long long out_stride = a.per_head ? kHeadDim : (long long)a.p.H * kHeadDim;
  T* rows = dst + (s.token - s.lo) * out_stride + (a.per_head ? 0 : s.h * kHeadDim) + 8 * c;   // row r of the page at r * out_stride
  const int step = blockDim.x >> 5;
  for (int r0 = s.lo + 2 * (warp >> 1) + pair; r0 < in.hi; r0 += 4 * step) {
    uint32_t w[4], scale[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = min(r0 + j * step, s.hi - 1), rt = r % kPageTile;
      const unsigned char* tile = tile_ptr(a.p, s.id, r / kPageTile);
      w[j] = *reinterpret_cast<const uint32_t*>(tile + (keys ? k_code_at(rt, c) : v_code_at(rt, c)));
      scale[j] = tile[keys ? k_scale_at(rt, c >> 1) : v_scale_at(rt, c >> 1)];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = r0 + j * step;
      if (r < in.lo || r >= in.hi) continue;
      uint32_t f[4], out[4];
      codes_to_f16(w[j], f);
      const uint32_t ss = scales_to_f16(scale[j] | scale[j] << 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 y = widen2<__half>(mul_f16x2(f[i], ss));
        out[i] = narrow2<T>(__fmul_rn(y.x, third), __fmul_rn(y.y, third));
      }
      *reinterpret_cast<uint4*>(rows + r * out_stride) = make_uint4(out[0], out[1], out[2], out[3]);
    }
  }
}

int check_rows(const mixkv_pages* c, int32_t type, int64_t num_tokens, const int32_t* offsets, int32_t per_head,
               int32_t max_new, RowArgs* a) {
  const int rc = check_pages(c, &a->p);
  if (rc != MIXKV_OK) return rc;
  if ((type != MIXKV_TYPE_BF16 && type != MIXKV_TYPE_FP16) || num_tokens < 0 || max_new < 1 || (per_head && !offsets) ||
      (reinterpret_cast<uintptr_t>(offsets) & 3u))
    return MIXKV_ERR_INVALID_ARG;
  if (max_new > (1 << 30)) return MIXKV_ERR_UNSUPPORTED;
  a->offsets = offsets, a->per_head = per_head != 0, a->max_new = offsets ? max_new : 1, a->num_tokens = num_tokens;
  // pages that a head's new rows can touch: one, and one more for every page_rows rows behind the first
  a->slots = (a->max_new - 1 + c->page_rows - 1) / c->page_rows + 1;
  if (a->slots > c->max_pages + 1) a->slots = c->max_pages + 1;   // (one past the table: rows there are reported)
  if ((long long)c->batch * c->kv_heads * a->slots > 0x7fffffffll) return MIXKV_ERR_UNSUPPORTED;
  return MIXKV_OK;
}
template <typename F, typename... Args>
int launch_rows(F kernel, const mixkv_pages* c, const RowArgs& a, void* stream, Args... args) {
  const int rc = device_check(nullptr);
  if (rc != MIXKV_OK) return rc;
  const dim3 grid((unsigned)(c->batch * c->kv_heads * a.slots)), block(a.max_new > 1 ? kRowThreads : 64);
  return launch_pdl(kernel, grid, block, 0, (cudaStream_t)stream, 1, a, args...) == cudaSuccess ? MIXKV_OK : MIXKV_ERR_CUDA;
}
template <typename T>
int append_as(const mixkv_pages* c, const RowArgs& a, const void* k, const void* v, const int rope, void* stream) {
  const T *kk = static_cast<const T*>(k), *vv = static_cast<const T*>(v);
  switch (rope) {
    case 0: return launch_rows(k_paged_append<T, 0>, c, a, stream, kk, vv);
    case 1: return launch_rows(k_paged_append<T, 1>, c, a, stream, kk, vv);
    default: return launch_rows(k_paged_append<T, 2>, c, a, stream, kk, vv);
  }
}
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace mixkv

using namespace mixkv;

extern "C" int mixkv_paged_page_bytes(int32_t page_rows, size_t* bytes) {
  if (!bytes || page_rows < kPageTile || page_rows % kPageTile || page_rows > MIXKV_PAGE_MAX_ROWS)
    return MIXKV_ERR_INVALID_ARG;
  *bytes = (size_t)(page_rows / kPageTile) * kTileBytes;
  return MIXKV_OK;
}

extern "C" int mixkv_paged_append(const mixkv_pages* c, const void* k, const void* v, int32_t type, int64_t num_tokens,
                                  int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride,
                                  int64_t v_head_stride, const int32_t* offsets_opt, int32_t offsets_per_head,
                                  int32_t max_new, const float* cos_opt, const float* sin_opt, int32_t table_len,
                                  int32_t rot_dim, int32_t interleaved, const int32_t* positions_opt,
                                  int32_t* status_dev, void* stream) {
  RowArgs a = {};
  const int rc = check_rows(c, type, num_tokens, offsets_opt, offsets_per_head, max_new, &a);
  if (rc != MIXKV_OK) return rc;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return MIXKV_ERR_INVALID_ARG;
  for (const int64_t stride : {k_row_stride, k_head_stride, v_row_stride, v_head_stride})
    if (stride < 0 || stride % 8) return MIXKV_ERR_INVALID_ARG;
  const bool rope = cos_opt != nullptr;
  if (rope != (sin_opt != nullptr)) return MIXKV_ERR_INVALID_ARG;
  if (rope) {
    if (!positions_opt || table_len < 1 || !aligned16(cos_opt) || !aligned16(sin_opt) || rot_dim < 1 || rot_dim > kHeadDim ||
        (reinterpret_cast<uintptr_t>(positions_opt) & 3u))
      return MIXKV_ERR_INVALID_ARG;
    if (rot_dim % 16) return MIXKV_ERR_UNSUPPORTED;
  }
  a.k_row = k_row_stride, a.k_head = k_head_stride, a.v_row = v_row_stride, a.v_head = v_head_stride;
  a.cosv = cos_opt, a.sinv = sin_opt, a.positions = positions_opt, a.table_len = table_len, a.rot = rot_dim;
  a.status = status_dev;
  const int mode = !rope ? 0 : interleaved ? 2 : 1;
  return type == MIXKV_TYPE_BF16 ? append_as<__nv_bfloat16>(c, a, k, v, mode, stream)
                                 : append_as<__half>(c, a, k, v, mode, stream);
}

extern "C" int mixkv_paged_read(const mixkv_pages* c, void* k_out, void* v_out, int32_t type, int64_t num_tokens,
                                const int32_t* offsets_opt, int32_t offsets_per_head, int32_t max_new, void* stream) {
  RowArgs a = {};
  const int rc = check_rows(c, type, num_tokens, offsets_opt, offsets_per_head, max_new, &a);
  if (rc != MIXKV_OK) return rc;
  if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return MIXKV_ERR_INVALID_ARG;
  if (type == MIXKV_TYPE_BF16)
    return launch_rows(k_paged_read<__nv_bfloat16>, c, a, stream, static_cast<__nv_bfloat16*>(k_out),
                       static_cast<__nv_bfloat16*>(v_out));
  return launch_rows(k_paged_read<__half>, c, a, stream, static_cast<__half*>(k_out), static_cast<__half*>(v_out));
}
