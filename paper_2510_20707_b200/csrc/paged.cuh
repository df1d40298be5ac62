// The paged 4-bit cache (format: include/mixkv.h): where things lie, and the small conversions its kernels share.
#pragma once

#include <cfloat>

#include <cuda_fp16.h>

#include "internal_api.h"
#include "tc_common.cuh"

namespace mixkv {

constexpr int kPageTile = 16;                                // rows of a tile
constexpr int kTileBytes = MIXKV_PAGE_TILE_BYTES;
constexpr int kTileV = 1024, kTileKs = 2048, kTileVs = 2176;  // V codes, K scales, V scales inside a tile
static_assert(kTileBytes == kTileVs + 128, "a tile");
constexpr int kMostListed = 1 << 20;                         // longest page list

// n / d for 0 <= n < 2^31 as a product: with l = ceil(log2 d) and m = floor(2^(31 + l) / d) + 1, n m exceeds n 2^(31 + l) / d by
// less than 2^(31 + l) / d (n < 2^31, and m d - 2^(31 + l) <= 2^l).  A division of the hardware's kind is a chain of some twenty
// instructions; a kernel of a few microseconds begins and ends with a handful of them.
struct Divider {
  uint32_t d, mul;
  int shift;
  Divider() = default;
  explicit Divider(const uint32_t by) : d(by), mul(0), shift(0) {
    int l = 0;
    while ((1ull << l) < by) ++l;
    if (l) mul = (uint32_t)((1ull << (31 + l)) / by + 1), shift = l - 1;
  }
  __device__ __forceinline__ int div(const int n) const { return mul ? (int)(__umulhi((uint32_t)n, mul) >> shift) : n; }
};

// What kernels take of a mixkv_pages.
struct PagePool {
  unsigned char* pool;
  __half* bounds;
  const int* table;
  const int* rows;
  long long num_pages;
  int max_pages, page_rows, tiles;   // tiles of a page
  int H;
  float k_scale, v_scale;
  Divider by_heads, by_rows, by_tiles;   // of kv_heads, page_rows, tiles
};

inline bool aligned(const void* p, const unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

inline int check_pages(const mixkv_pages* c, PagePool* p) {
  if (!c || !c->pool || !c->table || !c->rows) return MIXKV_ERR_INVALID_ARG;
  // (of a subnormal scale the reciprocal is infinite, and a block of zeros would be NaN)
  const auto is_scale = [](const float x) { return x >= FLT_MIN && x <= 3e38f; };
  if (c->num_pages < 1 || c->max_pages < 1 || c->batch < 1 || c->kv_heads < 1 || !is_scale(c->k_scale) || !is_scale(c->v_scale))
    return MIXKV_ERR_INVALID_ARG;
  if (c->page_rows < kPageTile || c->page_rows % kPageTile || c->page_rows > MIXKV_PAGE_MAX_ROWS)
    return MIXKV_ERR_INVALID_ARG;
  if (!aligned(c->pool, 16) || !aligned(c->bounds_opt, 16) || !aligned(c->table, 4) || !aligned(c->rows, 4))
    return MIXKV_ERR_INVALID_ARG;
  if (c->head_dim != kHeadDim) return MIXKV_ERR_UNSUPPORTED;
  if ((long long)c->batch * c->kv_heads > (1 << 24) || (long long)c->max_pages * c->page_rows > (1ll << 30) ||
      c->num_pages > 0x7fffffffll / (c->page_rows / kPageTile))
    return MIXKV_ERR_UNSUPPORTED;
  *p = PagePool{static_cast<unsigned char*>(c->pool), static_cast<__half*>(c->bounds_opt), c->table, c->rows,
                c->num_pages, c->max_pages, c->page_rows, c->page_rows / kPageTile, c->kv_heads, c->k_scale, c->v_scale, Divider(c->kv_heads),
                Divider(c->page_rows), Divider(c->page_rows / kPageTile)};
  return MIXKV_OK;
}

// First byte of tile `t` of page `id` (a pool has at most 2^31 tiles, 2^42 bytes).
__device__ __forceinline__ unsigned char* tile_ptr(const PagePool& p, const int id, const int t) {
  return p.pool + (long long)(id * p.tiles + t) * kTileBytes;
}

// The larger of two words' halves, as unsigned numbers of 16 bits.
__device__ __forceinline__ uint32_t max_u16x2(const uint32_t a, const uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Two adjacent 16-bit values of a word, widened.
template <typename T>
__device__ __forceinline__ float2 widen2(uint32_t w);
template <>
__device__ __forceinline__ float2 widen2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 widen2<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <typename T>
__device__ __forceinline__ uint32_t narrow2(float x, float y);   // x in the low half
template <>
__device__ __forceinline__ uint32_t narrow2<__nv_bfloat16>(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t narrow2<__half>(float x, float y) {
  const __half2 v = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// What an earlier kernel of the stream may have written while this one was already resident (it waits in pdl_wait) is read by ordinary
// loads: the read-only path is for data that does not change in a kernel's lifetime, and an SM's copy of it may be from before.
template <typename T>
__device__ __forceinline__ T fresh(const T* p) { return *p; }

// This CTA's cluster in the grid (a CTA outside of one: its own number).
__device__ __forceinline__ int cluster_id() {
  uint32_t r;
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(r));
  return (int)r;
}

// The four bytes of a word, two codes each, as four fp16 pairs (low code in the low half).
__device__ __forceinline__ void codes_to_f16(const uint32_t w, uint32_t (&r)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(w));
}
// Two scales (the halves of a 16-bit word) as an fp16 pair.
__device__ __forceinline__ uint32_t scales_to_f16(const uint32_t w16) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)w16));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(const uint32_t a, const uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

__device__ __forceinline__ f32x2 mul2(const f32x2 a, const f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

}  // namespace mixkv
