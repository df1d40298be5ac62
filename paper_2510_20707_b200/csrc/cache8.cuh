// The paged 8-bit cache (format: include/mixkv.h): where things lie, and the conversions its kernels share.
#pragma once

#include <cfloat>

#include <cuda_fp16.h>

#include "internal_api.h"
#include "paged.cuh"
#include "tc_common.cuh"

namespace mixkv {

constexpr int kBlockRows = 16;                               // rows of a tile, which is a block
constexpr int kBlockBytes = MIXKV_CACHE8_TILE_BYTES;
constexpr int kBlockV = 2048, kBlockScales = 4096;           // V codes, the two scales inside a tile

// What kernels take of a mixkv_cache8.
struct CachePool {
  unsigned char* pool;
  float* mass;
  const int* table;
  int* rows;
  long long num_pages;
  int max_pages, page_rows, tiles;   // tiles of a page
  int H;
  Divider by_heads, by_rows, by_tiles;   // of kv_heads, page_rows, tiles
};

inline int check_cache(const mixkv_cache8* c, CachePool* p) {
  if (!c || !c->pool || !c->table || !c->rows) return MIXKV_ERR_INVALID_ARG;
  if (c->num_pages < 1 || c->max_pages < 1 || c->batch < 1 || c->kv_heads < 1 ||
      (c->code != MIXKV_CODE_INT8 && c->code != MIXKV_CODE_E4M3))
    return MIXKV_ERR_INVALID_ARG;
  if (c->page_rows < kBlockRows || c->page_rows % kBlockRows || c->page_rows > MIXKV_PAGE_MAX_ROWS)
    return MIXKV_ERR_INVALID_ARG;
  if (!aligned(c->pool, 16) || !aligned(c->mass_opt, 4) || !aligned(c->table, 4) || !aligned(c->rows, 4))
    return MIXKV_ERR_INVALID_ARG;
  if (c->head_dim != kHeadDim) return MIXKV_ERR_UNSUPPORTED;
  if ((long long)c->batch * c->kv_heads > (1 << 24) || (long long)c->max_pages * c->page_rows > (1ll << 30) ||
      c->num_pages > 0x7fffffffll / (c->page_rows / kBlockRows))
    return MIXKV_ERR_UNSUPPORTED;
  const int tiles = c->page_rows / kBlockRows;
  *p = CachePool{static_cast<unsigned char*>(c->pool), c->mass_opt, c->table, c->rows, c->num_pages, c->max_pages, c->page_rows,
                 tiles, c->kv_heads, Divider(c->kv_heads), Divider(c->page_rows), Divider(tiles)};
  return MIXKV_OK;
}

// First byte of tile `t` of page `id` (a pool has at most 2^31 tiles, 2^43 bytes).
__device__ __forceinline__ unsigned char* block_ptr(const CachePool& p, const int id, const int t) {
  return p.pool + ((long long)id * p.tiles + t) * kBlockBytes;
}
// Sixteen codes, dimensions 16 g and on, of row r of a tile's K (V: kBlockV further on).  Eight lanes that read one piece of
// eight rows, or eight pieces of a row, meet in no bank of shared memory.
__device__ __forceinline__ int piece_at(const int r, const int g) { return 128 * r + 16 * (g ^ (r & 7)); }

// The 32 bytes at p, a lane's sixteen values of 16 bits.
struct Sixteen {
  uint32_t w[8];
};
__device__ __forceinline__ void load_sixteen(Sixteen& r, const void* p) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store_sixteen(void* p, const Sixteen& r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]),
               "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7])
               : "memory");
}

// Two codes (the low or the high half of a word) as an fp16 pair: exact.
// int8: a byte plus 128 behind the exponent of 1024 is 1152 + code.
template <bool E4M3>
__device__ __forceinline__ void codes_to_half(const uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (E4M3) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  } else {
    const uint32_t x = w ^ 0x80808080u;
    const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
  }
}
// Four codes as fp32 numbers.  int8: a byte plus 128 in the low bits of 2^23.
template <bool E4M3>
__device__ __forceinline__ void codes_to_float(const uint32_t w, f32x2& a, f32x2& b) {
  if constexpr (E4M3) {
    uint32_t lo, hi;
    codes_to_half<true>(w, lo, hi);
    const float2 x = widen2<__half>(lo), y = widen2<__half>(hi);
    a = pack2(x.x, x.y), b = pack2(y.x, y.y);
  } else {
    const uint32_t x = w ^ 0x80808080u;
    const f32x2 off = pack2(-8388736.f, -8388736.f);
    a = add2(pack2(__uint_as_float(__byte_perm(x, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7441))), off);
    b = add2(pack2(__uint_as_float(__byte_perm(x, 0x4b000000u, 0x7442)), __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7443))), off);
  }
}

// Scale of a block whose largest magnitude is m (a NaN or an infinity: NaN).
template <bool E4M3>
__device__ __forceinline__ float scale_of_largest(const float m) {
  const float s = __fmul_rn(m, E4M3 ? 1.f / 448.f : 1.f / 127.f);
  return !(m < INFINITY) ? NAN : s < FLT_MIN ? 0.f : s;
}
__device__ __forceinline__ float larger_scale(const float a, const float b) { return a != a || b != b ? NAN : fmaxf(a, b); }
// What values are multiplied by; zero (all codes are zero) for a scale of zero or NaN.
__device__ __forceinline__ float by_scale(const float s) { return s > 0.f ? __frcp_rn(s) : 0.f; }
// Codes of four values.  by > 0: they are finite, and no product is beyond the largest code by more than its own rounding.
// int8: 1.5 * 2^23 + y has the nearest whole number to y, ties to even, in its low bits.  (The sums are taken one by one: of packed
// products and a packed sum the compiler makes multiply-adds.)
template <bool E4M3>
__device__ __forceinline__ uint32_t encode4(const f32x2 a, const f32x2 b, const float by) {
  float ya, yb, yc, yd;
  unpack2(mul2(a, pack2(by, by)), ya, yb), unpack2(mul2(b, pack2(by, by)), yc, yd);
  uint32_t r;
  if constexpr (E4M3) {
    asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 y, %4, %3;\n\t"
        "mov.b32 %0, {x, y};\n\t}"
        : "=r"(r)
        : "f"(ya), "f"(yb), "f"(yc), "f"(yd));
  } else {
    constexpr float magic = 12582912.f;
    const uint32_t x = __float_as_uint(__fadd_rn(ya, magic)), y = __float_as_uint(__fadd_rn(yb, magic));
    const uint32_t z = __float_as_uint(__fadd_rn(yc, magic)), w = __float_as_uint(__fadd_rn(yd, magic));
    r = __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
  }
  return by > 0.f ? r : 0u;
}
template <typename T>
__device__ __forceinline__ f32x2 widen_pair(const uint32_t w) {
  const float2 v = widen2<T>(w);
  return pack2(v.x, v.y);
}
template <>
__device__ __forceinline__ f32x2 widen_pair<__nv_bfloat16>(const uint32_t w) { return bf16x2_wide(w); }
template <typename T, bool E4M3>
__device__ __forceinline__ uint4 encode16(const Sixteen& x, const float by) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = encode4<E4M3>(widen_pair<T>(x.w[2 * i]), widen_pair<T>(x.w[2 * i + 1]), by);
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// Sixteen codes under scale `s` as fp32(code * s).
template <bool E4M3>
__device__ __forceinline__ void values16(const uint4& c, const float s, f32x2 (&x)[8]) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x2 a, b;
    codes_to_float<E4M3>(w[i], a, b);
    x[2 * i] = mul2(a, pack2(s, s)), x[2 * i + 1] = mul2(b, pack2(s, s));
  }
}
template <bool E4M3>
__device__ __forceinline__ uint4 encode16(const f32x2 (&x)[8], const float by) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = encode4<E4M3>(x[2 * i], x[2 * i + 1], by);
  return make_uint4(r[0], r[1], r[2], r[3]);
}

}  // namespace mixkv
