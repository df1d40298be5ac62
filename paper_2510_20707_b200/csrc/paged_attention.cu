// Attention of the newest tokens over the paged 4-bit cache (format: include/mixkv.h).
//
// A warp takes two tiles of 16 cache rows per step, 2304 contiguous bytes each, brought by bulk copies into a ring of its own.
// The codes are widened to fp16 by the hardware's conversion and multiplied by their scale: exact.  The products
// run as m16n8k16 with the CACHE on the sixteen-row side and the query rows (tokens x heads of the group) on the
// eight-column side: with up to eight query rows (one token of seven heads) nothing is padded but the eighth, where
// query rows on the sixteen side would leave more than half of every instruction empty (32 instead of 16 instructions a tile).
//   S^T[row, query]  = K q^T      A: rows 4 (g / 2) + 2 j + g % 2, a lane the dimensions 32 t .. 32 t + 31 of two rows
//   O^T[dim, query] += V^T P^T    A: dimensions 16 g + 2 m, + 1 of rows 4 t .. 4 t + 3; P^T from S^T by a transposing move
// Codes of two rows are interleaved (V) by one select per eight values before they are widened, so that a pair is two rows.
//
// Softmax: a running reference per query row, moved only when a logit exceeds it by more than 2^kLag (one vote a
// step instead of a reduction); weights are fp16 times 2^kLift, so that what is 2^-20 of the largest is still a normal
// number; sums are fp32.  The weights enter the sum of values as ONE fp16 number, the sum of weights unrounded.  As two parts they
// double the products of the values: 256 heads of 1021 to 16384 rows 82.7 us a call for 75.9, a draft of 35 query rows 36.7 for 31.1.  What
// that would buy is seen in fp16 outputs alone, 2.1e-4 from 64 bits (their own rounding) in place of 2.8e-4 with the draft; bf16 outputs
// are 1.7e-3 from them in both.
//
// What bounds it.  A row pair is 144 bytes; a tile of 16 costs a warp 303 instructions (43.3 M for 142 848 tiles): 64 conversions (two
// clocks each, as the fp16 products), 64 products with scales, 16 matrix instructions (eight clocks), 16 selects.  256 heads of 1021 to
// 16384 rows (329 MB) take 74 us in this kernel under the profiler: 4.5 TB/s, an instruction issued in 60 % of the clocks, the arithmetic
// pipe busy in 52, the tensor pipe in 25; the same copies without the arithmetic take 57 us.  Two tiles a softmax step instead of one: 54
// instructions a tile fewer, and 8 % of the time of such calls, 10 % with 32 query rows.  Twelve warps an SM with 159 registers are as
// fast as sixteen with 128; asking for values ahead of the vote, one copy for two tiles that follow one another, rings of three: no gain.
// With query rows on the sixteen side, one tile a step and a chunk per CTA the same call took 129 us, and now 76.
#include <cfloat>

#include <cooperative_groups.h>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace mixkv {
namespace {

constexpr int kAttWarps = 4;                   // of a CTA of which an SM holds several
constexpr int kAttWide = 16;                   // of one that has an SM for itself (one group of query rows)
constexpr int kAttDepth = 2;                   // steps of a warp on their way or in work
constexpr int kStepBytes = 2 * kTileBytes;
constexpr int kNoRow = 0x3fffffff;             // first row of a tile that is not there: beyond all
constexpr int kAttPitch = kHeadDim / 2 + 4;    // floats between the query rows of half a warp's sums
constexpr int kAttGroups = 4;                  // most groups of eight query rows a CTA takes
constexpr int kAttUnits = 1024;                // most units whose steps are dealt out evenly
constexpr int kAttFew = 2, kAttFewRows = 8, kAttWideSteps = 8, kAttManySteps = 20;   // steps of a warp (att_shape)
constexpr float kLag = 8.f, kLift = 6.f;       // largest weight 2^14
constexpr float kNoRef = -FLT_MAX;             // reference before the first row: no logit is below, and it is finite

// rings of the warps (a cluster's CTA: then its sums); half of the warps' sums; references and sums of the warps, the CTA,
// the cluster; barriers and rows of the rings
__host__ __device__ constexpr size_t att_smem(int NT, int W) {
  return W * (kAttDepth * kStepBytes + 8 * NT * kAttPitch * 4) + (2 * W + 2 + 2 * kMaxCluster) * 8 * NT * 4 +
         W * kAttDepth * 16 + 16;
}
// CTAs of an SM, which sets the registers of a thread.  One group of query rows: comment above.  Two groups: three CTAs of 168 registers
// spill 124 bytes, two spill nothing and are 2 to 10 % faster (16 query rows, us: 64 heads of 4096 rows 20.7 with three, 18.6 with two, 256
// of 2048 35.5 and 32.9, of 8192 95.4 and 93.4): not taken so far.  Three groups: two CTAs of 249 registers, no spills; three spill 544
// bytes (24 rows, 256 heads of 2048: 42.4 with two, 62.2 with three).  Four: 255 registers, the most there are, spill 348 bytes with two,
// 1760 with three (32 rows: 59.1 and 155.7).
__host__ __device__ constexpr int att_per_sm(int NT, int W) { return W > kAttWarps ? 1 : NT == 1 ? 4 : NT == 2 ? 3 : 2; }

struct AttArgs {
  PagePool p;
  const void* q;
  long long q_batch, q_token;
  int T, G, R;               // tokens, heads of a group, T * G
  Divider by_group;          // of G
  int max_rows;
  const int *list, *counts;  // nullptr: all pages
  int top;
  int units;
  int ctas;                  // that share all steps evenly; 0: a cluster has a unit
  int per;                   // fours of outputs of a CTA of such a cluster
  float scale_log2e;         // k_scale included
  int2* spans;               // [units]: first CTA with a share of a unit, times two, plus one if its run begins before the unit; last CTA
  float* part;               // [2 ctas][R][128]: sums of a unit's share, where it is not the whole
  float2* part_mz;           // [2 ctas][R]: (reference, sum)
  void* out;
};

// Steps (pairs of tiles) of a unit, and its rows that the call sees.
struct UnitTiles {
  int n, tiles, steps;
};
__device__ __forceinline__ UnitTiles unit_tiles(const AttArgs& a, const int u) {
  UnitTiles r;
  int n = fresh(a.p.rows + u);
  n = min(n, a.max_rows);
  n = (int)min((long long)n, (long long)a.p.max_pages * a.p.page_rows);
  r.n = max(n, 0);
  r.tiles = a.list ? max(0, min(fresh(a.counts + u), a.top)) * a.p.tiles : (r.n + kPageTile - 1) >> 4;
  r.steps = (r.tiles + 1) >> 1;
  return r;
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2,
                                        const uint32_t a3, const uint32_t b0, const uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(const uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float column_max(float v) {   // over the eight lanes that hold a query row's logits
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor_sync(0xffffffffu, v, 4);
  v += __shfl_xor_sync(0xffffffffu, v, 8);
  return v + __shfl_xor_sync(0xffffffffu, v, 16);
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, const uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// Place in the pool and first row of tile `t` of a unit (-1, kNoRow: none).  The table is asked before the unit's rows are looked at:
// both may be on their way.
struct TileAt {
  int tile, row;
};
__device__ __forceinline__ TileAt tile_at(const AttArgs& a, const int u, const UnitTiles& ut, const int t) {
  const int slot = a.p.by_tiles.div(t), in = t - slot * a.p.tiles;
  int page = slot;
  if (a.list) page = slot < a.top ? fresh(a.list + (long long)u * a.top + slot) : -1;
  const int id = page >= 0 && page < a.p.max_pages ? fresh(a.p.table + (long long)u * a.p.max_pages + page) : -1;
  const int row = page * a.p.page_rows + in * kPageTile;
  if (id < 0 || id >= a.p.num_pages || t >= ut.tiles || row >= ut.n) return TileAt{-1, kNoRow};
  return TileAt{id * a.p.tiles + in, row};
}

// Steps of a CTA when `ctas` of them share `total`: CTA c has those from c * share on, the last ones may have none.
__device__ __forceinline__ int share_of(const int total, const int ctas) { return (total + ctas - 1) / ctas; }

// Row of the output that query row r of a unit has.
__device__ __forceinline__ long long out_row(const AttArgs& a, const int u, const int r) {
  const int b = a.p.by_heads.div(u), h = u - b * a.p.H, token = a.by_group.div(r);
  return ((long long)b * a.T + token) * ((long long)a.p.H * a.G) + h * a.G + (r - token * a.G);
}

__device__ __forceinline__ void add_scaled(float4& sum, const float4& x, const float by) {
  sum.x = fmaf(x.x, by, sum.x), sum.y = fmaf(x.y, by, sum.y), sum.z = fmaf(x.z, by, sum.z), sum.w = fmaf(x.w, by, sum.w);
}
// Four outputs: sums of weighted values over the sum of weights (zeros where there were none), times v_scale.  (The quotient of the two
// factors could be subnormal.)
template <typename T>
__device__ __forceinline__ void store_row(T* to, const float4& num, const float den, const float v_scale) {
  const float by = den == 0.f ? 0.f : 1.f / den;
  *reinterpret_cast<uint2*>(to) = make_uint2(narrow2<T>(num.x * by * v_scale, num.y * by * v_scale),
                                             narrow2<T>(num.z * by * v_scale, num.w * by * v_scale));
}

// The first `keep` of the four scales of a word, zeros for the others.
__device__ __forceinline__ uint32_t keep_scales(const uint32_t w, const int keep) {
  return keep >= 4 ? w : keep <= 0 ? 0u : w & ((1u << (8 * keep)) - 1u);
}
// A fragments of V^T, dimensions 16 g + 2 m and + 1 (m = 0 .. 7) of rows 4 t .. 4 t + 3, handed to f(m, ...) one by one.
template <typename F>
__device__ __forceinline__ void values(const uint4 (&v)[2], const uint32_t vs, const F& f) {
  const uint32_t s0 = scales_to_f16(vs & 0xffffu), s1 = scales_to_f16(vs >> 16);   // rows 4 t, + 1; 4 t + 2, + 3
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t a0 = i ? v[0].y : v[0].x, b0 = i ? v[0].w : v[0].z;
    const uint32_t a1 = i ? v[1].y : v[1].x, b1 = i ? v[1].w : v[1].z;
    constexpr uint32_t low = 0x0f0f0f0fu;
    uint32_t e0[4], o0[4], e1[4], o1[4];   // even and odd dimensions of the rows' pairs
    codes_to_f16((a0 & low) | ((b0 << 4) & ~low), e0);
    codes_to_f16(((a0 >> 4) & low) | (b0 & ~low), o0);
    codes_to_f16((a1 & low) | ((b1 << 4) & ~low), e1);
    codes_to_f16(((a1 >> 4) & low) | (b1 & ~low), o1);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      f(4 * i + e, mul_f16x2(e0[e], s0), mul_f16x2(o0[e], s0), mul_f16x2(e1[e], s1), mul_f16x2(o1[e], s1));
  }
}
// Token of query row r of a unit (rows of the padding: the last).
__device__ __forceinline__ int token_of(const AttArgs& a, const int r) { return a.by_group.div(min(r, a.R - 1)); }

template <typename T, int NT>
struct AttState {
  uint32_t q[NT][8][2];     // B fragments: query row g, dimensions 32 t + 4 s .. + 3
  float f[NT][2];           // logits to log2 units: query rows 2 t, 2 t + 1
  float acc[NT][8][4];      // dimensions 16 g + 2 m (0, 1), 16 g + 2 m + 1 (2, 3) of query rows 2 t, 2 t + 1
  float ref[NT][2], z[NT][2];   // weights are 2^(logit - ref)

  // Query rows first .. first + 8 NT - 1 of a unit.  bf16 rows are divided by a power of two that brings their largest
  // magnitude to [1, 2): exact as fp16 but for what is 2^-24 of it; the power goes into f.
  __device__ __forceinline__ void start(const AttArgs& a, const int u, const int first, const int g, const int t) {
    const int b = a.p.by_heads.div(u), h = u - b * a.p.H;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = first + 8 * nt + g;
      uint4 raw[4];
      const bool on = r < a.R;
      const int token = on ? a.by_group.div(r) : 0;
      const T* src = static_cast<const T*>(a.q) + b * a.q_batch + token * a.q_token +
                     (long long)(h * a.G + (on ? r - token * a.G : 0)) * kHeadDim + 32 * t;
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i] = on ? fresh(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0, 0, 0, 0);
      float most = 0.f;
      bool odd = false;    // a NaN or an infinity
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = widen2<T>(w[e]);
          most = fmaxf(most, fmaxf(fabsf(x.x), fabsf(x.y)));
          odd |= !(fabsf(x.x) < INFINITY) || !(fabsf(x.y) < INFINITY);
        }
      }
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      // 2^e <= most < 2^(e + 1) (subnormal: 2^-126); down = 2^-e
      const uint32_t e = max(__float_as_uint(most) >> 23, 1u);
      const bool scaled = sizeof(T) == 2 && __float_as_uint(most) != 0 && most < INFINITY && IsBf16;
      const float down = scaled ? __uint_as_float((254u - min(e, 253u)) << 23) : 1.f;
      float up = scaled ? __uint_as_float(min(e, 253u) << 23) : 1.f;
      odd |= __shfl_xor_sync(0xffffffffu, (int)odd, 1) != 0;
      odd |= __shfl_xor_sync(0xffffffffu, (int)odd, 2) != 0;
      if (odd) up = NAN;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int e2 = 0; e2 < 4; ++e2) {
          if constexpr (IsBf16) {
            const float2 x = widen2<T>(w[e2]);
            q[nt][2 * i + (e2 >> 1)][e2 & 1] = odd ? 0u : narrow2<__half>(x.x * down, x.y * down);
          } else {
            q[nt][2 * i + (e2 >> 1)][e2 & 1] = odd ? 0u : w[e2];
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float by = __shfl_sync(0xffffffffu, up, 4 * (2 * t + c)) * a.scale_log2e;
        f[nt][c] = by < 1.2e-38f ? 1.2e-38f : by;    // (a NaN stays; never zero: times minus infinity it is the logit of a masked row)
        ref[nt][c] = kNoRef, z[nt][c] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[nt][i][c] = 0.f;
    }
  }
  static constexpr bool IsBf16 = std::is_same<T, __nv_bfloat16>::value;

  // s[2 j + c] += products of row 4 (g / 2) + 2 j + g % 2 of the tile and query row 8 nt + 2 t + c
  __device__ __forceinline__ void logits(const unsigned char* tile, const int lane, float (&s)[NT][4]) const {
    const uint4 k[2] = {*reinterpret_cast<const uint4*>(tile + 16 * lane), *reinterpret_cast<const uint4*>(tile + 512 + 16 * lane)};
    const uint32_t ks = *reinterpret_cast<const uint32_t*>(tile + kTileKs + 4 * lane);
    const uint32_t s0 = scales_to_f16(ks & 0xffffu), s1 = scales_to_f16(ks >> 16);   // (block 2 t, block 2 t + 1) of row j
    const uint32_t sc[2][2] = {{__byte_perm(s0, 0, 0x1010), __byte_perm(s0, 0, 0x3232)},
                               {__byte_perm(s1, 0, 0x1010), __byte_perm(s1, 0, 0x3232)}};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t x[4], y[4];
      codes_to_f16(i == 0 ? k[0].x : i == 1 ? k[0].y : i == 2 ? k[0].z : k[0].w, x);
      codes_to_f16(i == 0 ? k[1].x : i == 1 ? k[1].y : i == 2 ? k[1].z : k[1].w, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = mul_f16x2(x[e], sc[0][i >> 1]), y[e] = mul_f16x2(y[e], sc[1][i >> 1]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma_f16(s[nt], x[0], y[0], x[1], y[1], q[nt][2 * i][0], q[nt][2 * i][1]);
        mma_f16(s[nt], x[2], y[2], x[3], y[3], q[nt][2 * i + 1][0], q[nt][2 * i + 1][1]);
      }
    }
  }

  // Two tiles, whose first rows are row[], of a unit of n rows; `first`: the CTA's first query row.  edge: rows may lie
  // beyond what a query row sees.  (A flag and not a second copy of the code: a step that was alone in its kind waited for its
  // instructions for longer than it took.)
  __device__ __forceinline__ void step(const AttArgs& a, const unsigned char* tiles, const int (&row)[2], const bool edge,
                                       const int n, const int first, const int lane) {
    const int g = lane >> 2, t = lane & 3;
    float s[2][NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][nt][i] = 0.f;
      logits(tiles + h * kTileBytes, lane, s[h]);
    }
    if (edge) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int sees = n - a.T + 1 + token_of(a, first + 8 * nt + 2 * t + c) - 4 * (g >> 1) - (g & 1);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = c; i < 4; i += 2)
              if (row[h] + 2 * (i >> 1) >= sees) s[h][nt][i] = -INFINITY;
        }
    }
    // (A logit is rounded before the reference, itself a logit, is taken from it: of a product that is not, equal logits beyond 2^24 would
    // differ from it by their last bits, whole powers of two.)
    bool above = false;
    float y[2][NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[h][nt][i] = __fsub_rn(__fmul_rn(s[h][nt][i], f[nt][i & 1]), ref[nt][i & 1]);
          above |= y[h][nt][i] > kLag + kLift;
        }
    if (__any_sync(0xffffffffu, above)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float mx = -INFINITY;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = c; i < 4; i += 2) {
              y[h][nt][i] = __fmul_rn(s[h][nt][i], f[nt][c]);
              mx = fmaxf(mx, y[h][nt][i]);
            }
          const float to = fmaxf(ref[nt][c], column_max(mx) - kLift);
          const float shrink = ex2(ref[nt][c] - to);
          ref[nt][c] = to, z[nt][c] *= shrink;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = c; i < 4; i += 2) y[h][nt][i] = __fsub_rn(y[h][nt][i], to);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[nt][i][c] *= shrink, acc[nt][i][2 + c] *= shrink;
        }
    }
    uint32_t p[2][NT][2];   // B fragments: query row g, tile rows 4 t, 4 t + 1 and 4 t + 2, 4 t + 3
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[h][nt][i] = ex2(y[h][nt][i]), z[nt][i & 1] += y[h][nt][i];
        p[h][nt][0] = transpose8x8(narrow2<__half>(y[h][nt][0], y[h][nt][1]));
        p[h][nt][1] = transpose8x8(narrow2<__half>(y[h][nt][2], y[h][nt][3]));
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned char* tile = tiles + h * kTileBytes;
      const uint4 v[2] = {*reinterpret_cast<const uint4*>(tile + kTileV + 16 * lane),
                          *reinterpret_cast<const uint4*>(tile + kTileV + 512 + 16 * lane)};
      uint32_t vs = *reinterpret_cast<const uint32_t*>(tile + kTileVs + 4 * lane);
      // Rows that were never written can hold anything, a scale of NaN as well: their scales become zero.  A NaN in a row
      // that some of the query rows see must not reach the others through a weight of zero: such a tile is taken once per
      // token, with the rows that this token sees, and added to its own query rows alone.
      if (edge) {
        vs = keep_scales(vs, n - row[h] - 4 * t);
        const bool nan = ((((vs & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u)) != 0;   // a byte of 0x7f
        if (a.T > 1 && __any_sync(0xffffffffu, nan)) {
          for (int token = 0; token < a.T; ++token) {
            const uint32_t seen = keep_scales(vs, n - a.T + 1 + token - row[h] - 4 * t);
            values(v, seen, [&](const int m, const uint32_t x0, const uint32_t x1, const uint32_t x2, const uint32_t x3) {
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float d[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(d, x0, x1, x2, x3, p[h][nt][0], p[h][nt][1]);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                  if (token_of(a, first + 8 * nt + 2 * t + (c & 1)) == token) acc[nt][m][c] += d[c];
              }
            });
          }
          continue;
        }
      }
      values(v, vs, [&](const int m, const uint32_t x0, const uint32_t x1, const uint32_t x2, const uint32_t x3) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_f16(acc[nt][m], x0, x1, x2, x3, p[h][nt][0], p[h][nt][1]);
      });
    }
  }
};

// W warps.  grid.x: units * S in clusters of S (ctas == 0), or ctas; grid.y: groups of 8 NT query rows
template <typename T, int NT, int W>
__global__ void __launch_bounds__(32 * W, att_per_sm(NT, W)) k_paged_attention(const AttArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int Q = 8 * NT, kSums = Q * kAttPitch, kThreads = 32 * W;
  float* xo = reinterpret_cast<float*>(smem);   // [Q][128]: a cluster's CTA has its sums where its rings were
  static_assert(Q * kHeadDim * 4 <= W * kAttDepth * kStepBytes, "sums of a CTA fit the rings");
  float* sums = reinterpret_cast<float*>(smem + W * kAttDepth * kStepBytes);   // [warps][Q][pitch]
  float* wm = sums + W * kSums;      // [warps][Q]
  float* wz = wm + W * Q;            // [warps][Q]
  float* xm = wz + W * Q;            // [Q]
  float* xz = xm + Q;                        // [Q]
  float* allm = xz + Q;                      // [8][Q]
  float* allz = allm + kMaxCluster * Q;      // [8][Q]
  uint64_t* bars = reinterpret_cast<uint64_t*>(allz + kMaxCluster * Q);   // [warps][depth]
  int2* rows = reinterpret_cast<int2*>(bars + W * kAttDepth);   // [warps][depth]: first rows of a step's tiles
  int* abort = reinterpret_cast<int*>(rows + W * kAttDepth);
  __shared__ int starts[kAttUnits + 1];      // first step of every unit
  __shared__ int warp_total[W];
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const bool shares = a.ctas > 0;
  const int S = shares ? 1 : (int)cluster.num_blocks(), crank = shares ? 0 : (int)cluster.block_rank();
  const int first = blockIdx.y * Q, live = min(Q, a.R - first);
  uint64_t* bar = bars + warp * kAttDepth;
  if (lane == 0) {
    for (int d = 0; d < kAttDepth; ++d) mbar_init(&bar[d], 1);
    mbar_init_fence();
    if (warp == 0) *abort = 0;
  }
  __syncthreads();
  pdl_wait();

  // steps lo .. hi - 1: of a cluster's unit, or of all units one after the other
  int u = shares ? 0 : cluster_id(), lo = crank * W, hi;
  if (shares) {
    // first steps of all units: a thread takes consecutive ones
    constexpr int kEach = kAttUnits / kThreads;
    int mine[kEach], sum = 0;
    const int u0 = tid * kEach;
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine[i] = u0 + i < a.units ? unit_tiles(a, u0 + i).steps : 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += mine[i];
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_total[warp] = upto;
    __syncthreads();
    int at = upto - sum, total = 0;
    for (int w = 0; w < W; ++w) {
      if (w < warp) at += warp_total[w];
      total += warp_total[w];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (u0 + i < a.units) starts[u0 + i] = at;
      at += mine[i];
    }
    if (tid == 0) starts[a.units] = total;
    __syncthreads();
    if (blockIdx.x + 1 == gridDim.x && blockIdx.y == 0) {      // (the CTA whose run is the shortest)
      const int share = max(1, share_of(total, a.ctas));
      for (int i = tid; i < a.units; i += kThreads) {
        const int from = starts[i], to = starts[i + 1], c0 = from / share;
        a.spans[i] = from < to ? make_int2(2 * c0 + (c0 * share < from), (to - 1) / share) : make_int2(0, -1);
      }
    }
    const int share = share_of(total, a.ctas);
    lo = blockIdx.x * share, hi = min(lo + share, total);
    if (lo >= hi) return;
    int x = 0, y = a.units;     // the last unit that begins at or before lo
    while (y - x > 1) {
      const int m = (x + y) >> 1;
      (starts[m] <= lo ? x : y) = m;
    }
    u = x;
  } else {
    hi = unit_tiles(a, u).steps;
  }
  const int stride = S * W, begin = lo + warp;
  const int count = begin < hi ? (hi - begin + stride - 1) / stride : 0;   // steps of this warp
  unsigned char* ring = smem + warp * kAttDepth * kStepBytes;
  int2* ring_rows = rows + warp * kAttDepth;

  TileAt ahead[2] = {};      // lane l knows the tiles of step 32 n + l of the warp, 32 n the last multiple at or before `sent`
  auto locate = [&](const int i) {
    int f = begin + i * stride, v = u;
    if (shares) {
      if (i >= count) return;
      int y = a.units;
      while (y - v > 1) {
        const int m = (v + y) >> 1;
        (starts[m] <= f ? v : y) = m;
      }
      f -= starts[v];
    }
    const UnitTiles ut = unit_tiles(a, v);
    ahead[0] = tile_at(a, v, ut, 2 * f), ahead[1] = tile_at(a, v, ut, 2 * f + 1);
  };
  locate(lane);
  int sent = 0, slot_out = 0;
  auto send = [&]() {   // the copies of the warp's step `sent`
    if ((sent & 31) == 0 && sent) locate(sent + lane);
    if (lane == (sent & 31)) {
      uint64_t* full = &bar[slot_out];
      unsigned char* to = ring + slot_out * kStepBytes;
      ring_rows[slot_out] = make_int2(ahead[0].row, ahead[1].row);
      const uint32_t bytes = (ahead[0].tile >= 0 ? kTileBytes : 0) + (ahead[1].tile >= 0 ? kTileBytes : 0);
      if (bytes) mbar_expect_tx(full, bytes);
      else mbar_arrive(full);    // nothing to come
      if (ahead[0].tile >= 0) bulk_load(to, a.p.pool + (long long)ahead[0].tile * kTileBytes, kTileBytes, full);
      if (ahead[1].tile >= 0) bulk_load(to + kTileBytes, a.p.pool + (long long)ahead[1].tile * kTileBytes, kTileBytes, full);
    }
    ++sent, slot_out = slot_out + 1 == kAttDepth ? 0 : slot_out + 1;
  };
  while (sent < min(count, kAttDepth)) send();
  int slot = 0;
  uint32_t parity = 0;
  bool lost = false;

  for (int f = begin;;) {     // one unit after the other
    int end = hi;
    if (shares) {
      while (starts[u + 1] <= max(lo, starts[u])) ++u;    // (units without tiles)
      end = min(hi, starts[u + 1]);
    }
    AttState<T, NT> st;
    st.start(a, u, first, g, t);
    const int n = unit_tiles(a, u).n;
    const int clear = n - a.T + 1;   // rows below are seen by all
    for (; f < end && !lost; f += stride) {
      if (!mbar_wait_warp(&bar[slot], parity, abort)) {
        lost = true;
        break;
      }
      const int2 at = ring_rows[slot];
      const unsigned char* tiles = ring + slot * kStepBytes;
      const bool inside = max(at.x, at.y) + kPageTile <= clear;
      const int row[2] = {at.x, at.y};
      st.step(a, tiles, row, !inside, n, first, lane);
      __syncwarp();     // every lane has read the slot
      if (sent < count) send();
      ++slot;
      if (slot == kAttDepth) slot = 0, parity ^= 1;
    }
    if (lost) {     // (once: the units that follow have no copies)
      if (lane == 0) drain_ring(bar, kAttDepth, sent);
      sent = 0;
    }

    pdl_launch_dependents();      // (the next kernel's CTAs, where this one's have ended)
    // ---- the warps merge through shared memory, the dimensions 16 g .. 16 g + 7 first and then the others
    float* own = sums + warp * kSums;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float z = column_sum(st.z[nt][c]);
        const int r = 8 * nt + 2 * t + c;
        if (g == 0) wm[warp * Q + r] = st.ref[nt][c], wz[warp * Q + r] = lost ? NAN : z;
      }
    const bool whole = shares ? lo <= starts[u] && end == starts[u + 1] : S == 1;
    const int share = 2 * blockIdx.x + (shares && lo < starts[u]);   // (the first unit of a CTA, or its last)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half) __syncthreads();
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int m = 0; m < 4; ++m)
            *reinterpret_cast<float2*>(own + (8 * nt + 2 * t + c) * kAttPitch + 8 * g + 2 * m) =
                make_float2(st.acc[nt][4 * half + m][c], st.acc[nt][4 * half + m][2 + c]);
      __syncthreads();
      for (int e = tid; e < live * (kHeadDim / 8); e += kThreads) {
        const int r = e / (kHeadDim / 8), x = 4 * (e % (kHeadDim / 8)), dim = 16 * (x >> 3) + 8 * half + (x & 7);
        float M = kNoRef;
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, wm[w * Q + r]);
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float sc = ex2(wm[w * Q + r] - M);
          add_scaled(num, *reinterpret_cast<const float4*>(sums + w * kSums + r * kAttPitch + x), sc);
          den = fmaf(wz[w * Q + r], sc, den);
        }
        if (whole) {
          store_row(static_cast<T*>(a.out) + out_row(a, u, first + r) * kHeadDim + dim, num, den, a.p.v_scale);
        } else if (shares) {
          const long long at = (long long)share * a.R + first + r;
          *reinterpret_cast<float4*>(a.part + at * kHeadDim + dim) = num;
          if (dim == 0) a.part_mz[at] = make_float2(M, den);
        } else {
          *reinterpret_cast<float4*>(xo + r * kHeadDim + dim) = num;
          if (dim == 0) xm[r] = M, xz[r] = den;
        }
      }
    }
    if (shares) {
      if (end == hi) return;
      __syncthreads();
      ++u;
      continue;
    }
    if (whole) return;

    // ---- the CTAs of the cluster merge through distributed shared memory, each a slice of the outputs
    cluster.sync();
    for (int e = tid; e < S * Q; e += kThreads) {
      const int k = e / Q, r = e % Q;
      allm[e] = *cluster.map_shared_rank(&xm[r], k);
      allz[e] = *cluster.map_shared_rank(&xz[r], k);
    }
    __syncthreads();
    for (int e = crank * a.per + tid; e < min((crank + 1) * a.per, live * (kHeadDim / 4)); e += kThreads) {
      const int r = e / (kHeadDim / 4), dim = 4 * (e % (kHeadDim / 4));
      float M = kNoRef;
      for (int k = 0; k < S; ++k) M = fmaxf(M, allm[k * Q + r]);
      float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
      float den = 0.f;
#pragma unroll 4
      for (int k = 0; k < S; ++k) {
        const float sc = ex2(allm[k * Q + r] - M);
        add_scaled(num, *reinterpret_cast<const float4*>(cluster.map_shared_rank(xo + r * kHeadDim + dim, k)), sc);
        den = fmaf(allz[k * Q + r], sc, den);
      }
      store_row(static_cast<T*>(a.out) + out_row(a, u, first + r) * kHeadDim + dim, num, den, a.p.v_scale);
    }
    cluster.sync();   // a CTA's shared memory stays alive until its peers have read it
    return;
  }
}

// Joins the shares of units that several CTAs had a part of, and writes zeros for units without rows.  per_row warps (a power
// of two) take the shares of a query row in turn, a few at once with a running reference: what a share holds comes in one
// round trip.  It costs a call 4 to 6 us (8 heads of 131072 rows: 36.4 with a join that does nothing, 40.3).  Joined by the last
// CTA of a unit instead, behind a fence and a count that a kernel before had to clear, 8 to 10.
constexpr int kJoinWarps = 16;
template <typename T>
__global__ void __launch_bounds__(kJoinWarps * 32) k_paged_join(const AttArgs a, const Divider per_row, const Divider blocks) {
  __shared__ float4 sums[kJoinWarps][32];
  __shared__ float2 stat[kJoinWarps];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int u = blocks.div(blockIdx.x), slot = per_row.div(warp), part = warp - slot * per_row.d;
  const int row = (blockIdx.x - u * blocks.d) * per_row.div(kJoinWarps) + slot;      // (blocks: CTAs of a unit)
  pdl_wait();
  const int2 span = __ldcg(a.spans + u);
  const int c0 = span.x >> 1, c1 = span.y;
  if (c0 == c1) return;     // written by that CTA
  const bool on = row < a.R;
  constexpr int kAtOnce = 5;
  float M = kNoRef, den = 0.f;
  float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int c = c0 + part; on && c <= c1; c += per_row.d * kAtOnce) {
    float4 x[kAtOnce];
    float2 mz[kAtOnce];
    float to = M;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int k = min(c + i * (int)per_row.d, c1);
      const long long at = (2LL * k + (k == c0 ? span.x & 1 : 0)) * a.R + row;
      mz[i] = __ldcg(a.part_mz + at);
      x[i] = __ldcg(reinterpret_cast<const float4*>(a.part + at * kHeadDim) + lane);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) to = fmaxf(to, mz[i].x);
    const float shrink = ex2(M - to);
    num.x *= shrink, num.y *= shrink, num.z *= shrink, num.w *= shrink, den *= shrink;
    M = to;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float sc = c + i * (int)per_row.d <= c1 ? ex2(mz[i].x - M) : 0.f;
      add_scaled(num, x[i], sc);
      den = fmaf(mz[i].y, sc, den);
    }
  }
  if (per_row.d > 1) {
    sums[warp][lane] = num;
    if (lane == 0) stat[warp] = make_float2(M, den);
    __syncthreads();
    if (part) return;
    float to = M;
    for (int w = 1; w < (int)per_row.d; ++w) to = fmaxf(to, stat[warp + w].x);
    const float shrink = ex2(M - to);
    num.x *= shrink, num.y *= shrink, num.z *= shrink, num.w *= shrink, den *= shrink;
    for (int w = 1; w < (int)per_row.d; ++w) {
      const float2 mz = stat[warp + w];
      const float sc = ex2(mz.x - to);
      add_scaled(num, sums[warp + w][lane], sc);
      den = fmaf(mz.y, sc, den);
    }
  }
  if (on) store_row(static_cast<T*>(a.out) + out_row(a, u, row) * kHeadDim + 4 * lane, num, den, a.p.v_scale);
}

using AttKernel = void (*)(AttArgs);
template <typename T>
AttKernel att_kernel(const int NT, const bool wide) {
  switch (NT) {
    case 1: return wide ? k_paged_attention<T, 1, kAttWide> : k_paged_attention<T, 1, kAttWarps>;
    case 2: return k_paged_attention<T, 2, kAttWarps>;
    case 3: return k_paged_attention<T, 3, kAttWarps>;
    default: return k_paged_attention<T, 4, kAttWarps>;
  }
}

// How the work is split.  units: (sequence, head) pairs; groups of query rows; steps of the longest unit, as its rows and `top` have it, and
// `most` that one can have on the device (what a list counts is the caller's word): the shares' sum over all units has 31 bits.
// narrow(n), wide(n): clusters of n CTAs of either kind that are resident at once.
//
// A cluster of small CTAs per unit, one of large CTAs that have an SM each, or all steps dealt out evenly and joined by a second
// kernel; us a call, one token of four query heads, heads of one length (and of lengths from one row to that):
//     heads x rows     small          large         shares
//     8 x 2048         7.5            8.2           10.3        two steps for every warp of eight small CTAs
//     8 x 4096         9.3            8.2           10.8
//     8 x 16384       19.8 (21.5)    14.3 (14.4)    15.4 (16.6)
//     8 x 65536       60.8 (67.7)    35.8 (36.7)    27.7 (23.4)
//     64 x 4096       14.9 (13.4)    14.7 (14.5)    20.0 (17.3)
//     64 x 8192       22.6 (19.8)    22.1 (22.4)    26.4 (21.0)   eight steps for every warp of two large CTAs
//     64 x 16384      39.5 (31.7)    38.3 (37.2)    41.8 (29.5)
//     256 x 2048      23.5 (20.2)    26.5 (21.7)    28.7 (36.2)   eight steps for every warp of two small CTAs
//     256 x 4096      40.5 (32.3)    43.7 (33.4)    43.0 (43.1)
//     256 x 16384    128.9 (102.5)  125.9 (98.1)   121.2 (88.2)
// and 896 heads of 70 to 1639 rows 39.7 by small CTAs, 43.2 by shares.  More query rows make a step longer and the join a smaller
// part (35 rows in two groups, small / shares: 8 heads of 2048 rows 13.3 / 16.8, of 8192 26.8 / 25.5, 32 of 8192 45.0 / 48.1).
struct AttShape {
  int S, ctas;      // CTAs of a cluster that has a unit; or, not 0, CTAs that share all steps
  bool wide;
};
int att_slots(const int NT, const int sms) { return att_per_sm(NT, kAttWarps) * sms; }
template <typename Narrow, typename Wide>
AttShape att_shape(const long long units, const int groups, const long long steps, const long long most, const int NT, const int sms,
                   const Narrow& narrow, const Wide& wide) {
  const long long slots = att_slots(NT, sms), all = units * groups;
  auto clusters = [&](const long long room, const int warps, const auto& fit) {
    long long S = room / all < kMaxCluster ? room / all : kMaxCluster;
    if (S > steps / warps) S = steps / warps;
    if (S < 1) S = 1;
    while (S > 1 && all > fit((int)S)) --S;
    return (int)S;
  };
  int S = clusters(slots, kAttWarps, narrow);
  const long long alone = (steps + S * kAttWarps - 1) / (S * kAttWarps);     // steps of a warp
  if (alone <= (NT == 1 ? kAttFew : kAttFewRows)) return {S, 0, false};
  if (NT == 1 && all <= sms) {
    const int B = clusters(sms, kAttWide, wide);
    if (steps <= (long long)B * kAttWide * kAttWideSteps) return {B, 0, true};
  } else if (NT == 1 && alone <= kAttManySteps) {
    return {S, 0, false};
  }
  if (units <= kAttUnits && groups < slots && units * most <= 0x7fffffffll) {
    const long long want = (units * steps + kAttWarps * 2 - 1) / (kAttWarps * 2);     // (two steps to a warp)
    return {1, (int)(want < slots / groups ? want : slots / groups), false};
  }
  return {S, 0, false};
}

int queries_of(const mixkv_pages* c, const int32_t q_tokens, const int32_t gqa, int* groups, int* NT) {
  if (q_tokens < 1 || gqa < 1) return MIXKV_ERR_INVALID_ARG;
  const long long R = (long long)q_tokens * gqa;
  if (R > MIXKV_PAGED_MAX_QUERIES) return MIXKV_ERR_UNSUPPORTED;
  const int eights = (int)((R + 7) / 8);
  *groups = (eights + kAttGroups - 1) / kAttGroups;
  *NT = (eights + *groups - 1) / *groups;
  if ((long long)c->batch * c->kv_heads * *groups > 1 << 24) return MIXKV_ERR_UNSUPPORTED;
  return MIXKV_OK;
}
// Workspace: part, part_mz, spans.
size_t part_bytes(const int ctas, const long long R) { return (size_t)ctas * 2 * R * (kHeadDim + 2) * 4; }
size_t att_workspace(const int NT, const int sms, const long long R) {
  return part_bytes(att_slots(NT, sms), R) + kAttUnits * sizeof(int2);
}

}  // namespace
}  // namespace mixkv

using namespace mixkv;

extern "C" void mixkv_internal_paged_shape(int64_t units, int32_t groups, int64_t steps, int32_t eights, int32_t sms,
                                           const int32_t* narrow, const int32_t* wide, int32_t* ctas, int32_t* large,
                                           int32_t* shared) {
  const AttShape s = att_shape(units, groups, steps, steps, eights, sms, [&](const int n) { return narrow[n]; },
                               [&](const int n) { return wide[n]; });
  *ctas = s.S, *large = s.wide, *shared = s.ctas;
}

extern "C" int mixkv_paged_workspace_size(const mixkv_pages* c, int32_t q_tokens, int32_t gqa_ratio, size_t* bytes) {
  PagePool p;
  int rc = check_pages(c, &p), groups, NT;
  if (rc != MIXKV_OK) return rc;
  if (!bytes) return MIXKV_ERR_INVALID_ARG;
  if ((rc = queries_of(c, q_tokens, gqa_ratio, &groups, &NT)) != MIXKV_OK) return rc;
  *bytes = att_workspace(NT, device_sm_count(), (long long)q_tokens * gqa_ratio);
  return MIXKV_OK;
}

extern "C" int mixkv_paged_attention(const mixkv_pages* c, const void* q, int32_t type, int64_t q_batch_stride,
                                     int64_t q_token_stride, int32_t q_tokens, int32_t gqa_ratio, float softmax_scale,
                                     int32_t max_rows, const int32_t* page_list_opt, const int32_t* counts_opt,
                                     int32_t top, void* workspace, size_t workspace_bytes, void* out, void* stream) {
  AttArgs a = {};
  int groups, NT;
  int rc = check_pages(c, &a.p);
  if (rc != MIXKV_OK) return rc;
  if (!q || !out || !workspace || (type != MIXKV_TYPE_BF16 && type != MIXKV_TYPE_FP16) || max_rows < 1 ||
      !(softmax_scale >= 0.f) || q_batch_stride < 0 || q_token_stride < 0 || q_batch_stride % 8 || q_token_stride % 8 ||
      (page_list_opt == nullptr) != (counts_opt == nullptr) || (page_list_opt && top < 1))
    return MIXKV_ERR_INVALID_ARG;
  if (page_list_opt && top > kMostListed) return MIXKV_ERR_UNSUPPORTED;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(page_list_opt, 4) || !aligned(counts_opt, 4))
    return MIXKV_ERR_INVALID_ARG;
  if ((rc = queries_of(c, q_tokens, gqa_ratio, &groups, &NT)) != MIXKV_OK) return rc;
  const long long units = (long long)c->batch * c->kv_heads;
  const int R = q_tokens * gqa_ratio, sms = device_sm_count();
  if (workspace_bytes < att_workspace(NT, sms, R)) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  if ((rc = device_check(nullptr)) != MIXKV_OK) return rc;
  const long long seen = max_rows < (long long)c->max_pages * c->page_rows ? max_rows : (long long)c->max_pages * c->page_rows;
  long long tiles = (seen + kPageTile - 1) / kPageTile;
  const long long listed = (long long)top * a.p.tiles, most = page_list_opt ? listed : tiles;
  if (page_list_opt && tiles > listed) tiles = listed;

  const bool bf16 = type == MIXKV_TYPE_BF16;
  static std::atomic<bool> done[4 * (kAttGroups + 1)][kMaxDevices];
  static ClusterFit fits[4 * (kAttGroups + 1)];   // (by variant, as `done`)
  const int dev = device_slot();
  auto variant = [&](const bool wide) { return 4 * NT + 2 * wide + bf16; };
  auto warps = [&](const bool wide) { return wide ? kAttWide : kAttWarps; };
  auto kernel_of = [&](const bool wide) { return bf16 ? att_kernel<__nv_bfloat16>(NT, wide) : att_kernel<__half>(NT, wide); };
  auto resident = [&](const bool wide) {
    return [&, wide](const int size) {
      const size_t smem = att_smem(NT, warps(wide));
      if (!answered(ensure_smem(kernel_of(wide), smem, done[variant(wide)], dev))) return 0;
      return fits[variant(wide)].ask(kernel_of(wide), 32 * warps(wide), smem, size, dev);
    };
  };
  const AttShape shape = att_shape(units, groups, (tiles + 1) / 2, (most + 1) / 2, NT, sms, resident(false), resident(true));
  const AttKernel kernel = kernel_of(shape.wide);
  const size_t smem = att_smem(NT, warps(shape.wide));
  if (ensure_smem(kernel, smem, done[variant(shape.wide)], dev) != cudaSuccess) return MIXKV_ERR_CUDA;
  a.q = q, a.q_batch = q_batch_stride, a.q_token = q_token_stride;
  a.T = q_tokens, a.G = gqa_ratio, a.R = R, a.by_group = Divider(gqa_ratio), a.max_rows = max_rows;
  a.list = page_list_opt, a.counts = counts_opt, a.top = top;
  a.units = (int)units, a.ctas = shape.ctas;
  a.scale_log2e = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)kHeadDim)) * kLog2e * c->k_scale;
  a.part = static_cast<float*>(workspace);
  a.part_mz = reinterpret_cast<float2*>(a.part + (size_t)shape.ctas * 2 * R * kHeadDim);
  a.spans = reinterpret_cast<int2*>(static_cast<unsigned char*>(workspace) + part_bytes(shape.ctas, R));
  a.out = out;
  a.per = ((R < 8 * NT ? R : 8 * NT) * (kHeadDim / 4) + shape.S - 1) / shape.S;
  const unsigned grid = shape.ctas ? (unsigned)shape.ctas : (unsigned)(units * shape.S);
  cudaError_t e = launch_pdl(kernel, dim3(grid, groups), dim3(32 * warps(shape.wide)), smem, (cudaStream_t)stream, shape.S, a);
  if (e == cudaSuccess && shape.ctas) {
    int per_row = 1;      // warps that go through the shares of one query row
    while (per_row < kJoinWarps && per_row * 2 * units < shape.ctas) per_row *= 2;
    const int at_once = kJoinWarps / per_row, blocks = (R + at_once - 1) / at_once;
    e = launch_pdl(bf16 ? k_paged_join<__nv_bfloat16> : k_paged_join<__half>, dim3((unsigned)(units * blocks)),
                   dim3(kJoinWarps * 32), 0, (cudaStream_t)stream, 1, a, Divider(per_row), Divider(blocks));
  }
  return e == cudaSuccess ? MIXKV_OK : MIXKV_ERR_CUDA;
}
