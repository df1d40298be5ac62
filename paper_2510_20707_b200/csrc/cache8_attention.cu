// Attention of the newest tokens over the paged 8-bit cache (format: include/mixkv.h), over all rows or over a sliding window and
// the first rows, and the weight that every row got of it.
//
// A warp takes a tile of 16 cache rows per step, brought by a bulk copy into a ring of its own.  Codes become fp16 exactly; the scale
// of a block is one number for the whole tile, so it multiplies logits and products, not codes.  The products run as m16n8k16 with the
// CACHE on the sixteen-row side and the query rows (tokens x heads of the group) on the eight-column side:
//   S^T[row, query]  = K q^T      A: rows g and g + 8 of the tile, a lane their dimensions 32 t .. 32 t + 31 (k-step s: 4 s .. 4 s + 3)
//   O^T[dim, query] += V^T P^T    A: dimensions 16 g + 2 m, + 1 of rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9; P^T from S^T by a transposing move
// Two rows of V are interleaved by byte moves before they are widened, so that a pair is two rows of one dimension.
//
// Softmax: a running reference per query row, moved only when a logit exceeds it by more than 2^kLag (one vote a step instead of
// a reduction); weights are fp16 times 2^kLift, sums are fp32.  For bf16 outputs a weight is ONE fp16 number: its rounding, 2^-11 of it, is an
// eighth of the output's own (0.0017 from 64 bits as with fp32 weights; two would cost 7 to 10 % of most calls' time, 1 % of one that counts
// weights over 256 long heads, 23 % with 32 query rows).  For fp16 outputs it would be as large as that (2.9e-4 from 64 bits where the outputs'
// rounding makes 2.1e-4, up to 1.7 times that where one row has most of the weight): there a weight is two of them, for 2 to 5 % of a call's
// time with one group of query rows, 12 with 35 rows, 24 with 32 over 64 heads.
//
// Weights of rows: what a row got is known when the sums are, so the logits go to the workspace as fp32 (R of them for a row of 257
// bytes), and the exponentials of one row's, taken in a fixed order, are added to the row's mass once all tiles have been read: by the
// clusters themselves, or by the kernel that joins the shares.
//
// What bounds it.  A row pair is 257 bytes, a tile of 16 costs a warp 426 instructions with int8, all told, and 335 with e4m3 (whose widening
// needs no subtraction).  256 heads of 1021 to 16384 rows (587 MB) take 104 us in this kernel under the profiler, weights counted: 5.7 TB/s, an
// instruction issued in 60 % of the clocks, the arithmetic pipe busy in 50, the tensor pipe in 18.  Without weights the call takes 101 us (an earlier
// build 103, and 93 with the same copies and no arithmetic); 8 heads of 131072 rows 49.2 (48.5 and 45).  Few or short heads are bounded by the chain
// from rows to table to tiles, the merge and the join (8 heads of 2048 rows 8.5 us; 8.7 and 5.2); drafts by eight warps an SM, which 255
// registers leave (35 query rows: issue slots 40 %, tensor pipe 33 %).  Loads that L2 evicts first: 8 heads of 131072 rows 49.6 us for 52.
//
// Measured and not taken, of earlier builds: two tiles a softmax step (256 heads 133 us for 131, 64 of 4096 rows 24.8 for 23.3); four warps in step on
// four tiles, each with 32 dimensions of all of them, so that warps need no merge (145 for 131, a draft 40 for 38: every warp then prepares every
// tile); forty query rows in one CTA, their queries in shared memory (a draft 42.6 for 36.5); two chains of products for two groups of query rows
// (nothing); weights in two parts only where a heavy one is among them (a draft 41.3 for 41.7, with 1.2 times the error).
#include <cfloat>

#include <cooperative_groups.h>

#include "attend.cuh"
#include "cache8.cuh"

namespace cg = cooperative_groups;

namespace mixkv {
namespace {

constexpr int kAttWarps = 4;
constexpr int kAttDepth = 2;                   // tiles of a warp on their way or in work
constexpr int kNoRow = 0x3fffffff;             // first row of a tile that is not there: beyond all
constexpr int kAttPitch = kHeadDim / 2 + 4;    // floats between the query rows of half a warp's sums
constexpr int kAttGroups = 4;                  // most groups of eight query rows a CTA takes
constexpr int kAttUnits = 1024;                // most units whose tiles are dealt out evenly
constexpr int kAttFew = 6, kAttMany = 16, kAttEven = 24;   // tiles of a warp (att_shape)
constexpr float kLag = 8.f, kLift = 6.f;       // largest weight 2^14
constexpr float kNoRef = -FLT_MAX;             // reference before the first row: no logit is below, and it is finite
// Sums of weighted values are kept times 2^8; those of a query row that has got something of a block with a scale above 2^64, times 2^-48:
// at 2^14 a weight, 2^30 rows and the largest values of either kind fit fp32, and what falls below its range is nothing beside either
// the smallest values (2^-126) or that block's own rounding.
constexpr float kWide = 0x1p64f, kFine = 0x1p8f, kCoarse = 0x1p-48f, kBack = 0x1p40f;

// Whether a warp has the queries in registers (with more of them there is no room).
__host__ __device__ constexpr bool att_held(int NT) { return NT <= 2; }
// rings of the warps (a cluster's CTA: then its averages); half of the warps' sums; references, sums of weights and units of the warps;
// references and sums of the CTA, the cluster; barriers and rows of the rings; what the queries were divided by, and they (or in
// the place of the sums)
__host__ __device__ constexpr size_t att_smem(int NT) {
  return kAttWarps * (kAttDepth * kBlockBytes + 8 * NT * kAttPitch * 4) + (3 * kAttWarps + 2 + 2 * kMaxCluster) * 8 * NT * 4 +
         kAttWarps * kAttDepth * 16 + 16 + 8 * NT * 4 + (att_held(NT) ? 0 : 8 * NT * kHeadDim * 2);
}
// CTAs of an SM, which sets the registers of a thread.  us a call, one token of four query heads unless said.
// One group of query rows, bf16: four of 128 registers for three, 256 heads of 1024 rows 18.7 for 20.7, of 2048 29.0 for 30.2, 32 of 4096
// 14.6 for 15.1; but 64 of one to 8192 rows 24.9 for 21.8 (att_shape then deals all tiles out), 8 of 2048 9.3 for 8.7.
// fp16, whose weights take more registers: three of 168 for four, which spill 28 bytes, 8 heads of 2048 8.8 for 9.7, 256 of 2048 31.4 for 31.7,
// of 8704 98.6 for 99.8, 64 of one to 8192 22.2 for 27.3; but 256 of 1024 21.3 for 20.0.
// Two groups (two tokens of seven query heads): two for three, which spill 48 bytes with bf16 and 60 with fp16, bf16 64 heads of 2048 16.1 for
// 17.5, 256 of 1024 21.9 for 28.3, of 70 to 1639 28.0 for 29.0, of 1639 36.7 for 36.2; fp16 64 of 2048 16.4 for 18.1, 256 of 70 to 1639
// 40.0 for 41.9, of 1024 34.2 for 33.1.  More groups: 255 registers, the most there are.
__host__ __device__ constexpr int att_per_sm(int NT, bool half) { return NT > 1 ? 2 : half ? 3 : 4; }
static_assert(att_per_sm(1, false) >= att_per_sm(1, true), "a workspace has room for the shares of bf16 outputs, whatever the type");

struct AttArgs {
  CachePool p;
  const void* q;
  long long q_batch, q_token;
  int T, G, R;               // tokens, heads of a group, T * G
  Divider by_group;          // of G
  int max_rows;
  int window, sinks;         // window 0: all rows
  int units;
  int ctas;                  // that share all tiles evenly; 0: a cluster has a unit
  int per;                   // fours of outputs of a CTA of such a cluster
  float scale_log2e;
  int2* spans;               // [units]: first CTA with a share of a unit, times two, plus one if its run begins before the unit; last CTA
  float* part;               // [2 ctas][R][128]: averages of a unit's share, where it is not the whole
  float2* part_mz;           // [2 ctas][R]: (reference, sum of weights)
  float2* stats;             // [units][R]: (reference, 1 / sum) of a query row
  bool inside;               // the weights are added up by the clusters
  float* logits;             // [units][cap][16][pitch], log2 units; nullptr: weights are not asked for
  int cap, pitch;            // tiles of a unit that a call can see; query rows, made even
  void* out;
};

// Tiles of a unit that the call sees, numbered 0 .. tiles - 1: tile i is number i, and from `sink` on i - gap.
struct UnitTiles {
  int n, tiles, sink, gap;
};
__device__ __forceinline__ UnitTiles unit_tiles(const AttArgs& a, const int u) {
  UnitTiles r;
  int n = fresh(a.p.rows + u);
  n = min(n, a.max_rows);
  n = (int)min((long long)n, (long long)a.p.max_pages * a.p.page_rows);
  r.n = n = max(n, 0);
  r.tiles = (n + kBlockRows - 1) >> 4;
  r.sink = r.tiles, r.gap = 0;
  if (a.window > 0) {     // token 0 sees the lowest rows of the window, from n - T - window + 1 on
    const int low = (int)max(0ll, (long long)n - a.T + 1 - a.window) >> 4, sink = (min(a.sinks, n) + kBlockRows - 1) >> 4;
    if (low > sink) r.sink = sink, r.gap = low - sink, r.tiles -= r.gap;
  }
  return r;
}
// Rows that query row's token (of T) sees: up to `last`, and from `low` on or below the sinks.
struct Seen {
  int last, low;
};
__device__ __forceinline__ Seen seen_by(const AttArgs& a, const int n, const int token) {
  const int p = n - a.T + token;
  return Seen{p, a.window > 0 ? (int)max((long long)p - a.window + 1, -1ll) : -1};
}

// Place in the pool and first row of tile number `i` of a unit (-1, kNoRow: none).
struct TileAt {
  int tile, row;
};
__device__ __forceinline__ TileAt tile_at(const AttArgs& a, const int u, const UnitTiles& ut, const int i) {
  // (without a window the table is asked before the unit's rows are looked at: both may be on their way)
  const int t = a.window > 0 && i >= ut.sink ? i + ut.gap : i, page = a.p.by_tiles.div(t), in = t - page * a.p.tiles;
  const int id = page < a.p.max_pages ? fresh(a.p.table + (long long)u * a.p.max_pages + page) : -1;
  if (i >= ut.tiles || id < 0 || id >= a.p.num_pages) return TileAt{-1, kNoRow};
  return TileAt{id * a.p.tiles + in, t * kBlockRows};
}

// Row of the output that query row r of a unit has.
__device__ __forceinline__ long long out_row(const AttArgs& a, const int u, const int r) {
  const int b = a.p.by_heads.div(u), h = u - b * a.p.H, token = a.by_group.div(r);
  return ((long long)b * a.T + token) * ((long long)a.p.H * a.G) + h * a.G + (r - token * a.G);
}
// Four outputs.
template <typename T>
__device__ __forceinline__ void store_row(T* to, const float4& x) {
  *reinterpret_cast<uint2*>(to) = make_uint2(narrow2<T>(x.x, x.y), narrow2<T>(x.z, x.w));
}
// (zero where there were no weights)
__device__ __forceinline__ float one_over(const float den) { return den == 0.f ? 0.f : 1.f / den; }
// The same but for two units of the last place (sums of weights are between 1 and 2^44), for the merge of a CTA's warps, which every unit
// goes through: a division there took 0.9 us of a draft's 41.8, 0.2 of eight heads' of 2048 rows.
__device__ __forceinline__ float about_one_over(const float den) { return den == 0.f ? 0.f : __fdividef(1.f, den); }
__device__ __forceinline__ void store_stat(const AttArgs& a, const int u, const int r, const float ref, const float by) {
  if (a.logits) a.stats[(long long)u * a.R + r] = make_float2(ref, by);
}
// Token of query row r of a unit (rows of the padding: the last).
__device__ __forceinline__ int token_of(const AttArgs& a, const int r) { return a.by_group.div(min(r, a.R - 1)); }

__device__ __forceinline__ uint32_t word_of(const uint4& v, const int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Query rows first .. first + 8 NT - 1 of a unit, as B fragments (k-step s of group nt and lane (g, t) at [nt][s][lane]: query row g,
// dimensions 32 t + 4 s .. + 3) and what they are to be multiplied by, into shared memory.  bf16 rows are divided by a power of two that
// brings their largest magnitude to [1, 2): exact as fp16 but for what is 2^-24 of it.  A row with a NaN or an infinity is zeros times NaN.
template <typename T, int NT>
__device__ __forceinline__ void stage_queries(const AttArgs& a, const int u, const int first, const int warp, const int lane, uint2* q,
                                              float* up) {
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  const int b = a.p.by_heads.div(u), h = u - b * a.p.H, g = lane >> 2, t = lane & 3;
  for (int nt = warp; nt < NT; nt += kAttWarps) {
    const int r = first + 8 * nt + g;
    uint4 raw[4];
    const bool on = r < a.R;
    const int token = on ? a.by_group.div(r) : 0;
    const T* src = static_cast<const T*>(a.q) + b * a.q_batch + token * a.q_token +
                   (long long)(h * a.G + (on ? r - token * a.G : 0)) * kHeadDim + 32 * t;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = on ? fresh(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0, 0, 0, 0);
    uint32_t bits = 0;       // magnitudes in the order of their bits, infinities and NaN above the others
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) bits = max_u16x2(bits, word_of(raw[i], e) & 0x7fff7fffu);
    bits = max(bits & 0xffffu, bits >> 16);
    bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 1));
    bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 2));
    const float most = widen2<T>(bits).x;
    const bool odd = !(most < INFINITY);
    // 2^e <= most < 2^(e + 1) (subnormal: 2^-126); down = 2^-e
    const uint32_t e = min(max(__float_as_uint(most) >> 23, 1u), 253u);
    const bool scaled = kBf16 && most > 0.f && !odd;
    const float down = scaled ? __uint_as_float((254u - e) << 23) : 1.f;
    if (t == 0) up[8 * nt + g] = odd ? NAN : scaled ? __uint_as_float(e << 23) : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t x[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        x[w] = word_of(raw[i], w);
        if constexpr (kBf16) {
          const float2 y = widen2<T>(x[w]);
          x[w] = narrow2<__half>(y.x * down, y.y * down);
        }
        if (odd) x[w] = 0u;
      }
      q[(nt * 8 + 2 * i) * 32 + lane] = make_uint2(x[0], x[1]);
      q[(nt * 8 + 2 * i + 1) * 32 + lane] = make_uint2(x[2], x[3]);
    }
  }
}

template <typename T, int NT, bool E4M3>
struct AttState {
  static constexpr bool kHeld = att_held(NT);
  static constexpr int kParts = std::is_same<T, __half>::value ? 2 : 1;      // of a weight
  uint2 q[kHeld ? NT : 1][8];
  const uint2* at;          // this lane's fragments in shared memory
  float f[NT][2];           // products of codes to log2 units, without the block's scale: query rows 2 t, 2 t + 1
  float acc[NT][8][4];      // dimensions 16 g + 2 m (0, 1), 16 g + 2 m + 1 (2, 3) of query rows 2 t, 2 t + 1
  float ref[NT][2], z[NT][2];   // weights are 2^(logit - ref)
  float unit[NT][2];            // acc is in units of one over it: kFine or kCoarse

  __device__ __forceinline__ void start(const AttArgs& a, const uint2* staged, const float* up, const int lane) {
    const int t = lane & 3;
    at = staged + lane;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if constexpr (kHeld) {
#pragma unroll
        for (int k = 0; k < 8; ++k) q[nt][k] = at[(nt * 8 + k) * 32];
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        f[nt][c] = up[8 * nt + 2 * t + c] * a.scale_log2e;
        ref[nt][c] = kNoRef, z[nt][c] = 0.f, unit[nt][c] = kFine;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[nt][i][c] = 0.f;
    }
  }

  // s[2 j + c] = product of row g + 8 j of the tile and query row 8 nt + 2 t + c
  __device__ __forceinline__ void products(const unsigned char* tile, const int g, const int t, float (&s)[NT][4]) const {
    float odd[4];      // (of one group of query rows, two chains of four instead of one of eight)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const unsigned char* rows = tile + piece_at(g, 2 * t + half);
      const uint4 lo = *reinterpret_cast<const uint4*>(rows), hi = *reinterpret_cast<const uint4*>(rows + 8 * 128);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t a0, a2, a1, a3;
        codes_to_half<E4M3>(word_of(lo, w), a0, a2);
        codes_to_half<E4M3>(word_of(hi, w), a1, a3);
        const int k = 4 * half + w;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float(&d)[4] = NT == 1 && (k & 1) ? odd : s[nt];
          uint2 b;
          if constexpr (kHeld) b = q[nt][k];
          else b = at[(nt * 8 + k) * 32];
          if (k == 0 || (NT == 1 && k == 1)) mma_f16_first(d, a0, a1, a2, a3, b.x, b.y);
          else mma_f16(d, a0, a1, a2, a3, b.x, b.y);
        }
      }
    }
    if constexpr (NT == 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[0][i] += odd[i];
    }
  }

  // A tile whose first row is `row`, of a unit of n rows; `first`: the CTA's first query row.  edge: some query row does not see some row.
  // logits: where they go (of row 0, the CTA's first query row), or nullptr.
  __device__ __forceinline__ void step(const AttArgs& a, const unsigned char* tile, const int row, const bool edge, const int n,
                                       const int first, const int lane, float* logits) {
    const int g = lane >> 2, t = lane & 3;
    float y[NT][4];
    products(tile, g, t, y);
    const float2 scale = *reinterpret_cast<const float2*>(tile + kBlockScales);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[nt][i] = __fmul_rn(y[nt][i], f[nt][i & 1] * scale.x);
    if (edge) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const Seen see = seen_by(a, n, token_of(a, first + 8 * nt + 2 * t + c));
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = row + g + 8 * j;
            if (r > see.last || (r < see.low && r >= a.sinks)) y[nt][2 * j + c] = -INFINITY;
          }
        }
    }
    if (logits) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (first + 8 * nt + 2 * t < a.R)
            *reinterpret_cast<float2*>(logits + (g + 8 * j) * a.pitch + 8 * nt + 2 * t) = make_float2(y[nt][2 * j], y[nt][2 * j + 1]);
    }
    // (A logit is rounded before the reference, itself a logit, is taken from it: of a product that is not, equal logits beyond 2^24 would
    // differ from it by their last bits, whole powers of two.)
    bool above = false;
    float x[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[nt][i] = __fsub_rn(y[nt][i], ref[nt][i & 1]);
        above |= x[nt][i] > kLag + kLift;
      }
    if (__any_sync(0xffffffffu, above)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float to = fmaxf(ref[nt][c], column_max(fmaxf(y[nt][c], y[nt][2 + c])) - kLift);
          const float shrink = ex2(ref[nt][c] - to);
          ref[nt][c] = to, z[nt][c] *= shrink;
          x[nt][c] = __fsub_rn(y[nt][c], to), x[nt][2 + c] = __fsub_rn(y[nt][2 + c], to);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[nt][i][c] *= shrink, acc[nt][i][2 + c] *= shrink;
        }
      bool coarse = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) coarse |= unit[nt][0] != kFine || unit[nt][1] != kFine;
      if (__any_sync(0xffffffffu, coarse)) {      // back to the finer unit where nothing large is left
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fmaxf(fabsf(acc[nt][i][c]), fabsf(acc[nt][i][2 + c])));
            const float by = column_max(most) < kBack && unit[nt][c] != kFine ? kFine / kCoarse : 1.f;
            if (by != 1.f) unit[nt][c] = kFine;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[nt][i][c] *= by, acc[nt][i][2 + c] *= by;
          }
      }
    }
    uint32_t p[kParts][NT][2];   // B fragments: query row g, tile rows 2 t, 2 t + 1 and 2 t + 8, 2 t + 9
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[nt][i] = ex2(x[nt][i]), z[nt][i & 1] += x[nt][i];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float lo = x[nt][2 * j], hi = x[nt][2 * j + 1];
        const uint32_t w = narrow2<__half>(lo, hi);
        p[0][nt][j] = transpose8x8(w);
        if constexpr (kParts > 1) {
          const float2 rounded = widen2<__half>(w);
          p[1][nt][j] = transpose8x8(narrow2<__half>(lo - rounded.x, hi - rounded.y));
        }
      }
    }
    // The block's scale multiplies the tile's products on their way into the sums.  (In the weights it would take them out of fp16's
    // range: of 16384 rows with 2^-17 of the heaviest one's weight, beside a block of values 3000 times as large, a quarter was lost.)  A
    // query row's sums are in a unit of their own: with one for all, values that one row sees would push those of the others out of fp32.
    if (__builtin_expect(!(scale.y <= kWide), 0)) {
      const bool nan = scale.y != scale.y;      // (it must not reach a query row that sees none of the block's rows)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const Seen see = seen_by(a, n, token_of(a, first + 8 * nt + 2 * t + c));
          const bool sees = row <= see.last && (row + kBlockRows - 1 >= see.low || row < a.sinks);
          const bool gets = column_max(fmaxf(x[nt][c], x[nt][2 + c])) > 0x1p-25f;      // (of less, fp16 is zero)
          const float by = nan ? (sees ? NAN : 1.f) : gets ? kCoarse / unit[nt][c] : 1.f;
          if (!nan && gets) unit[nt][c] = kCoarse;
#pragma unroll
          for (int m = 0; m < 8; ++m) acc[nt][m][c] *= by, acc[nt][m][2 + c] *= by;
        }
      if (nan) return;
    }
    uint4 v[2][2];       // 16 dimensions of rows 2 t + e + 8 h
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) v[h][e] = *reinterpret_cast<const uint4*>(tile + kBlockV + piece_at(2 * t + e + 8 * h, g));
    f32x2 by[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) by[nt] = mul2(pack2(scale.y, scale.y), pack2(unit[nt][0], unit[nt][1]));
#pragma unroll
    for (int m = 0; m < 8; ++m) {      // A fragments: dimensions 16 g + 2 m, + 1
      const uint32_t sel = (m & 1) ? 0x7362u : 0x5140u;
      uint32_t a0, a1, a2, a3;
      codes_to_half<E4M3>(__byte_perm(word_of(v[0][0], m >> 1), word_of(v[0][1], m >> 1), sel), a0, a1);
      codes_to_half<E4M3>(__byte_perm(word_of(v[1][0], m >> 1), word_of(v[1][1], m >> 1), sel), a2, a3);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float d[4];
        mma_f16_first(d, a0, a1, a2, a3, p[0][nt][0], p[0][nt][1]);
        if constexpr (kParts > 1) mma_f16(d, a0, a1, a2, a3, p[1][nt][0], p[1][nt][1]);
        float(&to)[4] = acc[nt][m];
        unpack2(fma2(pack2(d[0], d[1]), by[nt], pack2(to[0], to[1])), to[0], to[1]);
        unpack2(fma2(pack2(d[2], d[3]), by[nt], pack2(to[2], to[3])), to[2], to[3]);
      }
    }
  }
};

// Adds to the mass of a unit's rows what they got, a thread a row at a time: of the tiles number(0 .. n - 1) (a page's tiles lie one after
// the other in the pool and in the masses).  stat: (reference, 1 / sum) of the query rows, there once ready() has been called (by the whole
// CTA), which the first rows' logits do not wait for.  One addition a row of each unit, atomic since units may share a page: where they
// do not, there is no order in which it could differ.
template <int THREADS, typename Number, typename Ready>
__device__ __forceinline__ void add_weights(const AttArgs& a, const int u, const UnitTiles& ut, const float2* stat, const int n,
                                            const Number& number, const Ready& ready) {
  constexpr int kAtOnce = 4, kStep = THREADS / kBlockRows;       // rows of a thread on their way, eight query rows of each
  const int in = threadIdx.x % kBlockRows;
  const bool fours = (a.pitch & 3) == 0;
  int at[kAtOnce];
  const float* row[kAtOnce];
  float4 y[kAtOnce][2];
  const auto load = [&](const int r0) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + 4 * h;
        if (at[k] < 0 || r >= a.pitch) continue;
        if (fours) {
          y[k][h] = fresh(reinterpret_cast<const float4*>(row[k] + r));
        } else {
          const float2 lo = fresh(reinterpret_cast<const float2*>(row[k] + r));
          const float2 hi = r + 2 < a.pitch ? fresh(reinterpret_cast<const float2*>(row[k] + r + 2)) : make_float2(0.f, 0.f);
          y[k][h] = make_float4(lo.x, lo.y, hi.x, hi.y);
        }
      }
  };
  const auto begin = [&](const int i) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int tile = number(min(i + k * kStep, n - 1));
      const TileAt t = tile_at(a, u, ut, tile);
      at[k] = i + k * kStep < n && t.tile >= 0 && t.row + in < ut.n ? t.tile : -1;
      row[k] = a.logits + (((long long)u * a.cap + tile) * kBlockRows + in) * a.pitch;
    }
    load(0);
  };
  // (what a query row does not see gets nothing of it, if it is NaN either)
  const auto weight = [&](const float x, const int r) { return r < a.R && x != -INFINITY ? ex2(x - stat[r].x) * stat[r].y : 0.f; };
  int i = threadIdx.x / kBlockRows;
  if (i < n) begin(i);
  ready();
#pragma unroll 1
  while (i < n) {
    float sum[kAtOnce] = {};
#pragma unroll 1
    for (int r = 0;;) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (r + 4 * h < a.R) {
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k)
            sum[k] += weight(y[k][h].x, r + 4 * h) + weight(y[k][h].y, r + 4 * h + 1) + weight(y[k][h].z, r + 4 * h + 2) +
                      weight(y[k][h].w, r + 4 * h + 3);
        }
      r += 8;
      if (r >= a.R) break;
      load(r);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (at[k] >= 0) atomicAdd(a.p.mass + (long long)at[k] * kBlockRows + in, sum[k]);
    i += kAtOnce * kStep;
    if (i < n) begin(i);
  }
}

// grid.x: units * S in clusters of S (ctas == 0), or ctas; grid.y: groups of 8 NT query rows
template <typename T, int NT, bool E4M3>
__global__ void __launch_bounds__(32 * kAttWarps, att_per_sm(NT, std::is_same<T, __half>::value)) k_cache8_attention(const AttArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int W = kAttWarps, Q = 8 * NT, kSums = Q * kAttPitch, kThreads = 32 * W, kRing = kAttDepth * kBlockBytes;
  float* xo = reinterpret_cast<float*>(smem);   // [Q][128]: a cluster's CTA has its averages where its rings were
  static_assert(Q * kHeadDim * 4 <= W * kRing, "averages of a CTA fit the rings");
  static_assert(kBlockBytes % 16 == 0, "tiles in the ring are 16-byte aligned");
  float* sums = reinterpret_cast<float*>(smem + W * kRing);   // [warps][Q][pitch]
  float* wm = sums + W * kSums;      // [warps][Q]
  float* wz = wm + W * Q;            // [warps][Q]
  float* wu = wz + W * Q;            // [warps][Q]: what their sums of values are to be multiplied by
  float* xm = wu + W * Q;            // [Q]
  float* xz = xm + Q;                        // [Q]
  float* allm = xz + Q;                      // [8][Q]
  float* allz = allm + kMaxCluster * Q;      // [8][Q]
  uint64_t* bars = reinterpret_cast<uint64_t*>(allz + kMaxCluster * Q);   // [warps][depth]
  int* rows = reinterpret_cast<int*>(bars + W * kAttDepth);   // [warps][depth]: first rows of the tiles
  int* abort = rows + W * kAttDepth;         // [4]
  float* up = reinterpret_cast<float*>(abort + 4);      // [Q]
  uint2* queries = reinterpret_cast<uint2*>(att_held(NT) ? sums : up + Q);   // [NT][8][32]
  static_assert(NT * 2048 <= W * kSums * 4, "queries fit the place of the sums");
  __shared__ int starts[kAttUnits + 1];      // first tile of every unit
  __shared__ int warp_total[W];
  __shared__ float2 stat[Q];                 // (reference, 1 / sum) of a cluster's query rows
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

  // tiles lo .. hi - 1: of a cluster's unit, or of all units one after the other
  int u = shares ? 0 : cluster_id(), lo = crank * W, hi;
  if (shares) {
    // first tiles of all units: a thread takes consecutive ones
    constexpr int kEach = kAttUnits / kThreads;
    int mine[kEach], sum = 0;
    const int u0 = tid * kEach;
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine[i] = u0 + i < a.units ? unit_tiles(a, u0 + i).tiles : 0;
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
    const int share = share_of(total, a.ctas);
    if (blockIdx.x + 1 == gridDim.x && blockIdx.y == 0) {      // (the CTA whose run is the shortest)
      for (int i = tid; i < a.units; i += kThreads) {
        const int from = starts[i], to = starts[i + 1], c0 = from < to ? from / share : 0;
        a.spans[i] = from < to ? make_int2(2 * c0 + (c0 * share < from), (to - 1) / share) : make_int2(0, -1);
      }
    }
    lo = blockIdx.x * share, hi = min(lo + share, total);
    if (lo >= hi) return;
    int x = 0, y = a.units;     // the last unit that begins at or before lo
    while (y - x > 1) {
      const int m = (x + y) >> 1;
      (starts[m] <= lo ? x : y) = m;
    }
    u = x;
  } else {
    hi = unit_tiles(a, u).tiles;
  }
  const int stride = S * W, begin = lo + warp;
  const int count = begin < hi ? (hi - begin + stride - 1) / stride : 0;   // tiles of this warp
  unsigned char* ring = smem + warp * kRing;
  int* ring_rows = rows + warp * kAttDepth;

  TileAt ahead = {};      // lane l knows tile 32 n + l of the warp, 32 n the last multiple at or before `sent`
  auto locate = [&](const int i) {
    int f = begin + i * stride, v = u;
    if (i >= count) return;
    if (shares) {
      int y = a.units;
      while (y - v > 1) {
        const int m = (v + y) >> 1;
        (starts[m] <= f ? v : y) = m;
      }
      f -= starts[v];
    }
    ahead = tile_at(a, v, unit_tiles(a, v), f);
  };
  locate(lane);
  int sent = 0, slot_out = 0;
  auto send = [&]() {   // the copy of the warp's tile `sent`
    if ((sent & 31) == 0 && sent) locate(sent + lane);
    if (lane == (sent & 31)) {
      uint64_t* full = &bar[slot_out];
      ring_rows[slot_out] = ahead.row;
      if (ahead.tile >= 0) {
        mbar_expect_tx(full, kBlockBytes);
        bulk_load(ring + slot_out * kBlockBytes, a.p.pool + (long long)ahead.tile * kBlockBytes, kBlockBytes, full, l2_evict_first());
      } else {
        mbar_arrive(full);    // nothing to come
      }
    }
    ++sent, slot_out = slot_out + 1 == kAttDepth ? 0 : slot_out + 1;
  };
  while (sent < min(count, kAttDepth)) send();
  int slot = 0;
  uint32_t parity = 0;
  bool lost = false;

  for (int f = begin;;) {     // one unit after the other
    int end = hi, from = 0;
    if (shares) {
      while (starts[u + 1] <= max(lo, starts[u])) ++u;    // (units without tiles)
      end = min(hi, starts[u + 1]), from = starts[u];
    }
    AttState<T, NT, E4M3> st;
    stage_queries<T, NT>(a, u, first, warp, lane, queries, up);
    __syncthreads();
    st.start(a, queries, up, lane);
    if (att_held(NT)) __syncthreads();      // (before sums are written where they were)
    const int n = unit_tiles(a, u).n;
    const int clear = n - a.T + 1;                               // rows below are seen by all,
    const int low = a.window > 0 ? seen_by(a, n, a.T - 1).low : -1;   // from here on, or among the sinks
    float* logits = a.logits ? a.logits + (long long)u * a.cap * kBlockRows * a.pitch + first : nullptr;
    for (; f < end && !lost; f += stride) {
      if (!mbar_wait_warp(&bar[slot], parity, abort)) {
        lost = true;
        break;
      }
      const int row = ring_rows[slot];
      float* to = logits ? logits + (long long)(f - from) * (kBlockRows * a.pitch) : nullptr;
      if (row != kNoRow) {
        const bool inside = row + kBlockRows <= clear && (row >= low || row + kBlockRows <= a.sinks);
        st.step(a, ring + slot * kBlockBytes, row, !inside, n, first, lane, to);
      }
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
    // ---- the warps merge through shared memory, the dimensions 16 g .. 16 g + 7 first and then the others.  What is handed on are averages
    // of values, with the sum of weights that they stand for: no larger than the values, whatever the units were.
    float* own = sums + warp * kSums;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float z = column_sum(st.z[nt][c]);
        const int r = 8 * nt + 2 * t + c;
        if (g == 0) wm[warp * Q + r] = st.ref[nt][c], wz[warp * Q + r] = lost ? NAN : z;
        if (g == 0) wu[warp * Q + r] = st.unit[nt][c] == kFine ? 1.f / kFine : 1.f / kCoarse;
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
        float M = kNoRef, den = 0.f, sc[W];
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, wm[w * Q + r]);
#pragma unroll
        for (int w = 0; w < W; ++w) {
          sc[w] = ex2(wm[w * Q + r] - M);
          den = fmaf(wz[w * Q + r], sc[w], den);
        }
        const float by = about_one_over(den);
        float4 mean = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w)
          add_scaled(mean, *reinterpret_cast<const float4*>(sums + w * kSums + r * kAttPitch + x), sc[w] * by * wu[w * Q + r]);
        if (whole) {
          store_row(static_cast<T*>(a.out) + out_row(a, u, first + r) * kHeadDim + dim, mean);
          if (dim == 0) store_stat(a, u, first + r, M, by);
          if (dim == 0 && !shares) stat[r] = make_float2(M, by);
        } else if (shares) {
          const long long at = (long long)share * a.R + first + r;
          *reinterpret_cast<float4*>(a.part + at * kHeadDim + dim) = mean;
          if (dim == 0) a.part_mz[at] = make_float2(M, den);
        } else {
          *reinterpret_cast<float4*>(xo + r * kHeadDim + dim) = mean;
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
    // (a cluster that has all query rows of its unit adds up the weights of the tiles that its CTAs read)
    const auto weigh = [&]() {
      if (!a.inside) return;
      __syncthreads();
      const int mine = unit_tiles(a, u).tiles - crank * W, round = S * W;     // tiles from the CTA's first on; to its next ones
      const int tiles = mine <= 0 ? 0 : mine / round * W + min(mine % round, W);
      add_weights<kThreads>(a, u, unit_tiles(a, u), stat, tiles, [&](const int i) { return crank * W + i / W * round + i % W; }, [] {});
    };
    if (whole) {
      weigh();
      return;
    }

    // ---- the CTAs of the cluster merge through distributed shared memory, each a slice of the outputs
    cluster.sync();
    for (int e = tid; e < S * Q; e += kThreads) {
      const int k = e / Q, r = e % Q;
      allm[e] = *cluster.map_shared_rank(&xm[r], k);
      allz[e] = *cluster.map_shared_rank(&xz[r], k);
    }
    __syncthreads();
    if (a.inside) {
      for (int r = tid; r < live; r += kThreads) {
        float M = kNoRef, den = 0.f;
        for (int k = 0; k < S; ++k) M = fmaxf(M, allm[k * Q + r]);
        for (int k = 0; k < S; ++k) den = fmaf(allz[k * Q + r], ex2(allm[k * Q + r] - M), den);
        stat[r] = make_float2(M, one_over(den));
      }
    }
    for (int e = crank * a.per + tid; e < min((crank + 1) * a.per, live * (kHeadDim / 4)); e += kThreads) {
      const int r = e / (kHeadDim / 4), dim = 4 * (e % (kHeadDim / 4));
      float M = kNoRef, den = 0.f, share_z[kMaxCluster];
      float4 x[kMaxCluster];
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k)
        if (k < S) {
          M = fmaxf(M, allm[k * Q + r]);
          x[k] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(xo + r * kHeadDim + dim, k));
        }
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k)
        if (k < S) {
          const float sc = ex2(allm[k * Q + r] - M);
          share_z[k] = allz[k * Q + r] * sc, den = fmaf(allz[k * Q + r], sc, den);
        }
      const float by = one_over(den);
      float4 mean = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k)
        if (k < S) add_scaled(mean, x[k], share_z[k] * by);
      store_row(static_cast<T*>(a.out) + out_row(a, u, first + r) * kHeadDim + dim, mean);
      if (dim == 0) store_stat(a, u, first + r, M, by);
    }
    weigh();
    cluster.sync();   // a CTA's shared memory stays alive until its peers have read it
    return;
  }
}

// What is left when all tiles have been read.  grid.x: units, `join` + `add` CTAs to one.
//  - join: outputs of the query rows of units that several CTAs had a part of, `per_row.d` warps, a power of two, taking the shares of a
//    row in turn, and zeros for units without rows.
//  - add: what a run of the unit's rows got of the weights goes to their mass.
// Either works out the statistics of its query rows for itself: the outputs and the masses do not wait for one another, nor either of them for
// a launch and its first loads, which would cost as much as they do.
constexpr int kEndWarps = 8, kEndThreads = kEndWarps * 32, kEndPerSm = 3;
template <typename T>
__global__ void __launch_bounds__(kEndThreads, kEndPerSm) k_cache8_finish(const AttArgs a, const Divider by_unit, const int join, const int add,
                                                                         const Divider per_row) {
  __shared__ float4 sums[kEndWarps][32];
  __shared__ float2 stat[MIXKV_CACHE8_MAX_QUERIES];      // (reference, 1 / sum)
  __shared__ float2 of_warp[kEndWarps];                  // (reference, sum)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int u = by_unit.div(blockIdx.x), c = blockIdx.x - u * (int)by_unit.d;
  pdl_wait();
  const int2 span = a.ctas ? __ldcg(a.spans + u) : make_int2(0, 0);
  const int c0 = span.x >> 1, c1 = span.y;
  const bool joined = c0 != c1;
  const auto part_row = [&](const int k, const int r) { return (2LL * k + (k == c0 ? span.x & 1 : 0)) * a.R + r; };
  const auto statistics = [&]() {
    if (joined) {
      int lanes = 1;       // that share a query row
      while (lanes < 32 && lanes < c1 - c0 + 1) lanes *= 2;
      const int at = lane & (lanes - 1), at_once = 32 / lanes;
      for (int r = warp * at_once + lane / lanes; r - lane / lanes < a.R; r += kEndWarps * at_once) {
        float M = kNoRef, den = 0.f;
        for (int k = c0 + at; k <= c1 && r < a.R; k += lanes) {
          const float2 mz = __ldcg(a.part_mz + part_row(k, r));
          const float to = fmaxf(M, mz.x);
          den = fmaf(den, ex2(M - to), mz.y * ex2(mz.x - to));
          M = to;
        }
        float most = M;
        for (int o = 1; o < lanes; o *= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        den *= ex2(M - most);
        for (int o = 1; o < lanes; o *= 2) den += __shfl_xor_sync(0xffffffffu, den, o);
        if (at == 0 && r < a.R) stat[r] = make_float2(most, one_over(den));
      }
    } else {
      for (int r = tid; r < a.R; r += kEndThreads) stat[r] = __ldcg(a.stats + (long long)u * a.R + r);
    }
    __syncthreads();
  };
  if (c >= join) {
    const UnitTiles ut = unit_tiles(a, u);
    const int each = (ut.tiles + add - 1) / add, begin = min((c - join) * each, ut.tiles), n = min(each, ut.tiles - begin);
    if (n > 0) add_weights<kEndThreads>(a, u, ut, stat, n, [&](const int i) { return begin + i; }, statistics);
    return;
  }
  if (!joined) return;
  const int slot = per_row.div(warp), part = warp - slot * per_row.d, at_once = per_row.div(kEndWarps), r = c * at_once + slot;
  const bool on = r < a.R;
  float M = kNoRef, den = 0.f;
  float4 mean = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kAtOnce = 4;      // shares whose sums come in one round trip
#pragma unroll 1
  for (int k = c0 + part; on && k <= c1; k += kAtOnce * per_row.d) {
    float4 x[kAtOnce];
    float2 mz[kAtOnce];
    float to = M;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const long long at = part_row(min(k + i * (int)per_row.d, c1), r);
      mz[i] = __ldcg(a.part_mz + at);
      x[i] = __ldcg(reinterpret_cast<const float4*>(a.part + at * kHeadDim) + lane);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) to = fmaxf(to, mz[i].x);
    const float had = den * ex2(M - to);
    den = had;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      mz[i].y = k + i * (int)per_row.d <= c1 ? mz[i].y * ex2(mz[i].x - to) : 0.f;
      den += mz[i].y;
    }
    M = to;
    const float by = one_over(den), old = had * by;
    mean.x *= old, mean.y *= old, mean.z *= old, mean.w *= old;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) add_scaled(mean, x[i], mz[i].y * by);
  }
  if (per_row.d > 1) {
    sums[warp][lane] = mean;
    if (lane == 0) of_warp[warp] = make_float2(M, den);
    __syncthreads();
    if (part) return;
    float to = M;
    for (int w = 1; w < (int)per_row.d; ++w) to = fmaxf(to, of_warp[warp + w].x);
    const float mine = den * ex2(M - to);
    den = mine;
    for (int w = 1; w < (int)per_row.d; ++w) den = fmaf(of_warp[warp + w].y, ex2(of_warp[warp + w].x - to), den);
    const float by = one_over(den), old = mine * by;
    mean.x *= old, mean.y *= old, mean.z *= old, mean.w *= old;
    for (int w = 1; w < (int)per_row.d; ++w) add_scaled(mean, sums[warp + w][lane], of_warp[warp + w].y * ex2(of_warp[warp + w].x - to) * by);
  }
  if (on) store_row(static_cast<T*>(a.out) + out_row(a, u, r) * kHeadDim + 4 * lane, mean);
}

using AttKernel = void (*)(AttArgs);
template <typename T, bool E4M3>
AttKernel att_kernel_of(const int NT) {
  switch (NT) {
    case 1: return k_cache8_attention<T, 1, E4M3>;
    case 2: return k_cache8_attention<T, 2, E4M3>;
    case 3: return k_cache8_attention<T, 3, E4M3>;
    default: return k_cache8_attention<T, 4, E4M3>;
  }
}
AttKernel att_kernel(const bool bf16, const bool e4m3, const int NT) {
  return bf16 ? e4m3 ? att_kernel_of<__nv_bfloat16, true>(NT) : att_kernel_of<__nv_bfloat16, false>(NT)
              : e4m3 ? att_kernel_of<__half, true>(NT) : att_kernel_of<__half, false>(NT);
}

// How the work is split.  units: (sequence, head) pairs; groups of query rows; tiles of the longest unit; even: a window cuts long units
// to one length.  resident(n): clusters of n CTAs that are resident at once.
//
// A cluster per unit, or all tiles dealt out evenly and joined by a second kernel.  us a call, one token of four query heads, bf16, heads of
// one length (and of lengths from one row to that), clusters / shares:
//     heads x rows    no weights                        weights counted
//     8 x 2048         8.5 / 10.0   (8.4 / 11.3)                                        four tiles a warp on 64 CTAs (of 592 at once)
//     8 x 4096        11.7 / 10.4  (11.7 / 11.0)        14.0 / 11.5  (13.9 / 12.2)      eight on 64
//     32 x 4096       15.7 / 15.0  (13.4 / 14.1)        16.5 / 16.7  (16.2 / 16.0)      eight on 256
//     32 x 8192       24.5 / 20.8  (20.6 / 17.4)                                        sixteen on 256
//     64 x 4096       18.2 / 21.0  (15.8 / 17.2)        21.0 / 24.9  (18.6 / 20.5)      eight on 512
//     256 x 1024      18.3 / 21.4  (16.0 / 19.4)        21.0 / 25.4  (18.9 / 22.9)      eight on 512
//     64 x 8192       28.7 / 30.6  (24.3 / 21.9)        34.3 / 36.8  (29.7 / 26.8)      sixteen on 512
//     256 x 2048      28.6 / 30.7  (24.8 / 23.9)        34.3 / 36.6  (30.3 / 28.8)      sixteen on 512
// So clusters up to sixteen tiles a warp where they fill the GPU, and up to fewer where they do not, but for six; up to 24 where a window
// cuts the heads to one length (4096 rows seen: 128 heads 29.3 / 32.1, 64 heads 18.8 / 22.4; 2048 rows: 256 heads 29.5 / 32.1; 8192 rows:
// 32 heads, 64 tiles a warp, 25.5 / 22.0).
// More query rows, and a head's CTAs fewer: 32 of them, 64 x 8192 55.6 / 60.6 (52.2 / 43.9), 64 x 4096 32.9 / 40.0 (30.9 / 32.9), 8 x 8192 26.3 /
// 19.1 (25.9 / 20.6); fourteen, 256 x 1639 31.3 / 36.2 (29.9 / 27.3), 256 x 1024 21.6 / 27.1 (20.7 / 23.1).  The rule is the same: where it
// takes shares, heads of one length lose up to a seventh, and heads of unlike length, as budgets of their own leave them, gain as much.
// fp16, with three CTAs an SM: 256 x 1024 19.6 / 21.0 (17.9 / 18.0), 64 x 8192 30.8 / 31.5 (26.6 / 21.7), 256 x 2048 33.5 / 31.1 (31.6 / 23.1).
struct AttShape {
  int S, ctas;      // CTAs of a cluster that has a unit; or, not 0, CTAs that share all tiles
};
int att_slots(const int NT, const bool half, const int sms) { return att_per_sm(NT, half) * sms; }
template <typename Resident>
AttShape att_shape(const long long units, const int groups, const long long tiles, const bool even, const int NT, const bool half,
                   const int sms, const Resident& resident) {
  const long long slots = att_slots(NT, half, sms), all = units * groups;
  long long most = slots / all < kMaxCluster ? slots / all : kMaxCluster;
  if (most > tiles / kAttWarps) most = tiles / kAttWarps;
  int S = most < 1 ? 1 : (int)most;
  while (S > 1 && all > resident(S)) --S;
  const long long alone = (tiles + S * kAttWarps - 1) / (S * kAttWarps);     // tiles of a warp
  const long long full = even ? kAttEven : kAttMany, filled = full * all * S * 5 / (slots * 4);     // (0.8 of the slots count as all)
  const long long limit = filled > full ? full : filled < kAttFew ? kAttFew : filled;
  if (alone <= limit) return {S, 0};
  // (sums up to tiles + CTAs, and a step of a CTA's warps past the end, are kept in 32 bits)
  if (units <= kAttUnits && groups < slots && units * tiles <= 0x7fffffffll - slots - kAttWarps) {
    const long long want = (units * tiles + kAttWarps * 4 - 1) / (kAttWarps * 4);     // (four tiles to a warp)
    return {1, (int)(want < slots / groups ? want : slots / groups)};
  }
  return {S, 0};
}

// What a call with such arguments works with: its query rows, the rows it sees, its workspace.
struct AttPlan {
  int R, groups, NT, cap, pitch, sms;
  long long tiles;                    // of the longest unit
  bool even;                          // cut to that number by a window
  size_t part, spans, stats, logits, bytes;   // offsets: sums at 0, (reference, sum) at `part`
};
int att_plan(const mixkv_cache8* c, const int32_t q_tokens, const int32_t gqa, const int32_t max_rows, const int32_t window,
             const int32_t sinks, const bool accumulate, AttPlan* p) {
  if (q_tokens < 1 || gqa < 1 || max_rows < 1 || window < 0 || sinks < 0 || (accumulate && !c->mass_opt)) return MIXKV_ERR_INVALID_ARG;
  const long long R = (long long)q_tokens * gqa, units = (long long)c->batch * c->kv_heads;
  if (R > MIXKV_CACHE8_MAX_QUERIES) return MIXKV_ERR_UNSUPPORTED;
  const int eights = (int)((R + 7) / 8);
  p->R = (int)R, p->groups = (eights + kAttGroups - 1) / kAttGroups, p->NT = (eights + p->groups - 1) / p->groups;
  if (units * p->groups > 1 << 24) return MIXKV_ERR_UNSUPPORTED;
  const long long room = (long long)c->max_pages * c->page_rows, seen = max_rows < room ? max_rows : room;
  p->tiles = (seen + kBlockRows - 1) / kBlockRows, p->even = false;
  if (window > 0) {     // tiles of the sinks, of the window and of the tokens behind the first, each with a ragged end
    const long long some = ((long long)sinks + kBlockRows - 1) / kBlockRows +
                           ((long long)window + q_tokens - 1 + kBlockRows - 2) / kBlockRows + 1;
    p->even = some < p->tiles;
    if (p->even) p->tiles = some;
  }
  p->cap = (int)p->tiles, p->pitch = ((int)R + 1) & ~1, p->sms = device_sm_count();
  const auto up = [](const size_t x) { return (x + 127) & ~(size_t)127; };
  const size_t shares = 2 * (size_t)att_slots(p->NT, false, p->sms);     // (the workspace serves either type)
  p->part = up(shares * R * kHeadDim * 4);
  p->spans = up(p->part + shares * R * sizeof(float2));
  p->stats = up(p->spans + kAttUnits * sizeof(int2));
  p->logits = up(p->stats + (accumulate ? (size_t)units * R * sizeof(float2) : 0));
  p->bytes = p->logits + (accumulate ? (size_t)units * p->cap * kBlockRows * p->pitch * 4 : 0);
  return MIXKV_OK;
}

}  // namespace
}  // namespace mixkv

using namespace mixkv;

extern "C" void mixkv_internal_cache8_shape(int64_t units, int32_t groups, int64_t tiles, int32_t even, int32_t eights, int32_t half,
                                            int32_t sms, const int32_t* resident, int32_t* ctas, int32_t* shared) {
  const AttShape s = att_shape(units, groups, tiles, even != 0, eights, half != 0, sms, [&](const int n) { return resident[n]; });
  *ctas = s.S, *shared = s.ctas;
}

extern "C" int mixkv_cache_workspace_size(const mixkv_cache8* c, int32_t q_tokens, int32_t gqa_ratio, int32_t max_rows,
                                           int32_t window, int32_t sinks, int32_t accumulate, size_t* bytes) {
  CachePool pool;
  AttPlan p;
  int rc = check_cache(c, &pool);
  if (rc != MIXKV_OK) return rc;
  if (!bytes) return MIXKV_ERR_INVALID_ARG;
  if ((rc = att_plan(c, q_tokens, gqa_ratio, max_rows, window, sinks, accumulate != 0, &p)) != MIXKV_OK) return rc;
  *bytes = p.bytes;
  return MIXKV_OK;
}

extern "C" int mixkv_cache_attention(const mixkv_cache8* c, const void* q, int32_t type, int64_t q_batch_stride,
                                      int64_t q_token_stride, int32_t q_tokens, int32_t gqa_ratio, float softmax_scale,
                                      int32_t max_rows, int32_t window, int32_t sinks, int32_t accumulate, void* workspace,
                                      size_t workspace_bytes, void* out, void* stream) {
  AttArgs a = {};
  AttPlan p;
  int rc = check_cache(c, &a.p);
  if (rc != MIXKV_OK) return rc;
  if (!q || !out || !workspace || (type != MIXKV_TYPE_BF16 && type != MIXKV_TYPE_FP16) || !(softmax_scale >= 0.f) ||
      !(softmax_scale < INFINITY) || q_batch_stride < 0 || q_token_stride < 0 || q_batch_stride % 8 || q_token_stride % 8)
    return MIXKV_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16)) return MIXKV_ERR_INVALID_ARG;
  if ((rc = att_plan(c, q_tokens, gqa_ratio, max_rows, window, sinks, accumulate != 0, &p)) != MIXKV_OK) return rc;
  if (workspace_bytes < p.bytes) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  if ((rc = device_check(nullptr)) != MIXKV_OK) return rc;
  const long long units = (long long)c->batch * c->kv_heads;
  const bool bf16 = type == MIXKV_TYPE_BF16, e4m3 = c->code == MIXKV_CODE_E4M3;
  static std::atomic<bool> done[4 * (kAttGroups + 1)][kMaxDevices];
  static ClusterFit fits[4 * (kAttGroups + 1)];   // (by variant, as `done`)
  const int dev = device_slot(), variant = 4 * p.NT + 2 * e4m3 + bf16;
  const AttKernel kernel = att_kernel(bf16, e4m3, p.NT);
  const size_t smem = att_smem(p.NT);
  const AttShape shape = att_shape(units, p.groups, p.tiles, p.even, p.NT, !bf16, p.sms, [&](const int size) {
    if (!answered(ensure_smem(kernel, smem, done[variant], dev))) return 0;
    return fits[variant].ask(kernel, 32 * kAttWarps, smem, size, dev);
  });
  if (ensure_smem(kernel, smem, done[variant], dev) != cudaSuccess) return MIXKV_ERR_CUDA;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.q = q, a.q_batch = q_batch_stride, a.q_token = q_token_stride;
  a.T = q_tokens, a.G = gqa_ratio, a.R = p.R, a.by_group = Divider(gqa_ratio), a.max_rows = max_rows;
  a.window = window, a.sinks = sinks;
  a.units = (int)units, a.ctas = shape.ctas;
  a.scale_log2e = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)kHeadDim)) * kLog2e;
  a.part = reinterpret_cast<float*>(ws), a.part_mz = reinterpret_cast<float2*>(ws + p.part);
  a.spans = reinterpret_cast<int2*>(ws + p.spans), a.stats = reinterpret_cast<float2*>(ws + p.stats);
  a.logits = accumulate ? reinterpret_cast<float*>(ws + p.logits) : nullptr, a.cap = p.cap, a.pitch = p.pitch;
  a.out = out;
  a.inside = accumulate && !shape.ctas && p.groups == 1;
  a.per = ((p.R < 8 * p.NT ? p.R : 8 * p.NT) * (kHeadDim / 4) + shape.S - 1) / shape.S;
  const unsigned grid = shape.ctas ? (unsigned)shape.ctas : (unsigned)(units * shape.S);
  const cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = launch_pdl(kernel, dim3(grid, p.groups), dim3(32 * kAttWarps), smem, st, shape.S, a);
  if (e == cudaSuccess && (shape.ctas || (accumulate && !a.inside))) {
    int per_row = 1;      // warps that go through the shares of one query row
    while (per_row < kEndWarps && per_row * 2 * units < shape.ctas) per_row *= 2;
    const int at_once = kEndWarps / per_row, join = shape.ctas ? (p.R + at_once - 1) / at_once : 0;
    long long add = 0;
    if (accumulate && !a.inside) {       // sixty-four tiles to a CTA, where that is no more of them than twice those that are there at once
      const long long some = (p.tiles + 63) / 64, room = 2 * kEndPerSm * p.sms / units;
      add = some < room ? some : room < 1 ? 1 : room;
    }
    e = launch_pdl(bf16 ? k_cache8_finish<__nv_bfloat16> : k_cache8_finish<__half>, dim3((unsigned)(units * (join + add))),
                   dim3(kEndThreads), 0, st, 1, a, Divider((uint32_t)(join + add)), join, (int)add, Divider(per_row));
  }
  return e == cudaSuccess ? MIXKV_OK : MIXKV_ERR_CUDA;
}
