// Attention of the newest tokens over the paged 4-bit cache (format: include/mixkv.h).
//
// A warp takes a tile of 16 cache rows per step: 2304 contiguous bytes, brought by one bulk copy into a ring of its own.
// The codes are widened to fp16 by the hardware's conversion and multiplied by their scale: exact.  The products
// run as m16n8k16 with the CACHE on the sixteen-row side and the query rows (tokens x heads of the group) on the
// eight-column side: with up to eight query rows (one token of seven heads) nothing is padded but the eighth, where
// query rows on the sixteen side would leave more than half of every instruction empty (32 instead of 16 instructions a tile).
//   S^T[row, query]  = K q^T      A: rows 4 (g / 2) + 2 j + g % 2, a lane the dimensions 32 t .. 32 t + 31 of two rows
//   O^T[dim, query] += V^T P^T    A: dimensions 16 g + 2 m, + 1 of rows 4 t .. 4 t + 3; P^T from S^T by a transposing move
// Codes of two rows are interleaved (V) by one select per eight values before they are widened, so that a pair is two rows.
//
// Softmax: a running reference per query row, moved only when a logit exceeds it by more than 2^kLag (one vote a
// tile instead of a reduction); weights are fp16 times 2^kLift, so that what is 2^-20 of the largest is still a normal
// number; sums are fp32.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace mixkv {
namespace {

constexpr int kAttWarps = 4, kAttThreads = kAttWarps * 32;
constexpr int kAttDepth = 4;                   // tiles of a warp on their way or in work
constexpr int kAttPitch = kHeadDim + 4;        // floats between the query rows of a warp's sums
constexpr int kAttGroups = 4;                  // most groups of eight query rows a CTA takes
constexpr float kLag = 8.f, kLift = 6.f;       // largest weight 2^14

__host__ __device__ constexpr size_t att_warp_bytes(int NT) {
  return (size_t)(kAttDepth * kTileBytes > 8 * NT * kAttPitch * 4 ? kAttDepth * kTileBytes : 8 * NT * kAttPitch * 4);
}
// rings / sums of the warps; the CTA's sums; references and sums of the warps, the CTA, the cluster; barriers
__host__ __device__ constexpr size_t att_smem(int NT) {
  return kAttWarps * att_warp_bytes(NT) + 8 * NT * kHeadDim * 4 + (2 * kAttWarps + 2 + 2 * kMaxCluster) * 8 * NT * 4 +
         kAttWarps * kAttDepth * 8 + 16;
}
__host__ __device__ constexpr int att_per_sm(int NT) { return NT == 1 ? 4 : NT == 2 ? 3 : 2; }

struct AttArgs {
  PagePool p;
  const void* q;
  long long q_batch, q_token;
  int T, G, R;               // tokens, heads of a group, T * G
  int max_rows;
  const int *list, *counts;  // nullptr: all pages
  int top;
  int chunk, chunks;         // tiles of a work item and items of a unit; chunks == 1: a cluster has the unit
  float scale_log2e;         // k_scale included
  float* part;               // [unit][chunk][R][128] sums, then [unit][chunk][R][2] (reference, sum)
  float* part_mz;
  void* out;
};

// Tiles of a unit, and its rows that the call sees.
struct UnitTiles {
  int n, tiles, pages;
};
__device__ __forceinline__ UnitTiles unit_tiles(const AttArgs& a, const int u) {
  UnitTiles r;
  int n = a.p.rows[u];
  n = min(n, a.max_rows);
  n = (int)min((long long)n, (long long)a.p.max_pages * a.p.page_rows);
  r.n = max(n, 0);
  r.pages = a.list ? max(0, min(a.counts[u], a.top)) : (r.n + a.p.page_rows - 1) / a.p.page_rows;
  r.tiles = a.list ? r.pages * a.p.tiles : (r.n + kPageTile - 1) / kPageTile;
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

// Page of the pool and first row of tile `t` of a unit (id -1: none).
struct TileAt {
  int id, row;
};
__device__ __forceinline__ TileAt tile_at(const AttArgs& a, const int u, const UnitTiles& ut, const int t) {
  TileAt r = {-1, 0};
  if (t >= ut.tiles) return r;
  const int slot = t / a.p.tiles;
  const int page = a.list ? a.list[(long long)u * a.top + slot] : slot;
  if (page < 0 || page >= a.p.max_pages) return r;
  r.row = page * a.p.page_rows + (t - slot * a.p.tiles) * kPageTile;
  if (r.row >= ut.n) return r;
  const int id = a.p.table[(long long)u * a.p.max_pages + page];
  if (id >= 0 && id < a.p.num_pages) r.id = id;
  return r;
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
struct Tokens {   // of the CTA's query rows
  int n, T, G, R, first;
};

template <typename T, int NT>
struct AttState {
  uint32_t q[NT][8][2];     // B fragments: query row g, dimensions 32 t + 4 s .. + 3
  float f[NT][2];           // logits to log2 units: query rows 2 t, 2 t + 1
  float acc[NT][8][4];      // dimensions 16 g + 2 m (0, 1), 16 g + 2 m + 1 (2, 3) of query rows 2 t, 2 t + 1
  float m[NT][2], z[NT][2];

  // Query rows first .. first + 8 NT - 1 of a unit.  bf16 rows are divided by a power of two that brings their largest
  // magnitude to [1, 2): exact as fp16 but for what is 2^-24 of it; the power goes into f.
  __device__ __forceinline__ void start(const AttArgs& a, const int u, const int first, const int g, const int t) {
    const int b = u / a.p.H, h = u % a.p.H;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = first + 8 * nt + g;
      uint4 raw[4];
      const bool on = r < a.R;
      const T* src = static_cast<const T*>(a.q) + b * a.q_batch + (on ? r / a.G : 0) * a.q_token +
                     (long long)(h * a.G + (on ? r % a.G : 0)) * kHeadDim + 32 * t;
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i] = on ? __ldg(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0, 0, 0, 0);
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
        f[nt][c] = __shfl_sync(0xffffffffu, up, 4 * (2 * t + c)) * a.scale_log2e;
        m[nt][c] = -INFINITY, z[nt][c] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[nt][i][c] = 0.f;
    }
  }
  static constexpr bool IsBf16 = std::is_same<T, __nv_bfloat16>::value;

  // One tile.  k: codes of the lane's two K rows; ks: their scales; v, vs likewise.  EDGE: rows from `row` on may lie
  // beyond what a query row sees; limit[nt][c] rows it sees, `left` rows of the tile exist.
  template <bool EDGE>
  __device__ __forceinline__ void tile(const uint4 (&k)[2], const uint32_t ks, const uint4 (&v)[2], uint32_t vs,
                                       const int row, const int (&limit)[NT][2], const int left, const Tokens& tokens,
                                       const int g, const int t) {
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[nt][c] = 0.f;
    {
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
    // s[nt][2 j + c]: row 4 (g / 2) + 2 j + g % 2 of the tile, query row 8 nt + 2 t + c
    bool above = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[nt][i] *= f[nt][i & 1];
        if (EDGE && row + 4 * (g >> 1) + 2 * (i >> 1) + (g & 1) >= limit[nt][i & 1]) s[nt][i] = -INFINITY;
        above |= s[nt][i] > m[nt][i & 1] + kLag;
      }
    if (__any_sync(0xffffffffu, above)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float mx = fmaxf(m[nt][c], column_max(fmaxf(s[nt][c], s[nt][2 + c])));
          const float shrink = mx == -INFINITY ? 1.f : ex2(m[nt][c] - mx);
          m[nt][c] = mx, z[nt][c] *= shrink;
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[nt][i][c] *= shrink, acc[nt][i][2 + c] *= shrink;
        }
    }
    uint32_t p[NT][2];   // B fragments: query row g, tile rows 4 t, 4 t + 1 and 4 t + 2, 4 t + 3
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ref = m[nt][i & 1] == -INFINITY ? 0.f : m[nt][i & 1] - kLift;
        w[i] = ex2(s[nt][i] - ref);
        z[nt][i & 1] += w[i];
      }
      p[nt][0] = transpose8x8(narrow2<__half>(w[0], w[1]));
      p[nt][1] = transpose8x8(narrow2<__half>(w[2], w[3]));
    }
    // Rows that were never written can hold anything, a scale of NaN as well: their scales become zero.  A NaN in a row that
    // some of the query rows see must not reach the others through a weight of zero: such a tile is taken once per
    // token, with the rows that this token sees, and added to its own query rows alone.
    if (EDGE) {
      vs = keep_scales(vs, left - 4 * t);
      const bool nan = ((((vs & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u)) != 0;   // a byte of 0x7f
      if (tokens.T > 1 && __any_sync(0xffffffffu, nan)) {
        for (int token = 0; token < tokens.T; ++token) {
          const uint32_t seen = keep_scales(vs, tokens.n - tokens.T + 1 + token - row - 4 * t);
          values(v, seen, [&](const int m, const uint32_t x0, const uint32_t x1, const uint32_t x2, const uint32_t x3) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float d[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(d, x0, x1, x2, x3, p[nt][0], p[nt][1]);
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if (min(tokens.first + 8 * nt + 2 * t + (c & 1), tokens.R - 1) / tokens.G == token) acc[nt][m][c] += d[c];
            }
          });
        }
        return;
      }
    }
    values(v, vs, [&](const int m, const uint32_t x0, const uint32_t x1, const uint32_t x2, const uint32_t x3) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_f16(acc[nt][m], x0, x1, x2, x3, p[nt][0], p[nt][1]);
    });
  }
};

// grid.x: units * S in clusters of S (chunks == 1), or units * chunks; grid.y: groups of 8 NT query rows
template <typename T, int NT>
__global__ void __launch_bounds__(kAttThreads, att_per_sm(NT)) k_paged_attention(const AttArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int Q = 8 * NT;
  constexpr size_t kWarpBytes = att_warp_bytes(NT);
  float* xo = reinterpret_cast<float*>(smem + kAttWarps * kWarpBytes);   // [Q][128]
  float* wm = xo + Q * kHeadDim;             // [warps][Q]
  float* wz = wm + kAttWarps * Q;            // [warps][Q]
  float* xm = wz + kAttWarps * Q;            // [Q]
  float* xz = xm + Q;                        // [Q]
  float* allm = xz + Q;                      // [8][Q]
  float* allz = allm + kMaxCluster * Q;      // [8][Q]
  uint64_t* bars = reinterpret_cast<uint64_t*>(allz + kMaxCluster * Q);   // [warps][depth]
  int* abort = reinterpret_cast<int*>(bars + kAttWarps * kAttDepth);
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const bool split = a.chunks > 1;
  const int S = split ? 1 : (int)cluster.num_blocks(), crank = split ? 0 : (int)cluster.block_rank();
  const int u = split ? blockIdx.x / a.chunks : blockIdx.x / S;
  const int item = split ? blockIdx.x % a.chunks : 0;
  const int first = blockIdx.y * Q;
  uint64_t* bar = bars + warp * kAttDepth;
  if (lane == 0) {
    for (int d = 0; d < kAttDepth; ++d) mbar_init(&bar[d], 1);
    mbar_init_fence();
    if (warp == 0) *abort = 0;
  }
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait();
  const UnitTiles ut = unit_tiles(a, u);
  const int t0 = item * a.chunk, t1 = split ? min(ut.tiles, t0 + a.chunk) : ut.tiles;
  if (split && t0 >= t1 && (item > 0 || ut.tiles > 0)) return;   // (a unit without rows leaves its first item)
  const int stride = S * kAttWarps, begin = t0 + crank * kAttWarps + warp;
  const int count = begin < t1 ? (t1 - begin + stride - 1) / stride : 0;   // tiles of this warp
  unsigned char* ring = smem + warp * kWarpBytes;

  // lane l knows tile 32 n + l of the warp; `next` are those of n + 1
  TileAt now = tile_at(a, u, ut, lane < count ? begin + lane * stride : ut.tiles);
  auto issue = [&](const int i, const TileAt& from) {   // the copy of the warp's tile i
    const int id = __shfl_sync(0xffffffffu, from.id, i & 31), row = __shfl_sync(0xffffffffu, from.row, i & 31);
    if (lane == 0) {
      uint64_t* full = &bar[i % kAttDepth];
      if (id >= 0) {
        mbar_expect_tx(full, kTileBytes);
        bulk_load(ring + (i % kAttDepth) * kTileBytes, tile_ptr(a.p, id, row % a.p.page_rows / kPageTile), kTileBytes, full);
      } else {
        mbar_arrive(full);    // nothing to come
      }
    }
  };
  for (int i = 0; i < min(count, kAttDepth); ++i) issue(i, now);
  AttState<T, NT> st;
  st.start(a, u, first, g, t);
  int limit[NT][2];     // rows that a query row sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) limit[nt][c] = ut.n - a.T + 1 + min(first + 8 * nt + 2 * t + c, a.R - 1) / a.G;
  const int clear = ut.n - a.T + 1;   // rows below are seen by all
  const Tokens tokens = {ut.n, a.T, a.G, a.R, first};
  bool lost = false;
  int sent = min(count, kAttDepth);
  TileAt next = tile_at(a, u, ut, 32 + lane < count ? begin + (32 + lane) * stride : ut.tiles);
  for (int i = 0; i < count; ++i) {
    if (!mbar_wait(&bar[i % kAttDepth], (i / kAttDepth) & 1, abort)) {
      lost = true;
      break;
    }
    const int id = __shfl_sync(0xffffffffu, now.id, i & 31), row = __shfl_sync(0xffffffffu, now.row, i & 31);
    const unsigned char* slot = ring + (i % kAttDepth) * kTileBytes;
    const uint4 k[2] = {*reinterpret_cast<const uint4*>(slot + 16 * lane), *reinterpret_cast<const uint4*>(slot + 512 + 16 * lane)};
    const uint4 v[2] = {*reinterpret_cast<const uint4*>(slot + kTileV + 16 * lane),
                        *reinterpret_cast<const uint4*>(slot + kTileV + 512 + 16 * lane)};
    const uint32_t ks = *reinterpret_cast<const uint32_t*>(slot + kTileKs + 4 * lane);
    const uint32_t vs = *reinterpret_cast<const uint32_t*>(slot + kTileVs + 4 * lane);
    __syncwarp();     // every lane has read the slot
    if (sent < count) issue(sent++, (i & 31) + kAttDepth < 32 ? now : next);
    if (id >= 0) {
      if (row + kPageTile <= clear) st.template tile<false>(k, ks, v, vs, row, limit, kPageTile, tokens, g, t);
      else st.template tile<true>(k, ks, v, vs, row, limit, ut.n - row, tokens, g, t);
    }
    if ((i & 31) == 31) {
      now = next;
      const int ahead = i + 1 + 32 + lane;
      next = tile_at(a, u, ut, ahead < count ? begin + ahead * stride : ut.tiles);
    }
  }
  if (lost && lane == 0) drain_ring(bar, kAttDepth, sent);
  __syncwarp();

  // ---- the warps merge through shared memory
  float* mine = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float z = column_sum(st.z[nt][c]);
      const int r = 8 * nt + 2 * t + c;
#pragma unroll
      for (int m = 0; m < 8; ++m)
        *reinterpret_cast<float2*>(mine + r * kAttPitch + 16 * g + 2 * m) = make_float2(st.acc[nt][m][c], st.acc[nt][m][2 + c]);
      if (g == 0) wm[warp * Q + r] = st.m[nt][c], wz[warp * Q + r] = lost ? NAN : z;
    }
  }
  __syncthreads();
  const int live = min(Q, a.R - first);
  for (int e = tid; e < live * kHeadDim; e += kAttThreads) {
    const int r = e / kHeadDim, dim = e % kHeadDim;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kAttWarps; ++w) M = fmaxf(M, wm[w * Q + r]);
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < kAttWarps; ++w) {
      const float mw = wm[w * Q + r];
      const float sc = mw == -INFINITY ? (M == -INFINITY ? 1.f : 0.f) : ex2(mw - M);
      num = fmaf(reinterpret_cast<const float*>(smem + w * kWarpBytes)[r * kAttPitch + dim], sc, num);
      den = fmaf(wz[w * Q + r], sc, den);
    }
    if (split) {
      const long long at = ((long long)u * a.chunks + item) * a.R + first + r;
      a.part[at * kHeadDim + dim] = num;
      if (dim == 0) a.part_mz[2 * at] = M, a.part_mz[2 * at + 1] = den;
    } else {
      xo[e] = num;
      if (dim == 0) xm[r] = M, xz[r] = den;
    }
  }
  if (split) return;

  // ---- the CTAs of the cluster merge through distributed shared memory, each a slice of the outputs
  cluster.sync();
  for (int e = tid; e < S * live; e += kAttThreads) {
    const int k = e / live, r = e % live;
    allm[k * Q + r] = *cluster.map_shared_rank(&xm[r], k);
    allz[k * Q + r] = *cluster.map_shared_rank(&xz[r], k);
  }
  __syncthreads();
  const int per = (live * kHeadDim + S - 1) / S;
  const int b = u / a.p.H, h = u % a.p.H;
  for (int e = crank * per + tid; e < min((crank + 1) * per, live * kHeadDim); e += kAttThreads) {
    const int r = e / kHeadDim;
    float M = -INFINITY;
    for (int k = 0; k < S; ++k) M = fmaxf(M, allm[k * Q + r]);
    float num = 0.f, den = 0.f;
    for (int k = 0; k < S; ++k) {
      const float mk = allm[k * Q + r];
      const float sc = mk == -INFINITY ? (M == -INFINITY ? 1.f : 0.f) : ex2(mk - M);
      num = fmaf(*cluster.map_shared_rank(&xo[e], k), sc, num);
      den = fmaf(allz[k * Q + r], sc, den);
    }
    const int row = first + r;
    const long long at = ((long long)b * a.T + row / a.G) * ((long long)a.p.H * a.G) + (long long)h * a.G + row % a.G;
    static_cast<T*>(a.out)[at * kHeadDim + e % kHeadDim] = from_f32<T>(den == 0.f ? 0.f : num / den * a.p.v_scale);
  }
  cluster.sync();   // a CTA's shared memory stays alive until its peers have read it
}

// Joins the items of split units: one CTA per (unit, query row).
constexpr int kJoinWarps = 4;
template <typename T>
__global__ void __launch_bounds__(kJoinWarps * 32) k_paged_join(const AttArgs a) {
  __shared__ float4 sums[kJoinWarps][32];
  __shared__ float stat[kJoinWarps][2];
  pdl_launch_dependents();
  pdl_wait();
  const int u = blockIdx.x / a.R, row = blockIdx.x % a.R;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const UnitTiles ut = unit_tiles(a, u);
  const int items = max(1, min(a.chunks, (ut.tiles + a.chunk - 1) / a.chunk));
  const long long base = (long long)u * a.chunks * a.R + row;
  float M = -INFINITY;
  for (int i = lane; i < items; i += 32) M = fmaxf(M, a.part_mz[2 * (base + (long long)i * a.R)]);
  M = warp_max(M);
  float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
  float den = 0.f;
#pragma unroll 4
  for (int i = warp; i < items; i += kJoinWarps) {
    const long long at = base + (long long)i * a.R;
    const float2 mz = *reinterpret_cast<const float2*>(a.part_mz + 2 * at);
    const float4 x = *(reinterpret_cast<const float4*>(a.part + at * kHeadDim) + lane);
    const float sc = mz.x == -INFINITY ? (M == -INFINITY ? 1.f : 0.f) : ex2(mz.x - M);
    num.x = fmaf(x.x, sc, num.x), num.y = fmaf(x.y, sc, num.y), num.z = fmaf(x.z, sc, num.z), num.w = fmaf(x.w, sc, num.w);
    den = fmaf(mz.y, sc, den);
  }
  sums[warp][lane] = num;
  if (lane == 0) stat[warp][0] = den;
  __syncthreads();
  if (warp == 0) {
    for (int w = 1; w < kJoinWarps; ++w) {
      const float4 x = sums[w][lane];
      num.x += x.x, num.y += x.y, num.z += x.z, num.w += x.w;
      den += stat[w][0];
    }
    const float inv = den == 0.f ? 0.f : a.p.v_scale / den;
    const int b = u / a.p.H, h = u % a.p.H;
    const long long at = ((long long)b * a.T + row / a.G) * ((long long)a.p.H * a.G) + (long long)h * a.G + row % a.G;
    uint2 o;
    o.x = narrow2<T>(num.x * inv, num.y * inv), o.y = narrow2<T>(num.z * inv, num.w * inv);
    *(reinterpret_cast<uint2*>(static_cast<T*>(a.out) + at * kHeadDim) + lane) = o;
  }
}

using AttKernel = void (*)(AttArgs);
template <typename T>
AttKernel att_kernel(const int NT) {
  switch (NT) {
    case 1: return k_paged_attention<T, 1>;
    case 2: return k_paged_attention<T, 2>;
    case 3: return k_paged_attention<T, 3>;
    default: return k_paged_attention<T, 4>;
  }
}

// How the rows of a unit are split.  units: (sequence, head) pairs times groups of query rows; tiles: of the longest.
struct AttShape {
  int S, chunk, chunks;
};
constexpr int kAttItems = 2;        // work items per resident CTA, of split units
long long att_slots(const int NT, const int sms) { return (long long)att_per_sm(NT) * sms; }
int att_most_chunks(const long long units, const int NT, const int sms) {
  const long long n = (kAttItems * att_slots(NT, sms) + units - 1) / units;
  return (int)(n < 1 ? 1 : n);
}
template <typename Fit>
AttShape att_shape(const long long units, const long long tiles, const int NT, const int sms, const Fit& fit) {
  const long long slots = att_slots(NT, sms);
  int S = (int)(slots / units < kMaxCluster ? slots / units : kMaxCluster);
  if (S > tiles / kAttWarps) S = (int)(tiles / kAttWarps);
  if (S < 1) S = 1;
  while (S > 1 && units > fit(S)) --S;
  // Split over items that no cluster holds together once a warp has more steps than the join costs
  if (tiles > (long long)S * kAttWarps * 8) {
    int chunks = att_most_chunks(units, NT, sms);
    long long chunk = (tiles + chunks - 1) / chunks;
    if (chunk < 4 * kAttWarps) chunk = 4 * kAttWarps;
    chunks = (int)((tiles + chunk - 1) / chunk);
    if (chunks > 1) return {1, (int)chunk, chunks};
  }
  return {S, 0, 1};
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
size_t part_bytes(const long long units, const int chunks, const long long R) {
  return (size_t)(units * chunks * R) * (kHeadDim + 2) * 4;
}

}  // namespace
}  // namespace mixkv

using namespace mixkv;

extern "C" int mixkv_paged_workspace_size(const mixkv_pages* c, int32_t q_tokens, int32_t gqa_ratio, size_t* bytes) {
  PagePool p;
  int rc = check_pages(c, &p), groups, NT;
  if (rc != MIXKV_OK) return rc;
  if (!bytes) return MIXKV_ERR_INVALID_ARG;
  if ((rc = queries_of(c, q_tokens, gqa_ratio, &groups, &NT)) != MIXKV_OK) return rc;
  const long long units = (long long)c->batch * c->kv_heads;
  *bytes = part_bytes(units, att_most_chunks(units * groups, NT, device_sm_count()), (long long)q_tokens * gqa_ratio);
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
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(workspace)) & 15u)
    return MIXKV_ERR_INVALID_ARG;
  if ((rc = queries_of(c, q_tokens, gqa_ratio, &groups, &NT)) != MIXKV_OK) return rc;
  const long long units = (long long)c->batch * c->kv_heads;
  const int R = q_tokens * gqa_ratio, sms = device_sm_count();
  if (workspace_bytes < part_bytes(units, att_most_chunks(units * groups, NT, sms), R))
    return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  if ((rc = device_check(nullptr)) != MIXKV_OK) return rc;
  const long long seen = max_rows < (long long)c->max_pages * c->page_rows ? max_rows : (long long)c->max_pages * c->page_rows;
  long long tiles = (seen + kPageTile - 1) / kPageTile;
  if (page_list_opt && tiles > (long long)top * a.p.tiles) tiles = (long long)top * a.p.tiles;

  const bool bf16 = type == MIXKV_TYPE_BF16;
  static std::atomic<bool> done[2 * (kAttGroups + 1)][kMaxDevices];
  static ClusterFit fits[2 * (kAttGroups + 1)];   // (by variant, as `done`)
  const int variant = 2 * NT + bf16, dev = device_slot();
  const AttKernel kernel = bf16 ? att_kernel<__nv_bfloat16>(NT) : att_kernel<__half>(NT);
  const size_t smem = att_smem(NT);
  if (ensure_smem(kernel, smem, done[variant], dev) != cudaSuccess) return MIXKV_ERR_CUDA;
  const AttShape shape = att_shape(units * groups, tiles, NT, sms, [&](const int size) {
    return fits[variant].ask(kernel, kAttThreads, smem, size, dev);
  });
  a.q = q, a.q_batch = q_batch_stride, a.q_token = q_token_stride;
  a.T = q_tokens, a.G = gqa_ratio, a.R = R, a.max_rows = max_rows;
  a.list = page_list_opt, a.counts = counts_opt, a.top = top;
  a.chunk = shape.chunk, a.chunks = shape.chunks;
  a.scale_log2e = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)kHeadDim)) * kLog2e * c->k_scale;
  a.part = static_cast<float*>(workspace);
  a.part_mz = a.part + units * shape.chunks * R * kHeadDim;
  a.out = out;
  const unsigned per_unit = shape.chunks > 1 ? shape.chunks : shape.S;
  cudaError_t e = launch_pdl(kernel, dim3((unsigned)units * per_unit, groups), dim3(kAttThreads), smem, (cudaStream_t)stream,
                             shape.S, a);
  if (e == cudaSuccess && shape.chunks > 1)
    e = launch_pdl(bf16 ? k_paged_join<__nv_bfloat16> : k_paged_join<__half>, dim3((unsigned)(units * R)),
                   dim3(kJoinWarps * 32), 0, (cudaStream_t)stream, 1, a);
  return e == cudaSuccess ? MIXKV_OK : MIXKV_ERR_CUDA;
}
