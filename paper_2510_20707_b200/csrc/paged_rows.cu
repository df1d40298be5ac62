// Rows into the paged 4-bit cache and back (format and rounding: include/mixkv.h).
//
// A page of one head is one CTA's, or one warp's, so that its bounds have one owner and need no atomics.  A warp takes four rows at
// a time, eight lanes each, a lane 16 dimensions of V and of K: the largest magnitude, the scale and the codes of a block are one
// lane's.  Of K that is turned in pairs (i, i + rot_dim / 2) a lane has eight dimensions of either side instead, and the largest magnitudes
// are exchanged between the two lanes of two blocks; with a block per lane and the partner's dimensions fetched from it, every lane
// loaded the angles of sixteen pairs, and a call took 13 us longer than one without a rotation, where it takes 5.
// (Two rows at a time, half a block per lane and K and V in warps of their own took 262 instructions a row instead of 115, and half
// of the warps waited for the others.)
//
// What bounds it.  Append: latencies.  4 x 32768 rows in pages of 64 (67 MB in, 17 of angles, 19 out) take 27 us, 3.8 TB/s.  A step of
// a warp that has its SM for itself takes 0.8 us, a chain of about 1400 clocks (load, largest magnitude, scale, divisor, quotient, codes,
// 115 instructions a row); sixteen warps an SM, as registers allow, are in each other's way half of the time.  The angles come by
// asynchronous copies a step ahead, the positions two (31 us with loads while V is rounded).  All of a row by such copies, three
// steps ahead: 30; twenty warps with 96 registers: 32.  Divisors and reciprocals of the 127 scales come from a table that a CTA fills
// once.  Reading back: 16 us (19 MB in, 67 out), 5.4 TB/s; with 16-byte stores 20.
#include "paged.cuh"

namespace mixkv {
namespace {

constexpr int kRowThreads = 256;   // of a CTA that reads many rows of a page; one row per head: 64
constexpr int kAppThreads = 128, kAppPerSm = 4;   // of a CTA that may get many rows, and such CTAs per SM
constexpr int kAppAlone = 8;       // pages per SM above which a warp has a page alone (append_as)

struct RowArgs {
  PagePool p;
  const int* offsets;     // nullptr: token b
  int per_head, max_new, slots;
  Divider by_slots;
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
  int lo, hi;              // new rows of the page
  int first, last;         // those of them whose token is in the input
  long long token;         // token (or row of the input) of row 0 of the page; there may be none
  int id;                  // what the table says, -1 beyond it
  bool bad;                // a new row below row zero, or more of them than the call allows
};
__device__ __forceinline__ PageSpan page_span(const RowArgs& a, const int task) {
  PageSpan s;
  // heads of a token next to one another: they are in memory, and they are turned by the same angles
  const int at = a.p.by_heads.div(task), b = a.by_slots.div(at), slot = at - b * a.slots;
  s.h = task - at * a.p.H;
  s.u = b * a.p.H + s.h;
  const int rows = fresh(a.p.rows + s.u);
  int n = 1;
  bool over = false;
  long long first = b;
  if (a.offsets) {
    const int i = a.per_head ? s.u : b;
    const int from = fresh(a.offsets + i), to = fresh(a.offsets + i + 1);
    const unsigned all = to > from ? (unsigned)to - (unsigned)from : 0u;
    over = all > (unsigned)a.max_new;
    n = (int)min(all, (unsigned)a.max_new);
    first = (long long)to - n;
  }
  s.bad = rows < n;
  if (s.bad) first += n - max(rows, 0), n = max(rows, 0);      // (only the last rows have a place)
  s.bad |= over;
  const int r0 = rows - n;      // row of the first new token
  s.page = n > 0 ? a.p.by_rows.div(r0) + slot : 0;
  const long long begin = (long long)s.page * a.p.page_rows, end = begin + a.p.page_rows;
  const long long lo = r0 > begin ? r0 : begin, hi = rows < end ? rows : end;
  s.lo = n > 0 ? (int)(lo - begin) : 0, s.hi = n > 0 && hi > lo ? (int)(hi - begin) : s.lo;
  s.token = first + (begin - r0);
  // (rows r of the page with 0 <= token + r < num_tokens)
  const long long from = -s.token, to = a.num_tokens - s.token;
  s.first = from > s.lo ? (int)(from < s.hi ? from : s.hi) : s.lo;
  s.last = to < s.hi ? (int)(to > s.lo ? to : s.lo) : s.hi;
  s.id = s.lo < s.hi && s.page < a.p.max_pages ? fresh(a.p.table + (long long)s.u * a.p.max_pages + s.page) : -1;
  return s;
}

__device__ __forceinline__ float max3_nan(const float x, const float y, const float z) {   // NaN if one is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
// Of every scale byte: scale * third and its rounded reciprocal.
__device__ __forceinline__ void fill_divisors(float2* table, const float third) {
  for (int i = threadIdx.x; i < 128; i += blockDim.x) {
    const uint32_t wide = scales_to_f16(i);
    const float d = __fmul_rn(__low2float(*reinterpret_cast<const __half2*>(&wide)), third);
    table[i] = make_float2(d, __frcp_rn(d));
  }
}

// Largest magnitude of eight values.
__device__ __forceinline__ float largest8(const f32x2* x) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpack2(x[i], a, b);
    m = max3_nan(m, fabsf(a), fabsf(b));
  }
  return m;
}
// Scale byte of a block whose largest magnitude is m; inv6: 1 / (6 k_scale).
__device__ __forceinline__ uint32_t scale_of(const float m, const float inv6) {
  unsigned short s;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(s) : "f"(0.f), "f"(__fmul_rn(m, inv6)));
  return s & 0x7fu;
}
// Codes of eight values of a block.  div: its divisor and the rounded reciprocal; divide: by division.
//
// x / d is rounded to nearest by Markstein's correction of x times the rounded reciprocal: the remainder of that first quotient is
// exact, and one step with it rounds correctly while nothing over- or underflows: x / d stays below 1e36, and the remainder of
// an x that is no code of zero (above d / 8, 2^-63) is a multiple of 2^-47 x.  Blocks of infinities, of extreme values or scales (unsafe) are
// divided.  (A code of zero has either sign.)
__device__ __forceinline__ bool unsafe(const float m, const float2 div) { return !(m < 1e18f && div.x > 1e-18f); }   // (NaN, and d == 0, too)
template <bool DIVIDE>
__device__ __forceinline__ uint32_t codes8(const f32x2* x, const float2 div) {
  const f32x2 by = pack2(div.y, div.y), d = pack2(-div.x, -div.x);
  f32x2 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DIVIDE) {
      float a, b;
      unpack2(x[i], a, b);
      q[i] = div.x == 0.f ? 0ull : pack2(__fdiv_rn(a, div.x), __fdiv_rn(b, div.x));
    } else {
      const f32x2 first = mul2(x[i], by);
      q[i] = fma2(fma2(first, d, x[i]), by, first);
    }
  }
  // (joined by byte moves: with the four bytes packed by one move, the two upper ones came out wrong where the codes are widened
  // again for the bounds)
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpack2(q[i], a, b);
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(c[i]) : "f"(b), "f"(a));
  }
  return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
}
// Codes of sixteen values, eight of a block with largest magnitude ma and divisor da, eight of one with mb and db.
__device__ __forceinline__ uint2 codes16(const f32x2 (&x)[8], const float ma, const float2 da, const float mb, const float2 db) {
  if (unsafe(ma, da) || unsafe(mb, db)) return make_uint2(codes8<true>(x, da), codes8<true>(x + 4, db));
  return make_uint2(codes8<false>(x, da), codes8<false>(x + 4, db));
}

// Where the codes and the scale of block g of row r lie inside a tile.
__device__ __forceinline__ int k_codes_at(const int r, const int g) {
  return 512 * ((r >> 1) & 1) + 64 * ((r >> 2) * 2 + (r & 1)) + 8 * g;
}
__device__ __forceinline__ int v_codes_at(const int r, const int g) {
  return kTileV + 512 * ((r >> 1) & 1) + 64 * g + 16 * (r >> 2) + 8 * (r & 1);
}
__device__ __forceinline__ int k_scale_at(const int r, const int g) {
  return kTileKs + 16 * ((r >> 2) * 2 + (r & 1)) + 4 * (g >> 1) + 2 * ((r >> 1) & 1) + (g & 1);
}
__device__ __forceinline__ int v_scale_at(const int r, const int g) { return kTileVs + 16 * g + r; }
constexpr int kKCodesFour = 128, kVCodesFour = 16, kKScalesFour = 32, kVScalesFour = 4;     // from row r to row r + 4

struct Raw16 {   // 16 values of 16 bits
  uint4 a, b;
};
__device__ __forceinline__ uint32_t word16(const Raw16& r, const int i) {
  return i == 0 ? r.a.x : i == 1 ? r.a.y : i == 2 ? r.a.z : i == 3 ? r.a.w : i == 4 ? r.b.x : i == 5 ? r.b.y : i == 6 ? r.b.z : r.b.w;
}
// (Without a row the registers keep what they have: nothing of it is written.)
template <typename T>
__device__ __forceinline__ void load16(Raw16& r, const T* src, const bool on) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %9, 0;\n\t@p ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t}"
      : "+r"(r.a.x), "+r"(r.a.y), "+r"(r.a.z), "+r"(r.a.w), "+r"(r.b.x), "+r"(r.b.y), "+r"(r.b.z), "+r"(r.b.w)
      : "l"(src), "r"((uint32_t)on)
      : "memory");
}
template <typename T>
__device__ __forceinline__ void load8x2(Raw16& r, const T* a, const T* b, const bool on) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %10, 0;\n\t@p ld.global.v4.b32 {%0, %1, %2, %3}, [%8];\n\t"
      "@p ld.global.v4.b32 {%4, %5, %6, %7}, [%9];\n\t}"
      : "+r"(r.a.x), "+r"(r.a.y), "+r"(r.a.z), "+r"(r.a.w), "+r"(r.b.x), "+r"(r.b.y), "+r"(r.b.z), "+r"(r.b.w)
      : "l"(a), "l"(b), "r"((uint32_t)on)
      : "memory");
}
template <typename T>
__device__ __forceinline__ f32x2 wide2(const uint32_t w) {
  const float2 v = widen2<T>(w);
  return pack2(v.x, v.y);
}
template <>
__device__ __forceinline__ f32x2 wide2<__nv_bfloat16>(const uint32_t w) { return bf16x2_wide(w); }

// What lane g of a row has of K: eight dimensions from a on (x), eight from b on (y).  Pairs (i, i + rot / 2) lie in two blocks, and the
// two lanes of these blocks have eight pairs each (so neither needs the other's dimensions, nor the same cosines); else a lane
// has a block.
struct Eights {
  int a, b;
  bool split;
};
template <int ROPE>
__device__ __forceinline__ Eights eights_of(const int g, const int rot) {
  const int half = rot >> 1;
  if (ROPE != 1 || 16 * g >= rot) return Eights{16 * g, 16 * g + 8, false};
  return 16 * g < half ? Eights{16 * g, 16 * g + half, true} : Eights{16 * g + 8 - half, 16 * g + 8, true};
}
// Cosines and sines of a lane's eight pairs, ROPE 1: (i, i + rot / 2), 2: (2 i, 2 i + 1), from the token's row of the tables; a lane
// copies 16-byte pieces for itself (piece i at i * blockDim.x), and waits for all but its last group of them.
__device__ __forceinline__ void ask_turn(const RowArgs& a, uint4* to, const int pos, const int at, const bool on) {
  if (on) {
    const long long from = (long long)pos * (a.rot >> 1) + at;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to + i * blockDim.x)),
                   "l"((i < 2 ? a.cosv : a.sinv) + from + 4 * (i & 1))
                   : "memory");
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}
__device__ __forceinline__ void wait_turn() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// a + b and a - b in halves: of a packed sum and the packed products before it, .rn or not, the compiler makes multiply-adds.
__device__ __forceinline__ f32x2 add_rounded(const f32x2 a, const f32x2 b) {
  float ax, ay, bx, by;
  unpack2(a, ax, ay), unpack2(b, bx, by);
  return pack2(__fadd_rn(ax, bx), __fadd_rn(ay, by));
}
__device__ __forceinline__ f32x2 sub_rounded(const f32x2 a, const f32x2 b) {
  float ax, ay, bx, by;
  unpack2(a, ax, ay), unpack2(b, bx, by);
  return pack2(__fsub_rn(ax, bx), __fsub_rn(ay, by));
}
// The rotation of a lane's eight pairs by the pieces at `turn`; products and sums are rounded one by one.
template <int ROPE>
__device__ __forceinline__ void rotate8(f32x2 (&x)[8], const float4* turn) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4 cs = turn[i * blockDim.x], sn = turn[(2 + i) * blockDim.x];
    if constexpr (ROPE == 1) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const f32x2 c = e ? pack2(cs.z, cs.w) : pack2(cs.x, cs.y), s = e ? pack2(sn.z, sn.w) : pack2(sn.x, sn.y);
        const f32x2 u = x[2 * i + e], w = x[4 + 2 * i + e];
        x[2 * i + e] = sub_rounded(mul2(u, c), mul2(w, s));
        x[4 + 2 * i + e] = add_rounded(mul2(w, c), mul2(u, s));
      }
    } else {
      const float cc[4] = {cs.x, cs.y, cs.z, cs.w}, ss[4] = {sn.x, sn.y, sn.z, sn.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float p, q;
        unpack2(x[4 * i + e], p, q);
        x[4 * i + e] = add_rounded(mul2(x[4 * i + e], pack2(cc[e], cc[e])), mul2(pack2(-q, p), pack2(ss[e], ss[e])));
      }
    }
  }
}

// A CTA of two warps has one page, K and V of one row each.  Of four warps each has a page (alone), or all have one; every warp both
// K and V.
template <typename T, int ROPE>
__global__ void __launch_bounds__(kAppThreads, kAppPerSm)
k_paged_append(const RowArgs a, const T* k, const T* v, const int tasks, const bool alone) {
  extern __shared__ __align__(16) uint4 turns[];      // what K's next two rows (the one row) are turned by
  __shared__ float2 divisors[2][128];
  __shared__ __half2 part[kAppThreads / 32][8][17];   // of every warp: minima and maxima of a block's eight pairs of dimensions
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane & 7, sub = lane >> 3;
  fill_divisors(divisors[0], a.p.k_scale);
  fill_divisors(divisors[1], a.p.v_scale);
  pdl_wait();
  const bool single = blockDim.x == 64;
  const int team = single || alone ? 1 : blockDim.x >> 5, step = 4 * team;     // warps that share the page's rows
  const bool does_k = !single || warp == 0, does_v = !single || warp == 1;
  __syncthreads();
  const int task = alone ? blockIdx.x * (kAppThreads / 32) + warp : blockIdx.x;
  if (task >= tasks) return;      // (a warp that is alone)
  const float k6 = (float)(1.0 / (6.0 * (double)a.p.k_scale)), v6 = (float)(1.0 / (6.0 * (double)a.p.v_scale));
  const Eights own = eights_of<ROPE>(g, a.rot);
  const bool inside = ROPE && 16 * g < a.rot;
  const int partner = !own.split ? lane : own.a == 16 * g ? lane + (a.rot >> 5) : lane - (a.rot >> 5);
  const PageSpan s = page_span(a, task);
  const bool placed = s.id >= 0 && s.id < a.p.num_pages;
  bool bad = s.bad || (s.lo < s.hi && !placed);
  __half2 lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) lo[i] = __float2half2_rn(INFINITY), hi[i] = __float2half2_rn(-INFINITY);

  int r = s.lo + (team == 1 ? 0 : 4 * warp) + sub;
  bool on = r >= s.first && r < s.last;
  // (row r of the page is row s.token + r of the input)
  const T* kr = k + (a.per_head ? 0 : s.h * a.k_head) + (s.token + r) * a.k_row + own.a;
  const T* vr = v + (a.per_head ? 0 : s.h * a.v_head) + (s.token + r) * a.v_row + 16 * g;
  const int* positions = a.positions + (s.token + r);
  Raw16 kk = {}, vv = {};
  auto load_k = [&](const bool on) {
    if constexpr (ROPE == 1) load8x2(kk, kr, kr + (own.b - own.a), on);
    else load16(kk, kr, on);
  };
  load_k(on && does_k), load16(vv, vr, on && does_v);
  // a row's angles are on their way while the row before it is rounded, its position while the one before that is
  bool turned = true;
  int pos = 0, odd = 0;
  if constexpr (ROPE != 0) {
    const int now = on ? fresh(positions) : 0;
    positions += step;
    pos = r + step >= s.first && r + step < s.last ? fresh(positions) : 0;
    turned = now >= 0 && now < a.table_len;
    ask_turn(a, turns + tid, now, ROPE == 1 ? own.a : 8 * g, on && does_k && inside && turned);
  }
  // places of the lane's rows in a tile: those of row r % 4, and the same further on for every four rows
  unsigned char* const page = tile_ptr(a.p, placed ? s.id : 0, 0);
  const int k_at = k_codes_at(r & 3, ROPE == 1 ? 0 : g), v_at = v_codes_at(r & 3, g);
  const int ks_at = k_scale_at(r & 3, g), vs_at = v_scale_at(r & 3, g);
  for (; r - sub < s.hi; r += step) {
    const int next = r + step;
    const bool write = on && placed && turned;      // (a token is written whole or not at all)
    on = next >= s.first && next < s.last;
    kr += step * a.k_row, vr += step * a.v_row;
    if constexpr (ROPE != 0) {
      turned = pos >= 0 && pos < a.table_len;
      ask_turn(a, turns + (odd ^ 1) * 4 * blockDim.x + tid, pos, ROPE == 1 ? own.a : 8 * g, on && does_k && inside && turned);
      positions += step;
      if (next + step >= s.first && next + step < s.last) pos = fresh(positions);
    }
    bad |= r < s.hi && !write;
    unsigned char* tile = page + (r / kPageTile) * kTileBytes;
    const int four = (r % kPageTile) >> 2;
    if (does_v) {
      f32x2 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = wide2<T>(word16(vv, i));
      load16(vv, vr, on);      // the next row on its way
      const float m = max3_nan(largest8(x), largest8(x + 4), 0.f);
      const uint32_t scale = scale_of(m, v6);
      const float2 div = divisors[1][scale];
      const uint2 w = codes16(x, m, div, m, div);
      if (write) {
        *reinterpret_cast<uint2*>(tile + v_at + kVCodesFour * four) = w;
        tile[vs_at + kVScalesFour * four] = (unsigned char)scale;
      }
    }
    if (does_k) {
      f32x2 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = wide2<T>(word16(kk, i));
      load_k(on);
      if constexpr (ROPE != 0) {
        wait_turn();
        if (inside) rotate8<ROPE>(x, reinterpret_cast<const float4*>(turns + odd * 4 * blockDim.x + tid));
        odd ^= 1;
      }
      // of the two blocks that the lane has a part of (one and the same, if they are not split)
      float ma = largest8(x), mb = largest8(x + 4);
      if constexpr (ROPE == 1) {
        const float oa = __shfl_sync(0xffffffffu, ma, partner), ob = __shfl_sync(0xffffffffu, mb, partner);
        ma = max3_nan(ma, own.split ? oa : ob, 0.f), mb = max3_nan(mb, own.split ? ob : oa, 0.f);
      } else {
        ma = mb = max3_nan(ma, mb, 0.f);
      }
      const uint32_t sa = scale_of(ma, k6), sb = ROPE == 1 ? scale_of(mb, k6) : sa;
      const uint2 w = codes16(x, ma, divisors[0][sa], mb, divisors[0][sb]);
      if (write) {
        unsigned char* codes = tile + k_at + kKCodesFour * four;
        if constexpr (ROPE == 1) {
          *reinterpret_cast<uint32_t*>(codes + own.a / 2) = w.x, *reinterpret_cast<uint32_t*>(codes + own.b / 2) = w.y;
        } else {
          *reinterpret_cast<uint2*>(codes) = w;
        }
        tile[ks_at + kKScalesFour * four] = (unsigned char)(own.a >> 4 == g ? sa : sb);
        if (a.p.bounds) {
          uint32_t f[8];
          codes_to_f16(w.x, *reinterpret_cast<uint32_t(*)[4]>(&f[0]));
          codes_to_f16(w.y, *reinterpret_cast<uint32_t(*)[4]>(&f[4]));
          const uint32_t fa = scales_to_f16(sa | sa << 8), fb = ROPE == 1 ? scales_to_f16(sb | sb << 8) : fa;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t y = mul_f16x2(f[i], i < 4 ? fa : fb);
            lo[i] = __hmin2_nan(lo[i], *reinterpret_cast<const __half2*>(&y));
            hi[i] = __hmax2_nan(hi[i], *reinterpret_cast<const __half2*>(&y));
          }
        }
      }
    }
  }
  pdl_launch_dependents();      // (sooner, its CTAs would crowd the few multiprocessors that this one leaves free)
  if (bad && a.status) *a.status = MIXKV_ERR_INVALID_ARG;
  if (!a.p.bounds || !placed || s.lo >= s.hi) return;      // (all that share a page)
  if (does_k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int o = 8; o < 32; o <<= 1) {
        lo[i] = __hmin2_nan(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o));
        hi[i] = __hmax2_nan(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o));
      }
      if (sub == 0) {
        const int d = (i < 4 ? own.a : own.b) + 2 * (i & 3);
        part[warp][d >> 4][(d & 15) >> 1] = lo[i], part[warp][d >> 4][8 + ((d & 15) >> 1)] = hi[i];
      }
    }
  }
  if (alone) __syncwarp();
  else __syncthreads();
  const int first = alone ? warp : 0, warps = team == 1 ? 1 : min(team, (s.hi - s.lo + 3) / 4);    // those that had rows
  for (int e = alone ? lane : tid; e < 128; e += alone ? 32 : blockDim.x) {
    const bool most = e & 64;
    const int block = (e & 63) >> 3, i = (most ? 8 : 0) + (e & 7);
    __half2 x = part[first][block][i];
    for (int w = 1; w < warps; ++w) x = most ? __hmax2_nan(x, part[w][block][i]) : __hmin2_nan(x, part[w][block][i]);
    __half2* out = reinterpret_cast<__half2*>(a.p.bounds + ((long long)s.id * 2 + most) * kHeadDim) + (e & 63);
    if (s.lo > 0) x = most ? __hmax2_nan(x, *out) : __hmin2_nan(x, *out);
    *out = x;
  }
}

// A lane has a block of a row, as above.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_paged_read(const RowArgs a, T* k, T* v) {
  pdl_wait();
  const PageSpan s = page_span(a, blockIdx.x);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane & 7, sub = lane >> 3;
  pdl_launch_dependents();      // (not sooner: as above)
  if (s.id < 0 || s.id >= a.p.num_pages) return;
  const bool keys = (warp & 1) == 0;
  const float third = keys ? a.p.k_scale : a.p.v_scale;
  const long long stride = a.per_head ? kHeadDim : (long long)a.p.H * kHeadDim;
  T* rows = (keys ? k : v) + (a.per_head ? 0 : s.h * kHeadDim) + s.token * stride + 16 * g;   // row r of the page at r * stride
  const int step = 4 * (blockDim.x >> 6);
  for (int r0 = s.first + 4 * (warp >> 1) + sub; r0 < s.last; r0 += 2 * step) {
    uint2 w[2];
    uint32_t scale[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = min(r0 + j * step, s.last - 1), rt = r % kPageTile;
      const unsigned char* tile = tile_ptr(a.p, s.id, r / kPageTile);
      w[j] = *reinterpret_cast<const uint2*>(tile + (keys ? k_codes_at(rt, g) : v_codes_at(rt, g)));
      scale[j] = tile[keys ? k_scale_at(rt, g) : v_scale_at(rt, g)];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = r0 + j * step;
      if (r >= s.last) break;
      uint32_t f[8], out[8];      // (32 bytes a lane, one store)
      codes_to_f16(w[j].x, *reinterpret_cast<uint32_t(*)[4]>(&f[0]));
      codes_to_f16(w[j].y, *reinterpret_cast<uint32_t(*)[4]>(&f[4]));
      const uint32_t ss = scales_to_f16(scale[j] | scale[j] << 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 y = widen2<__half>(mul_f16x2(f[i], ss));
        float a, b;
        unpack2(mul2(pack2(y.x, y.y), pack2(third, third)), a, b);
        out[i] = narrow2<T>(a, b);
      }
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(rows + r * stride), "r"(out[0]), "r"(out[1]),
                   "r"(out[2]), "r"(out[3]), "r"(out[4]), "r"(out[5]), "r"(out[6]), "r"(out[7])
                   : "memory");
    }
  }
}

int check_rows(const mixkv_pages* c, int32_t type, int64_t num_tokens, const int32_t* offsets, int32_t per_head,
               int32_t max_new, RowArgs* a) {
  const int rc = check_pages(c, &a->p);
  if (rc != MIXKV_OK) return rc;
  if ((type != MIXKV_TYPE_BF16 && type != MIXKV_TYPE_FP16) || num_tokens < 0 || max_new < 1 || (per_head && !offsets) ||
      !aligned(offsets, 4))
    return MIXKV_ERR_INVALID_ARG;
  if (max_new > (1 << 30)) return MIXKV_ERR_UNSUPPORTED;
  a->offsets = offsets, a->per_head = per_head != 0, a->max_new = offsets ? max_new : 1, a->num_tokens = num_tokens;
  // pages that a head's new rows can touch: one, and one more for every page_rows rows behind the first
  a->slots = (a->max_new - 1 + c->page_rows - 1) / c->page_rows + 1;
  if (a->slots > c->max_pages + 1) a->slots = c->max_pages + 1;   // (one past the table: rows there are reported)
  if ((long long)c->batch * c->kv_heads * a->slots > 0x7fffffffll) return MIXKV_ERR_UNSUPPORTED;
  a->by_slots = Divider(a->slots);
  return MIXKV_OK;
}
int tasks_of(const mixkv_pages* c, const RowArgs& a) { return c->batch * c->kv_heads * a.slots; }
template <typename T>
int append_as(const mixkv_pages* c, const RowArgs& a, const void* k, const void* v, const int rope, void* stream) {
  const int rc = device_check(nullptr);
  if (rc != MIXKV_OK) return rc;
  void (*kernel)(RowArgs, const T*, const T*, int, bool) =
      rope == 0 ? k_paged_append<T, 0> : rope == 1 ? k_paged_append<T, 1> : k_paged_append<T, 2>;
  // A page to a warp or to four: four end a page sooner, but a page begins with a chain of loads (rows, table, first rows), which four
  // times as many CTAs go through.  Pages of 64 rows, us: 512 pages 18.3 alone / 9.9 by four, 1024 20.5 / 18.2, 2048 27.1 / 33.4; of 16
  // rows: 512 7.3 / 5.6, 1024 8.1 / 9.8, 2048 10.1 / 17.6.  (CTAs of one or two such warps: level.)
  const int tasks = tasks_of(c, a);
  const bool many = a.max_new > 1, alone = many && tasks > kAppAlone * device_sm_count();
  const int threads = many ? kAppThreads : 64;
  return launch_pdl(kernel, dim3((unsigned)(alone ? (tasks + kAppThreads / 32 - 1) / (kAppThreads / 32) : tasks)),
                    dim3(threads), rope == 0 ? 0 : (many ? 2 : 1) * 64 * threads, (cudaStream_t)stream, 1, a,
                    static_cast<const T*>(k), static_cast<const T*>(v), tasks, alone) == cudaSuccess
             ? MIXKV_OK
             : MIXKV_ERR_CUDA;
}
template <typename T>
int read_as(const mixkv_pages* c, const RowArgs& a, void* k, void* v, void* stream) {
  const int rc = device_check(nullptr);
  if (rc != MIXKV_OK) return rc;
  return launch_pdl(k_paged_read<T>, dim3((unsigned)tasks_of(c, a)), dim3(a.max_new > 1 ? kRowThreads : 64), 0,
                    (cudaStream_t)stream, 1, a, static_cast<T*>(k), static_cast<T*>(v)) == cudaSuccess
             ? MIXKV_OK
             : MIXKV_ERR_CUDA;
}

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
  if (!k || !v || !aligned(k, 32) || !aligned(v, 32) || !aligned(status_dev, 4)) return MIXKV_ERR_INVALID_ARG;
  for (const int64_t stride : {k_row_stride, k_head_stride, v_row_stride, v_head_stride})
    if (stride < 0 || stride % 16) return MIXKV_ERR_INVALID_ARG;
  const bool rope = cos_opt != nullptr;
  if (rope != (sin_opt != nullptr)) return MIXKV_ERR_INVALID_ARG;
  if (rope) {
    if (!positions_opt || table_len < 1 || !aligned(cos_opt, 16) || !aligned(sin_opt, 16) || rot_dim < 1 || rot_dim > kHeadDim ||
        !aligned(positions_opt, 4))
      return MIXKV_ERR_INVALID_ARG;
    if (rot_dim % (interleaved ? 16 : 32)) return MIXKV_ERR_UNSUPPORTED;
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
  if (!k_out || !v_out || !aligned(k_out, 32) || !aligned(v_out, 32)) return MIXKV_ERR_INVALID_ARG;
  return type == MIXKV_TYPE_BF16 ? read_as<__nv_bfloat16>(c, a, k_out, v_out, stream)
                                 : read_as<__half>(c, a, k_out, v_out, stream);
}
