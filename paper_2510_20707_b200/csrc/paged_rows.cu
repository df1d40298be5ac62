// Rows into the paged 4-bit cache and back (format and rounding: include/mixkv.h).
//
// One CTA has one page of one head, so a page's bounds have one owner and need no atomics.  A warp takes four rows at a
// time, eight lanes each, a lane one block of 16 dimensions: the largest magnitude, the scale and the codes of a block are
// one lane's (32 bytes in, 8 out).  The rotation's partner dimensions lie rot_dim / 2 on, in another lane's registers.
// (Two rows at a time, half a block per lane and K and V in warps of their own took 262 instructions a row instead of
// 150, and half of the warps waited for the others.)
//
// What bounds it.  Append: latencies and instructions together; 4 x 32768 rows (67 MB in, 19 out) take 39 us, 2.2 TB/s, an
// instruction in 49 % of the clocks with sixteen warps an SM, and as long with twelve.  The cosines and sines are on their way while V is
// rounded.  Divisors and reciprocals of the 127 scales come from a table that a CTA fills once.  Reading back: 16 us (19 MB in, 67
// out), 5.4 TB/s; with 16-byte stores 20.
#include "paged.cuh"

namespace mixkv {
namespace {

constexpr int kRowThreads = 256;   // of a CTA that reads many rows of a page; one row per head: 64
constexpr int kAppThreads = 128, kAppPerSm = 4;   // of a CTA that may get many rows, and such CTAs per SM

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
  bool bad;                // a new row below row zero
};
__device__ __forceinline__ PageSpan page_span(const RowArgs& a, const int task) {
  PageSpan s;
  s.u = a.by_slots.div(task);
  const int slot = task - s.u * a.slots, b = a.p.by_heads.div(s.u);
  s.h = s.u - b * a.p.H;
  const int rows = fresh(a.p.rows + s.u);
  int n = 1;
  long long first = b;
  if (a.offsets) {
    const int i = a.per_head ? s.u : b;
    const int from = fresh(a.offsets + i), to = fresh(a.offsets + i + 1);
    n = to > from ? (int)min((unsigned)to - (unsigned)from, (unsigned)a.max_new) : 0;
    first = (long long)to - n;
  }
  s.bad = rows < n;
  if (s.bad) first += n - max(rows, 0), n = max(rows, 0);      // (only the last rows have a place)
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

// A block of 16 values -> its codes, and *scale.
//
// x / d is rounded to nearest by Markstein's correction of x times the rounded reciprocal: the remainder of that first quotient is
// exact, and one step with it rounds correctly while nothing over- or underflows.  Blocks of infinities and of extreme scales
// are divided.  (A code of zero has either sign.)
__device__ __forceinline__ uint2 quantise16(const f32x2 (&x)[8], const float inv6, const float2* divisors, uint32_t* scale) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float a, b;
    unpack2(x[i], a, b);
    m = max3_nan(m, fabsf(a), fabsf(b));
  }
  unsigned short s;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(s) : "f"(0.f), "f"(__fmul_rn(m, inv6)));
  *scale = s & 0x7fu;
  const float2 div = divisors[s & 0x7fu];
  const f32x2 by = pack2(div.y, div.y), d = pack2(-div.x, -div.x);
  f32x2 q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const f32x2 first = mul2(x[i], by);
    q[i] = fma2(fma2(first, d, x[i]), by, first);
  }
  if (!(m < 1e30f && div.x > 1e-30f)) {     // (NaN, and d == 0, too)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a, b;
      unpack2(x[i], a, b);
      q[i] = div.x == 0.f ? 0ull : pack2(__fdiv_rn(a, div.x), __fdiv_rn(b, div.x));
    }
  }
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) unpack2(q[4 * i + e], v[2 * e], v[2 * e + 1]);
    // (packed by shifts: with the four bytes packed by one move, the two upper ones came out wrong where the codes are widened
    // again for the bounds)
    w[i] = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t c;
      asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}"
          : "=r"(c)
          : "f"(v[2 * e + 1]), "f"(v[2 * e]));
      w[i] |= c << (8 * e);
    }
  }
  return make_uint2(w[0], w[1]);
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

struct Raw16 {   // 16 values of 16 bits
  uint4 a, b;
};
__device__ __forceinline__ uint32_t word16(const Raw16& r, const int i) {
  return i == 0 ? r.a.x : i == 1 ? r.a.y : i == 2 ? r.a.z : i == 3 ? r.a.w : i == 4 ? r.b.x : i == 5 ? r.b.y : i == 6 ? r.b.z : r.b.w;
}
template <typename T>
__device__ __forceinline__ Raw16 load16(const T* src, const bool on) {
  Raw16 r = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  if (on)
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
        : "=r"(r.a.x), "=r"(r.a.y), "=r"(r.a.z), "=r"(r.a.w), "=r"(r.b.x), "=r"(r.b.y), "=r"(r.b.z), "=r"(r.b.w)
        : "l"(src)
        : "memory");
  return r;
}
template <typename T>
__device__ __forceinline__ f32x2 wide2(const uint32_t w) {
  const float2 v = widen2<T>(w);
  return pack2(v.x, v.y);
}
template <>
__device__ __forceinline__ f32x2 wide2<__nv_bfloat16>(const uint32_t w) { return bf16x2_wide(w); }

// What a lane's block g is rotated by: cosines and sines of its pairs (ROPE 2: eight of each), from the token's row of the tables.
// ROPE 1: pairs (i, i + rot / 2), 2: (2 i, 2 i + 1).
template <int ROPE>
struct Turn {
  float4 cs[ROPE == 1 ? 4 : 2], sn[ROPE == 1 ? 4 : 2];
};
template <int ROPE>
__device__ __forceinline__ Turn<ROPE> load_turn(const RowArgs& a, const int pos, const int g) {
  Turn<ROPE> t;
  const int half = a.rot >> 1;
  const int at = ROPE == 2 ? 8 * g : 16 * g < half ? 16 * g : 16 * g - half;
  const long long from = (long long)pos * half + (16 * g < a.rot ? at : 0);
#pragma unroll
  for (int i = 0; i < (ROPE == 1 ? 4 : 2); ++i)
    t.cs[i] = fresh(reinterpret_cast<const float4*>(a.cosv + from) + i), t.sn[i] = fresh(reinterpret_cast<const float4*>(a.sinv + from) + i);
  return t;
}

// a + b in halves: of a packed sum and the packed products before it, .rn or not, the compiler makes multiply-adds.
__device__ __forceinline__ f32x2 add_rounded(const f32x2 a, const f32x2 b) {
  float ax, ay, bx, by;
  unpack2(a, ax, ay), unpack2(b, bx, by);
  return pack2(__fadd_rn(ax, bx), __fadd_rn(ay, by));
}
// The rotation; products and sums are rounded one by one.  All lanes of the warp take part.
template <typename T, int ROPE>
__device__ __forceinline__ void rotate16(const Raw16& raw, f32x2 (&x)[8], const int g, const int rot, const Turn<ROPE>& turn) {
  const int half = rot >> 1, lane = threadIdx.x & 31;
  const bool inside = 16 * g < rot;
  if constexpr (ROPE == 1) {
    const bool low = 16 * g < half;
    const int from = !inside ? lane : low ? lane + (half >> 4) : lane - (half >> 4);
    const uint32_t flip = low ? 0x80008000u : 0u;     // x cos - y sin is x cos + (-y) sin
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xffffffffu, word16(raw, i), from) ^ flip;
    if (!inside) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 cs = turn.cs[i], sn = turn.sn[i];
      x[2 * i] = add_rounded(mul2(x[2 * i], pack2(cs.x, cs.y)), mul2(wide2<T>(y[2 * i]), pack2(sn.x, sn.y)));
      x[2 * i + 1] = add_rounded(mul2(x[2 * i + 1], pack2(cs.z, cs.w)), mul2(wide2<T>(y[2 * i + 1]), pack2(sn.z, sn.w)));
    }
  } else if (ROPE == 2 && inside) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 cs = turn.cs[i], sn = turn.sn[i];
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

// A CTA of two warps has one page, K and V of one row each; one of four warps has a run of pages (of a head mostly: what the next
// page needs of the tables is in L1), every warp both.
template <typename T, int ROPE>
__global__ void __launch_bounds__(kAppThreads, kAppPerSm)
k_paged_append(const RowArgs a, const T* k, const T* v, const int tasks, const int run) {
  __shared__ float2 divisors[2][128];
  __shared__ __half2 part[kAppThreads / 32][8][17];   // of every warp: minima and maxima of a block's eight pairs of dimensions
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane & 7, sub = lane >> 3;
  fill_divisors(divisors[0], a.p.k_scale);
  fill_divisors(divisors[1], a.p.v_scale);
  pdl_launch_dependents();
  pdl_wait();
  const bool single = blockDim.x == 64;
  const int step = single ? 4 : 4 * (blockDim.x >> 5);
  const bool does_k = !single || warp == 0, does_v = !single || warp == 1;
  __syncthreads();
  const float k6 = (float)(1.0 / (6.0 * (double)a.p.k_scale)), v6 = (float)(1.0 / (6.0 * (double)a.p.v_scale));
  bool bad = false;
  const int end = min((int)(blockIdx.x + 1) * run, tasks);
  for (int task = blockIdx.x * run; task < end; ++task) {
    const PageSpan s = page_span(a, task);
    const T* kr = k + (a.per_head ? 0 : s.h * a.k_head) + s.token * a.k_row + 16 * g;     // row r of the page at r * stride
    const T* vr = v + (a.per_head ? 0 : s.h * a.v_head) + s.token * a.v_row + 16 * g;
    const int* positions = a.positions + s.token;
    const bool placed = s.id >= 0 && s.id < a.p.num_pages;
    bad |= s.bad || (s.lo < s.hi && !placed);
    __half2 lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = __float2half2_rn(INFINITY), hi[i] = __float2half2_rn(-INFINITY);

    int r = s.lo + (single ? 0 : 4 * warp) + sub;
    bool on = r >= s.first && r < s.last;
    Raw16 kk = load16(kr + r * a.k_row, on && does_k), vv = load16(vr + r * a.v_row, on && does_v);
    int pos = ROPE && on ? fresh(positions + r) : 0;
    for (; r - sub < s.hi; r += step) {
      const Raw16 kx = kk, vx = vv;
      const int at = pos;
      const bool have = on;
      if (r - sub + step < s.hi) {      // the next rows on their way
        const int next = r + step;
        on = next >= s.first && next < s.last;
        kk = load16(kr + next * a.k_row, on && does_k), vv = load16(vr + next * a.v_row, on && does_v);
        pos = ROPE && on ? fresh(positions + next) : 0;
      }
      const bool turned = at >= 0 && at < a.table_len;
      const bool write = have && placed && (!ROPE || turned);      // (a token is written whole or not at all)
      bad |= r < s.hi && !write;
      unsigned char* tile = tile_ptr(a.p, placed ? s.id : 0, r / kPageTile);
      const int rt = r % kPageTile;
      Turn<ROPE> turn;      // (on its way while V is rounded)
      if (ROPE && does_k) turn = load_turn<ROPE>(a, turned ? at : 0, g);
      if (does_v) {
        f32x2 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = wide2<T>(word16(vx, i));
        uint32_t scale;
        const uint2 w = quantise16(x, v6, divisors[1], &scale);
        if (write) {
          *reinterpret_cast<uint2*>(tile + v_codes_at(rt, g)) = w;
          tile[v_scale_at(rt, g)] = (unsigned char)scale;
        }
      }
      if (does_k) {
        f32x2 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = wide2<T>(word16(kx, i));
        if constexpr (ROPE != 0) {
          rotate16<T, ROPE>(kx, x, g, a.rot, turn);
        }
        uint32_t scale;
        const uint2 w = quantise16(x, k6, divisors[0], &scale);
        if (write) {
          *reinterpret_cast<uint2*>(tile + k_codes_at(rt, g)) = w;
          tile[k_scale_at(rt, g)] = (unsigned char)scale;
          if (a.p.bounds) {
            uint32_t f[8];
            codes_to_f16(w.x, *reinterpret_cast<uint32_t(*)[4]>(&f[0]));
            codes_to_f16(w.y, *reinterpret_cast<uint32_t(*)[4]>(&f[4]));
            const uint32_t ss = scales_to_f16(scale | scale << 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t y = mul_f16x2(f[i], ss);
              lo[i] = __hmin2_nan(lo[i], *reinterpret_cast<const __half2*>(&y));
              hi[i] = __hmax2_nan(hi[i], *reinterpret_cast<const __half2*>(&y));
            }
          }
        }
      }
    }
    if (!a.p.bounds || !placed || s.lo >= s.hi) continue;
    if (does_k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int o = 8; o < 32; o <<= 1) {
          lo[i] = __hmin2_nan(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o));
          hi[i] = __hmax2_nan(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o));
        }
        if (sub == 0) part[warp][g][i] = lo[i], part[warp][g][8 + i] = hi[i];
      }
    }
    __syncthreads();
    const int warps = single ? 1 : min((int)(blockDim.x >> 5), (s.hi - s.lo + 3) / 4);    // those that had rows
    for (int e = tid; e < 128; e += blockDim.x) {
      const bool most = e & 64;
      const int block = (e & 63) >> 3, i = (most ? 8 : 0) + (e & 7);
      __half2 x = part[0][block][i];
      for (int w = 1; w < warps; ++w) x = most ? __hmax2_nan(x, part[w][block][i]) : __hmin2_nan(x, part[w][block][i]);
      __half2* out = reinterpret_cast<__half2*>(a.p.bounds + ((long long)s.id * 2 + most) * kHeadDim) + (e & 63);
      if (s.lo > 0) x = most ? __hmax2_nan(x, *out) : __hmin2_nan(x, *out);
      *out = x;
    }
    if (task + 1 < end) __syncthreads();    // `part` is written again
  }
  if (bad && a.status) *a.status = MIXKV_ERR_INVALID_ARG;
}

// A lane has a block of a row, as above.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_paged_read(const RowArgs a, T* k, T* v) {
  pdl_launch_dependents();
  pdl_wait();
  const PageSpan s = page_span(a, blockIdx.x);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane & 7, sub = lane >> 3;
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
      (reinterpret_cast<uintptr_t>(offsets) & 3u))
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
  void (*kernel)(RowArgs, const T*, const T*, int, int) =
      rope == 0 ? k_paged_append<T, 0> : rope == 1 ? k_paged_append<T, 1> : k_paged_append<T, 2>;
  // Two pages to a CTA: one leaves the tables it fills first to be filled more often, an equal share of a whole wave (four and
  // eight pages here) lets it wait for the last.  4 x 32768 rows in pages of 64 55.6 / 55.2 / 54.7 us on one, two and four
  // pages (append and read back), 8 ragged chunks in pages of 32 45.4 / 43.4 / 48.8.
  const int tasks = tasks_of(c, a), run = tasks > kAppPerSm * device_sm_count() ? 2 : 1;
  return launch_pdl(kernel, dim3((unsigned)((tasks + run - 1) / run)), dim3(a.max_new > 1 ? kAppThreads : 64), 0,
                    (cudaStream_t)stream, 1, a, static_cast<const T*>(k), static_cast<const T*>(v), tasks, run) == cudaSuccess
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
bool aligned(const void* p, const unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

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
  if (!k || !v || !aligned(k, 32) || !aligned(v, 32)) return MIXKV_ERR_INVALID_ARG;
  for (const int64_t stride : {k_row_stride, k_head_stride, v_row_stride, v_head_stride})
    if (stride < 0 || stride % 16) return MIXKV_ERR_INVALID_ARG;
  const bool rope = cos_opt != nullptr;
  if (rope != (sin_opt != nullptr)) return MIXKV_ERR_INVALID_ARG;
  if (rope) {
    if (!positions_opt || table_len < 1 || !aligned(cos_opt, 16) || !aligned(sin_opt, 16) || rot_dim < 1 || rot_dim > kHeadDim ||
        (reinterpret_cast<uintptr_t>(positions_opt) & 3u))
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
