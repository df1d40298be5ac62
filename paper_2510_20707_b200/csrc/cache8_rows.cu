// Rows into the paged 8-bit cache and back (format: include/mixkv.h).
//
// A warp has the K or the V rows of one tile.  Lane (sub, g) has dimensions 16 g .. 16 g + 15 of rows 4 i + sub, 32 bytes of each as they
// come and 16 as they are kept: eight lanes read 256 contiguous bytes and write 128.  The block's largest magnitude is one
// reduction over the warp, on the bits of the 16-bit values (a magnitude's bits are in its order, infinities and NaN above all numbers).
// Nothing is pipelined: a warp has four rows a lane in flight, and an SM holds enough warps.
//
// What bounds it: 32768 rows of four heads are appended in 17.9 us (100 MB, 5.6 TB/s; an instruction issued in 70 % of the clocks, and no
// faster without the search for the largest magnitude), read back in 14.6 (100 MB, 6.9 TB/s).  One token of a head costs its tile, 4
// KB read and, where the scale grows, written: 512 heads 4.8 us, the call's host time.
#include "cache8.cuh"

namespace mixkv {
namespace {

constexpr int kRowWarps = 4;
// CTAs of an SM that appends, which sets the registers of a thread: 32768 rows of four heads 17.9 us with ten (48 registers, 24 bytes
// spilt), 20.3 with six (79, what the compiler takes), 21.7 and 22.0 with eight and nine (56, 8 bytes), 22.9 with twelve (40, 132 bytes), 31
// with sixteen.
constexpr int kAppendPerSm = 10;

struct RowArgs {
  CachePool p;
  const int* offsets;      // nullptr: one token per sequence
  bool per_head;
  int max_new;
  int slots;               // tiles of a head that its new rows can touch
  Divider by_slots;
  long long num_tokens;
  long long k_row, k_head, v_row, v_head;   // strides, elements
  int* status;
};

// The new rows of a unit (head h of sequence b) that lie on one tile.
struct TileSpan {
  int u, h;
  int lo, hi;              // new rows of the tile; none: hi <= lo
  int first, last;         // those of them whose token is in the input
  long long token;         // token (or row of the input) of row 0 of the tile; there may be none
  int id, in;              // what the table says, -1 beyond it; tile of the page
  bool begun;              // the tile has rows from before the call
  bool bad;                // a new row below row zero, or more of them than the call allows
};
__device__ __forceinline__ TileSpan tile_span(const RowArgs& a, const int task) {
  TileSpan s;
  // heads of a token next to one another: they are in memory
  const int at = a.p.by_heads.div(task), b = a.by_slots.div(at), slot = at - b * a.slots;
  s.h = task - at * a.p.H;
  s.u = b * a.p.H + s.h;
  const int rows = fresh(a.p.rows + s.u);
  int n = 1;
  unsigned all = 1;
  long long first = b;
  if (a.offsets) {
    const int i = a.per_head ? s.u : b;
    const int from = fresh(a.offsets + i), to = fresh(a.offsets + i + 1);
    all = to > from ? (unsigned)to - (unsigned)from : 0u;
    n = (int)min(all, (unsigned)a.max_new);
    first = (long long)to - n;
  }
  s.bad = rows < n;
  if (s.bad) first += n - max(rows, 0), n = max(rows, 0);      // (only the last rows have a place)
  s.bad |= all > (unsigned)a.max_new;
  const int r0 = rows - n, t = (r0 >> 4) + slot;      // row of the first token that is written, the tile
  const long long begin = (long long)t * kBlockRows, end = begin + kBlockRows;
  const long long hi = rows < end ? rows : end;
  s.lo = n > 0 ? (int)((r0 > begin ? r0 : begin) - begin) : 0, s.hi = n > 0 ? (int)(hi - begin) : 0;
  s.begun = begin < (long long)rows - (long long)all;      // (rows beyond max_new are new as well)
  s.token = first + (begin - r0);
  const long long from = -s.token, to = a.num_tokens - s.token;
  s.first = from > s.lo ? (int)(from < s.hi ? from : s.hi) : s.lo;
  s.last = to < s.hi ? (int)(to > s.lo ? to : s.lo) : s.hi;
  const int page = n > 0 ? a.p.by_tiles.div(t) : 0;
  s.in = t - page * a.p.tiles;
  s.id = s.lo < s.hi && page < a.p.max_pages ? fresh(a.p.table + (long long)s.u * a.p.max_pages + page) : -1;
  return s;
}

template <typename T, bool E4M3>
__global__ void __launch_bounds__(kRowWarps * 32, kAppendPerSm) k_cache8_append(const RowArgs a, const T* k, const T* v, const int tasks) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane & 7, sub = lane >> 3;
  const int job = blockIdx.x * kRowWarps + warp;
  pdl_wait();
  if (job >= 2 * tasks) return;
  const bool values = job & 1;
  const TileSpan s = tile_span(a, job >> 1);
  if (s.lo >= s.hi) {
    if (s.bad && a.status && lane == 0) *a.status = MIXKV_ERR_INVALID_ARG;
    return;
  }
  const long long row = values ? a.v_row : a.k_row, head = a.per_head ? 0 : s.h * (values ? a.v_head : a.k_head);
  const T* from = (values ? v : k) + head + 16 * g;
  Sixteen x[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {       // (on their way before it is known where they go)
    const int r = 4 * i + sub;
    if (r >= s.first && r < s.last) load_sixteen(x[i], from + (s.token + r) * row);
  }
  const bool placed = s.id >= 0 && s.id < a.p.num_pages;
  if ((s.bad || !placed || s.first > s.lo || s.last < s.hi) && a.status && lane == 0) *a.status = MIXKV_ERR_INVALID_ARG;
  if (!placed) return;
  unsigned char* tile = block_ptr(a.p, s.id, s.in);
  unsigned char* codes = tile + (values ? kBlockV : 0);
  float* scale_at = reinterpret_cast<float*>(tile + kBlockScales) + values;
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max_u16x2(most, x[i].w[j] & 0x7fff7fffu);
  most = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
  const float was = s.begun ? *scale_at : 0.f;
  const float scale = larger_scale(was, scale_of_largest<E4M3>(widen2<T>(most).x)), by = by_scale(scale);
  const bool grown = !(scale == was);      // (or NaN: its codes are zero)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + sub;
    const bool is_new = r >= s.first && r < s.last;
    uint4* at = reinterpret_cast<uint4*>(codes + piece_at(r, g));
    if (is_new || !s.begun) {      // (rows that are not there: zeros)
      *at = encode16<T, E4M3>(x[i], by);
    } else if (grown) {            // an old row, of which each lane has its own piece
      f32x2 y[8];
      values16<E4M3>(*at, was, y);
      *at = encode16<E4M3>(y, by);
    }
  }
  if (lane == 0 && (grown || !s.begun)) *scale_at = scale;
  if (values && a.p.mass && lane >= s.first && lane < s.last)
    a.p.mass[(long long)s.id * a.p.page_rows + s.in * kBlockRows + lane] = 0.f;
}

template <typename T, bool E4M3>
__global__ void __launch_bounds__(kRowWarps * 32) k_cache8_read(const RowArgs a, T* k, T* v, const int tasks) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane & 7, sub = lane >> 3;
  const int job = blockIdx.x * kRowWarps + warp;
  pdl_wait();
  if (job >= 2 * tasks) return;
  const bool values = job & 1;
  const TileSpan s = tile_span(a, job >> 1);
  if (s.first >= s.last || s.id < 0 || s.id >= a.p.num_pages) return;
  const unsigned char* tile = block_ptr(a.p, s.id, s.in);
  const float scale = *(reinterpret_cast<const float*>(tile + kBlockScales) + values);
  const long long row = a.per_head ? kHeadDim : (long long)a.p.H * kHeadDim;
  T* to = (values ? v : k) + (a.per_head ? 0 : s.h * kHeadDim) + 16 * g;
  uint4 codes[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) codes[i] = *reinterpret_cast<const uint4*>(tile + (values ? kBlockV : 0) + piece_at(4 * i + sub, g));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + sub;
    if (r < s.first || r >= s.last) continue;
    f32x2 y[8];
    values16<E4M3>(codes[i], scale, y);
    Sixteen out;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float lo, hi;
      unpack2(y[j], lo, hi);
      out.w[j] = narrow2<T>(lo, hi);
    }
    store_sixteen(to + (s.token + r) * row, out);
  }
}

int check_rows(const mixkv_cache8* c, int32_t type, int64_t num_tokens, const int32_t* offsets, int32_t per_head,
               int32_t max_new, RowArgs* a) {
  const int rc = check_cache(c, &a->p);
  if (rc != MIXKV_OK) return rc;
  if ((type != MIXKV_TYPE_BF16 && type != MIXKV_TYPE_FP16) || num_tokens < 0 || max_new < 1 || (per_head && !offsets) ||
      !aligned(offsets, 4))
    return MIXKV_ERR_INVALID_ARG;
  if (max_new > (1 << 30)) return MIXKV_ERR_UNSUPPORTED;
  a->offsets = offsets, a->per_head = per_head != 0, a->max_new = offsets ? max_new : 1, a->num_tokens = num_tokens;
  // tiles that a head's new rows can touch: one, and one more for every sixteen rows behind the first
  a->slots = (a->max_new - 1 + kBlockRows - 1) / kBlockRows + 1;
  const long long all = (long long)c->max_pages * a->p.tiles + 1;   // (one past the table: rows there are reported)
  if (a->slots > all) a->slots = (int)all;
  if ((long long)c->batch * c->kv_heads * a->slots > 0x3fffff00ll) return MIXKV_ERR_UNSUPPORTED;
  a->by_slots = Divider(a->slots);
  return MIXKV_OK;
}
template <typename T, typename Kernel>
int launch_rows(const mixkv_cache8* c, const RowArgs& a, Kernel int8, Kernel e4m3, T* k, T* v, void* stream) {
  const int rc = device_check(nullptr);
  if (rc != MIXKV_OK) return rc;
  const int tasks = c->batch * c->kv_heads * a.slots;
  return launch_pdl(c->code == MIXKV_CODE_E4M3 ? e4m3 : int8, dim3((unsigned)((2LL * tasks + kRowWarps - 1) / kRowWarps)),
                    dim3(kRowWarps * 32), 0, (cudaStream_t)stream, 1, a, k, v, tasks) == cudaSuccess
             ? MIXKV_OK
             : MIXKV_ERR_CUDA;
}
template <typename T>
int append_as(const mixkv_cache8* c, const RowArgs& a, const void* k, const void* v, void* stream) {
  return launch_rows(c, a, k_cache8_append<T, false>, k_cache8_append<T, true>, static_cast<const T*>(k),
                     static_cast<const T*>(v), stream);
}
template <typename T>
int read_as(const mixkv_cache8* c, const RowArgs& a, void* k, void* v, void* stream) {
  return launch_rows(c, a, k_cache8_read<T, false>, k_cache8_read<T, true>, static_cast<T*>(k), static_cast<T*>(v), stream);
}

}  // namespace
}  // namespace mixkv

using namespace mixkv;

extern "C" int mixkv_cache_page_bytes(int32_t page_rows, size_t* bytes) {
  if (!bytes || page_rows < kBlockRows || page_rows % kBlockRows || page_rows > MIXKV_PAGE_MAX_ROWS)
    return MIXKV_ERR_INVALID_ARG;
  *bytes = (size_t)(page_rows / kBlockRows) * kBlockBytes;
  return MIXKV_OK;
}

extern "C" int mixkv_cache_append(const mixkv_cache8* c, const void* k, const void* v, int32_t type, int64_t num_tokens,
                                   int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride,
                                   int64_t v_head_stride, const int32_t* offsets_opt, int32_t offsets_per_head,
                                   int32_t max_new, int32_t* status_dev, void* stream) {
  RowArgs a = {};
  const int rc = check_rows(c, type, num_tokens, offsets_opt, offsets_per_head, max_new, &a);
  if (rc != MIXKV_OK) return rc;
  if (!k || !v || !aligned(k, 32) || !aligned(v, 32) || !aligned(status_dev, 4)) return MIXKV_ERR_INVALID_ARG;
  for (const int64_t stride : {k_row_stride, k_head_stride, v_row_stride, v_head_stride})
    if (stride < 0 || stride % 16) return MIXKV_ERR_INVALID_ARG;
  a.k_row = k_row_stride, a.k_head = k_head_stride, a.v_row = v_row_stride, a.v_head = v_head_stride;
  a.status = status_dev;
  return type == MIXKV_TYPE_BF16 ? append_as<__nv_bfloat16>(c, a, k, v, stream) : append_as<__half>(c, a, k, v, stream);
}

extern "C" int mixkv_cache_read(const mixkv_cache8* c, void* k_out, void* v_out, int32_t type, int64_t num_tokens,
                                 const int32_t* offsets_opt, int32_t offsets_per_head, int32_t max_new, void* stream) {
  RowArgs a = {};
  const int rc = check_rows(c, type, num_tokens, offsets_opt, offsets_per_head, max_new, &a);
  if (rc != MIXKV_OK) return rc;
  if (!k_out || !v_out || !aligned(k_out, 32) || !aligned(v_out, 32)) return MIXKV_ERR_INVALID_ARG;
  return type == MIXKV_TYPE_BF16 ? read_as<__nv_bfloat16>(c, a, k_out, v_out, stream)
                                 : read_as<__half>(c, a, k_out, v_out, stream);
}
