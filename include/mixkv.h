/*
 * mixkv.h -- C ABI of the B200 (sm_100a) MixKV prefill KV-cache compression library.
 *
 * The library implements one step of LVLM / LLM inference: at the end of prefill, for
 * one transformer layer, score every cached key of every KV head, keep the best B per
 * head and copy the kept K/V rows into a compact cache (MixKV, arxiv 2510.20707,
 * Sec. 3.1 "KV Cache Compression", Sec. 3.2-3.3, Algorithm 1).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - All tensor pointers are DEVICE pointers unless the name ends in `_host`.
 *    bf16 tensors must be 16-byte aligned, fp32 / int32 tensors 4-byte aligned.
 *  - The caller owns every buffer, including the workspace.  The library allocates no
 *    device memory and never synchronises the stream: every call only enqueues kernels
 *    on `stream` (a cudaStream_t passed as void*; NULL is the default stream).  Host
 *    state kept between calls is limited to per-device caches of attributes (SM count,
 *    compute capability, shared-memory opt-in, clusters resident at once).  The workspace needs no initialisation
 *    and no clearing between calls (every word a kernel reads was written earlier in the
 *    same call; nothing is counted across CTAs), and may be reused for other shapes.  It belongs
 *    to one call at a time: calls whose kernels may overlap on the GPU need one each, and so do calls that
 *    several host threads make at once, on one stream even (a call enqueues several kernels, and those of
 *    another thread's call may come between them; mixkv_scores_static takes care of that itself).
 *  - Shapes.  H = kv_heads, G = gqa_ratio, d = head_dim (128), W = window.
 *      K, V      [H, Ltot, d] bf16, row-major.  Ltot = L for one sequence, else
 *                cu_seqlens_host[batch]; sequence b owns rows cu[b] .. cu[b+1]-1.
 *      Qwin      [batch, H*G, W, d] bf16: the last W prompt queries (post-RoPE) of every
 *                query head; query head q attends KV head q / G.  Window row j sits at
 *                sequence position P + j (P = L - W) and sees keys 0 .. P + j.
 *      scores    [H, Ptot] fp32, Ptot = Ltot - batch*W: the P_b = L_b - W candidate
 *                (non-window) positions of sequence b start at column cu[b] - b*W.
 *      rbar      [batch, H] fp32.
 *  - cu_seqlens_host: HOST pointer to batch+1 ascending int32 offsets, read during the
 *    call (not retained).  NULL means one sequence of length L (batch must be 1).
 *  - Return value: 0 on success, a negative mixkv_status otherwise.  Argument errors
 *    (INVALID_ARG, UNSUPPORTED, WORKSPACE_TOO_SMALL) enqueue nothing; MIXKV_ERR_CUDA means a
 *    launch failed, earlier kernels of the call may already be enqueued and the outputs are
 *    undefined.  A device whose compute capability is not 10.x gives MIXKV_ERR_UNSUPPORTED (the
 *    kernels use tcgen05 / tensor memory; see mixkv_device_check).  Conditions only the
 *    device can see (a bounded wait inside a kernel expired) are written to *status_dev
 *    (device int32, optional, must be zeroed by the caller) as MIXKV_ERR_TIMEOUT; kernels
 *    never trap.
 *  - CUDA graphs: a call may be recorded into a stream capture and replayed, provided the
 *    same entry point ran once on that device outside capture (its first use sets function
 *    attributes); the host arrays (cu_seqlens_host) are read at capture time only.
 *  - Limits: head_dim == 128; 16 <= G*W <= 240 and G*W % 16 == 0; batch <= 64;
 *    every sequence needs L_b >= W + 1; budget > W; odd pool_kernel <= 63.
 */
#ifndef MIXKV_H_
#define MIXKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MIXKV_OK = 0,
  MIXKV_ERR_INVALID_ARG = -1,
  MIXKV_ERR_UNSUPPORTED = -2,
  MIXKV_ERR_WORKSPACE_TOO_SMALL = -3,
  MIXKV_ERR_CUDA = -4,
  MIXKV_ERR_TIMEOUT = -5,
  MIXKV_ERR_STATIC_SCRATCH_EXCEEDED = -6
} mixkv_status;

enum { MIXKV_MIX_HEADWISE = 0, MIXKV_MIX_IMPORTANCE_ONLY = 1, MIXKV_MIX_DIVERSITY_ONLY = 2,
       MIXKV_MIX_PLAIN_SUM = 3 };
enum { MIXKV_POOL_AVG = 0, MIXKV_POOL_MAX = 1 };
enum { MIXKV_BUDGET_FIXED = 0, MIXKV_BUDGET_ADAPTIVE = 1 };
enum { MIXKV_INTRINSIC_NONE = 0, MIXKV_INTRINSIC_VNORM = 1, MIXKV_INTRINSIC_KNORM = 2 };

typedef struct mixkv_params {
  int32_t kv_heads;     /* H */
  int32_t gqa_ratio;    /* G: query heads per KV head */
  int32_t head_dim;     /* d: must be 128 */
  int32_t window;       /* W: observation window, paper default 32 (Sec. 3.2) */
  int32_t pool_kernel;  /* odd k >= 1; 1-D pooling of the attention score, 1 = none */
  int32_t pool_mode;    /* MIXKV_POOL_AVG (zero padded, divides by k) or MIXKV_POOL_MAX */
  int32_t use_vnorm;    /* intrinsic importance added in Eq. 2: MIXKV_INTRINSIC_VNORM (value norm,
                           the paper's default), _KNORM (minus the key norm: the KNorm variant of
                           Sec. 3.2 and of the ablation table), _NONE */
  int32_t mix_mode;     /* MIXKV_MIX_*: Eq. 5, or one of the ablation variants of Table 4 */
  int32_t budget_mode;  /* MIXKV_BUDGET_FIXED: B per head; _ADAPTIVE: B*H per sequence */
  int32_t budget;       /* B: rows kept per head INCLUDING the W window rows (Alg. 1) */
  float ada_floor;      /* adaptive: fraction of B - W guaranteed to every head (0..1) */
  float eps;            /* epsilon of the two min-max normalisations (Sec. 3.2, 3.3) */
  float softmax_scale;  /* 0 => 1/sqrt(d) */
} mixkv_params;

/* Fills *p with the paper's defaults: W 32, average pooling k 7, VNorm on, Eq. 5 mixing,
 * fixed budget, ada_floor 0.2, eps 1e-6, scale 1/sqrt(d).  Sets H, G and B as given. */
void mixkv_default_params(mixkv_params* p, int32_t kv_heads, int32_t gqa_ratio, int32_t budget);

/* Bytes of device workspace the three entry points below need for a batch whose sequence
 * lengths sum to total_tokens (max single length max_seq_len).  Host-only; no CUDA call. */
int mixkv_workspace_size(const mixkv_params* p, int32_t batch, int64_t total_tokens,
                         int32_t max_seq_len, size_t* bytes);

/* The same for a call that handles n_layers layers at once (mixkv_compress_layers). */
int mixkv_workspace_size_layers(const mixkv_params* p, int32_t n_layers, int32_t batch,
                                int64_t total_tokens, int32_t max_seq_len, size_t* bytes);

/* Scores of every candidate key (Sec. 3.2-3.3; Algorithm 1 step 1 and the mixing of step 2):
 *   s_ex   = pool_k( sum over the G query heads of the mean over the W window rows of the
 *            causal softmax attention weight on key i )             (extrinsic importance)
 *   s_imp  = s_ex + VNorm_i min-max normalised, rescaled to mean(s_ex)            (Eq. 2)
 *   s_div  = - cos(K_i, mean over all L keys of the unit keys)                  (diversity)
 *   rbar   = (L^2 |mean unit key|^2 - L) / (L (L-1))                            (Eq. 3-4)
 *   s_comp = (1 - rbar) s_imp + rbar * (s_div min-max normalised, rescaled to mean(s_imp))
 *                                                                                 (Eq. 5)
 * Key geometry (mean unit key, rbar) uses all L keys of the sequence; score vectors and
 * their min / max / mean use the P candidate positions.
 *   s_comp        out, required, [H, Ptot]
 *   s_ex_opt      out, optional (NULL to skip), pooled attention score [H, Ptot]
 *   s_div_opt     out, optional, raw diversity score [H, Ptot]
 *   rbar_opt      out, optional, [batch, H]
 *   rbar_in_opt   in, optional, [batch, H]: redundancy to mix with instead of the computed
 *                 one (head weights calibrated offline, Sec. 4.3)
 *   V may be NULL unless use_vnorm == MIXKV_INTRINSIC_VNORM.
 * NaN or infinite values in K, V or Q can make every score of their head NaN, in their sequence and in the one before
 * it in the batch.  Selection takes any scores: a NaN ranks by its bits, above every number or (sign set) below, and
 * budgets, offsets and index lists are those of such scores, within the outputs' sizes. */
int mixkv_scores(const void* K, const void* V, const void* Qwin,
                 const int32_t* cu_seqlens_host, int32_t batch, int32_t L,
                 const mixkv_params* p, void* workspace, size_t workspace_bytes,
                 float* s_comp, float* s_ex_opt, float* s_div_opt, float* rbar_opt,
                 const float* rbar_in_opt, int32_t* status_dev, void* stream);

/* mixkv_scores for callers that cannot obtain device memory for a workspace (the paper has
 * no counterpart; this is a packaging variant of mixkv_scores, same kernels, same results).
 * Typical users: a serving engine that hands every free byte of HBM to its own paged KV pool
 * at start-up, so that a later cudaMalloc fails or fragments the pool; a plug-in running
 * inside somebody else's step loop, where cudaMalloc / cudaFree would stall the whole device
 * with their implicit synchronisation; a host language binding that can pass pointers it
 * was given but owns no allocator.  Such callers still pass their inputs and outputs; only
 * the scratch the kernels need between them comes from the library: a fixed array of
 * MIXKV_STATIC_SCRATCH_BYTES that lives in the library's device image, so every GPU that
 * loads the library sets that much memory aside until the process exits.
 *  - Problems whose workspace (mixkv_workspace_size) would exceed the array are refused with
 *    MIXKV_ERR_STATIC_SCRATCH_EXCEEDED before anything is enqueued (the size is worked out on
 *    the host; the only CUDA calls before the refusal are attribute queries).  As a guide the array covers
 *    about 128k (head, token) pairs, e.g. H = 4 at L = 32768 or H = 8 at L = 16384.
 *  - The call performs no cudaMalloc / cudaFree and calls no allocating library routine.
 *  - The first call on each device looks up the array's device address (once per device, with
 *    that device current) and keeps it for later calls; make that first call outside any
 *    stream capture.  The kept address does not survive cudaDeviceReset: a process that resets
 *    a device must not call this entry point on it afterwards.
 *  - All calls on one device share the one array, and it keeps whatever the previous call
 *    left in it.  Nothing in it needs to start from zero (every cell is written before it is
 *    read inside a call), but two calls whose kernels overlap on the GPU (different streams
 *    without an ordering between them) race on it: order such calls yourself.  Several host threads
 *    may call at once: the kernels of one call are enqueued together, and a call waits on the host
 *    while another thread's is being enqueued on that device.
 * Arguments are those of mixkv_scores without workspace / workspace_bytes. */
#define MIXKV_STATIC_SCRATCH_BYTES (12u << 20)
int mixkv_scores_static(const void* K, const void* V, const void* Qwin,
                        const int32_t* cu_seqlens_host, int32_t batch, int32_t L,
                        const mixkv_params* p, float* s_comp, float* s_ex_opt, float* s_div_opt,
                        float* rbar_opt, const float* rbar_in_opt, int32_t* status_dev,
                        void* stream);

/* TopB of Sec. 3.1 / Algorithm 1 on caller-supplied scores [H, Ptot]: per (sequence, head)
 * the b_h highest scores among the P_b candidates, ties to the lower position, written in
 * ascending position order.  b_h = min(B - W, P_b) for fixed budgets.  Adaptive budgets
 * (per sequence): every head is guaranteed f = floor(ada_floor * (B - W)); the remaining
 * H * (B - W - f) slots go to the highest scores of the H heads taken together (ties to the
 * lower (head, position)); b_h = min(f + share_h, P_b).
 *   idx          out, packed in (b, h) order; capacity batch * H * (B - W) int32 is always
 *                enough
 *   counts       out, [batch * H], b_h
 *   idx_offsets  out, [batch * H + 1], exclusive prefix sum of counts
 * status_dev is accepted for symmetry and never written: the kernels of this entry point
 * contain no bounded waits. */
int mixkv_select(const float* scores, const int32_t* cu_seqlens_host, int32_t batch, int32_t L,
                 const mixkv_params* p, void* workspace, size_t workspace_bytes,
                 int32_t* idx, int32_t* counts, int32_t* idx_offsets,
                 int32_t* status_dev, void* stream);

/* The whole per-layer step of Algorithm 1: mixkv_scores, mixkv_select, then the gather:
 * for every (b, h) the selected rows of K and V in ascending position order followed by the
 * W window rows, packed in (b, h) order.
 *   K_out, V_out      out, [rows, d] bf16; capacity batch * H * B rows is always enough
 *   out_row_offsets   out, [batch * H + 1]: first output row of each (b, h); last = rows
 *   idx_opt / counts_opt / idx_offsets_opt / s_comp_opt   optional outputs as above (NULL:
 *                     kept in the workspace) */
int mixkv_compress_layer(const void* K, const void* V, const void* Qwin,
                         const int32_t* cu_seqlens_host, int32_t batch, int32_t L,
                         const mixkv_params* p, void* workspace, size_t workspace_bytes,
                         const float* rbar_in_opt, void* K_out, void* V_out,
                         int32_t* out_row_offsets, int32_t* idx_opt, int32_t* counts_opt,
                         int32_t* idx_offsets_opt, float* s_comp_opt,
                         int32_t* status_dev, void* stream);

/* Measurement hook (no counterpart in the paper): mixkv_compress_layer with CUDA events
 * recorded on `stream` around its kernels.  events_host is a HOST array of n_events
 * cudaEvent_t handles created by the caller with timing enabled: events_host[i] is recorded
 * just before the i-th kernel and events_host[k] after the last of the k kernels
 * (k = mixkv_launches_per_layer); entries beyond n_events are skipped, so n_events = 2
 * brackets the first kernel only.  Everything else is as mixkv_compress_layer. */
int mixkv_compress_layer_traced(const void* K, const void* V, const void* Qwin,
                                const int32_t* cu_seqlens_host, int32_t batch, int32_t L,
                                const mixkv_params* p, void* workspace, size_t workspace_bytes,
                                const float* rbar_in_opt, void* K_out, void* V_out,
                                int32_t* out_row_offsets, int32_t* idx_opt, int32_t* counts_opt,
                                int32_t* idx_offsets_opt, float* s_comp_opt,
                                int32_t* status_dev, void* stream,
                                void* const* events_host, int32_t n_events);

/* mixkv_compress_layer for n_layers layers of identical shape in ONE set of kernel launches
 * (Algorithm 1's "for each layer l and head h" loop taken whole): a serving engine that keeps the
 * prefill KV of all layers resident can compress them together at the end of prefill, which
 * spreads the per-launch costs over all layers and keeps every SM busy in the selection and
 * gather step.  The layers are an outer batch dimension; each is processed exactly as
 * mixkv_compress_layer would.
 *   K, V              [n_layers, H, Ltot, d] bf16; kv_layer_stride = elements between the
 *                     tensors of consecutive layers (0: packed, H * Ltot * d; otherwise a
 *                     multiple of 8 and at least that)
 *   Qwin              [n_layers, batch, H*G, W, d] bf16; q_layer_stride likewise (0: packed)
 *   rbar_in_opt       optional, [n_layers, batch, H]
 *   K_out, V_out      [n_layers, batch * H * B, d]: layer l starts at row l * batch * H * B and
 *                     is packed inside its slice as mixkv_compress_layer packs it
 *   out_row_offsets   [n_layers, batch * H + 1], rows relative to the layer's slice
 *   idx_opt           [n_layers, cap], cap = sum over sequences of H * min(B - W, P_b)
 *   counts_opt        [n_layers, batch * H];  idx_offsets_opt [n_layers, batch * H + 1]
 *   s_comp_opt        [n_layers, H, Ptot]
 *   workspace         mixkv_workspace_size_layers bytes
 *   events_host       optional measurement hook as in mixkv_compress_layer_traced (NULL, 0: off)
 * n_layers <= 1024. */
int mixkv_compress_layers(const void* K, const void* V, const void* Qwin, int32_t n_layers,
                          int64_t kv_layer_stride, int64_t q_layer_stride,
                          const int32_t* cu_seqlens_host, int32_t batch, int32_t L,
                          const mixkv_params* p, void* workspace, size_t workspace_bytes,
                          const float* rbar_in_opt, void* K_out, void* V_out,
                          int32_t* out_row_offsets, int32_t* idx_opt, int32_t* counts_opt,
                          int32_t* idx_offsets_opt, float* s_comp_opt, int32_t* status_dev,
                          void* stream, void* const* events_host, int32_t n_events);

/* mixkv_compress_layers with the budgets chosen outside the library: the paper plugs its scores
 * into compressors that differ only in how many rows a layer or a head may keep (Section 4.1 and
 * the related-work appendix: PyramidKV gives lower layers more than higher ones, SparseMM / HeadKV
 * give every head its own static share).  Scores, selection and gather are exactly those of
 * mixkv_compress_layers; only the number of candidates taken per head comes from the caller.
 *   head_budgets   device, [n_layers, batch * H] int32: rows to keep for that (layer, sequence,
 *                  head), window included.  A value is used as min(max(v - W, 0), B - W, P_b)
 *                  selected candidates plus the W window rows; p->budget (B) is the largest
 *                  budget any head may get and sizes the outputs as in mixkv_compress_layers.
 *   p->budget_mode must be MIXKV_BUDGET_FIXED (else MIXKV_ERR_INVALID_ARG).
 * Outputs are ragged as with adaptive budgets: rows of (b, h) start at out_row_offsets[l][b*H+h]
 * of layer l's slice; counts_opt receives the candidates actually selected. */
int mixkv_compress_layers_budgeted(const void* K, const void* V, const void* Qwin,
                                   int32_t n_layers, int64_t kv_layer_stride,
                                   int64_t q_layer_stride, const int32_t* cu_seqlens_host,
                                   int32_t batch, int32_t L, const mixkv_params* p,
                                   void* workspace, size_t workspace_bytes,
                                   const float* rbar_in_opt, const int32_t* head_budgets,
                                   void* K_out, void* V_out, int32_t* out_row_offsets,
                                   int32_t* idx_opt, int32_t* counts_opt, int32_t* idx_offsets_opt,
                                   float* s_comp_opt, int32_t* status_dev, void* stream);

/* Host-side layer schedule in the manner of PyramidKV (named in the paper's related work; the
 * paper gives no formula, this is the build's reading): budgets fall linearly with depth and
 * their sum stays n_layers * budget.  With B' = budget - window candidates per head and
 * t = taper_permille / 1000 (0 <= taper_permille <= 999), layer l of n gets
 * floor(B' * (1 + t * (1 - 2 l / (n - 1)))) candidates; the candidates lost to rounding go to
 * the lowest layers, one each; window is added back.  budgets_host [n_layers] (host memory)
 * receives the rows to keep per head of each layer: layer 0 gets the most.  Fill a
 * [n_layers, batch * H] array with them for mixkv_compress_layers_budgeted and pass
 * budgets_host[0] as p->budget.  No device work. */
int mixkv_layer_budget_schedule(int32_t n_layers, int32_t budget, int32_t window,
                                int32_t taper_permille, int32_t* budgets_host);

/* Redundancy analysis: the pairwise cosine similarity of the keys (or values) of a head, which
 * the paper plots as heat maps and summarises per head (Sec. 1, Sec. 3.1, the redundancy
 * figures), at block resolution.
 *   X          device, [heads, L, head_dim] bf16, 16-byte aligned (head_dim must be 128)
 *   block      rows per map cell (>= 1); T = ceil(L / block) cells per side (T <= 65535)
 *   cells      device, [heads, T, T] fp32: mean of cos(x_i, x_j) over i in block I, j in block J,
 *              pairs i == j left out (a diagonal cell averages n (n - 1) pairs, 0 if n == 1)
 *   mean_opt   device, [heads] fp32 or NULL: mean over all ordered pairs i != j of the head,
 *              the redundancy of Eq. 4
 *   workspace  device, mixkv_similarity_workspace_size bytes, 16-byte aligned, caller-owned
 * A zero row has cosine 0 with every row.  The cells come from the Gram matrix of the
 * per-block sums of unit rows (one streaming pass over X, then the upper triangle of tiles on the
 * tensor cores, the sums as two 16-bit parts).  Errors as for the other entry
 * points, but for a bounded wait that expires inside a kernel: there is no status word, the cells it
 * concerns are NaN. */
int mixkv_similarity_workspace_size(int32_t heads, int32_t L, int32_t block, size_t* bytes);
int mixkv_similarity_map(const void* X, int32_t heads, int32_t L, int32_t head_dim, int32_t block,
                         void* workspace, size_t workspace_bytes, float* cells, float* mean_opt,
                         void* stream);

/* The step after compression: one new query token per sequence attends over the compact cache
 * that mixkv_compress_layers wrote (paper Sec. 3.1: decoding continues on the compressed K, V),
 * all layers in one launch.  softmax(q . K^T * scale) V per query head over the rows kept for
 * its KV head, fp32 accumulation.
 *   K_cache, V_cache   device, [n_layers, rows_cap, d] bf16: K_out / V_out of the compression
 *   out_row_offsets    device, [n_layers, batch * H + 1]: rows of (b, h) inside a layer's slice
 *   rows_cap           rows between the slices of consecutive layers (batch * H * B)
 *   q                  device, [n_layers, batch, H * G, d] bf16: the token's query per layer
 *   max_rows           upper bound on the rows of one (layer, b, h), e.g. B, or L for a cache
 *                      that was not compressed; rows beyond it are not read.  It only steers
 *                      how many CTAs share one head (the warps of a cluster of 1 to 8
 *                      CTAs take the rows 16 at a time, each with a running softmax), so any
 *                      length is accepted
 *   out                device, [n_layers, batch, H * G, d] fp32; a head without rows gets zeros
 * softmax_scale 0 means 1 / sqrt(d).  d must be 128, G <= 16 (else MIXKV_ERR_UNSUPPORTED). */
int mixkv_decode_attention(const void* K_cache, const void* V_cache,
                           const int32_t* out_row_offsets, int64_t rows_cap, const void* q,
                           int32_t n_layers, int32_t batch, int32_t kv_heads, int32_t gqa_ratio,
                           int32_t head_dim, float softmax_scale, int32_t max_rows, float* out,
                           void* stream);

/* A paged KV cache held in 4 bits: where decoding puts the rows of new tokens, and what it attends over when nothing,
 * or not everything, is compressed away (no counterpart in the paper, whose caches stop growing at the end of
 * prefill).  A page holds page_rows rows of K and V of ONE KV head, because compression leaves the heads of a sequence with
 * different numbers of rows.
 *
 * Format.  The 128 values of a row are eight blocks of 16.  A value is a 4-bit code (a sign and one of 0, 0.5, 1, 1.5, 2, 3,
 * 4, 6; the sign is the top bit) times the scale of its block (e4m3) times k_scale or v_scale.  A page is a run of
 * tiles of 16 rows, MIXKV_PAGE_TILE_BYTES each, laid out as the matrix fragments of a warp take them; row
 * 4 a + 2 j + b of a tile (a < 4; j, b < 2) has
 *   K codes    at 512 j + 64 (2 a + b): 64 bytes, dimension 2 i in the low half of byte i
 *   V codes    of block g at 1024 + 512 j + 64 g + 16 a + 8 b: 8 bytes, likewise
 *   K scales   of blocks 2 t, 2 t + 1 at 2048 + 16 (2 a + b) + 4 t + 2 j
 *   V scales   of block g at 2176 + 16 g + 4 a + 2 j + b
 * code * scale has at most six significant bits: it is exact in fp16 and bf16. */
enum { MIXKV_TYPE_BF16 = 0, MIXKV_TYPE_FP16 = 1 };
#define MIXKV_PAGE_TILE_BYTES 2304
#define MIXKV_PAGE_MAX_ROWS 256
#define MIXKV_PAGES_MAX 32768      /* columns of a page table that a page selection takes */
#define MIXKV_PAGED_MAX_QUERIES 128  /* q_tokens * gqa_ratio */

typedef struct mixkv_pages {
  void* pool;            /* device, 16-byte aligned: page p at p * mixkv_paged_page_bytes */
  void* bounds_opt;      /* device fp16 [num_pages, 2, 128], 16-byte aligned, or NULL: elementwise minimum and maximum of
                            the K values that a page has had since it began, without k_scale (exact) */
  const int32_t* table;  /* device [batch, kv_heads, max_pages]: page of a head's rows p * page_rows .. */
  const int32_t* rows;   /* device [batch, kv_heads]: rows of every head, those that a call appends included */
  int64_t num_pages;     /* pages in the pool */
  int32_t max_pages;     /* columns of the table */
  int32_t page_rows;     /* a multiple of 16, at most 256 */
  int32_t batch, kv_heads;
  int32_t head_dim;      /* 128 */
  float k_scale, v_scale; /* 1.2e-38 (normal numbers) to 3e38: a third factor of all values, for caches whose blocks are far from
                            the range of e4m3 (largest magnitudes of 0.1 to 2000 need none) */
} mixkv_pages;

/* Bytes of a page.  Host-only. */
int mixkv_paged_page_bytes(int32_t page_rows, size_t* bytes);

/* Appends rows to the cache: the last n rows of every head, where the n new rows of sequence b are tokens
 * offsets[b] .. offsets[b + 1] - 1 of k and v (n = rows after the call minus rows before it: the caller counts them into
 * c->rows first).  K is rotated by the tokens' positions on the way.
 *   k, v            device, type `type`: head h of token i at i * row_stride + h * head_stride elements (both multiples of
 *                   16; 32-byte aligned), num_tokens tokens
 *   offsets_opt     device int32 [batch + 1], ascending; NULL: one token per sequence.  offsets_per_head != 0:
 *                   [batch * kv_heads + 1], every head its own range of rows, head_stride is not used: K_out, V_out and
 *                   out_row_offsets of a compressed layer as they are
 *   max_new         upper bound on n; of more, a head's last max_new are written, and the others reported as those without a
 *                   place are
 *   cos_opt, sin_opt  device fp32 [table_len, rot_dim / 2], 16-byte aligned; both NULL: no rotation.  Dimension i of a
 *                   pair becomes x cos - y sin, its partner y cos + x sin, in fp32; pairs are (i, i + rot_dim / 2), or
 *                   with interleaved != 0 (2 i, 2 i + 1), below rot_dim (at most 128; a multiple of 32,
 *                   interleaved of 16)
 *   positions_opt   device int32 [num_tokens], needed with cos_opt: row of the tables.  It is not the row in the cache: a
 *                   compressed cache has fewer rows than its sequence has tokens
 * Rounding: the scale of a block is e4m3(min(max |x| c, 448)), nearest even, with c the fp32 number nearest to 1 / (6 k_scale) and the
 * product in fp32 (not the quotient, which at ties can have another byte where k_scale is no power of two); a code is the nearest to
 * x / (scale k_scale), ties to the even code, largest magnitude 6 (the sign of a code of zero is not defined); a block of zeros, or one that is too small for e4m3,
 * is zero; one that holds a NaN is NaN.  Every operation is rounded by itself, so codes are the same wherever
 * they are computed.
 * Bounds (if there are any) of a page that begins with a new row are set, those of a page that had rows are widened.  Rows are taken back
 * (a draft's rejected tokens) by counting them out of c->rows; the next append writes over them.  Bounds of a page that keeps rows are
 * not narrowed: they hold for the rows there are, as wide as for those that were taken back too, until the page begins anew (with a NaN
 * among these the page is selected first until then).
 * Pages are written by one call at a time.  A token whose page (table entry outside the pool, row beyond the table or
 * below zero), position or place in k lies outside, and one beyond max_new, gives MIXKV_ERR_INVALID_ARG in *status_dev and is not
 * written. */
int mixkv_paged_append(const mixkv_pages* c, const void* k, const void* v, int32_t type, int64_t num_tokens,
                       int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride,
                       const int32_t* offsets_opt, int32_t offsets_per_head, int32_t max_new, const float* cos_opt,
                       const float* sin_opt, int32_t table_len, int32_t rot_dim, int32_t interleaved,
                       const int32_t* positions_opt, int32_t* status_dev, void* stream);

/* The last n rows of every head back as dense rows: what mixkv_paged_append was given, rounded (and rotated).  offsets_opt,
 * offsets_per_head and max_new as there (n = the number of rows reads the whole head; of more than max_new the last are read).
 *   k_out, v_out    device, type `type`, 32-byte aligned: [num_tokens, kv_heads, 128], or [num_tokens, 128] with
 *                   offsets_per_head; rows that do not exist are not written */
int mixkv_paged_read(const mixkv_pages* c, void* k_out, void* v_out, int32_t type, int64_t num_tokens,
                     const int32_t* offsets_opt, int32_t offsets_per_head, int32_t max_new, void* stream);

/* Pages of every (sequence, KV head) that a query would miss most: a page's score is the largest, over the query rows
 * of the head, of sum_d max(q_d lo_d, q_d hi_d), with lo and hi its bounds: no key of the page has a larger product with q.
 * The 128 terms are summed as neighbouring pairs, seven times over, in fp32 (the products are exact, for queries up to 1e35): the
 * same scores wherever they are computed.  A query row that holds a NaN or an infinity has a score of NaN; a page outside the pool
 * counts as one whose bounds are zero.  The first keep_first and the last keep_last pages go first, then NaN, then by score; ties go
 * to the lower page.
 *   q               device, type `type`: [batch, q_tokens, kv_heads * gqa_ratio, 128], strides in elements of the first
 *                   two dimensions (multiples of 8), 16-byte aligned
 *   max_rows        upper bound on c->rows; rows beyond it do not exist for this call
 *   top             pages to list, at most 2^20
 *   page_list       out, int32 [batch, kv_heads, top]: ascending columns of the page table, -1 behind the last
 *   counts          out, int32 [batch, kv_heads]: min(top, pages of the head)
 * Needs c->bounds_opt; at most MIXKV_PAGES_MAX pages per head (of max_rows), and 4 bytes for every page and 1 KB for every query
 * row (a multiple of eight) within 219 KB, else MIXKV_ERR_UNSUPPORTED. */
int mixkv_paged_select(const mixkv_pages* c, const void* q, int32_t type, int64_t q_batch_stride,
                       int64_t q_token_stride, int32_t q_tokens, int32_t gqa_ratio, int32_t max_rows, int32_t top,
                       int32_t keep_first, int32_t keep_last, int32_t* page_list, int32_t* counts, void* stream);

/* Workspace of mixkv_paged_attention (any max_rows, with or without a list).  Asks the device for its SMs. */
int mixkv_paged_workspace_size(const mixkv_pages* c, int32_t q_tokens, int32_t gqa_ratio, size_t* bytes);

/* softmax(q K^T scale) V over the cache: q_tokens new tokens per sequence, the last of its rows (append theirs first).
 * Token t attends to rows 0 .. rows - q_tokens + t of its KV head; a token that has no row gets zeros.
 *   q               as in mixkv_paged_select; q_tokens * gqa_ratio <= MIXKV_PAGED_MAX_QUERIES
 *   page_list_opt   device int32 [batch, kv_heads, top], counts_opt [batch, kv_heads]: attend to the rows of these
 *                   pages only (ascending, as mixkv_paged_select lists them; counts_opt entries, at most top, are looked at, and
 *                   those that are no page of the head have no rows); NULL, NULL, 0: to all
 *   max_rows        upper bound on c->rows; rows beyond it do not exist for this call.  It steers how the rows of a head are
 *                   split
 *   out             device, type `type`, contiguous [batch, q_tokens, kv_heads * gqa_ratio, 128], 16-byte aligned
 * Logits, softmax statistics and sums are fp32, the weights enter the value sum as fp16.  softmax_scale 0 means
 * 1 / sqrt(128).  A page outside the pool counts as a page without rows.  A query row that holds a NaN or an infinity, or one that
 * sees a NaN, is NaN, and so is what a wait inside the kernel ran out on (there is no status word). */
int mixkv_paged_attention(const mixkv_pages* c, const void* q, int32_t type, int64_t q_batch_stride,
                          int64_t q_token_stride, int32_t q_tokens, int32_t gqa_ratio, float softmax_scale,
                          int32_t max_rows, const int32_t* page_list_opt, const int32_t* counts_opt, int32_t top,
                          void* workspace, size_t workspace_bytes, void* out, void* stream);

/* A paged KV cache held in 8 bits that keeps count of attention: closer to the 16-bit rows than the 4-bit pages above, and with an
 * eviction that keeps what has been attended to most while the model answers (no counterpart in the paper, whose selection ends with
 * prefill).  Pages, table and rows are as in mixkv_pages.
 *
 * Format.  A page is a run of tiles of 16 rows, MIXKV_CACHE8_TILE_BYTES each.  A tile is a block: a value is a code of 8 bits times
 * the block's scale, one for its 16 rows of K and one for those of V.  Row r of a tile has the code of dimension d of K at
 * 128 r + 16 ((d >> 4) ^ (r & 7)) + (d & 15) and of V 2048 bytes behind; the fp32 scale of K is at 4096, that of V at 4100, and eight
 * bytes behind them have no meaning.  Codes are int8 (-127 .. 127: equal steps, finer where no few dimensions are far larger than the
 * others) or e4m3 (a relative error of at most 2^-4 for each value above scale / 64).
 * Rounding: scale = max |x| c with c the fp32 number nearest to 1 / 127 or 1 / 448, product in fp32, zero if below 2^-126; code = the
 * nearest to the fp32 product of x and the rounded reciprocal of the scale, ties to even (int8) or to the even code (e4m3).  A block
 * that gets a NaN or an infinity has a scale of NaN, and so all its values, until it begins anew.  Every operation is rounded by
 * itself: codes are the same wherever they are computed. */
enum { MIXKV_CODE_INT8 = 0, MIXKV_CODE_E4M3 = 1 };
#define MIXKV_CACHE8_TILE_BYTES 4112
#define MIXKV_CACHE8_MAX_QUERIES 128  /* q_tokens * gqa_ratio */

typedef struct mixkv_cache8 {
  void* pool;            /* device, 16-byte aligned: page p at p * mixkv_cache_page_bytes */
  float* mass_opt;       /* device [num_pages, page_rows] or NULL: accumulated attention weight of every row */
  const int32_t* table;  /* device [batch, kv_heads, max_pages]: page of a head's rows p * page_rows .. */
  int32_t* rows;         /* device [batch, kv_heads]: rows of every head, those that a call appends included */
  int64_t num_pages;     /* pages in the pool */
  int32_t max_pages;     /* columns of the table */
  int32_t page_rows;     /* a multiple of 16, at most 256 */
  int32_t batch, kv_heads;
  int32_t head_dim;      /* 128 */
  int32_t code;          /* MIXKV_CODE_* */
} mixkv_cache8;

/* Bytes of a page.  Host-only. */
int mixkv_cache_page_bytes(int32_t page_rows, size_t* bytes);

/* Appends rows to the cache, as mixkv_paged_append does (the caller counts them into c->rows first; K comes as it is to be
 * attended to): tokens offsets[b] .. offsets[b + 1] - 1 of k and v are the last rows of sequence b, or with offsets_per_head of one
 * head.  Strides in elements, multiples of 16; k and v 32-byte aligned.
 * Rows that join a block which has rows: its scale becomes the larger of its own and that of the new rows, and if it grows, the codes of
 * its old rows are rounded again, from fp32(code * old scale).  A block that begins with a new row is set, whatever was there.  The mass
 * of new rows (if there is any) is set to zero; a caller who has scores for them writes these behind the call.
 * Rows are taken back (a draft's rejected tokens) by counting them out of c->rows; the scale of a block that keeps rows stays, and so does
 * what the rows' queries have added to masses.
 * Of more than max_new new rows of a head the last are written.  These others, and tokens whose place (table entry outside the pool, row
 * beyond the table or below zero, token not in k) does not exist, are not written and give MIXKV_ERR_INVALID_ARG in *status_dev.
 * Pages are written by one call at a time. */
int mixkv_cache_append(const mixkv_cache8* c, const void* k, const void* v, int32_t type, int64_t num_tokens,
                        int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride,
                        const int32_t* offsets_opt, int32_t offsets_per_head, int32_t max_new, int32_t* status_dev,
                        void* stream);

/* The last n rows of every head back as dense rows, fp32(code * scale) rounded to `type`; arguments as in mixkv_paged_read. */
int mixkv_cache_read(const mixkv_cache8* c, void* k_out, void* v_out, int32_t type, int64_t num_tokens,
                      const int32_t* offsets_opt, int32_t offsets_per_head, int32_t max_new, void* stream);

/* Workspace of a mixkv_cache_attention call with these arguments, or with a smaller max_rows.  With accumulate it holds the
 * logits of all rows that a call sees: 4 bytes for each of the query rows (an even number) and every row of every head, as if all
 * heads had the most that max_rows, or sinks and window, let them see.  Asks the device for its SMs. */
int mixkv_cache_workspace_size(const mixkv_cache8* c, int32_t q_tokens, int32_t gqa_ratio, int32_t max_rows, int32_t window,
                                int32_t sinks, int32_t accumulate, size_t* bytes);

/* softmax(q K^T scale) V over the cache: q_tokens new tokens per sequence, the last of its rows (append theirs first).  Token t
 * is row p = rows - q_tokens + t of its KV head and attends to rows j <= p; with window > 0 to those of them that have j < sinks or
 * j > p - window: the last `window` rows, itself included, and the first `sinks` (rows are counted in the cache: what was evicted has
 * no place).  A token that has no row gets zeros.
 *   q               device, type `type`: [batch, q_tokens, kv_heads * gqa_ratio, 128], strides in elements of the first
 *                   two dimensions (multiples of 8), 16-byte aligned; q_tokens * gqa_ratio <= MIXKV_CACHE8_MAX_QUERIES
 *   max_rows        upper bound on c->rows; rows beyond it do not exist for this call.  It steers how the rows of a head are
 *                   split
 *   accumulate      nonzero: adds to the mass of every row that a query row sees the weights it got, of all tokens and heads of
 *                   the group (needs c->mass_opt; sums in one order, the same every time).  A page that the table names for several heads
 *                   or sequences (a prompt that they share) gets what each of them gives, one after the other in any order: the last bits
 *                   of its masses may differ from call to call.  A mass below 2^-126 may become zero.  What a call has added
 *                   stays: a draft's tokens that are rejected afterwards leave their weights on the rows they saw (a caller who does
 *                   not want that checks the draft without, counts the rejected rows out and calls again for the tokens that
 *                   stay), and a row that has a mass of NaN keeps it, which an eviction ranks above all others
 *   out             device, type `type`, contiguous [batch, q_tokens, kv_heads * gqa_ratio, 128], 16-byte aligned
 * Logits, softmax statistics and sums are fp32; the weights enter the value sum as fp16 (for fp16 outputs as two such numbers; one below
 * 2^-31 of its query row's largest may be lost there) and the mass as fp32.  softmax_scale 0 means 1 / sqrt(128).  A page outside the
 * pool counts as a page without rows.  A query row that holds a NaN or an infinity, or one that sees a block of NaN, is NaN (and, unless
 * the NaN is among the values, gives NaN to the mass of the rows it sees), and so is what a wait inside the kernel ran out on (there
 * is no status word). */
int mixkv_cache_attention(const mixkv_cache8* c, const void* q, int32_t type, int64_t q_batch_stride,
                           int64_t q_token_stride, int32_t q_tokens, int32_t gqa_ratio, float softmax_scale,
                           int32_t max_rows, int32_t window, int32_t sinks, int32_t accumulate, void* workspace,
                           size_t workspace_bytes, void* out, void* stream);

/* Eviction by accumulated attention weight: of every head the first keep_first rows, the last keep_last and, of the others, those of
 * the largest mass are written to `into`, in their order: min(rows, budget) of them.  A NaN ranks above every number, ties go
 * to the lower row.  c stays as it is (its pages may be shared with other sequences); the pages of `into` must not be among those that
 * c's rows lie on.  Kept rows are read as fp32(code * scale) and written as an append to an empty cache writes them; their mass goes with
 * them (if into->mass_opt is given), and into->rows is set.
 *   into            batch, kv_heads, code as in c; its own table and rows; the pool and the page size may be c's
 *   budget          rows to keep of a head, at least keep_first + keep_last and 1
 *   budgets_opt     device int32 [batch, kv_heads] or NULL: budgets of the heads' own, used as
 *                   min(max(value, keep_first + keep_last), budget)
 *   max_rows        upper bound on c->rows; rows beyond it do not exist for this call
 *   idx             out, device int32 [batch, kv_heads, budget]: rows that were kept, ascending, -1 behind the last
 *   status_dev      device int32, optional: MIXKV_ERR_INVALID_ARG where a kept row has no place in `into` (its table names no page
 *                   of the pool, or is too short); that row is not written
 * Needs c->mass_opt.  A row on a page outside c's pool has a mass below all others and is zeros if it is kept. */
int mixkv_cache_evict(const mixkv_cache8* c, const mixkv_cache8* into, int32_t budget, const int32_t* budgets_opt,
                       int32_t keep_first, int32_t keep_last, int32_t max_rows, int32_t* idx, int32_t* status_dev,
                       void* stream);

/* Number of kernels one mixkv_compress_layer[s] call WITH events enqueues, and the name of the
 * i-th of them (NULL when i is out of range), for the measurement hook.  The route depends on the
 * shape: fixed budgets take three kernels (pass1, pass2, tail; max pooling adds poolsum) while
 * the candidates of the longest sequence fit the tail kernel's shared memory (P_b <= 131072)
 * and add the unfused mix kernel beyond that; adaptive budgets take the unfused route with
 * the budget kernel.  Without events, calls of few heads with adaptive budgets share them out in the
 * tail kernel: mixpool and budget are not launched, the results are the same bit for bit, and the
 * hook cannot time that tail.  The _for variants take the shape and follow the route a call with
 * events takes; the short forms assume the fused route where it exists. */
int mixkv_launches_per_layer(const mixkv_params* p);
const char* mixkv_stage_name(const mixkv_params* p, int32_t i);
int mixkv_launches_for(const mixkv_params* p, int32_t n_layers, int32_t batch,
                       int32_t max_seq_len);
const char* mixkv_stage_name_for(const mixkv_params* p, int32_t n_layers, int32_t batch,
                                 int32_t max_seq_len, int32_t i);

/* Whether the current device can run the library (no counterpart in the paper): MIXKV_OK for
 * compute capability 10.x, MIXKV_ERR_UNSUPPORTED for any other device, MIXKV_ERR_CUDA when no
 * device can be queried.  *cc_major_opt receives the major compute capability (0 when unknown).
 * Every enqueueing entry point performs the same check (cached per device). */
int mixkv_device_check(int32_t* cc_major_opt);

/* Diagnostic (no counterpart in the paper): enqueues a one-CTA kernel that waits, through the
 * same bounded-wait helper as the pass kernels, on a barrier nothing arrives on.  After the
 * wait limit (2 s) the kernel writes MIXKV_ERR_TIMEOUT to *status_dev and, if waited_ns_dev is
 * not NULL, the time it waited; it never traps and the context stays usable.  For tests of the
 * error path. */
int mixkv_selftest_bounded_wait(int32_t* status_dev, unsigned long long* waited_ns_dev,
                                void* stream);

/* Static, human-readable name of a status code. */
const char* mixkv_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* MIXKV_H_ */
