/*
 * tra.h — C ABI of the Token Radius Attention hot path for NVIDIA B200 (sm_100a).
 *
 * One GPU, one stream per call.  The library allocates device memory only inside
 * tra_plan_create (plan-owned tables, freed by tra_plan_destroy); every tensor is
 * owned by the caller.  Unless stated otherwise a pointer is a DEVICE pointer to
 * contiguous memory, 16-byte aligned.  All calls are asynchronous on `stream`
 * (a cudaStream_t passed as void*, NULL = default stream) and return a status
 * code; none of them synchronises the device or throws.
 *
 * The structures carry neither size nor version, and new fields come at their ends: a caller is compiled against the header of the library that it
 * loads, and clears a structure before it fills the fields it knows.
 *
 * Token order.  N = T*H*W video tokens.  Every token-indexed array handed to the
 * four hot calls is in TILE-MAJOR order (Section 3.3, "Flash Radius Mask Kernel":
 * each H x W frame is cut into tile_h x tile_w tiles, edge tiles clipped; tokens
 * are listed frame by frame, tile by tile, row-major inside a tile).  A block is
 * `block` consecutive tile-major positions (Algorithm 1: q = u*b + i, q < N);
 * NB = ceil(N / block).  tra_tile_major_gather / _scatter move tensors between
 * raster order (n = (t*H + y)*W + x) and tile-major order.  A plan created with
 * TRA_ORDER_RASTER takes Q, K, V and O in raster order instead and needs no such pass
 * (TRA_ORDER_RASTER_QO: Q and O only).
 *
 * Joint text-video attention (Section 3.2, last paragraph; Algorithm 1).  With cfg.n_text > 0 a
 * sequence is the N video tokens followed by n_text text tokens, S = N + n_text; S takes the place
 * of N in every shape below and NB = ceil(S / block).  The first B_v = floor(N / block) blocks, made
 * of video tokens only, are the video blocks; a block pair with u >= B_v or v >= B_v is always kept
 * (this includes the block that holds both the last video and the first text tokens, so that every
 * text key stays visible to every query and a text query sees every key), the gather/scatter leaves
 * text tokens where they are, and text positions get budget S, radius +inf and the last candidate
 * index.  Without text the ragged last block is a video block like any other.
 *
 * Shapes.  Q, K, V, O: bf16 [B, heads, N, head_dim].  entropy, budget, radius,
 * ridx: [B, heads, N].  block_mask: uint8 [B, heads, NB, NB].  row_ptr: int32
 * [B*heads*NB + 1]; col_idx: int32 [nnz], key blocks ascending inside a row.
 */
#ifndef TRA_H_
#define TRA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* status codes */
#define TRA_OK 0
#define TRA_ERR_INVALID_ARG (-1) /* NULL / misaligned pointer, non-positive size, bad flag     */
#define TRA_ERR_UNSUPPORTED (-2) /* head_dim, block or grid size outside what the kernels take */
#define TRA_ERR_CAPACITY (-3)    /* col_idx capacity too small (reported by tra_plan_status)   */
#define TRA_ERR_CUDA (-4)        /* a CUDA runtime / driver call failed                        */
#define TRA_ERR_TIMEOUT (-5)     /* a bounded device-side wait expired (reported by tra_plan_status) */
#define TRA_ERR_BOUNDS (-6)      /* debug build (-DTRA_DEBUG) only: a kernel computed an index outside its   */
                                 /* array, or its roles disagree on the work they walked; the access was    */
                                 /* skipped (reported by tra_plan_status)                                    */

/* plan flags */
#define TRA_KEEP_DIAGONAL 1u /* force block_mask[u][u] = 1 (a token always sees itself, Eq. 15) */
#define TRA_ORDER_RASTER 2u  /* Q, K, V and O of the attention calls (and of tra_hot_path_host) are in RASTER   */
                             /* order, n = (t*H + y)*W + x: the kernels fetch every run of 16 tile-major     */
                             /* positions, which is 16 consecutive raster rows, with a TMA box of its own and */
                             /* write O rows where they belong, so no gather / scatter pass is needed         */
                             /* (Section 3.3 reorders explicitly).  entropy, lse, budget, radius, ridx and    */
                             /* the mask stay in tile-major order: they only travel between this library's    */
                             /* calls.  Needs W, tile_w and block to be multiples of 16 (else                  */
                             /* tra_plan_create returns TRA_ERR_UNSUPPORTED).                                 */
#define TRA_ORDER_RASTER_QO 4u /* only Q and O are in raster order; K and V are tile-major (gathered by the     */
                               /* caller).  Q is loaded once per thread block and O rows are stored one by one */
                               /* anyway, so this costs nothing in the launches and saves the gather of Q and  */
                               /* the scatter of O; the many K / V tile loads keep their two large boxes.      */
                               /* Same conditions as TRA_ORDER_RASTER, which takes precedence.                 */

/* entropy-to-budget maps */
#define TRA_BUDGET_UNIFORM 0   /* K = ceil(tau exp(H)): the uniform-support map of Eq. 8 (the paper's choice) */
#define TRA_BUDGET_LOGNORMAL 1 /* K = ceil(N Phibar(sqrt(2 (log N - H)) - Phi^-1(tau))): Appendix,           */
                               /* "Entropy-identified Lognormal mapping"                                    */

/* candidate-radius policies for the set R of Eq. 14 when cfg.radii == NULL */
#define TRA_RADII_EXTENDED 0 /* 0..D (D = ceil(frame diagonal)), then D*exp(gamma*m), m = 1..T-1 */
#define TRA_RADII_LITERAL 1  /* 0..D and +infinity as the full-support radius                    */

typedef struct tra_plan tra_plan_t; /* opaque: grid geometry, thresholds, count table, block boxes */

typedef struct {
  int T, H, W;         /* latent grid (Section 2.1); 1 <= T,H,W <= 1023                          */
  int head_dim;        /* d: 64 or 128                                                          */
  int block;           /* b of Algorithm 1: 16..128 for the budget/radius/mask calls; the        */
                       /* attention calls take 33..128; the token mask inside blocks (ridx)     */
                       /* needs 64 or 128                                                       */
  int tile_h, tile_w;  /* tile shape of the tile-major order (Section 3.3)                       */
  double tau;          /* target attention mass of Eq. 4, in (0, 1]                              */
  double gamma;        /* temporal decay rate of Eq. 10, >= 0                                    */
  const double* radii; /* HOST pointer: optional strictly ascending candidate radii; the last    */
                       /* one must reach full support (may be +inf).  NULL = radius_policy       */
  int n_radii;
  int radius_policy;   /* TRA_RADII_* (used when radii == NULL)                                  */
  unsigned flags;      /* TRA_KEEP_DIAGONAL | TRA_ORDER_RASTER | TRA_ORDER_RASTER_QO             */
  int budget_map;      /* TRA_BUDGET_* used by tra_budget_radius                                 */
  int n_text;          /* text tokens that follow the video tokens in every sequence (>= 0)     */
} tra_config_t;

/* ---- plan ---------------------------------------------------------------------------- */

/* Builds the plan for one grid / gamma / candidate set on the current device: tile-major
 * coordinates, the squared-distance thresholds floor(r^2 exp(-2 gamma delta)) of Eq. 15, the
 * boundary-aware count table C_grid of Eq. 13 for every (token coordinate, candidate) — the
 * lookup table of Section 3.2 — and per-block bounding boxes (Section 3.3).  Work is enqueued
 * on `stream`; the call returns after the tables are built (it synchronises that stream).
 * *out is owned by the caller and released with tra_plan_destroy. */
int tra_plan_create(tra_plan_t** out, const tra_config_t* cfg, void* stream);
int tra_plan_destroy(tra_plan_t* plan);

/* Geometry queries (host). */
int tra_plan_num_tokens(const tra_plan_t* plan);   /* S = N + n_text: tokens per sequence */
int tra_plan_num_video_tokens(const tra_plan_t* plan); /* N = T*H*W */
int tra_plan_num_blocks(const tra_plan_t* plan);   /* NB */
int tra_plan_num_radii(const tra_plan_t* plan);    /* |R| */
int tra_plan_num_tile_pairs(const tra_plan_t* plan); /* entries per (batch, head) of the tile-pair table of
                                                        tra_build_block_mask: ceil(NT / 2); 0 for blocks <= 32 */
/* Copies plan tables to HOST buffers (synchronises): radii[|R|] (double), theta[|R|*T]
 * (int32, theta[k*T + delta]), coord[N*3] (int32 t,y,x per tile-major position).  Any may be NULL. */
int tra_plan_tables(const tra_plan_t* plan, double* radii, int32_t* theta, int32_t* coord);
/* Copies the count table to a HOST buffer uint32 [T*H*W*|R|], indexed ((t*H+y)*W+x)*|R| + k. */
int tra_plan_count_table(const tra_plan_t* plan, uint32_t* counts);

/* Reads and clears the plan's device status word (synchronises `stream`): TRA_OK, or the
 * first TRA_ERR_CAPACITY / TRA_ERR_TIMEOUT / TRA_ERR_BOUNDS a kernel of this plan recorded since the
 * last call. */
int tra_plan_status(tra_plan_t* plan, void* stream);

const char* tra_status_string(int status);

/* Self-test of the device-side error path (the paper has no counterpart): launches one warp that
 * waits, with the same bounded wait the attention kernels use, on a barrier nothing arrives on.
 * After limit_ms (1..1000) the wait gives up and records TRA_ERR_TIMEOUT in the plan status; the
 * kernel then returns normally and the context stays usable.  Asynchronous on `stream`. */
int tra_selftest_wait_timeout(tra_plan_t* plan, int limit_ms, void* stream);

/* ---- layout (Section 3.3: Q, K, V are reordered before attention, O restored after) -- */

/* dst[bh, p, :] = src[bh, raster(p), :] for every tile-major position p.  row_bytes = bytes of
 * one token row (multiple of 16); n_bh = B*heads.  src and dst must not overlap. */
int tra_tile_major_gather(const tra_plan_t* plan, const void* src_raster, void* dst_tile_major,
                          int n_bh, int row_bytes, void* stream);
/* dst[bh, raster(p), :] = src[bh, p, :] — the inverse. */
int tra_tile_major_scatter(const tra_plan_t* plan, const void* src_tile_major, void* dst_raster,
                           int n_bh, int row_bytes, void* stream);

/* ---- the four hot calls ------------------------------------------------------------- */

/* Dense attention of Eq. 1 fused with the attention entropy of Eq. 2, accumulated from the
 * online-softmax state as in Algorithm 2 (H = m + log l - a/l, nats).
 *   Q, K, V : bf16 [B, heads, N, head_dim], 128-byte aligned.
 *   O       : bf16, same shape (written).
 *   entropy : fp32 [B, heads, N] or NULL (NULL = plain dense attention, no entropy work).
 *   lse     : fp32 [B, heads, N] or NULL; log sum_j exp(s_ij), exact to fp32 rounding (the row sum
 *             of the unrounded probabilities is kept next to the bf16-rounded one that normalises O).
 *   sm_scale: multiplies q.k; pass 1/sqrt(head_dim) for Eq. 1. */
int tra_entropy_attn(const tra_plan_t* plan, const void* Q, const void* K, const void* V, void* O,
                     float* entropy, float* lse, int B, int heads, float sm_scale, void* stream);

/* Entropy -> token budget -> radius (Eq. 8 and Eq. 14; Appendix "Entropy-to-budget-to-radius
 * lookup"): budget = clamp(ceil(tau * exp(entropy)), 1, N) evaluated in fp64 (or the lognormal
 * map of the appendix when the plan was created with TRA_BUDGET_LOGNORMAL); ridx = index of
 * the smallest candidate radius whose C_grid at the token's coordinate reaches the budget;
 * radius = that candidate as fp32 (+inf for an infinite full-support radius).
 *   entropy: fp32 [B, heads, N];  budget: int32 or NULL;  radius: fp32 or NULL;  ridx: uint16. */
int tra_budget_radius(const tra_plan_t* plan, const float* entropy, int32_t* budget, float* radius,
                      uint16_t* ridx, int B, int heads, void* stream);

/* Algorithm 1: block mask from per-query radii.  For every (head, query block u, key block v):
 * c_j = number of valid queries of u whose disk (Eq. 15) holds key column j; keep the pair iff
 * some c_j > 0 and 10*#{c_j > b/3} > 6*#{c_j > 0}.  Block bounding boxes only skip pairs whose
 * vote is already decided; the result equals the unpruned vote bit for bit.
 *   ridx      : uint16 [B, heads, N] from tra_budget_radius.
 *   block_mask: uint8 [B, heads, NB, NB] (written, 0/1).
 *   row_ptr   : int32 [B*heads*NB + 1] (written); col_idx: int32 [col_idx_capacity] (written,
 *               ascending inside a row).  If nnz exceeds the capacity, TRA_ERR_CAPACITY is recorded
 *               in the plan status, col_idx holds the first `capacity` entries and every row_ptr
 *               offset is clamped to the capacity, so that a later tra_sparse_attn stays inside
 *               col_idx (its result is then incomplete; read the status).
 *   nnz_out   : device int64 or NULL; total retained blocks.
 *   tile_pairs: int32 [B*heads, ceil(NT/2), 2] or NULL, NT = ceil(NB / G) query tiles, G = 2 blocks
 *               per tile for blocks of up to 64 tokens, else 1 (written).  The paper has
 *               no counterpart: tra_sparse_attn gives each thread block two query tiles (128 rows of
 *               tensor-core work each, of which the first G * block hold queries) that
 *               share the key/value tiles they both retain, and this table pairs tiles whose block
 *               lists are similar (entry -1 = no second tile).  Pass it to tra_sparse_attn together
 *               with row_ptr / col_idx; it changes the speed of that call, never its result.
 *               Blocks of 32 tokens or fewer have no attention launch and no query tiles:
 *               with such a plan a non-NULL tile_pairs returns TRA_ERR_UNSUPPORTED (nothing is run).
 *               The pairing kernel runs beside the list kernels on a stream the plan owns, forked from and
 *               joined to `stream` by two plan-owned events (this also works inside a stream capture):
 *               everything the call writes is complete for later work on `stream`, but calls with
 *               tile_pairs on ONE plan must not be issued from several host threads at once. */
int tra_build_block_mask(const tra_plan_t* plan, const uint16_t* ridx, uint8_t* block_mask,
                         int32_t* row_ptr, int32_t* col_idx, int64_t col_idx_capacity,
                         int64_t* nnz_out, int32_t* tile_pairs, int B, int heads, void* stream);

/* The active-block list for callers that cannot allocate (the paper has no counterpart: this is
 * about how the library is embedded, not about the method).  Some users of this library may not
 * call cudaMalloc, or any allocator, at the point where the mask is rebuilt: code that runs as a
 * plugin inside another framework's memory pool, a server that hands out all device memory at
 * start-up, a latency-critical thread that must stay out of the allocator's lock.  Such a caller
 * needs row_ptr / col_idx / tile_pairs for tra_sparse_attn and has no use for the Boolean mask, which
 * is then scratch; this call keeps that scratch in a fixed array of TRA_STATIC_BLOCK_MASK_BYTES
 * (16 MiB) inside the library's device image.  Every GPU on which the library is loaded holds those
 * 16 MiB until the process exits.
 *   Arguments and results as tra_build_block_mask without `block_mask`: the same row_ptr, col_idx,
 *   nnz_out and tile_pairs, bit for bit; the same recorded errors.
 *   Limit: B * heads * NB * NB <= TRA_STATIC_BLOCK_MASK_BYTES, else TRA_ERR_CAPACITY is returned and
 *   nothing runs (the 75.6K-token, 40-head shape with 128-token blocks needs 13.97 MB).
 *   The call itself allocates nothing: no cudaMalloc / cudaFree and no allocating library routine.
 *   The first call on a device looks up the array's device address (once per device, with that device
 *   current); make that first call before starting any stream capture.
 *   All calls on a device share the one array, which keeps the last call's mask: two calls whose
 *   kernels can overlap on the GPU (different streams without an ordering between them) race; order
 *   them.  Nothing needs clearing between calls: a call writes every mask entry it later reads.
 * Errors: TRA_ERR_INVALID_ARG (NULL pointer, non-positive count, a current device other than the
 * plan's), TRA_ERR_CAPACITY (mask larger than the array, see above; or, recorded in the plan status,
 * col_idx too small), TRA_ERR_UNSUPPORTED / TRA_ERR_CUDA as for tra_build_block_mask. */
#define TRA_STATIC_BLOCK_MASK_BYTES (16u << 20)
int tra_build_block_list_static(const tra_plan_t* plan, const uint16_t* ridx, int32_t* row_ptr,
                                int32_t* col_idx, int64_t col_idx_capacity, int64_t* nnz_out,
                                int32_t* tile_pairs, int B, int heads, void* stream);

/* Block-sparse attention (Eq. 16 as executed: Section 3.2, last paragraph, and "Limitations"):
 * softmax attention of each query over the valid keys of the retained key blocks of its block row.
 *   ridx == NULL: retained blocks are evaluated in full, no token mask inside them (what the
 *                 paper's block-sparse execution does);
 *   ridx != NULL: uint16 [B, heads, N] from tra_budget_radius; inside the retained blocks a video
 *                 query additionally sees only the video keys inside its disk (the token mask of
 *                 Eq. 15 on top of the block list); text keys and text queries are not masked.
 *   row_ptr == NULL and col_idx == NULL (only with ridx != NULL): Eq. 16 itself, no block list — a
 *                 video query sees exactly the video keys inside its disk, text keys and text
 *                 queries are not masked.  The kernel finds the key blocks a query block can reach
 *                 from the plan's block boxes; no [heads, NB, NB] mask is needed.
 * A query that is left with no visible key gets O = 0 and lse = -inf.
 *   row_ptr, col_idx: the CSR list written by tra_build_block_mask (reusable across calls:
 *   Section 3.3, warm-up reuse).  tile_pairs: the table the same call wrote, or NULL (consecutive
 *   tiles share a thread block); any table in which every tile 0 .. NT-1 of a (batch, head) appears
 *   exactly once gives the same result.  Q, K, V, O as in tra_entropy_attn.  lse: fp32 or NULL, exact
 *   to fp32 rounding. */
int tra_sparse_attn(const tra_plan_t* plan, const void* Q, const void* K, const void* V,
                    const int32_t* row_ptr, const int32_t* col_idx, const uint16_t* ridx,
                    const int32_t* tile_pairs, void* O, float* lse, int B, int heads, float sm_scale,
                    void* stream);

/* ---- the whole pass over HOST tensors (the paper has no counterpart: plumbing around the calls
 * above for callers whose Q, K, V and O live in host memory) ----------------------------- */

/* One pass of the hot path — tile-major layout, dense attention + entropy, budget / radius, block
 * mask, block-sparse attention (retained blocks in full), layout back — over
 *   Q_host, K_host, V_host : HOST pointers, bf16 [heads, S, head_dim], RASTER token order (read),
 *   O_host                 : HOST pointer, same shape and order (written): the block-sparse output.
 * Heads are independent problems, so the pass runs in groups of at most `group` heads (the first
 * group holds `first_group` <= group heads, so that the kernels start early, the following ones
 * twice as many as the one before until `group` is reached, and the last group is split so that
 * little output is left to copy after the last kernel); the host-to-device copy of
 * the next group and the device-to-host copy of the previous one run on two copy streams owned by
 * the plan while the kernels of the current group run on `stream`.  Pinned (page-locked) host
 * memory is needed for the copies to overlap; pageable memory works but serialises.
 *   workspace : DEVICE memory, 256-byte aligned, at least tra_hot_path_host_workspace_bytes(plan,
 *               group) bytes; owned by the caller, free to reuse once `stream` has passed the call.
 * The call allocates no device memory (on its first uses it creates the plan's two copy streams and
 * a pool of events, which later calls reuse).  The current device must be the one the plan was
 * created on.  It returns after enqueueing; `stream` completes after the last copy in
 * either direction, so synchronising `stream` (or an event recorded on it) makes O_host valid.
 * Calls that share a plan or a workspace must be ordered on `stream`.
 * Errors: TRA_ERR_INVALID_ARG (NULL / misaligned pointer, non-positive count or scale, another
 * current device), TRA_ERR_CAPACITY (workspace too small), TRA_ERR_CUDA; kernel-side errors as for
 * the four calls.  After a non-OK return part of the pass may already be enqueued, with the copy
 * streams and `stream` waiting on one another: synchronise `stream` before the workspace or the
 * host buffers are reused. */
size_t tra_hot_path_host_workspace_bytes(const tra_plan_t* plan, int group);
int tra_hot_path_host(tra_plan_t* plan, const void* Q_host, const void* K_host, const void* V_host,
                      void* O_host, void* workspace, size_t workspace_bytes, int heads, int group,
                      int first_group, float sm_scale, void* stream);

/* ---- head norm, rotary positions and token order, before the attention and back (the paper starts from the
 * Q, K and V its models hand to the attention; this is the step that makes them) ------------ */

/* One call turns the projections' Q, K and V into what the attention calls take, and one call takes the
 * gradients back.  A row is one (token, head), d = head_dim channels x.
 *   norm    : n = x (TRA_NORM_NONE), x r (TRA_NORM_RMS) or (x - mean) r (TRA_NORM_LAYER) with
 *             r = (mean square [of x, or of x - mean] + eps)^-1/2 over the d channels; z = weight n + bias,
 *             weight and bias [d], shared by all heads, of the tensors' type (NULL = 1 and 0; bias with
 *             TRA_NORM_LAYER only).
 *   rotary  : d / 2 channel pairs, pair p = channels (2p, 2p + 1), or (p, p + d/2) with `halves`; pair p belongs to
 *             axis axis[p] and turns by the angle pos[axis[p]] * inv_freq[p]:
 *             (z1, z2) -> (z1 cos - z2 sin, z1 sin + z2 cos).  inv_freq[p] = 0 leaves a pair as it is.
 *             Angles are reduced by whole turns before they are rounded: off by 2^-23 at most for every int32 position.
 *   order   : see TRA_ROTARY_TILE_MAJOR.
 * All arithmetic is fp32 and rounded once, to the tensors' type. */
#define TRA_ROTARY_MAX_HEAD_DIM 256

/* types of the tensors of the rotary and packed-attention calls */
#define TRA_BF16 0
#define TRA_FP16 1
#define TRA_FP32 2

#define TRA_NORM_NONE 0
#define TRA_NORM_RMS 1
#define TRA_NORM_LAYER 2

typedef struct tra_rotary tra_rotary_t; /* opaque, host memory only: frequencies, axes, norm */

typedef struct {
  int head_dim;           /* d: a multiple of 16, 16 .. 256                               */
  int n_axes;             /* 1 .. 4                                                       */
  const int* axis;        /* HOST [d / 2]: 0 .. n_axes - 1                                */
  const double* inv_freq; /* HOST [d / 2]: radians per position, finite, below 2^64 in magnitude */
  int halves;             /* how channels pair: 0 = (2p, 2p + 1), 1 = (p, p + d/2)        */
  int norm;               /* TRA_NORM_*                                                   */
  double eps;             /* of the norm, >= 0                                            */
} tra_rotary_config_t;

#define TRA_ROTARY_ROTATE 1u     /* norm and rotate (Q, K); without it the rows are only moved (V)              */
#define TRA_ROTARY_TILE_MAJOR 2u /* the attention side (dst of the forward call, src of the backward call) is in */
                                 /* the plan's tile-major order; the other side is in raster order               */

typedef struct {           /* one tensor of a call: [B, tokens, heads, d] behind strides, channels contiguous */
  const void* src;         /* forward: x.  backward: the gradient of the forward's dst              */
  void* dst;               /* forward: y.  backward: the gradient of the forward's src              */
  const void* x;           /* backward with a norm: the forward's src (NULL otherwise)              */
  const void* weight;      /* [d] or NULL                                                          */
  const void* bias;        /* [d] or NULL (read by the forward call only)                          */
  float* weight_grad;      /* backward with a norm: fp32 [d] (written) or NULL                     */
  float* bias_grad;        /* backward with TRA_NORM_LAYER: fp32 [d] (written) or NULL             */
  int64_t src_stride[3];   /* batch, token, head, in elements; multiples of 16 bytes               */
  int64_t dst_stride[3];
  int64_t x_stride[3];
  int heads;
  unsigned flags;          /* TRA_ROTARY_ROTATE | TRA_ROTARY_TILE_MAJOR                            */
} tra_rotary_tensor_t;

int tra_rotary_create(tra_rotary_t** out, const tra_rotary_config_t* cfg);
int tra_rotary_destroy(tra_rotary_t* rot);

/* Up to three tensors (HOST array), one launch.
 *   plan : NULL, or the grid: tokens must then be its S (video tokens in raster order, then text).  Needed for
 *          TRA_ROTARY_TILE_MAJOR and for positions from the grid.  Its device must be the current one.
 *   pos  : int32 [tokens, n_axes], the position of every token in the order of the projection side, shared by the
 *          batch entries; or NULL: video token (t*H + y)*W + x of the plan has position (t, y, x) (n_axes = 3) and
 *          text tokens are normed and not turned.
 * Pointers 16-byte aligned.  B and tokens are at least 1.  src (and x) and dst must not overlap, except that a tensor
 * that is not TILE_MAJOR may be worked on in place (dst = src with the same strides).
 * Errors: TRA_ERR_INVALID_ARG, TRA_ERR_UNSUPPORTED, TRA_ERR_CUDA. */
int tra_rotary_forward(const tra_rotary_t* rot, const tra_plan_t* plan, const int32_t* pos,
                       const tra_rotary_tensor_t* tensors, int n_tensors, int B, int tokens, int dtype,
                       void* stream);

/* The gradients.  weight_grad = sum over rows of u n, bias_grad = sum of u, u = the gradient turned back: summed in
 * fp32 in a fixed order (the same bits every time) through `workspace`, device memory of at least
 * tra_rotary_backward_workspace_bytes, 16-byte aligned, owned by the caller and free to reuse once `stream` has passed the call
 * (NULL when no weight_grad or bias_grad is asked for; TRA_ERR_CAPACITY when it is too small). */
size_t tra_rotary_backward_workspace_bytes(const tra_rotary_t* rot);
int tra_rotary_backward(const tra_rotary_t* rot, const tra_plan_t* plan, const int32_t* pos,
                        const tra_rotary_tensor_t* tensors, int n_tensors, int B, int tokens, int dtype,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---- attention over packed sequences (the paper's layer attends inside one clip; this is attention for the
 * sequences around it: prompts and clips of different lengths in one batch, chunks behind a cache, one new token) ---- */

/* Tokens of all sequences lie one after the other: Q, O [total_q, heads, d], K, V [total_k, kv_heads, d], bf16 or fp16, channels
 * contiguous, tokens and heads behind strides.  Query heads g * group .. g * group + group - 1 share key/value head g,
 * group = heads / kv_heads.  Sequence s has the queries cu_q[s] .. cu_q[s + 1] - 1 and the keys k_begin[s] .. k_end[s] - 1
 * (device int32; ranges of keys may leave gaps and may be shared).  With `causal`, query i of a sequence sees its keys
 * 0 .. i + (number of keys - number of queries): the last query sees every key.
 *   O = softmax(sm_scale Q K^T) V,  lse = log sum exp of the scores a query sees, fp32 [total_q, heads].
 * A query that sees no key, or only scores of -inf, gets O = 0 and lse = -inf.  Rows of O and lse in front of cu_q[0]
 * and behind cu_q[n_seq] are left as they were.  What lies in K and V outside a sequence's range, or in Q outside of all, is never used and may be
 * anything, NaN too.  (Inside a sequence a NaN among the scores that a query sees makes its O and lse NaN; a hidden key's weight is
 * 0, but 0 * NaN is NaN: a value that is not finite can reach queries that do not see its key.)
 * What a call writes overlaps neither what it reads nor its other results. */
typedef struct tra_packed tra_packed_t; /* opaque: head layout, type, order, a device status word */

typedef struct {
  int heads, kv_heads; /* heads a multiple of kv_heads, group <= 128 */
  int head_dim;        /* 64 or 128                                  */
  int dtype;           /* TRA_BF16 or TRA_FP16                       */
  int causal;
  int window;          /* 0: none.  Else (with causal) a query sees the last `window` keys up to its own position and the   */
  int sinks;           /* first `sinks` keys of its sequence (0: none): at position p = i + keys - queries, key j with      */
                       /* j <= p and (j > p - window or j < sinks).  What lies behind the first tokens and in front of    */
                       /* every window costs nothing                                                                     */
} tra_packed_config_t;

typedef struct {
  const void *q, *k, *v;  /* 16-byte aligned                                                     */
  void* o;                /* forward: written; backward: read                                     */
  float* lse;             /* forward: written, or NULL; backward: read                            */
  int64_t q_stride[2], k_stride[2], v_stride[2], o_stride[2]; /* token, head: elements, multiples of 8 */
  const int32_t *cu_q;    /* device [n_seq + 1], ascending                                        */
  const int32_t *k_begin, *k_end; /* device [n_seq]; packed keys: cu_k and cu_k + 1               */
  int n_seq, total_q, total_k;
  int max_q, max_k;       /* upper bounds of the sequences' queries and keys, at most total_q and total_k */
  float sm_scale;
  void* o_rest;           /* what rounding took from o, in o's type, [total_q, heads, d] contiguous, 16-byte aligned,   */
                          /* or NULL.  Forward, with lse only: written.  Backward: read; the sums of dO O are then those */
                          /* of the unrounded o, without which the gradients of a short or peaked row are mostly the     */
                          /* rounding of o                                                                             */
} tra_packed_args_t;

/* Creates the handle on the current device (allocates its status word). */
int tra_packed_create(tra_packed_t** out, const tra_packed_config_t* cfg);
int tra_packed_destroy(tra_packed_t* packed);
/* Reads and clears the handle's device status word (synchronises `stream`): TRA_OK, TRA_ERR_TIMEOUT, or
 * TRA_ERR_INVALID_ARG: a range on the device lay outside its tensor, ran backwards or was longer than the stated maximum; it was
 * cut to fit and the results of that call are incomplete. */
int tra_packed_status(tra_packed_t* packed, void* stream);

/* Forward.  The launch follows from the sizes alone: sequences of at most 16 rows (max_q * group) go to a kernel for few
 * rows over many keys, others to 128-row tensor-core tiles; either splits the keys over thread blocks when there
 * are too few rows to fill the GPU.  Many parts are joined by a second launch and lie in `workspace`: device memory of
 * tra_packed_attn_workspace_bytes (0: none needed, pass NULL), 16-byte aligned, owned by the caller and free to reuse once
 * `stream` has passed the call.  The current device must be the handle's.
 * Errors: TRA_ERR_INVALID_ARG, TRA_ERR_UNSUPPORTED, TRA_ERR_CAPACITY (workspace too small), TRA_ERR_CUDA. */
size_t tra_packed_attn_workspace_bytes(const tra_packed_t* packed, int n_seq, int total_q, int max_q, int max_k);
int tra_packed_attn(const tra_packed_t* packed, const tra_packed_args_t* args, void* workspace, size_t workspace_bytes,
                    void* stream);

/* Gradients of a forward call over PACKED keys (args->k_end must be args->k_begin + 1: ascending bounds, so that no key
 * belongs to two sequences).  args as in the forward call, with its o and lse.  dq, dk, dv are written for the rows of the
 * sequences (zeros where nothing is seen) and left alone elsewhere; sums of gradients that heads share are formed in fp32
 * inside one thread block: the same bits every time.  d_o outside the sequences may be anything.
 * fp16: the probabilities and their gradients are rounded for their products as multiples by powers of two that follow the
 * largest rows of d_o and v of a key/value head, so that the relative precision does not depend on the size of d_o.
 * The launch follows from max_q, max_k and total_q, not from the lengths, and with a window so does how dS is rounded for its products: dq is 1.1 to 1.3 times as
 * far off as its own rounding, but 1.5 times at head_dim 128 where max_k is above 1,024 and the window hides nothing of that many keys; dk
 * is 1.05 times where the window or max_q spans at most three tiles of 128 rows, else 1.4 to 1.6 over a few dozen keys.  Loose bounds cost that much, and time.
 *   workspace: device memory of tra_packed_attn_backward_workspace_bytes, as for the forward call. */
typedef struct {
  const void* d_o;        /* the gradient of o */
  void *dq, *dk, *dv;     /* written           */
  int64_t do_stride[2], dq_stride[2], dk_stride[2], dv_stride[2];
} tra_packed_grads_t;

size_t tra_packed_attn_backward_workspace_bytes(const tra_packed_t* packed, int total_q);
int tra_packed_attn_backward(const tra_packed_t* packed, const tra_packed_args_t* args, const tra_packed_grads_t* grads,
                             void* workspace, size_t workspace_bytes, void* stream);

/* ---- a cache of 4 bits: keys and values quantised as they are written, read back, and attended over (long streams whose
 * cache would not fit, or whose reading bounds every new token) ---- */

/* Heads, head_dim and type are those of a tra_packed_t.  A row (one token of one key/value head) is held in groups of 32 channels:
 *   low = the group's smallest element, step = the smallest number of the type with 15 step >= largest - low,
 *   code = floor((x - low) / step + 1/2) in 0 .. 15; it stands for low + code step, so that it is off by step / 2 at most.
 * Differences and quotients are fp32's, and a quotient less than 2^-22 of itself below a half may go up: step / 2 (1 + 2^-16) at most.  A group that holds a NaN or an infinity reads back as NaN.  Where the codes lie inside a row is the library's affair: rows are
 * written and read by these calls.  A row takes d / 2 + d / 8 bytes, for keys and for values each. */
typedef struct {
  void *k, *v;             /* [kv_heads, tokens, d / 2] bytes, 16-byte aligned                                          */
  void *k_step, *v_step;   /* [kv_heads, tokens, 2, d / 32] of the type: steps, then lowest values; 16-byte aligned     */
  int tokens;              /* rows of every head: even, at most 2^30                                                   */
} tra_cache4_t;

/* Token i of k and v ([n, kv_heads, d] behind strides (token, head), elements, multiples of 8; 16-byte aligned) goes to row slots[i] of the
 * cache (device int32 [n]); a negative slot is left out, one past the cache is left out and reported (tra_packed_status:
 * TRA_ERR_INVALID_ARG).  The slots of one call are distinct; what a slot that is named twice holds afterwards is not specified.
 * Errors: TRA_ERR_INVALID_ARG, TRA_ERR_UNSUPPORTED, TRA_ERR_CUDA. */
int tra_cache4_write(const tra_packed_t* packed, const tra_cache4_t* cache, const void* k, const void* v, const int64_t* k_stride,
                     const int64_t* v_stride, const int32_t* slots, int n, void* stream);

/* The way back: rows slots[i] of the cache, rounded once to the type (to its largest number where low + 15 step passes that), to token i of k
 * and v.  Tokens of slots that are left out stay as they are.  A slot may be named several times. */
int tra_cache4_read(const tra_packed_t* packed, const tra_cache4_t* cache, void* k, void* v, const int64_t* k_stride, const int64_t* v_stride,
                    const int32_t* slots, int n, void* stream);

/* Attention over the cache: tra_packed_attn with the values that the codes stand for as keys and values (not rounded to the type; where a
 * sequence has more than 64 rows per key/value head, they are read back, rounded, into the workspace first, half a gigabyte or one sequence
 * at a time).  k_begin, k_end: rows of the cache.  args->k, v and their strides are not used, total_k is the cache's tokens; o_rest must be
 * NULL (there are no gradients with respect to a cache).  What lies in rows outside the sequences' ranges may be anything.  Products are fp16's,
 * of multiples that follow a head's largest value and a row's largest query element: bf16 values 2^-26 and query elements 2^-24 of the largest, hidden keys
 * included, begin to lose bits.  Workspace, status and errors as for tra_packed_attn; the workspace query is 0 for sizes that the call refuses. */
size_t tra_packed_attn_cache4_workspace_bytes(const tra_packed_t* packed, int n_seq, int total_q, int max_q, int max_k);
int tra_packed_attn_cache4(const tra_packed_t* packed, const tra_packed_args_t* args, const tra_cache4_t* cache, void* workspace,
                           size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TRA_H_ */
