/*
 * memfine.h - C ABI of the MI355X (gfx950) chunked MoE expert layer.
 *
 * The layer is the per-GPU hot path of MemFine (memory-aware fine-grained
 * scheduling for MoE training): on one GPU's share of expert-parallel work it
 * runs dispatch (group the received token-slots by local expert), the expert
 * SwiGLU FFN on every expert's rows, and the gate-weighted combine, over C
 * contiguous token chunks (paper Section 4.1, Eq. (6)); the backward
 * recomputes each chunk before back-propagating it (Eq. (7)).  C comes from
 * the paper's activation-memory model (Section 4.2, Eq. (8), Eq. (9), bins).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Pointers named d_* are device pointers, h_* host pointers.  Every buffer
 *   is owned by the caller; the library keeps no state between calls except a
 *   lazily created per-process profiling table; the launch options of
 *   memfine_set_launch_options (one process-wide setting); for calls made
 *   with a NULL allocator, one workspace block per (device, stream), carved
 *   into each chunk's buffers and reused by the next chunk in stream order
 *   (grown from a per-device stream-ordered pool when a call needs more,
 *   kept until memfine_workspace_trim or the end of the process: see
 *   memfine_workspace_held), and, for such calls made while their stream is
 *   being captured into a graph, blocks that belong to that capture alone and
 *   stay until the process ends (a caller that captures often passes an
 *   allocator whose memory lives as long as its graphs); one pinned host buffer of 1025 ints per device
 *   for memfine_count; and, only when the side-stream launch option is on,
 *   two side streams and three events per device (kept until the process
 *   ends).
 * - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *   Device work is enqueued asynchronously on it; only memfine_count and
 *   memfine_profile_end synchronise (with the stream / the recorded events).
 * - Return value: MEMFINE_OK (0) or a negative status.  Argument errors are
 *   detected on the host and returned before anything is enqueued.  A HIP
 *   failure returns MEMFINE_ERR_HIP; an allocator that returns NULL gives
 *   MEMFINE_ERR_OOM.  After a failed call the outputs are unspecified, and
 *   every internal allocation has been handed back.
 * - Shapes (memfine_shape): T received tokens, h hidden size, F expert FFN
 *   size (g_e in the paper), E local experts, k slots per token (top-k).
 *   Requirements: T >= 0, T*k < 2^31, h % 64 == 0, F % 64 == 0, h, F >= 64,
 *   1 <= k, 1 <= E <= 1024.
 * - Layouts, all row-major and contiguous:
 *     idx    int32 [T, k]       expert of each slot, 0 <= idx < E
 *     gates  float [T, k]       score of each slot (need not sum to 1)
 *     X, Y, dY, dX   dtype [T, h]
 *     W1     dtype [E, 2F, h]   rows 0..F-1: SiLU gate, rows F..2F-1: up
 *     W2     dtype [E, h, F]
 *     dW1, dW2  float, shaped like W1, W2;   dgates float [T, k]
 *   dtype is bf16 (MEMFINE_BF16, raw 16-bit storage) or float (MEMFINE_F32).
 *   Per slot (token t, slot j, expert e = idx[t,j], g = gates[t,j]):
 *     u = W1[e] X[t];  a = silu(u[0:F]) * u[F:2F];  Y[t] += g * (W2[e] a).
 *   Arithmetic: fp32 accumulation everywhere; on the bf16 path the per-chunk
 *   intermediates are stored as bf16.
 */
#ifndef MEMFINE_H
#define MEMFINE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* status codes */
#define MEMFINE_OK                0
#define MEMFINE_ERR_INVALID_ARG  (-1)
#define MEMFINE_ERR_UNSUPPORTED  (-2)
#define MEMFINE_ERR_BUDGET       (-3)
#define MEMFINE_ERR_OOM          (-4)
#define MEMFINE_ERR_HIP          (-5)
#define MEMFINE_ERR_SCRATCH      (-6)

/* element types */
#define MEMFINE_BF16  0
#define MEMFINE_F32   1

/* passes for memfine_workspace_bytes */
#define MEMFINE_PASS_FWD  0
#define MEMFINE_PASS_BWD  1

typedef struct memfine_shape {
  int64_t T;      /* received tokens (rows of X)                       */
  int32_t h;      /* hidden size                                        */
  int32_t F;      /* expert FFN size (SwiGLU width; FC1 has 2F rows)    */
  int32_t E;      /* local experts                                      */
  int32_t k;      /* slots per token (top-k)                            */
  int32_t dtype;  /* MEMFINE_BF16 or MEMFINE_F32                        */
} memfine_shape;

/*
 * Optional device-memory provider for the per-chunk working buffers.
 * alloc(bytes, stream, ctx) returns a device pointer (256-byte aligned) that
 * is usable in stream order on `stream`, or NULL on failure; release(ptr,
 * bytes, stream, ctx) gives it back in stream order.  When the allocator
 * argument of a call is NULL the library takes the chunk's buffers from its
 * cached workspace block for the call's stream (see the conventions above):
 * the block's size is the largest per-chunk workspace asked for on that
 * stream since it was last trimmed, and it stays allocated after the call
 * returns (memfine_workspace_held / memfine_workspace_trim).
 */
typedef struct memfine_allocator {
  void* (*alloc)(size_t bytes, void* stream, void* ctx);
  void (*release)(void* ptr, size_t bytes, void* stream, void* ctx);
  void* ctx;
} memfine_allocator;

/* Output of the planner (all fields filled on MEMFINE_OK and on
 * MEMFINE_ERR_BUDGET). */
typedef struct memfine_plan_info {
  int64_t s_recv;        /* s'': received slots, the sum of the counts      */
  int64_t beta;          /* bytes per received slot used by Eq. (8)         */
  int64_t avail;         /* budget - fixed, the numerator of Eq. (8)        */
  double s_max;          /* Eq. (8): avail / beta (for reporting only)      */
  int64_t c_theory;      /* Eq. (9): ceil(s'' / s'_max); -1 if avail <= 0   */
  int32_t chunks;        /* chosen chunk count (a bin)                      */
  int32_t fits;          /* 1 if the call returned MEMFINE_OK               */
  int64_t paper_peak_bytes; /* beta_paper * slots of the largest chunk      */
  int64_t beta_paper;    /* Table 2 rows 11-13: D_t (2h + 2F)               */
  int64_t beta_impl;     /* this library's backward bytes per slot          */
  int64_t workspace_bytes; /* memfine_workspace_bytes(chunks, backward)     */
  int32_t paper_chunks;  /* the bin Eq. (8)/(9) give with beta_paper alone  */
  int32_t reserved;
} memfine_plan_info;

/*
 * Launch options, for measurements and tests.  Every GEMM setting (tile,
 * raster, split_tail, pair, streams) gives bit-identical results (each
 * output element is one lane's fp32 sum in one fixed K order whatever the
 * tiling); chunk_order changes the order of the sums that form Y and dX.
 * Process-wide; a layer call reads them once when it starts, and
 * memfine_workspace_bytes (hence memfine_plan) follows chunk_order.
 */
#define MEMFINE_TILE_AUTO    0   /* per problem (the default)                  */
#define MEMFINE_TILE_128     1   /* 128 x 128 tiles, 4 waves                   */
#define MEMFINE_TILE_256     2   /* 256 x 256 tiles, 8 waves, direct copies    */
#define MEMFINE_TILE_256_REG 3   /* 256 x 256 tiles, 8 waves, register-staged  */
/*
 * Chunk order.  MEMFINE_CHUNK_TOKENS (the default) is the paper's split,
 * Eq. (6): chunk i holds the slots of tokens [i T / C, (i + 1) T / C).
 * MEMFINE_CHUNK_EXPERTS, a variant that is not in the paper: one dispatch
 * groups all T k slots by expert, and chunk c holds rows [c N / C,
 * (c + 1) N / C) of that grouping (N = T k), i.e. a run of whole experts
 * with at most the first and last split.  An expert's weights are then read,
 * and its fp32 dW written, in one chunk (two for a split expert) instead of
 * in every chunk; in exchange Y and dX are sums over chunks: the chunk that
 * holds a token's first row writes its partial sum, later chunks add theirs
 * to the stored value (one rounding to the storage type per chunk), so
 * these two outputs are not bit-identical across C or to the token order,
 * while dW, dgates and the per-chunk peak (at most ceil(N / C) rows plus
 * the layer's routing tables) follow the same definitions.
 */
#define MEMFINE_CHUNK_TOKENS  0
#define MEMFINE_CHUNK_EXPERTS 1
typedef struct memfine_launch_options {
  int32_t tile;        /* MEMFINE_TILE_*                                       */
  int32_t raster;      /* -1 per problem; 0 row-major by workgroup id; 1..3
                          XCD blocks with groups of 4, 8, 16 m-tiles; 4 XCD
                          blocks row-major                                     */
  int32_t split_tail;  /* 1: a short last round of a GEMM runs as quarter tiles */
  int32_t pair;        /* 1: FC1 dgrad and FC1 wgrad in one launch             */
  int32_t streams;     /* 1: the weight gradients on two side streams          */
  int32_t chunk_order; /* MEMFINE_CHUNK_* (changes results: see above)         */
} memfine_launch_options;

/* NULL restores the defaults {AUTO, -1, 1, 0, 0, TOKENS}.
 * MEMFINE_ERR_INVALID_ARG on a value out of range (the setting is then
 * unchanged). */
int memfine_set_launch_options(const memfine_launch_options* opts);
int memfine_get_launch_options(memfine_launch_options* opts_out);

/*
 * Expert counts over all T tokens: the "first notification" of the paper's
 * Section 4.2 that delivers the number of received slots s''.
 *   d_idx     int32 [T, k] device
 *   d_work    int32 [E + 1] device scratch owned by the caller; on return
 *             d_work[e] = slots routed to expert e and d_work[E] = number of
 *             ids outside [0, E)
 *   h_counts  int64 [E] host output
 * Synchronises `stream`.  Returns MEMFINE_ERR_INVALID_ARG when any id is out
 * of range (h_counts then counts only the valid ids).
 */
int memfine_count(const memfine_shape* shape, const int32_t* d_idx, int32_t* d_work,
                  int64_t* h_counts, void* stream);

/*
 * Dispatch of one chunk, tokens [t0, t1) (the "dispatch" of Eq. (4)), exposed
 * so that tests can check the exact permutation the layer uses.  With
 * n = (t1 - t0) * k and global slot id s = t * k + j:
 *   d_counts       int32 [E]       slots of expert e in the chunk
 *   d_offsets      int32 [E + 1]   exclusive prefix sum, d_offsets[E] = n
 *   d_sorted_slot  int32 [n]       slot ids grouped by expert; ascending
 *                                  slot id inside an expert (stable)
 *   d_row_of_slot  int32 [n]       row of slot t0*k + i in that order
 * Precondition: ids already validated (memfine_count).  Scratch comes from
 * `alloc` (NULL = the library's workspace block for the stream).  Asynchronous.
 */
int memfine_dispatch(const memfine_shape* shape, const int32_t* d_idx, int64_t t0, int64_t t1,
                     int32_t* d_counts, int32_t* d_offsets, int32_t* d_sorted_slot,
                     int32_t* d_row_of_slot, const memfine_allocator* alloc, void* stream);

/*
 * Memory-aware chunk tuning (paper Section 4.2).  Pure host arithmetic, exact
 * in integers.
 *   h_counts      int64 [E]   slots per local expert (memfine_count)
 *   budget_bytes  the numerator of Eq. (8): memory left for this layer's
 *                 chunked MoE activations (alpha*M_GPU - M_sta - non-MoE)
 *   fixed_bytes   subtracted from the budget first (>= 0)
 *   beta_bytes    bytes per received slot, see below
 *   bins, nbins   allowed chunk counts (each >= 1), e.g. {1, 2, 4, 8}
 * Chooses s'' = sum(counts), s'_max = (budget - fixed) / beta (Eq. (8)),
 * c = ceil(s'' / s'_max) (Eq. (9)), then the smallest bin >= c (decided
 * exactly as bin * (budget - fixed) >= s'' * beta).
 *   beta_bytes > 0: that beta; the paper's model alone decides.
 *   beta_bytes = 0 (default): beta = max(beta_paper, beta_impl), the larger
 *     of Table 2 rows 11-13, D_t (2h + 2F), and this library's own backward
 *     bytes per slot; then, so that Eq. (3) holds for the memory the layer
 *     really takes, the chosen bin moves up to the next bin while
 *     memfine_workspace_bytes(bin, backward) > budget - fixed (the rounding
 *     of the chunk split and the per-chunk metadata are not in Eq. (9)).
 *     On MEMFINE_OK the chunk's workspace therefore fits the budget.
 * If no bin is large enough, or budget - fixed <= 0, *chunks_out = the
 * largest bin and the call returns MEMFINE_ERR_BUDGET.  s'' = 0 gives the
 * smallest bin.  `info` may be NULL; info->paper_chunks reports the bin that
 * the paper's beta alone would give.
 */
int memfine_plan(const memfine_shape* shape, const int64_t* h_counts, int64_t budget_bytes,
                 int64_t fixed_bytes, int64_t beta_bytes, const int32_t* bins, int32_t nbins,
                 int32_t* chunks_out, memfine_plan_info* info);

/*
 * Bytes of working memory the layer allocates for its largest chunk (the
 * per-chunk buffers of memfine_moe_fwd or memfine_moe_bwd, pass =
 * MEMFINE_PASS_FWD / MEMFINE_PASS_BWD) - the activation peak of the chunked
 * layer that Section 4.1 says replaces the unchunked one.  Under
 * MEMFINE_CHUNK_EXPERTS it adds the layer's routing tables, held for the
 * whole call.  Returns < 0 on invalid arguments.
 */
int64_t memfine_workspace_bytes(const memfine_shape* shape, int32_t chunks, int32_t pass);

/*
 * The library's cached workspace block for calls with a NULL allocator
 * (paper Section 4.1: the layer's activation peak is the largest chunk's).
 * memfine_workspace_held: bytes of the block kept for (the current device,
 * `stream`); 0 if none.  memfine_workspace_trim: if that block is larger than
 * keep_bytes, it is released in stream order (after the work enqueued on
 * `stream` so far) and, when keep_bytes > 0, replaced by a block of
 * keep_bytes; afterwards the held bytes are at most keep_bytes.  A caller
 * that raises the chunk count to free memory trims to
 * memfine_workspace_bytes(new chunks, MEMFINE_PASS_BWD).  Not to be called
 * while a layer call runs on the same stream from another thread, and refused
 * (MEMFINE_ERR_INVALID_ARG) while the stream is being captured.  The blocks of
 * captured calls are neither counted nor released.
 */
int memfine_workspace_held(void* stream, int64_t* bytes_out);
int memfine_workspace_trim(void* stream, int64_t keep_bytes);

/*
 * High-water mark of the library's per-device stream-ordered pool (the
 * bytes its blocks held at most at once, on the current device) since the
 * pool was created or last reset (reset = 1 resets it after reading).  0
 * before the first call that needed a block.
 */
int memfine_pool_high_water(int64_t* bytes_out, int32_t reset);

/* ------------------------------------------------------------------------
 * MACT from the model configuration (paper Section 3 and Section 4.2).
 * Pure host arithmetic, exact (128-bit integers); no device state.
 *
 * The memory model uses the symbols of the paper's notation table; every
 * size is an element count and D_t the bytes per activation element.
 */
typedef struct memfine_model {
  int64_t b, s;            /* micro-batch size, sequence length                */
  int64_t h, a, h_d, k_a;  /* hidden size, heads, head dim, kv heads           */
  int64_t e_n, g_e;        /* router output width, expert FFN size (F)         */
  int32_t t, c;            /* tensor- and context-parallel sizes (>= 1)        */
  int32_t v, p;            /* pipeline stages per GPU, pipeline size (>= 1)    */
  int32_t D_t;             /* activation bytes per element (>= 1)              */
  int32_t full_recompute;  /* 1: m_g = 1; 0: m_g = v p + p - 2 r_pp - 1        */
} memfine_model;

/*
 * Eq. (1): static memory = (D_para + D_grad + 4 D_opt) * v * l * sum(S_para),
 * parameters, gradients and four optimizer-state copies of the m_n weighted
 * modules of a layer (S_para[i] elements each), v stages of l layers.
 * *bytes_out receives the total.  MEMFINE_ERR_INVALID_ARG on a negative or
 * zero size factor, a negative S_para, or a result beyond int64.
 */
int memfine_static_memory(const int64_t* S_para, int32_t m_n, int32_t v, int32_t l,
                          int32_t D_para, int32_t D_grad, int32_t D_opt, int64_t* bytes_out);

/*
 * Eq. (2): peak activation bytes at pipeline rank r_pp (0 <= r_pp < p) with
 * s_recv received slots, m_g/(t c) D_t b (s (5h + a h_d + 2 k_a h_d + e_n)
 * + s_recv (2h + 2 g_e)), rounded up to whole bytes.  With chunking, s_recv
 * is the largest chunk's slots.  MEMFINE_ERR_INVALID_ARG on invalid fields,
 * m_g < 1, or a result beyond int64.
 */
int memfine_activation_memory(const memfine_model* m, int32_t r_pp, int64_t s_recv,
                              int64_t* bytes_out);

/*
 * MACT set-up, once per pipeline rank before training: the threshold table
 * of the bins.  s'_max is Eq. (8) with alpha = alpha_num / alpha_den, GPU
 * memory M_gpu and static memory M_sta (bytes); thresholds_out[i] is the
 * largest s'' for which bins[i] chunks keep Eq. (3), floor(bins[i] * s'_max),
 * or -1 when the part of Eq. (2) that does not depend on s'' alone exceeds
 * alpha M_gpu - M_sta.  Values beyond int64 are clamped to INT64_MAX.
 */
int memfine_mact_thresholds(const memfine_model* m, int32_t r_pp, int64_t M_gpu, int64_t alpha_num,
                            int64_t alpha_den, int64_t M_sta, const int32_t* bins, int32_t nbins,
                            int64_t* thresholds_out);

/*
 * MACT at run time, per iteration and layer: the smallest bin whose
 * threshold admits the received slots s_recv (the threshold form of Eq. (9)
 * followed by the bin choice).  When no bin admits them, *chunks_out is the
 * largest bin and the call returns MEMFINE_ERR_BUDGET.
 */
int memfine_mact_select(const int32_t* bins, const int64_t* thresholds, int32_t nbins,
                        int64_t s_recv, int32_t* chunks_out);

/*
 * Chunked forward, Eq. (6): Y = concat(F_w(X_1), ..., F_w(X_C)), with
 * F_w = combine(expert(dispatch(.))) of Eq. (4) on tokens
 * [floor(i*T/C), floor((i+1)*T/C)).  Every chunk's buffers are allocated
 * before and released after its kernels.  Nothing is kept for the backward.
 * Y is overwritten.  `chunks` >= 1 (chunks > T behaves like T).  A slot whose
 * id lies outside [0, E) is dropped: it contributes nothing to Y (and, in the
 * backward, nothing to dX or dW; its dgates entry is 0).
 */
int memfine_moe_fwd(const memfine_shape* shape, int32_t chunks, const void* d_X,
                    const int32_t* d_idx, const float* d_gates, const void* d_W1,
                    const void* d_W2, void* d_Y, const memfine_allocator* alloc, void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the
 * chunked forward of memfine_moe_fwd, same arguments (no allocator) and
 * bit-identical results, with every chunk's working buffers in one static
 * device array of MEMFINE_NOALLOC_SCRATCH_BYTES (64 MiB) that the library's
 * code object carries; each GPU the library runs on holds its own copy until
 * the process ends.  The call allocates and frees nothing (no hipMalloc,
 * pool or allocator call; the array's address is looked up once per device
 * with hipGetSymbolAddress).  A call whose largest chunk needs more than the
 * array, memfine_workspace_bytes(shape, chunks, MEMFINE_PASS_FWD) >
 * MEMFINE_NOALLOC_SCRATCH_BYTES, returns MEMFINE_ERR_SCRATCH before anything
 * is enqueued: raise `chunks`.  Nothing in the array needs to start at zero
 * (every buffer is written before it is read).  All calls on one GPU share
 * its array: calls that overlap on one GPU (other streams, other threads)
 * race, and the caller must order them (e.g. one stream).
 */
#define MEMFINE_NOALLOC_SCRATCH_BYTES (64ll << 20)
int memfine_moe_fwd_noalloc(const memfine_shape* shape, int32_t chunks, const void* d_X,
                            const int32_t* d_idx, const float* d_gates, const void* d_W1,
                            const void* d_W2, void* d_Y, void* stream);

/*
 * Chunked-recompute backward, Eq. (7): for each chunk in ascending order,
 * recompute its forward, then back-propagate dY's rows of that chunk.
 * Overwrites dX and dgates.  dW1/dW2 are overwritten when accumulate_dW == 0
 * and added to when accumulate_dW == 1.
 */
int memfine_moe_bwd(const memfine_shape* shape, int32_t chunks, const void* d_X,
                    const int32_t* d_idx, const float* d_gates, const void* d_W1,
                    const void* d_W2, const void* d_dY, void* d_dX, float* d_dW1, float* d_dW2,
                    float* d_dgates, int32_t accumulate_dW, const memfine_allocator* alloc,
                    void* stream);

/* ------------------------------------------------------------------------
 * Router in front of the expert layer (Table 2 rows 9-10 store its input and
 * its logits; the gates it produces are the scores that multiply the expert
 * outputs, Table 2 "score mul").  `shape` is the layer's shape; the router
 * needs k <= 16 and k <= E <= 256 (MEMFINE_ERR_UNSUPPORTED otherwise): up to
 * the 256 routed experts of the paper's Table 3 models.
 *
 * Forward: logits = X Wr^T (fp32 accumulation), softmax over the E experts,
 * the k largest logits (equal logits: the lower expert id first), and the
 * gates renormalised over the selected k (the full softmax denominator
 * cancels, so gates_j = exp(z_j - z_max) / sum over the selected).
 *   d_X       dtype [T, h];   d_Wr  dtype [E, h]
 *   d_idx     int32 [T, k] out, largest logit first
 *   d_gates   float [T, k] out
 *   d_logits  float [T, E] out, may be NULL
 * Asynchronous.  Up to 64 logits (or E not a multiple of 32) one fused
 * kernel, no working memory; wider routers compute the logits as a grouped
 * GEMM and select from them, taking, when d_logits is NULL, the [T, E] fp32
 * logits from the library's per-stream workspace (as a layer call with a
 * NULL allocator does); MEMFINE_ERR_OOM if that fails.
 */
int memfine_router_fwd(const memfine_shape* shape, const void* d_X, const void* d_Wr,
                       int32_t* d_idx, float* d_gates, float* d_logits, void* stream);

/*
 * Backward from the expert layer's dgates (memfine_moe_bwd's output), with
 * the selection held fixed: per token, with c = sum_j g_j dg_j,
 *   dlogits[t, idx_j] = g_j (dg_j - c), 0 for the unselected experts;
 *   dX  = dlogits Wr   (accumulate_dX = 1 adds it into d_dX, e.g. the
 *                       layer's dX; 0 overwrites)
 *   dWr = dlogits^T X  (float [E, h]; accumulate_dWr as above)
 * Slots whose id lies outside [0, E) pass no gradient.  Working memory
 * (dense dlogits rows and split-K partials of dWr) comes from `alloc`.
 */
int memfine_router_bwd(const memfine_shape* shape, const void* d_X, const void* d_Wr,
                       const int32_t* d_idx, const float* d_gates, const float* d_dgates,
                       void* d_dX, float* d_dWr, int32_t accumulate_dX, int32_t accumulate_dWr,
                       const memfine_allocator* alloc, void* stream);

/* ------------------------------------------------------------------------
 * Around the layer: the norm in front of it, routing from logits, and the
 * layer's forward with 4-bit weights.  Pointers must be 16-byte aligned
 * (MEMFINE_ERR_INVALID_ARG otherwise, as for a null pointer that is not
 * optional), but for the activations' scales d_XS and the row-major scales
 * d_row_scales, which may lie anywhere, and the experts' d_idx and d_gates,
 * aligned as their elements; T = 0 does nothing but what is said below.
 *
 * The MX formats hold blocks of 32 consecutive values of a row and one scale
 * byte s per block, 2^(s - 127): MX8 has e4m3 values (one byte each), MX4 has
 * e2m1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; two to a byte,
 * the first in the low half).  The scale is the smallest power of two, at
 * least 2^-127, that keeps the block's largest magnitude within 448 (MX8) or 6
 * (MX4) times it; values are rounded to nearest, ties to even.  (Not the
 * conversion of the OCP specification, which takes the power of two below the
 * largest magnitude, over 256 or 4, and lets what is then past the largest value
 * saturate; matrices that were rounded so are packed as they are.)  A block that
 * holds a NaN or an infinity gets s = 255, and all its values are NaN, in every
 * product too.
 */

/*
 * Residual addition and root-mean-square norm of T rows of h elements (h a
 * multiple of 64, else MEMFINE_ERR_INVALID_ARG; h <= 16384 and T < 2^31, else
 * MEMFINE_ERR_UNSUPPORTED):
 *   S = X + R            rounded to dtype; without R (null) S is X
 *   Y = S / sqrt(mean(S^2) + eps) * w
 *   d_X, d_R  dtype [T, h];   d_w  dtype [h];   eps >= 0
 *   d_S   dtype [T, h] out, may be null (must be null without R); may be d_X
 *         or d_R itself
 *   d_Y   dtype [T, h] out, may be null;
 *   d_Q, d_QS  uint8 [T, h], [T, h / 32] out: the MX8 form of the unrounded
 *         Y; both or neither
 * At least one of d_Y and d_Q is asked for.  fp32 arithmetic.
 */
int memfine_norm_fwd(int64_t T, int32_t h, int32_t dtype, float eps, const void* d_X,
                     const void* d_R, const void* d_w, void* d_S, void* d_Y, uint8_t* d_Q,
                     uint8_t* d_QS, void* stream);

/*
 * Its gradient.  With r = 1 / sqrt(mean(X^2) + eps), X the norm's input (the
 * forward's S):
 *   dX = r (dY w - X r^2 mean(dY w X)) + dS    dtype [T, h]: the gradient of X
 *        and, with a residual, of R alike; d_dS (the gradient that reaches S
 *        from elsewhere) may be null; d_dX may be d_dY or d_dS itself
 *   dw = sum over rows of dY X r               float [h], added to d_dw when
 *        accumulate_dw = 1, else overwriting it (T = 0: zeros)
 * Sums over rows are formed in a fixed order.  Working memory (partial sums of
 * dw) comes from `alloc` as for the layer's calls.
 */
int memfine_norm_bwd(int64_t T, int32_t h, int32_t dtype, float eps, const void* d_X,
                     const void* d_w, const void* d_dY, const void* d_dS, void* d_dX, float* d_dw,
                     int32_t accumulate_dw, const memfine_allocator* alloc, void* stream);

/* The values of an MX8 tensor, d_Q [T, h] with d_QS [T, h / 32] (h a multiple
 * of 32), as d_out, dtype [T, h]: exact in float, and in bf16 unless a value is
 * below its subnormals. */
int memfine_mx_values(int64_t T, int32_t h, const uint8_t* d_Q, const uint8_t* d_QS,
                       int32_t dtype, void* d_out, void* stream);

/* ------------------------------------------------------------------------
 * Routing from logits, for routers other than the renormalised softmax top-k
 * of memfine_router_fwd.  Per token:
 *   p_e = softmax over the E experts, or sigmoid, of the logits
 *   v_e = p_e + bias_e (no bias: p_e); selects, and enters nothing else
 *   groups > 1: the experts form `groups` runs of E / groups; a group's score
 *     is the sum of its two largest v (its v, when E = groups), and only
 *     experts of the top_groups best groups (equal: the lower one) are left
 *   the k experts of largest v, in that order (equal: the lower id)
 *   gate_j = scale p_j, or, with renorm, scale p_j / (sum of the selected p)
 * A logit of -inf, of the lowest finite float or a NaN masks its expert: p = 0,
 * and it is selected, with gate 0, only when fewer than k others are left
 * (a token without any other gets k masked experts and zero gates).  +inf
 * counts as the largest finite float.  A bias of -inf or NaN makes its expert
 * the last choice alike, with its own gate.  p and v are floats: in the
 * selection a p below 2^-126 counts as 0 (equal values: the lower id), while
 * renormalised gates keep the ratios of such p.
 * 1 <= E <= 256, 1 <= k <= 16 (MEMFINE_ERR_UNSUPPORTED otherwise), k <=
 * top_groups E / groups, groups <= 16 dividing E.
 */
#define MEMFINE_SCORE_SOFTMAX 0
#define MEMFINE_SCORE_SIGMOID 1
typedef struct memfine_gating {
  int32_t E, k;
  int32_t score;       /* MEMFINE_SCORE_*                                  */
  int32_t groups;      /* 1: no groups                                     */
  int32_t top_groups;  /* 1 <= top_groups <= groups                        */
  int32_t renorm;      /* 0 or 1                                           */
  float scale;         /* finite                                           */
} memfine_gating;

/* d_logits float [T, E]; d_bias float [E] or null; d_idx int32 [T, k] and
 * d_gates float [T, k] out. */
int memfine_route_fwd(int64_t T, const memfine_gating* g, const float* d_logits,
                      const float* d_bias, int32_t* d_idx, float* d_gates, void* stream);

/* The gradient of the gates, with the selection held fixed: d_dlogits float
 * [T, E] is overwritten, from the forward's d_logits and d_idx and d_dgates
 * float [T, k].  Softmax gates without renorm reach every logit, the others
 * those of the selected experts alone.  Slots whose id lies outside [0, E)
 * pass no gradient; slots of one token with the same id add up. */
int memfine_route_bwd(int64_t T, const memfine_gating* g, const float* d_logits,
                      const int32_t* d_idx, const float* d_dgates, float* d_dlogits, void* stream);

/* The router's product by itself, for routing from logits: d_logits = X Wr^T,
 * float [T, E] (shapes, types and limits of memfine_router_fwd; k is not
 * used; no working memory), and its gradients dX = dlogits Wr, dWr = dlogits^T
 * X (as memfine_router_bwd, working memory from `alloc` as there; dlogits are
 * rounded to the shape's dtype for the products). */
int memfine_router_logits(const memfine_shape* shape, const void* d_X, const void* d_Wr,
                          float* d_logits, void* stream);
int memfine_router_logits_bwd(const memfine_shape* shape, const void* d_X, const void* d_Wr,
                              const float* d_dlogits, void* d_dX, float* d_dWr,
                              int32_t accumulate_dX, int32_t accumulate_dWr,
                              const memfine_allocator* alloc, void* stream);

/* ------------------------------------------------------------------------
 * MX4 matrices.  W [N, K] (N a multiple of 16, K of 32; N <= 2^22, K <= 2^20) is held
 * in the matrix cores' order in two buffers of memfine_mxw_code_bytes(N, K)
 * and memfine_mxw_scale_bytes(N, K) bytes (< 0: invalid sizes); E matrices of
 * one size follow each other in both.  memfine_mxw_pack lays out row-major codes
 * uint8 [E, N, K / 2] and scales uint8 [E, N, K / 32] as a checkpoint holds
 * them; memfine_mxw_quantize rounds values dtype [E, N, K];
 * memfine_mxw_unpack gives the values back, dtype [E, N, K].
 */
int64_t memfine_mxw_code_bytes(int32_t N, int32_t K);
int64_t memfine_mxw_scale_bytes(int32_t N, int32_t K);
int memfine_mxw_pack(int32_t E, int32_t N, int32_t K, const uint8_t* d_row_codes,
                     const uint8_t* d_row_scales, uint8_t* d_codes, uint8_t* d_scales,
                     void* stream);
int memfine_mxw_quantize(int32_t E, int32_t N, int32_t K, int32_t dtype, const void* d_W,
                         uint8_t* d_codes, uint8_t* d_scales, void* stream);
int memfine_mxw_unpack(int32_t E, int32_t N, int32_t K, const uint8_t* d_codes,
                       const uint8_t* d_scales, int32_t dtype, void* d_W, void* stream);

/*
 * Y [T, N] = X [T, K] W^T with W in MX4 (d_codes, d_scales), T < 2^31.
 *   d_X  bf16 [T, K] when d_XS is null, else e4m3 bytes [T, K] with the scales
 *        d_XS [T, K / 32] (MX8, as memfine_norm_fwd gives them)
 *   d_Y  y_dtype [T, N], MEMFINE_BF16 or MEMFINE_F32
 * Sums in fp32, in an order that depends on T, N, K, the activations' format and
 * the device's compute units alone.  On bf16 activations the products are those
 * of the held values; on MX8 the matrix core cuts each product off, towards
 * zero, at 2^-13 of the power of two at or below the largest of eight
 * neighbouring ones.  A reduction of K > 4096 over few rows (T <= 64, or blocks
 * of 32 rows x 256 columns for less than half the compute units) is split and
 * takes ceil(K / 4096) T N floats of working memory,
 * memfine_linear_mxw_workspace_bytes (0: none; mx8 = 1: with d_XS; < 0: invalid
 * arguments).  It comes from `alloc` as for the layer's calls; memfine_linear_mxw
 * is the call with a null allocator.
 */
int memfine_linear_mxw(int64_t T, int32_t N, int32_t K, const void* d_X, const uint8_t* d_XS,
                       const uint8_t* d_codes, const uint8_t* d_scales, int32_t y_dtype, void* d_Y,
                       void* stream);
int memfine_linear_mxw_alloc(int64_t T, int32_t N, int32_t K, const void* d_X, const uint8_t* d_XS,
                             const uint8_t* d_codes, const uint8_t* d_scales, int32_t y_dtype,
                             void* d_Y, const memfine_allocator* alloc, void* stream);
int64_t memfine_linear_mxw_workspace_bytes(int64_t T, int32_t N, int32_t K, int32_t mx8);

/*
 * The chunked forward, memfine_moe_fwd, with W1 and W2 in MX4 (E matrices
 * [2F, h] and [h, F]); shape.dtype must be MEMFINE_BF16 (Y's type).
 *   d_X  bf16 [T, h] when d_XS is null; the SwiGLU output is then rounded to
 *        bf16 for the second product.  With d_XS: MX8, e4m3 [T, h] and scales
 *        [T, h / 32]; the SwiGLU output is then rounded to MX8 as well.
 * The second product's rows stay fp32 up to Y, but on MX8 activations may, in
 * chunks of more than 4096 rows, be rounded to fp16 times a power of two for each
 * 64 columns: by 2^-12 of a value, or 2^-41 of the largest of its 64 columns.
 * Everything else as memfine_moe_fwd, but at most 2^31 - 257 slots a chunk
 * (MEMFINE_ERR_UNSUPPORTED beyond).  memfine_moe_mxw_workspace_bytes: the
 * working memory of the chunk that needs the most (mx8 = 1: with d_XS).
 */
int memfine_moe_fwd_mxw(const memfine_shape* shape, int32_t chunks, const void* d_X,
                        const uint8_t* d_XS, const int32_t* d_idx, const float* d_gates,
                        const uint8_t* d_W1_codes, const uint8_t* d_W1_scales,
                        const uint8_t* d_W2_codes, const uint8_t* d_W2_scales, void* d_Y,
                        const memfine_allocator* alloc, void* stream);
int64_t memfine_moe_mxw_workspace_bytes(const memfine_shape* shape, int32_t chunks, int32_t mx8);

/* ------------------------------------------------------------------------
 * Attention in front of the layer.  A row holds heads of `dim` elements, one
 * after the other; rows of queries, keys, values, their gradients and of what
 * memfine_rope reads and writes lie ld elements apart (ld_* >= their heads times
 * dim, a multiple of 16 bytes, at most 2^20, UNSUPPORTED beyond), so that
 * they may be columns of one projection's output; O and dO are contiguous.
 * Head j uses key-value head j / (heads / kv_heads).
 *
 * Packed sequences: sequence b is rows [d_offsets[b], d_offsets[b + 1]) of T,
 * d_offsets int32 [seqs + 1] on the device, ascending, within [0, T] (what lies
 * outside is neither read nor written, whatever the offsets hold); a sequence may be
 * empty, and rows of none are left as they were.  T, its sequences rounded up to 32
 * rows, times heads is at most 2^27 for the attention (UNSUPPORTED beyond).
 *
 * Pointers as above (16 bytes), but d_offsets, d_table, d_lengths and d_lse, aligned
 * as their elements.  dim is 64 or 128, heads at most 1024
 * (MEMFINE_ERR_UNSUPPORTED otherwise).
 */
typedef struct memfine_attn {
  int32_t heads, kv_heads;   /* heads a multiple of kv_heads                    */
  int32_t dim;
  int32_t dtype;             /* MEMFINE_BF16 or MEMFINE_F32                     */
  int32_t causal;            /* 1: token i sees j <= i                          */
  int32_t window;            /* w > 0 (causal only): and j > i - w; 0: no limit */
  float scale;               /* of the products; finite, > 0                    */
} memfine_attn;

/*
 * Attention over packed sequences.  Per head, over the tokens j that token i sees:
 *   s_ij = scale q_i . k_j;  lse_i = log sum_j exp(s_ij);
 *   O_i = sum_j exp(s_ij - lse_i) v_j
 *   d_Q  dtype [T, heads, dim];  d_K, d_V  dtype [T, kv_heads, dim]
 *   d_O  dtype [T, heads, dim] out;  d_lse  float [heads, T] out, may be null
 * Products and sums in fp32; in bf16 the weights exp(.) are rounded to bf16 for
 * the product with V (their sum is not), as the ds of the gradient for theirs.
 * A NaN or an infinity in a row reaches any token of its sequence.
 */
int memfine_attn_fwd(int64_t T, int32_t seqs, const memfine_attn* a, const int32_t* d_offsets,
                     const void* d_Q, int64_t ld_q, const void* d_K, int64_t ld_k, const void* d_V,
                     int64_t ld_v, void* d_O, float* d_lse, void* stream);

/*
 * Its gradient, from the forward's O and lse and from dO:
 *   delta_i = dO_i . O_i;  p_ij = exp(s_ij - lse_i)
 *   ds_ij = scale p_ij (dO_i . v_j - delta_i)
 *   dQ_i = sum_j ds_ij k_j;  dK_j = sum_i ds_ij q_i;  dV_j = sum_i p_ij dO_i
 * dK and dV add up over the heads that share a key-value head.  dQ, dK and dV are
 * overwritten, rows of no sequence left as they were; they must not overlap the
 * inputs.  Every sum, here and in the forward, has a fixed order, which depends on T, seqs,
 * what `a` holds, the sequence's own length and the device's compute units alone.  Working
 * memory (two floats a row and head, and partial dK and dV where keys are few:
 * memfine_attn_bwd_workspace_bytes, < 0: invalid arguments) comes from `alloc` as for the
 * layer's calls.
 */
int memfine_attn_bwd(int64_t T, int32_t seqs, const memfine_attn* a, const int32_t* d_offsets,
                     const void* d_Q, int64_t ld_q, const void* d_K, int64_t ld_k, const void* d_V,
                     int64_t ld_v, const void* d_O, const float* d_lse, const void* d_dO,
                     void* d_dQ, int64_t ld_dq, void* d_dK, int64_t ld_dk, void* d_dV,
                     int64_t ld_dv, const memfine_allocator* alloc, void* stream);
int64_t memfine_attn_bwd_workspace_bytes(int64_t T, int32_t seqs, const memfine_attn* a);

/*
 * Rotation by position, of rows of packed sequences (position: the row's place in
 * its sequence), for the pairs (a, b) = (i, i + dim / 2) of every head, or with
 * interleaved = 1 (2 i, 2 i + 1), 0 <= i < dim / 2, c and s their cosine and sine:
 *   y_a = x_a c - x_b s;  y_b = x_b c + x_a s     (inverse = 1: -s, the gradient)
 *   d_cos, d_sin  float [positions, dim / 2]; rows past the tables become NaN
 *   d_X, d_Y  dtype [T, heads, dim], Y may be X (with X's ld)
 */
typedef struct memfine_rotary {
  const float *d_cos, *d_sin;
  int64_t positions;
  int32_t interleaved;       /* 0 or 1                                          */
} memfine_rotary;
int memfine_rope(int64_t T, int32_t seqs, const int32_t* d_offsets, int32_t heads, int32_t dim,
                 int32_t dtype, const memfine_rotary* r, int32_t inverse, const void* d_X,
                 int64_t ld_x, void* d_Y, int64_t ld_y, void* stream);

/*
 * Keys and values of served sequences, in pages of `page` tokens (a power of two, 16 to
 * 65536):
 *   d_k, d_v    bf16 [pages, kv_heads, page, dim] when d_ks and d_vs are null, else
 *               MX8: e4m3 bytes and scales d_ks, d_vs uint8 [pages, kv_heads,
 *               page, dim / 32]
 * Token t of sequence b is token t % page of page d_table[b][t / page], d_table
 * int32 [seqs, width] on the device (width page <= 2^30), d_lengths int32 [seqs] the tokens
 * that each sequence has (cut to [0, width page]).  Entries of the table past a sequence's
 * last page are not used.  An entry outside [0, pages) stands for no page: nothing
 * is written to it, and its tokens are left out of the attention.
 */
typedef struct memfine_cache {
  int32_t kv_heads, dim;     /* dim 64 or 128                                   */
  int32_t page;
  int64_t pages;             /* 1 .. 2^31 - 1                                   */
  void *d_k, *d_v;
  uint8_t *d_ks, *d_vs;
} memfine_cache;

/*
 * New tokens into the cache: d_lengths counts them already, row i of the n that
 * sequence b brings is its token d_lengths[b] - n + i (a negative one is dropped, and one
 * that the table's width has no page for).
 *   d_offsets  the sequences' rows, packed as above, or null: T = seqs, row b is
 *              sequence b's
 *   d_K, d_V   bf16 [T, kv_heads, dim];  K is turned on its way if r is not null,
 *              by the token's position, V is not; MX8 holds the unrounded K
 *   d_Q        bf16 [T, heads, dim] or null (heads = 0); turned likewise into
 *   d_R        bf16 [T, heads, dim], which may be d_Q when that is contiguous.
 *              Rows that are dropped are left as they were.
 * No page may be a sequence's twice, or that of two sequences that write to it.
 */
int memfine_kv_write(const memfine_cache* c, int64_t T, int32_t seqs, int32_t width,
                     const int32_t* d_table, const int32_t* d_lengths, const int32_t* d_offsets,
                     const memfine_rotary* r, const void* d_K, int64_t ld_k, const void* d_V,
                     int64_t ld_v, int32_t heads, const void* d_Q, int64_t ld_q, void* d_R,
                     void* stream);

/*
 * Attention of one token a sequence over its cached tokens (its own among them;
 * with a->window, the last `window`): O_b and lse_b as memfine_attn_fwd's for the
 * last token of sequence b, but with the weights of the product with V to 2^-16 of
 * each.  A sequence without tokens gets zeros (lse -inf).
 *   a      kv_heads and dim as the cache's, dtype MEMFINE_BF16; causal 0 and 1 are the
 *          same here, but a window is for causal = 1 alone, as everywhere
 *   d_Q    bf16 [seqs, heads, dim];  d_O  bf16 [seqs, heads, dim] out
 *   d_lse  float [seqs, heads] out, may be null
 * What pages hold past a sequence's tokens does not matter.  Sums are formed in an order
 * that depends on all lengths, the sizes and the device's compute units alone.
 * Working memory (the parts of sequences that several workgroups share,
 * memfine_attn_decode_workspace_bytes; < 0: invalid arguments) comes from `alloc` as
 * for the layer's calls.
 */
int memfine_attn_decode(const memfine_attn* a, const memfine_cache* c, int32_t seqs, int32_t width,
                        const int32_t* d_table, const int32_t* d_lengths, const void* d_Q,
                        int64_t ld_q, void* d_O, float* d_lse, const memfine_allocator* alloc,
                        void* stream);
int64_t memfine_attn_decode_workspace_bytes(const memfine_attn* a, const memfine_cache* c,
                                            int32_t seqs, int32_t width);

/* Static, human-readable text for a status code. */
const char* memfine_status_str(int status);

/*
 * Kernel timing for performance reports.  memfine_profile_begin(mask) makes
 * later calls record a pair of HIP events around every launch of the kernels
 * whose id bit is set in `mask` (ids: MEMFINE_K_*).  memfine_profile_end waits
 * for those events and returns, per kernel id, the number of launches, the
 * summed launch durations in milliseconds, and the algorithmic flops and HBM
 * bytes of those launches; then it stops recording.
 */
#define MEMFINE_K_COUNT       0
#define MEMFINE_K_DISPATCH    1
#define MEMFINE_K_FC1         2   /* forward FC1 + SwiGLU                    */
#define MEMFINE_K_FC2         3   /* forward FC2                             */
#define MEMFINE_K_COMBINE     4
#define MEMFINE_K_FC1_RECOMP  5   /* backward: FC1 recompute + SwiGLU bwd    */
#define MEMFINE_K_FC2_DGRAD   6   /* backward: dA = dY W2                    */
#define MEMFINE_K_FC2_WGRAD   7
#define MEMFINE_K_FC1_WGRAD   8
#define MEMFINE_K_FC1_DGRAD   9
#define MEMFINE_K_UNPERMUTE  10   /* dX sum over slots and gate gradient     */
#define MEMFINE_K_FC1_BWD    11   /* FC1 dgrad with FC1 wgrad, or with both wgrads, in one launch */
#define MEMFINE_K_ROUTER_FWD 12   /* router logits, softmax, top-k, gates    */
#define MEMFINE_K_ROUTER_BWD_DX 13 /* router: dz per token, dX contribution */
#define MEMFINE_K_ROUTER_WGRAD 14 /* router: split-K partials of dz^T X     */
#define MEMFINE_K_ROUTER_REDUCE 15 /* router: sum of the partials into dWr  */
#define MEMFINE_K_NORM_FWD   16
#define MEMFINE_K_NORM_BWD   17
#define MEMFINE_K_ROUTE_FWD  18 /* routing from logits                      */
#define MEMFINE_K_ROUTE_BWD  19
#define MEMFINE_K_MX_LINEAR  20 /* MX4: the single linear map               */
#define MEMFINE_K_MX_FC1     21 /* MX4: FC1 + SwiGLU                        */
#define MEMFINE_K_MX_FC2     22
#define MEMFINE_K_MX_COMBINE 23
#define MEMFINE_K_ATTN_FWD   24 /* attention: flops are counted as 0 (they depend */
#define MEMFINE_K_ATTN_BWD   25 /* on lengths that the host does not see)        */
#define MEMFINE_K_ATTN_DECODE 26
#define MEMFINE_K_ROPE       27
#define MEMFINE_K_KV_WRITE   28
#define MEMFINE_K_NUM        29

typedef struct memfine_kernel_stat {
  int64_t launches;
  double total_ms;
  double flops;   /* algorithmic floating-point operations, all launches */
  double bytes;   /* algorithmic HBM bytes, all launches                  */
} memfine_kernel_stat;

int memfine_profile_begin(uint32_t mask);
int memfine_profile_end(memfine_kernel_stat* out /* [MEMFINE_K_NUM] */);

#ifdef __cplusplus
}
#endif

#endif /* MEMFINE_H */
