/*
 * pblock.h — C ABI of the MI355X (gfx950) parallel transformer block library.
 *
 * The block is Eq. 2 of MegaScale (Section 3.1):
 *
 *     y = x + MLP(LN(x)) + Attention(LN(x))
 *
 * with ONE LayerNorm whose output h feeds both branches, a fused in-projection
 * Z = h W_in^T + b_in whose columns are [Q | K | V | U], causal sliding-window
 * attention (Section 3.1, "Sliding window attention") on Q, K, V, the GeLU MLP
 * activation G = gelu(U), and one fused out-projection over C = [O | G]:
 *
 *     y = x + C W_out^T + b_out.
 *
 * Window rule: query i attends to key j of the same batch row iff
 * 0 <= i - j < window (window keys, the query's own position included);
 * window >= seq is ordinary causal attention.  Scores are scaled by
 * 1/sqrt(head_dim).  LayerNorm uses the biased variance with eps inside the
 * square root.  GeLU is the tanh form when gelu_tanh != 0, else the erf form.
 *
 * Section 3.3 replaces attention with FlashAttention-2 and LN/GeLU with fused
 * kernels; this library does the same on gfx950 (banded flash-style attention
 * that skips key tiles outside the window, MFMA GEMMs with fused bias / GeLU /
 * residual epilogues).  None of that changes the result beyond rounding.
 *
 * ---------------------------------------------------------------- layouts
 * All tensors are dense, row-major, in device memory (HBM), 16-byte aligned.
 * Let T = batch*seq, H = hidden, A = heads*head_dim, F = ffn,
 *     N_in = 3A + F, K_out = A + F.
 *   x, y, dy, dx  [T, H]          activation dtype (bf16 or fp32), token-major
 *   ln_gamma/beta [H]             activation dtype
 *   w_in          [N_in, H]       activation dtype; rows Q | K | V | MLP-up;
 *                                 head h owns rows h*d .. h*d+d-1 of each of
 *                                 Q, K and V (d = head_dim)
 *   b_in          [N_in]          activation dtype
 *   w_out         [H, K_out]      activation dtype; columns attention-out |
 *                                 MLP-down (the two output projections of
 *                                 Eq. 2, side by side)
 *   b_out         [H]             activation dtype: the sum of the attention
 *                                 and MLP output biases (only their sum enters
 *                                 Eq. 2)
 *   dgamma, dbeta [H], dw_in [N_in, H], db_in [N_in], dw_out [H, K_out],
 *   db_out [H]                    fp32, always
 *
 * Saved stash (forward -> backward), regions in this order, each starting at
 * a 256-byte boundary (see pblock_saved_offsets):
 *   h     [T, H]      act   LN output
 *   z     [T, N_in]   act   Q | K | V | U  (U before GeLU)
 *   c     [T, K_out]  act   O | G          (attention output, GeLU output)
 *   mean  [T]         fp32  LN row mean
 *   rstd  [T]         fp32  LN row 1/sqrt(var + eps)
 *   lse   [batch, heads, seq] fp32  log of each softmax denominator, in the
 *                     scaled-score domain
 *
 * ---------------------------------------------------------------- ownership
 * The caller allocates every buffer (inputs, outputs, the stash, the
 * workspace).  The library allocates no device memory and keeps no state
 * between calls: the HIP events that the pipelined all-gather and
 * reduce-scatter order their streams with live in a pb_tp_context that the
 * caller creates and destroys, and the step events of the *_timed calls are
 * passed with each call.  (pblock_swattn_forward_noalloc alone uses a
 * library-owned device array; see there.)  Every call is
 * asynchronous on the given HIP stream; buffers must stay valid until the
 * stream has passed the call.  Other calls on disjoint buffers may run
 * concurrently.  Parameter gradients are overwritten, not accumulated.
 * The block's forward and backward calls (parallel and serial) only launch
 * kernels on the given stream (no allocation, memset, copy or
 * synchronisation), so a caller may capture them into a HIP graph and
 * replay it.
 *
 * ---------------------------------------------------------------- errors
 * Functions return a pb_status.  Arguments are checked on the host before any
 * HIP call is made; on a failed check nothing is launched and
 * pblock_last_error() describes the problem.  PB_ERR_HIP reports a launch
 * failure (hipGetLastError after the launches).  Nothing throws, aborts or
 * exits across this interface.
 */
#ifndef PBLOCK_H
#define PBLOCK_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PB_BF16 = 0, PB_F32 = 1 } pb_dtype;

typedef enum {
  PB_OK = 0,
  PB_ERR_INVALID_ARG = 1, /* null/misaligned pointer, non-positive size ... */
  PB_ERR_UNSUPPORTED = 2, /* a shape this build has no kernel for          */
  PB_ERR_WORKSPACE = 3,   /* workspace smaller than pblock_workspace_bytes */
  PB_ERR_HIP = 4          /* a kernel launch failed                        */
} pb_status;

typedef struct {
  int batch;     /* >= 1                                                    */
  int seq;       /* >= 1                                                    */
  int hidden;    /* H >= 8, multiple of 8, <= 32768                         */
  int heads;     /* >= 1                                                    */
  int head_dim;  /* 64, 96 or 128                                           */
  int ffn;       /* F >= 8, multiple of 8                                   */
  int window;    /* >= 1; keys seen per query, itself included              */
  float ln_eps;  /* > 0, e.g. 1e-5                                          */
  int gelu_tanh; /* 1: tanh form of GeLU, 0: erf form                      */
  pb_dtype dtype;/* storage type of activations and parameters              */
} pb_config;

/* Checks a configuration on the host.  Makes no HIP call. */
pb_status pblock_validate(const pb_config* cfg);

/* Bytes of the forward -> backward stash described above (0 on a bad cfg). */
size_t pblock_saved_bytes(const pb_config* cfg);

/* Byte offsets of the stash regions, in the order h, z, c, mean, rstd, lse.
 * offsets must hold 6 entries.  Host only. */
pb_status pblock_saved_offsets(const pb_config* cfg, size_t* offsets);

/* Workspace sizes.  mode:
 *   PB_WS_FORWARD             pblock_forward with a caller stash (saved != NULL)
 *   PB_WS_FORWARD_WITH_STASH  pblock_forward with saved == NULL: the stash is
 *                             kept at the start of ws
 *   PB_WS_BACKWARD            pblock_backward
 * The sizes include a region for the partial tiles of GEMMs split along K
 * (the last, partial wave of output tiles, or all tiles of a small grid, so
 * the chip stays full; fp32 and bf16, also inside shared launches).
 * That region is optional: a smaller ws (down to 0 bytes for PB_WS_FORWARD,
 * the stash for PB_WS_FORWARD_WITH_STASH, and the size without the region
 * for PB_WS_BACKWARD) also works, unsplit (results then differ only in
 * rounding order).  0 on a bad cfg. */
enum { PB_WS_FORWARD_WITH_STASH = 0, PB_WS_BACKWARD = 1, PB_WS_FORWARD = 2 };
size_t pblock_workspace_bytes(const pb_config* cfg, int mode);

/* Steps of the forward and backward passes, for the *_timed calls. */
typedef enum {
  PB_STEP_LN_FWD = 0, /* LayerNorm of x                                     */
  PB_STEP_IN_PROJ,    /* Z = h W_in^T + b_in, G = gelu(U)                   */
  PB_STEP_ATTN_FWD,   /* sliding-window attention, O and lse                */
  PB_STEP_OUT_PROJ,   /* y = x + C W_out^T + b_out                          */
  PB_STEP_DC,         /* dC = dy W_out; dU = dC_mlp * gelu'(U)              */
  PB_STEP_DW_OUT,     /* dW_out = dy^T C                                    */
  PB_STEP_DB_OUT,     /* empty: db_out is summed with dgamma and dbeta in
                         the LN backward step's column sums              */
  PB_STEP_ATTN_BWD,   /* dQ, dK, dV                                         */
  PB_STEP_DH,         /* dh = dZ W_in                                       */
  PB_STEP_DW_IN,      /* dW_in = dZ^T h                                     */
  PB_STEP_DB_IN,      /* db_in = sum over tokens of dZ; empty when formed
                         in dW_in's launch, shared with dh or its own     */
  PB_STEP_LN_BWD,     /* dx = dy + LN backward; dgamma, dbeta, db_out       */
  PB_STEP_COUNT
} pb_step;

/* Per-call step events (benchmarking).  pblock_forward_timed and
 * pblock_backward_timed record begin[i] on their stream just before the
 * launches of step i and end[i] just after them; NULL entries, and a NULL
 * pb_step_events, are skipped.  The events belong to the caller and are
 * only recorded, never waited on.  A step whose work shares a launch with
 * another step records nothing between its events (PB_STEP_DW_OUT and
 * PB_STEP_DW_IN when pblock_backward_pairs reports the pair; PB_STEP_DB_IN
 * where dW_in's launch forms it; PB_STEP_DB_OUT always). */
typedef struct {
  hipEvent_t begin[PB_STEP_COUNT];
  hipEvent_t end[PB_STEP_COUNT];
} pb_step_events;

/* Forward pass of the block (Eq. 2).  Writes y [T, H].  When saved is not
 * NULL it also fills the stash that pblock_backward reads, and ws (NULL or
 * up to pblock_workspace_bytes(cfg, PB_WS_FORWARD) bytes) only holds GEMM
 * partial tiles.  When saved is NULL (inference) the stash goes to the start
 * of ws, which must then hold at least the stash
 * (pblock_workspace_bytes(cfg, PB_WS_FORWARD_WITH_STASH) for full speed). */
pb_status pblock_forward(const pb_config* cfg, const void* x,
                         const void* ln_gamma, const void* ln_beta,
                         const void* w_in, const void* b_in,
                         const void* w_out, const void* b_out,
                         void* y, void* saved, void* ws, size_t ws_bytes,
                         hipStream_t stream);
/* pblock_forward, recording step_ev (NULL: none) around each step. */
pb_status pblock_forward_timed(const pb_config* cfg, const void* x,
                               const void* ln_gamma, const void* ln_beta,
                               const void* w_in, const void* b_in,
                               const void* w_out, const void* b_out,
                               void* y, void* saved, void* ws,
                               size_t ws_bytes, hipStream_t stream,
                               const pb_step_events* step_ev);

/* Byte offsets, within the backward workspace, of the intermediates that
 * pblock_backward leaves there, in the order:
 *   d_o [T, A]     act  the attention output's gradient (dC[:, :A])
 *   dz  [T, N_in]  act  dQ | dK | dV | dU, the in-projection's output
 *                       gradient (dQ, dK, dV from the attention backward)
 *   dh  [T, H]     act  the LayerNorm output's gradient
 *   delta [batch, heads, seq] fp32  the attention backward's row terms
 *                       rowsum(dO O) per head
 * They hold these values once the backward call has passed on its stream,
 * until the workspace is used again.  offsets must hold 4 entries.  Host
 * only; for inspection and tests. */
pb_status pblock_workspace_offsets(const pb_config* cfg, size_t* offsets);

/* Backward pass: the gradients of sum(y * dy) with respect to x and every
 * parameter, given the stash of the matching forward call.  dx is in the
 * activation dtype; the six parameter gradients are fp32 and overwritten.
 * ws should hold pblock_workspace_bytes(cfg, PB_WS_BACKWARD) bytes (fewer,
 * down to the size without the GEMM partial-tile region, also works).
 * Where dC and dW_out (dh and dW_in) share a launch of whole 256 x 256 tiles,
 * that launch is persistent: one workgroup per CU takes tiles from per-XCD
 * queues whose heads live in ws and are zeroed by the call itself, so ws
 * needs no initialisation and two calls in flight at once need separate
 * workspaces (as for every other region of ws). */
pb_status pblock_backward(const pb_config* cfg, const void* x,
                          const void* ln_gamma, const void* ln_beta,
                          const void* w_in, const void* b_in,
                          const void* w_out, const void* b_out,
                          const void* saved, const void* dy, void* dx,
                          float* dgamma, float* dbeta, float* dw_in,
                          float* db_in, float* dw_out, float* db_out,
                          void* ws, size_t ws_bytes, hipStream_t stream);
/* pblock_backward, recording step_ev (NULL: none) around each step. */
pb_status pblock_backward_timed(const pb_config* cfg, const void* x,
                                const void* ln_gamma, const void* ln_beta,
                                const void* w_in, const void* b_in,
                                const void* w_out, const void* b_out,
                                const void* saved, const void* dy, void* dx,
                                float* dgamma, float* dbeta, float* dw_in,
                                float* db_in, float* dw_out, float* db_out,
                                void* ws, size_t ws_bytes, hipStream_t stream,
                                const pb_step_events* step_ev);

/* ------------------------------------------------------- launch planning
 * Host-only queries of how the calls above launch their GEMMs (for
 * benchmarks and profilers that attribute kernel time to steps).  They make
 * no HIP call.
 *
 * pblock_gemm_plan: the launch of one GEMM C[M, N] = A[M, K] B[K, N] in
 * dtype, given a full GEMM workspace (as the block's calls have).  256 x 256
 * output tiles; when the last wave of tiles is partial (or the whole grid is
 * smaller than the 256 compute units), each of its `tail` tiles is split
 * into `splits` K-slices whose fp32 partial tiles a second kernel sums.
 * Small bf16 grids take whole 64 x 64 tiles instead (tiles counts those).
 * Fills tiles, n_full (tiles computed whole), tail, splits (1: no split),
 * workgroups (of the GEMM kernel: n_full + tail * splits) and threads (per
 * workgroup).  fp32 GEMMs have tiles of 64 x 64, all of them split along K
 * where that is estimated to be faster (n_full is 0 then, and tail counts the
 * 256 x 256 blocks of the output that the workspace holds `splits` times), or,
 * in small grids, whole tiles of 16 x 64.
 *
 * pblock_backward_pairs: which backward GEMMs share one launch with the
 * weight-gradient GEMM after them (1) or launch alone (0).  block 0, the
 * parallel block: paired[0] = dC with dW_out, paired[1] = dh with dW_in.
 * block 1, the serial block: paired[0..3] = dG with dW_down, dh2 with
 * dW_up, dO with dW_o, dh1 with dW_qkv.  A shared launch of whole tiles has
 * one workgroup per tile of either GEMM, or one per CU where it is
 * persistent; where the first GEMM's few tiles are split along K it has one
 * per slice of each, and the smallest pairs take 64 x 64 tiles. */
typedef struct {
  int tiles, n_full, tail, splits, workgroups, threads;
} pb_gemm_plan;
pb_status pblock_gemm_plan(pb_dtype dtype, int M, int N, int K,
                           pb_gemm_plan* plan);
pb_status pblock_backward_pairs(const pb_config* cfg, int block, int* paired);

/* How the pairs of pblock_backward_pairs launch (same block and order; host
 * only) when the backward call is given a workspace of ws_bytes: apart, or
 * together in whole 256 x 256 tiles, in 256 x 256 tiles with each of the first
 * GEMM's cut into `splits` K-slices, or in 64 x 64 tiles.  splits is 1 unless
 * the kind is PB_PAIR_SPLIT. */
typedef enum { PB_PAIR_APART = 0, PB_PAIR_WHOLE, PB_PAIR_SPLIT, PB_PAIR_SMALL } pb_pair_kind;
typedef struct {
  int kind, splits;
} pb_pair_launch;
pb_status pblock_backward_launches(const pb_config* cfg, int block, size_t ws_bytes,
                                   pb_pair_launch* launch);

/* ---------------------------------------------------------- serial block
 * The standard pre-LN block that Eq. 2 replaces (Section 3.1, Eq. 1), for
 * comparison and for models that keep it:
 *
 *     x1 = x + Attention(LN1(x)) W_o^T + b_o
 *     y  = x1 + gelu(LN2(x1) W_up^T + b_up) W_down^T + b_down
 *
 * The second residual adds x1 (the paper's printed Eq. 1 writes x there; the
 * block it describes, and the one this computes, carries x1).  Weights use
 * the parallel block's packed layouts as slices: W_qkv = w_in rows 0..3A-1,
 * W_up = rows 3A..N_in-1 (b_in likewise); W_o = w_out columns 0..A-1, W_down
 * = columns A..K_out-1.  Two LayerNorms (ln1_*, ln2_*, activation dtype [H])
 * and two output biases (b_o, b_down, activation dtype [H]); the same window
 * rule, scaling, LayerNorm and GeLU as above.
 *
 * Stash regions, in this order, each at a 256-byte boundary
 * (pblock_serial_saved_offsets, 10 entries):
 *   h1 [T, H] act, z [T, N_in] act (Q | K | V | U), c [T, K_out] act (O | G),
 *   mean1 [T] fp32, rstd1 [T] fp32, lse [batch, heads, seq] fp32,
 *   x1 [T, H] act, h2 [T, H] act, mean2 [T] fp32, rstd2 [T] fp32.
 *
 * Workspace modes, ownership, asynchrony and errors are those of the
 * parallel block's calls (pblock_serial_workspace_bytes takes the same
 * PB_WS_* modes).  Gradients dln1_*, dln2_*, dw_in, db_in, dw_out, db_o,
 * db_down are fp32, in the layouts of their parameters, and overwritten. */
size_t pblock_serial_saved_bytes(const pb_config* cfg);
pb_status pblock_serial_saved_offsets(const pb_config* cfg, size_t* offsets);
size_t pblock_serial_workspace_bytes(const pb_config* cfg, int mode);
pb_status pblock_serial_forward(const pb_config* cfg, const void* x,
                                const void* ln1_gamma, const void* ln1_beta,
                                const void* ln2_gamma, const void* ln2_beta,
                                const void* w_in, const void* b_in,
                                const void* w_out, const void* b_o,
                                const void* b_down, void* y, void* saved,
                                void* ws, size_t ws_bytes, hipStream_t stream);
pb_status pblock_serial_backward(const pb_config* cfg, const void* x,
                                 const void* ln1_gamma, const void* ln1_beta,
                                 const void* ln2_gamma, const void* ln2_beta,
                                 const void* w_in, const void* b_in,
                                 const void* w_out, const void* b_o,
                                 const void* b_down, const void* saved,
                                 const void* dy, void* dx, float* dln1_gamma,
                                 float* dln1_beta, float* dln2_gamma,
                                 float* dln2_beta, float* dw_in, float* db_in,
                                 float* dw_out, float* db_o, float* db_down,
                                 void* ws, size_t ws_bytes, hipStream_t stream);

/* Causal sliding-window attention alone (Section 3.1 SWA; the exact
 * FlashAttention-2 result of Section 3.3), for all heads of all batch rows.
 * q, k, v: element (b, s, head, e) at ptr[(b*seq + s)*ld + head*head_dim + e],
 * ld in elements (>= heads*head_dim, multiple of 8).  o uses ld_o the same
 * way.  lse [batch, heads, seq] fp32 as in the stash.  Reads cfg->batch, seq,
 * heads, head_dim, window and dtype only.
 *
 * Workspace (pblock_swattn_workspace_bytes, by mode):
 *   PB_ATTN_WS_FORWARD      optional space for the forward: when batch*heads
 *                           is too small to fill the GPU, the key range of
 *                           each query block is split over several
 *                           workgroups whose fp32 partial results are merged
 *                           afterwards.  ws may be NULL (or smaller), which
 *                           runs unsplit; 0 means no split is planned.
 *   PB_ATTN_WS_BACKWARD_MIN bytes the backward requires (one fp32 softmax row
 *                           term per query).
 *   PB_ATTN_WS_BACKWARD     the same plus the split backward's partials; any
 *                           size from _MIN up works, below this one unsplit.
 * Results of the split and unsplit runs agree to fp32 rounding; each is
 * deterministic (fixed merge order, no atomics). */
enum { PB_ATTN_WS_FORWARD = 0, PB_ATTN_WS_BACKWARD_MIN = 1, PB_ATTN_WS_BACKWARD = 2 };
size_t pblock_swattn_workspace_bytes(const pb_config* cfg, int mode);
pb_status pblock_swattn_forward(const pb_config* cfg, const void* q,
                                const void* k, const void* v, int ld_qkv,
                                void* o, int ld_o, float* lse, void* ws,
                                size_t ws_bytes, hipStream_t stream);

/* pblock_swattn_forward without a workspace, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation).  Same arguments, layouts and results as
 * pblock_swattn_forward with a full PB_ATTN_WS_FORWARD workspace (the same
 * kernels and split plan; bitwise the same output).  The split partials
 * live in a device array inside the library, PB_NOALLOC_SCRATCH_BYTES per
 * GPU, held from the first call on that GPU (made with it current) until the
 * process ends.  Nothing is allocated per call and nothing in it needs
 * clearing.  A shape whose split plan needs more scratch than that is
 * rejected with PB_ERR_UNSUPPORTED before any HIP call.  Every call on one
 * GPU shares that GPU's scratch: calls that overlap on one GPU (on
 * different streams, or from several host threads) race and must be
 * ordered by the caller. */
#define PB_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)
pb_status pblock_swattn_forward_noalloc(const pb_config* cfg, const void* q,
                                        const void* k, const void* v,
                                        int ld_qkv, void* o, int ld_o,
                                        float* lse, hipStream_t stream);

/* Gradient of pblock_swattn_forward: given q, k, v, o (ld_o), lse and the
 * output gradient d_o (ld_do), writes dq, dk, dv (ld_dqkv).  ws: see above
 * (at least PB_ATTN_WS_BACKWARD_MIN bytes, else PB_ERR_WORKSPACE). */
pb_status pblock_swattn_backward(const pb_config* cfg, const void* q,
                                 const void* k, const void* v, int ld_qkv,
                                 const void* o, int ld_o, const void* d_o,
                                 int ld_do, const float* lse, void* dq,
                                 void* dk, void* dv, int ld_dqkv, void* ws,
                                 size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------ tensor-parallel context
 * The HIP events with which pblock_ag_in_proj and pblock_rs_out_proj order
 * their copy streams against the GEMM stream, created by
 * pblock_tp_context_create on the device current at that call, with timing
 * disabled.  A context serves calls with the same tp on that device, one
 * after another (re-recording an event between calls is safe: a stream
 * that waits on it has already taken the earlier state); calls from several
 * host threads need one context each.  pblock_tp_context_destroy may be
 * called once the calls that used it have been issued (HIP keeps a recorded
 * event alive until its work has passed); NULL is ignored.
 * Errors: PB_ERR_INVALID_ARG for tp outside 1..64 or ctx NULL, PB_ERR_HIP
 * when an event cannot be created (nothing is left allocated). */
typedef struct pb_tp_context pb_tp_context;
pb_status pblock_tp_context_create(int tp, pb_tp_context** ctx);
void pblock_tp_context_destroy(pb_tp_context* ctx);

/* How the pipelined calls below copy a shard or chunk from src to dst (host
 * only): *by_kernel is 1 for a copy kernel, used where both are memory that
 * this process allocated on the context's device, and 0 for the DMA engines
 * (peers' memory opened by IPC handles, and anything else).  The copies of one
 * launch on one comm stream take the kernel only where it holds for all. */
pb_status pblock_tp_copies_by_kernel(const pb_tp_context* ctx, const void* src,
                                     const void* dst, int* by_kernel);

/* ------------------------------------------- in-projection + all-gather
 * Section 3.2 ("Overlapping in tensor/sequence parallelism", Fig. 3):
 * under sequence parallelism the LayerNorm output h is sharded along the
 * tokens over tp ranks and all-gathered before the column-parallel
 * in-projection; the paper breaks that GEMM into chunks and pipelines them
 * with the communication.  Here the shards are copied into h on the comm
 * streams in ring order from `rank` (rank, rank + 1, ...; the k-th on
 * comm_streams[k % n_comm]), and the in-projection runs on `stream` in
 * launches of shards_per_launch shards each, every launch waiting (by
 * event) only for its own shards.  Shards already in place at the head of
 * that order (this rank's own LayerNorm output, say) need no copy and form
 * a first launch of their own, which runs while the first copies land.
 * shards_per_launch = tp is the unpipelined order: all copies, then one
 * GEMM.
 *
 * shards[j]: rank j's rows of h, [T / tp, H] in the activation dtype (on
 *   one GPU, buffers in local memory; across GPUs, peer memory opened by IPC
 *   handles).  A shard already in place (shards[j] == h + j (T / tp) H) is
 *   not copied.  h: [T, H], the gathered LN output.
 * z [T, N_in], c [T, K_out]: written as pblock_forward writes the stash's
 *   Z and the G half of C (bias, and GeLU of the MLP-up columns); the
 *   result does not depend on tp, rank or the launch grouping beyond the
 *   rounding of K-split tiles.
 * Requirements: T % tp == 0, 1 <= tp <= 64, 0 <= rank < tp,
 *   1 <= shards_per_launch <= tp, 1 <= n_comm <= 8, comm streams distinct
 *   from each other and from `stream`.
 * ws: optional GEMM split region of pblock_ag_in_proj_workspace_bytes(cfg,
 *   tp, shards_per_launch) bytes (NULL/0 runs every launch unsplit).
 * ctx: a pb_tp_context made for this tp on the current device.
 * The copies start after the work already on `stream`; later work on
 *   `stream` follows every copy and GEMM. */
size_t pblock_ag_in_proj_workspace_bytes(const pb_config* cfg, int tp,
                                         int shards_per_launch);
pb_status pblock_ag_in_proj(const pb_config* cfg, int tp, int rank,
                            const void* const* shards, void* h,
                            const void* w_in, const void* b_in, void* z,
                            void* c, int shards_per_launch, void* ws,
                            size_t ws_bytes, hipStream_t stream, int n_comm,
                            const hipStream_t* comm_streams,
                            pb_tp_context* ctx);

/* The same overlap in the backward pass (the mirror of the forward's
 * reduce-scatter): the output gradient dy arrives sharded along the tokens
 * and is all-gathered before dC = dy W_out, the first GEMM of the backward.
 * pblock_ag_dc copies dy_shards[j] ([T / tp, H], rank j's rows) into dy
 * [T, H] exactly as pblock_ag_in_proj copies the LayerNorm shards, and runs
 * dC over groups of shards_per_launch landed shards, writing d_o [T, A]
 * (= dC[:, :A]) and the MLP part of dz [T, N_in] (dz[:, 3A:] = dC[:, A:] *
 * gelu'(U), U read from z [T, N_in], the stash's Z) as pblock_backward
 * writes them.  w_out [H, K_out] as in pblock_forward.  Requirements, ws
 * (pblock_ag_dc_workspace_bytes) and ctx as for pblock_ag_in_proj.  The
 * weight gradient dW_out = dy^T C needs every shard and is left to the
 * caller (after the call, dy holds them all). */
size_t pblock_ag_dc_workspace_bytes(const pb_config* cfg, int tp,
                                    int shards_per_launch);
pb_status pblock_ag_dc(const pb_config* cfg, int tp, int rank,
                       const void* const* dy_shards, void* dy,
                       const void* w_out, const void* z, void* d_o, void* dz,
                       int shards_per_launch, void* ws, size_t ws_bytes,
                       hipStream_t stream, int n_comm,
                       const hipStream_t* comm_streams, pb_tp_context* ctx);

/* --------------------------------------- out-projection + reduce-scatter
 * Section 3.2 ("Overlapping in tensor/sequence parallelism", Fig. 3), the
 * other half of the pattern above: after the row-parallel out-projection
 * every rank holds a partial sum P_r = C_r W_out,r^T of every token row
 * (C_r, W_out,r: its own columns of the out-projection input and weight),
 * and a reduce-scatter leaves rank j with the sum over ranks of its own
 * rows.  The paper pipelines that GEMM in chunks with the communication.
 *
 * pblock_rs_out_proj (the sending side of rank `rank`) computes P_r on
 * `stream` in row chunks of T / tp rows, in ring order from rank + 1 (this
 * rank's own chunk last), shards_per_launch chunks per launch; each chunk
 * j is copied to dst[j] on comm_streams[k % n_comm] (k its position in that
 * order) as soon as its launch has finished.  shards_per_launch = tp is the
 * unpipelined order: one GEMM, then all copies.
 *   c [T, K_out], w_out [H, K_out]: as in pblock_forward, in the activation
 *     dtype; cfg describes this rank's share (A, F its own widths).
 *   partial [T, H]: P_r in the activation dtype (rounded from the fp32
 *     accumulation).  dst[j]: [T / tp, H], where rank j receives this
 *     rank's chunk (on one GPU, local buffers; across GPUs, peer memory
 *     opened by IPC handles).  A chunk already in place (dst[j] == partial
 *     + j (T / tp) H) is not copied.
 *   Requirements as for pblock_ag_in_proj; ws: optional GEMM split region
 *   of pblock_rs_out_proj_workspace_bytes(cfg, tp, shards_per_launch)
 *   bytes (NULL/0 runs every launch unsplit); ctx as for pblock_ag_in_proj.
 *   Later work on `stream` follows every GEMM and copy.
 *
 * pblock_rs_reduce (the receiving side of one rank): y_shard = x_shard +
 * b_out + sum over q = 0 .. tp-1 of parts[q], summed in fp32 in the order
 * of q and rounded once; parts[q], x_shard, y_shard: [T / tp, H] in the
 * activation dtype, 16-byte aligned; b_out: [H].  x_shard and b_out may
 * each be NULL (left out of the sum).  With parts[q] the chunk
 * rank q sent here, y_shard is this rank's rows of the block output of
 * Eq. 2 (the out-projection of all ranks, the bias and the residual). */
size_t pblock_rs_out_proj_workspace_bytes(const pb_config* cfg, int tp,
                                          int shards_per_launch);
pb_status pblock_rs_out_proj(const pb_config* cfg, int tp, int rank,
                             const void* c, const void* w_out, void* partial,
                             void* const* dst, int shards_per_launch, void* ws,
                             size_t ws_bytes, hipStream_t stream, int n_comm,
                             const hipStream_t* comm_streams,
                             pb_tp_context* ctx);

/* The backward's mirror of the forward's all-gather: the column-parallel
 * in-projection leaves every rank a partial sum of the LayerNorm output's
 * gradient, dh_r = dZ_r W_in,r (dZ_r, W_in,r: its own columns of dZ and
 * rows of W_in), and a reduce-scatter leaves rank j the sum of its own rows
 * (the sequence-parallel dh that the LayerNorm backward of its shard needs).
 * pblock_rs_dh computes dh_r = dz [T, N_in] w_in [N_in, H] into partial
 * [T, H] (activation dtype) in row chunks and sends them to dst exactly as
 * pblock_rs_out_proj does; the receiving side is pblock_rs_reduce with
 * x_shard = b_out = NULL.  Requirements, ws (pblock_rs_dh_workspace_bytes)
 * and ctx as for pblock_rs_out_proj. */
size_t pblock_rs_dh_workspace_bytes(const pb_config* cfg, int tp,
                                    int shards_per_launch);
pb_status pblock_rs_dh(const pb_config* cfg, int tp, int rank, const void* dz,
                       const void* w_in, void* partial, void* const* dst,
                       int shards_per_launch, void* ws, size_t ws_bytes,
                       hipStream_t stream, int n_comm,
                       const hipStream_t* comm_streams, pb_tp_context* ctx);
pb_status pblock_rs_reduce(const pb_config* cfg, int tp,
                           const void* const* parts, const void* x_shard,
                           const void* b_out, void* y_shard,
                           hipStream_t stream);

/* ------------------------------------------------------------- LAMB step
 * One step of the LAMB optimizer the paper trains with (Section 3.1, "LAMB
 * optimizer"; the layer-wise method of You et al., 2020) over up to
 * PB_LAMB_MAX_TENSORS tensors, each its own trust-ratio "layer".  For each
 * tensor, with t = cfg->step:
 *
 *   g  = grad_scale * grad
 *   m  = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   u  = (m / c1) / (sqrt(v / c2) + eps) + weight_decay * w
 *        c1 = 1 - beta1^t, c2 = 1 - beta2^t (1 and 1 when bias_correction = 0)
 *   r  = ||w|| / ||u|| over the whole tensor (1 if either norm is 0)
 *   w  = w - lr * r * u
 *
 * param, exp_avg (m) and exp_avg_sq (v) are fp32 and updated in place; grad
 * is fp32 (as pblock_backward writes it).  param_copy, when not NULL,
 * receives the updated weights in copy_dtype (bf16: round to nearest even),
 * e.g. the block's bf16 parameters.  Every pointer is device memory, 16-byte
 * aligned; the five arrays of a tensor must not overlap.  trust_ratio, when
 * not NULL, is a device array of n_tensors floats that receives r.
 * Tensors with numel = 0 are allowed (nothing is touched).  More tensors:
 * call again; tensors are independent, so the result is the same.
 *
 * ws must hold pblock_lamb_workspace_bytes(n_tensors, tensors) bytes (per-
 * chunk partial norms and the ratios).  Asynchronous on the stream; the
 * result does not depend on timing (fixed reduction order, no atomics).
 * Errors: PB_ERR_INVALID_ARG for a bad config (lr or grad_scale not finite,
 * beta outside [0, 1), eps <= 0, step < 1, negative or non-finite decay,
 * n_tensors outside 1..16), a NULL or misaligned pointer, or too many
 * elements; PB_ERR_WORKSPACE for a small ws. */
#define PB_LAMB_MAX_TENSORS 16
typedef struct {
  float lr;
  float beta1, beta2;
  float eps;
  float grad_scale;
  int step;            /* t >= 1 */
  int bias_correction; /* 0 or 1 */
} pb_lamb_config;
typedef struct {
  float* param;        /* [numel] fp32 master weights */
  const float* grad;   /* [numel] fp32 */
  float* exp_avg;      /* [numel] fp32 */
  float* exp_avg_sq;   /* [numel] fp32 */
  void* param_copy;    /* NULL or [numel] in copy_dtype */
  size_t numel;
  float weight_decay;  /* lambda of this tensor (0 for biases and norms, say) */
} pb_lamb_tensor;
size_t pblock_lamb_workspace_bytes(int n_tensors, const pb_lamb_tensor* tensors);
pb_status pblock_lamb_step(const pb_lamb_config* cfg, int n_tensors,
                           const pb_lamb_tensor* tensors, pb_dtype copy_dtype,
                           float* trust_ratio, void* ws, size_t ws_bytes,
                           hipStream_t stream);

/* ------------------------------------------------------- rotary positions
 * The block has no positional terms of its own, and pblock_forward and
 * pblock_backward run from their inputs to their outputs, with no place for another
 * operator between their steps.  A block with rotated Q and K is put together from the
 * calls of its parts (with tp = 1 on one GPU): pblock_ag_in_proj, pblock_rope_forward on
 * Q and K of the packed Z, pblock_swattn_forward, pblock_rs_out_proj, pblock_rs_reduce;
 * and pblock_ag_dc, pblock_swattn_backward, pblock_rope_backward on dQ and dK of the
 * packed dZ, pblock_rs_dh.  Z then holds the rotated Q and K, and dZ the gradients of
 * the unrotated ones; the weights' gradients, dZ^T h and dy^T C, are the caller's.  (A
 * root-mean-square norm, below, takes its place before and after these in the same way.)
 *
 * The leading rot_dim elements of each head turn in pairs, i = 0 .. rot_dim/2 - 1:
 * elements (2i, 2i + 1) when interleaved, else (i, i + rot_dim/2), with
 *
 *   f_i = base^(-2i / rot_dim)                    PB_ROPE_PLAIN
 *   f_i / factor                                  PB_ROPE_LINEAR
 *   f_i (g + (1 - g) / factor)                    PB_ROPE_BY_PARTS
 *       g = clamp((orig_len f_i / 2 pi - low_turns) / (high_turns - low_turns), 0, 1)
 *   t = position f_i
 *   forward:   (y_a, y_b) = magnitude (x_a cos t - x_b sin t, x_b cos t + x_a sin t)
 *   backward:  the transposed map (t negated, the same magnitude): from the
 *              gradient of y to that of x
 *
 * By parts: pairs that turn often within the trained length orig_len keep their
 * frequency, the slow ones are interpolated (Peng et al. 2023); magnitude is the
 * attention's rescaling that goes with it (1 for none).  The other elements of a
 * head are passed through.  Angles are formed in 64 bits; sine, cosine (good to 1.5
 * 2^-24) and the rotation in 32, rounded once.
 *
 * tensors[k] (1 to PB_ROPE_MAX_TENSORS, e.g. Q and K, of their own head counts):
 *   element (token, head, e) of in at in[token*ld_in + head*head_dim + e], ld_in in
 *   elements (>= heads*head_dim), out likewise.  out may be in with ld_out = ld_in
 *   (in place; elements past rot_dim are then left alone); otherwise no memory of
 *   any out may be in any other in or out or in positions (refused; tensors may
 *   interleave row by row).  Pointers are aligned to the element;
 *   16-byte aligned pieces (head_dim, ld and rot_dim, or rot_dim/2 when not
 *   interleaved, multiples of 16 bytes) run fastest.
 * positions: int64 per token, device memory, any value (negative ones turn the
 *   other way; beyond 2^31 the angles lose accuracy).  NULL: token t is at position
 *   t mod seq.  seq is read only then.
 * tokens may be 0 (nothing is launched, and no pointer, position or seq is needed).
 * Errors: PB_ERR_INVALID_ARG for a bad config (a frequency that is not finite among
 * them) or pointer, PB_ERR_UNSUPPORTED for head_dim > 256, or too many tokens or heads. */
#define PB_ROPE_MAX_TENSORS 4
typedef enum { PB_ROPE_PLAIN = 0, PB_ROPE_LINEAR = 1, PB_ROPE_BY_PARTS = 2 } pb_rope_scaling;
typedef struct {
  int head_dim;      /* even, 2 .. 256                                        */
  int rot_dim;       /* even, 2 .. head_dim                                   */
  int interleaved;   /* 0 or 1                                                */
  int scaling;       /* pb_rope_scaling                                       */
  double base;       /* > 0, finite                                           */
  double factor;     /* > 0, finite; not read by PB_ROPE_PLAIN                */
  double orig_len;   /* > 0; this and the next two by PB_ROPE_BY_PARTS only   */
  double low_turns;  /* 0 <= low_turns < high_turns                           */
  double high_turns;
  double magnitude;  /* > 0, finite, in fp32                                  */
  pb_dtype dtype;
} pb_rope_config;
typedef struct {
  const void* in;
  void* out;
  size_t ld_in, ld_out;
  int heads;         /* 1 .. 8192                                             */
} pb_rope_tensor;
pb_status pblock_rope_forward(const pb_rope_config* cfg, int n_tensors,
                              const pb_rope_tensor* tensors, int64_t tokens,
                              int64_t seq, const int64_t* positions,
                              hipStream_t stream);
pb_status pblock_rope_backward(const pb_rope_config* cfg, int n_tensors,
                               const pb_rope_tensor* tensors, int64_t tokens,
                               int64_t seq, const int64_t* positions,
                               hipStream_t stream);

/* ------------------------------------------------- root-mean-square norm
 * Per row of a dense [rows, cols] matrix (any cols from 1 to 32768):
 *
 *   s = x + resid                    (resid NULL: s = x)
 *   r = 1 / sqrt(mean(s^2) + eps)
 *   y = s r gamma
 *
 * y is formed from the unrounded s, in 32 bits (64 with q8, and for the mean), and
 * rounded once.
 * Outputs, each left out when NULL, but y or q8 must be there:
 *   sum  [rows, cols] act   s rounded, the next residual (NULL unless resid is
 *                           given; may be x or resid)
 *   y    [rows, cols] act   (may be x or resid, whichever sum is not)
 *   q8   [rows, cols] OCP e4m3, with scales: q8 = y / scale rounded to fp32 and
 *        that to e4m3, each to nearest even (as a cast does),
 *        scale = max(max|y| / 448, 2^-126) in fp32 over each group of
 *        `group` columns of a row (32, 64 or 128; the last group of a row may be
 *        short) or over the row (0).  scales [rows, ceil(cols / group)] (or
 *        [rows]).  A NaN in y has a NaN code and is passed over by its scale; an
 *        infinite y (of an infinite gamma) makes its scale infinite, its own code
 *        NaN and the others of its group 0.
 *   rstd [rows] fp32        r, for the backward
 * gamma [cols] act.  A NaN in a row of s makes the row of y NaN, an infinity makes r 0:
 * y is NaN there and 0 beside it.  (eps 0: a row whose root mean square is under 3e-39,
 * past which r leaves fp32, is infinite or NaN; in q8 a row of zeros alone.)
 *
 * pblock_rmsnorm_backward: s [rows, cols] act is the forward's sum (x without a
 * residual), dy the gradient of y, dsum (may be NULL) the gradient that reaches s
 * from elsewhere (the residual's other use).  With g = dy gamma,
 *   dx = dsum + r (g - s r^2 mean(g s))   act: the gradient of x, and of resid
 *   dgamma = sum over rows of dy s r      [cols] fp32, overwritten; summed in fp32
 *            (off by 1e-7 of its norm at 8192 rows, 4e-7 at 10^6)
 * dx may be dy, dsum or s, as a whole.  Every other sharing of memory by an output
 * and another tensor (or ws) is refused, in both calls.  ws:
 * pblock_rmsnorm_workspace_bytes(cfg) bytes, 256-byte aligned, one for each call that
 * may overlap another.  Results do not depend on timing (fixed order, no atomics).
 *
 * Pointers are aligned to their element; cols a multiple of 8 with 16-byte aligned
 * pointers (8 for q8) runs fastest.  rows may be 0 (the backward then writes zeros
 * to dgamma).  Errors as above. */
typedef struct {
  int64_t rows;      /* 0 .. 2^31 - 1                                         */
  int cols;          /* 1 .. 32768                                            */
  int group;         /* q8 only: 0, 32, 64 or 128                             */
  float eps;         /* >= 0, finite                                          */
  pb_dtype dtype;
} pb_rmsnorm_config;
pb_status pblock_rmsnorm_forward(const pb_rmsnorm_config* cfg, const void* x,
                                 const void* resid, const void* gamma,
                                 void* sum, void* y, uint8_t* q8,
                                 float* scales, float* rstd,
                                 hipStream_t stream);
size_t pblock_rmsnorm_workspace_bytes(const pb_rmsnorm_config* cfg);
pb_status pblock_rmsnorm_backward(const pb_rmsnorm_config* cfg, const void* s,
                                  const void* gamma, const float* rstd,
                                  const void* dy, const void* dsum, void* dx,
                                  float* dgamma, void* ws, size_t ws_bytes,
                                  hipStream_t stream);

/* ------------------------------- attention with terms in its scores
 * Attention as a block with position biases, capped scores, packed documents or shared
 * key heads has it, next to pblock_swattn_forward / _backward (plain scores, causal
 * window, equal heads), whose place it takes among the calls of a block's parts.
 *
 * The seq_q queries of a batch row are the last of its seq_k positions: query i is at
 * p = i + seq_k - seq_q (seq_q = seq_k in training; 1 for a new token over kept keys).
 * Query head h reads key head h / (heads / kv_heads).
 *
 *   u = scale q.k
 *   c = cap tanh(u / cap)                           (cap 0: c = u)
 *   s = c - slopes[h] |p - j|                       with slopes
 *   s = c + table[bucket(p - j)][h]                 with a table
 *   P = softmax of s over the visible keys,  o = P v,  lse = log sum e^s
 *
 * Key j of the row is visible to query p when both are in one document and
 *   0 <= p - j < window (causal), or |p - j| < window (not causal),
 *   or j is in the document's prefix.
 * docs: n_docs + 1 ascending offsets into the batch * seq_k tokens; document d is
 *   tokens docs[d] .. docs[d + 1] - 1 (empty ones allowed), cut where a batch row ends.
 *   NULL: each batch row is a document, and n_docs is ignored.  Tokens before the first
 *   and behind the last document see nothing and are seen by none.
 * prefix: the leading tokens of each document ([n_docs], or [batch] without docs) that
 *   all its queries see, ahead of them or outside their window too.
 * Both are read on the device; offsets out of range are clamped (nothing outside the
 * tensors is touched).  What a mask hides does not enter any result, whatever it holds
 * (infinities and NaN too).  A query that sees nothing has o = 0, lse = -infinity and
 * no part in any gradient; so has one whose every score is -infinity.  A table entry
 * below -1e38 (the lowest value, as some programs mask with) counts as -infinity.
 *
 * bucket(n), of n = p - j: the first half of the buckets is of one distance each, the
 * others grow in the logarithm up to max_distance, from which on all is the last
 * bucket.  Causal: of max(n, 0), all buckets.  Not causal: of |n| among the first half
 * of the buckets where n >= 0, else among the second half.  With N buckets (of a side)
 * and E = N / 2, distance d >= E is in bucket
 *   E + floor((N - E) log(d / E) / log(max_distance / E)), at most N - 1,
 * in exact arithmetic: pblock_score_attn_borders gives the first distance of each
 * bucket (of a side; a bucket that no distance falls into has that of the next).
 *
 * Element (b, t, head, e) of a tensor is at ptr[(b*seq + t)*ld + head*head_dim + e],
 * in cfg->dtype, 16-byte aligned, ld in elements (>= its heads*head_dim, a multiple of
 * 16 bytes, < 2^24): q, o, d_o, dq with heads and seq_q; k, v, dk, dv with kv_heads and
 * seq_k.  lse [batch, heads, seq_q] fp32; slopes [heads], table and dtable [buckets,
 * heads] fp32.
 *
 * The backward gives the gradients of sum(o d_o): dq, dk, dv (dk and dv summed over the
 * heads that share a key head) and, when dtable is not NULL, dtable (fp32); all are
 * overwritten.  Where no query sees two keys (seq_k 1; window 1 without prefixes) dq, dk
 * and dtable are 0 to the bit.
 *
 * products, of PB_BF16 tensors (PB_F32 ones have fp32 products either way): the factors
 * that a call computes, P and its gradient, are not values of the type.  PB_F32 keeps 16
 * bits of them (a bf16 value and its remainder, two matrix products for one) and forms
 * the softmax's row term sum P dP from unrounded values, so that o, dq, dk and dv are
 * off by their own rounding.  PB_BF16 rounds them to bf16, and takes the row term from o
 * as it is kept (dtable has the unrounded one): as pblock_swattn_forward / _backward.
 * In norm, where a result's rounding alone is 1.66e-3, PB_BF16 gives o 1.7e-3 to 2.1e-3,
 * dv 2.1e-3 to 2.4e-3, dq and dk 2.6e-3 to 2.8e-3 over rows of 500 keys and more, 5.2e-3
 * over rows of two (normal values, scores of a standard deviation of 2; of 6: 4.4e-3).
 * Its forward takes 0.75 to 0.9 of PB_F32's time, its backward 0.63 to 0.75.
 * (A backward over a part of the rows' keys, with o and lse of all of them, needs the row
 * term from o: PB_BF16 or PB_F32 tensors; without dtable, and the latter without a table.)
 *
 * ws, 256-byte aligned, pblock_score_attn_workspace_bytes(cfg, mode): the PB_ATTN_WS_*
 * modes.  PB_ATTN_WS_FORWARD is optional as for pblock_swattn_forward (less runs
 * unsplit, the same result up to fp32 rounding), PB_ATTN_WS_BACKWARD_MIN is needed,
 * PB_ATTN_WS_BACKWARD for full speed.  Nothing in it outlives the call; calls that may
 * overlap (two captured graphs too) need one each.  Outputs may share no memory with any
 * other tensor of the call (refused).  Results do not depend on timing (fixed order, no
 * atomics between waves).
 *
 * Errors: PB_ERR_INVALID_ARG for a bad config, pointer or ld, PB_ERR_UNSUPPORTED for
 * another head_dim and for sizes past the kernels' (batch*seq_q*heads and
 * batch*seq_k*kv_heads <= 2^26, batch*heads <= 2^21, buckets*heads < 2^26), PB_ERR_WORKSPACE for a small ws. */
#define PB_SCORE_MAX_BUCKETS 64
typedef struct {
  int batch;         /* >= 1                                                  */
  int seq_q, seq_k;  /* 1 <= seq_q <= seq_k                                   */
  int heads;         /* a multiple of kv_heads                                */
  int kv_heads;      /* >= 1                                                  */
  int head_dim;      /* 64, 96 or 128                                         */
  int causal;        /* 0 or 1                                                */
  int window;        /* >= 1                                                  */
  float scale;       /* > 0, finite                                           */
  float cap;         /* 0 (none), or scale / 2^12 .. scale 2^120, <= 2^100    */
  int buckets;       /* 0 without a table; else 2 .. 64, or even, 4 .. 64,
                        when not causal                                       */
  int max_distance;  /* > half the buckets (of a side), <= 2^20               */
  pb_dtype dtype;
  pb_dtype products; /* PB_F32 or PB_BF16; of dtype PB_BF16                   */
} pb_score_attn_config;
/* What enters the scores beside q and k, in device memory; NULL where there is none.
 * At most one of slopes and table, which goes with cfg->buckets. */
typedef struct {
  const int32_t* docs;    /* [n_docs + 1]                                     */
  int n_docs;             /* >= 0                                             */
  const int32_t* prefix;  /* [n_docs], or [batch] without docs                */
  const float* slopes;    /* [heads]                                          */
  const float* table;     /* [buckets, heads]                                 */
} pb_score_terms;
/* first: an entry for each bucket (of a side, when not causal).  Host only. */
pb_status pblock_score_attn_borders(const pb_score_attn_config* cfg, int* first);
size_t pblock_score_attn_workspace_bytes(const pb_score_attn_config* cfg, int mode);
/* terms may be NULL (none). */
pb_status pblock_score_attn_forward(const pb_score_attn_config* cfg,
                                    const pb_score_terms* terms, const void* q,
                                    size_t ld_q, const void* k, const void* v,
                                    size_t ld_kv, void* o, size_t ld_o, float* lse,
                                    void* ws, size_t ws_bytes, hipStream_t stream);
pb_status pblock_score_attn_backward(const pb_score_attn_config* cfg,
                                     const pb_score_terms* terms, const void* q,
                                     size_t ld_q, const void* k, const void* v,
                                     size_t ld_kv, const void* o, size_t ld_o,
                                     const void* d_o, size_t ld_do, const float* lse,
                                     void* dq, size_t ld_dq, void* dk, void* dv,
                                     size_t ld_dkv, float* dtable, void* ws,
                                     size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------- Muon step
 * An optimizer step that treats each weight as a matrix (Jordan et al. 2024), next
 * to pblock_lamb_step: the momentum's update, made nearly orthogonal by `steps`
 * Newton-Schulz steps, moves the weight.  Per matrix, with g = grad_scale grad:
 *
 *   M = momentum M + g
 *   U = g + momentum M (nesterov), else M
 *   X = U / (||U||_F + eps)
 *   steps times: A = X X^T, X = a X + (b A + c A A) X,
 *                (a, b, c) = (3.4445, -4.7750, 2.0315)
 *   w = w (1 - lr weight_decay) - lr scale X
 *
 * (a matrix with more rows than columns goes through the products transposed; the
 * result is the same).  param, momentum and grad are fp32, param and momentum
 * updated in place; param_copy, when not NULL, receives the updated weights in
 * copy_dtype.  Each is [rows, cols] with ld elements from row to row: a slice of a
 * packed weight (rows of w_in; columns of w_out, ld = K_out) is a matrix of its
 * own.  scale is the caller's rule for the shape (0.2 sqrt(max(rows, cols)), say).
 * Matrices with rows = 0 or cols = 0 are allowed (nothing is touched).  No param,
 * momentum, param_copy or ws may share memory with another of them or with a grad
 * (refused; they may interleave row by row).
 *
 * products: PB_F32 carries 22 bits of every factor (each fp16 value with its
 * remainder, three matrix products for one).  PB_BF16 rounds the factors to fp16 (11
 * bits), one product: a step of 5120 x 5120 in 0.41 of PB_F32's time, of 2048 x 2048 in
 * 0.65, of 256 x 256 in 0.8.  Sums, norms, M and w are fp32 (or more) either way;
 * matrices with fewer than 64 rows or columns have PB_F32's products.  How far X is off
 * after five steps, as a share of its norm, grows with the spread of U's singular
 * values (which the steps raise up to 480 times, and roundings with them).  At most,
 * by the elements of the noise beside U's strongest directions as a share of theirs:
 *
 *                              PB_F32    PB_BF16   (in fp32)
 *   noise alone, or as large   5e-6      5e-3      1e-5
 *   a tenth                    5e-5      3e-2      3e-5
 *   a hundredth and less       5e-4      2e-1      6e-4      (U nearly of low rank)
 *
 * measured at 64 to 5120 rows, beside the same steps by fp32 library products.  Elements
 * of X are kept to 2^-40: an update whose norm is far below eps, which stays far from
 * orthogonal, is good to 2^-30 absolute.
 * Sizes and company decide tiles, cuts along K and whether steps go in pairs (which
 * moves X by up to 2.5 times the error of single ones): a matrix's last bits, with
 * PB_BF16 those within the table, may differ with the other matrices of the call.  The
 * same call gives the same bits.
 *
 * pblock_orthogonalize: X alone, from in to out (may be the same memory with the
 * same ld, else apart), both in dtype; PB_F32's products for either type, and the
 * result rounded once.
 *
 * ws: the *_workspace_bytes, 256-byte aligned; nothing in it outlives the call, and
 * calls that may overlap need one each (so do two captured graphs that may).
 * Errors: PB_ERR_INVALID_ARG for a bad config, size, pointer (aligned to its
 * element) or ld < cols, PB_ERR_UNSUPPORTED for a matrix too large, PB_ERR_WORKSPACE
 * for a small ws.  Results do not depend on timing (fixed order, no atomics). */
#define PB_MUON_MAX_TENSORS 16
typedef struct {
  float lr;            /* finite                                              */
  float momentum;      /* 0 <= momentum < 1                                   */
  float grad_scale;    /* finite                                              */
  float eps;           /* > 0, finite                                         */
  int nesterov;        /* 0 or 1                                              */
  int steps;           /* 1 .. 16                                             */
  pb_dtype products;
} pb_muon_config;
typedef struct {
  float* param;
  const float* grad;
  float* momentum;
  void* param_copy;    /* NULL or in copy_dtype                               */
  int rows, cols;      /* min <= 65536, max <= 2^20                           */
  size_t ld;           /* >= cols                                             */
  float weight_decay;  /* >= 0, finite                                        */
  float scale;         /* finite                                              */
} pb_muon_tensor;
size_t pblock_muon_workspace_bytes(const pb_muon_config* cfg, int n_tensors,
                                   const pb_muon_tensor* tensors);
pb_status pblock_muon_step(const pb_muon_config* cfg, int n_tensors,
                           const pb_muon_tensor* tensors, pb_dtype copy_dtype,
                           void* ws, size_t ws_bytes, hipStream_t stream);
typedef struct {
  const void* in;
  void* out;
  int rows, cols;
  size_t ld_in, ld_out;
} pb_ortho_tensor;
size_t pblock_orthogonalize_workspace_bytes(int n_tensors,
                                            const pb_ortho_tensor* tensors,
                                            pb_dtype dtype);
pb_status pblock_orthogonalize(int n_tensors, const pb_ortho_tensor* tensors,
                               pb_dtype dtype, int steps, float eps, void* ws,
                               size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------ AdamW step
 * One step of Adam with decoupled weight decay (Loshchilov and Hutter 2019) over many
 * tensors at once, next to pblock_lamb_step and pblock_muon_step (whose matrices leave
 * the biases, norm gains and bias tables to a step like this one).  Per element, with
 * t = cfg->step:
 *
 *   g = grad_scale grad
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   w = w (1 - lr weight_decay) - lr (m c1) / (sqrt(v c2) + eps)
 *       c1 = 1 / (1 - beta1^t), c2 = 1 / (1 - beta2^t) (1 and 1 without bias_correction)
 *
 * in fp32, each operation rounded by itself (one quotient in 2^32 to the next to
 * nearest).  param and grad are fp32, param updated in place; param_copy, when not NULL,
 * receives the updated weights in copy_dtype (bf16: round to nearest even).  state:
 *
 *   PB_ADAMW_F32   exp_avg is m and exp_avg_sq v, fp32.
 *   PB_ADAMW_E4M3  exp_avg holds m and exp_avg_sq sqrt(v) as OCP e4m3 codes, one byte
 *       an element, with fp32 scales for each PB_ADAMW_BLOCK elements (the last block may
 *       be short): value = code scale.  scale = max(largest magnitude (1 / 448), 2^-126)
 *       of the block's updated values, 1 / 448 rounded to fp32.  A code is one of the two
 *       neighbours of value / scale, the upper as often as it is near (a moving average
 *       that moves by less than half a code's step would stand still under rounding to
 *       nearest).  sqrt(v) above 0 keeps a code above 0.  Which one is taken follows from
 *       16 bits of a hash of (seed, number of the element), the upper half of 32 for m and
 *       the lower for sqrt(v): the same seed gives the same codes, so give each tensor and
 *       step its own.  The step itself uses the updated values before they are rounded.
 *       All zeros (codes and scales) are states of zero.  A value that is not finite makes
 *       its block's scale infinite or NaN, and the block's states with it.
 *
 * A captured step replays with the lr, step and seeds that it was captured with.
 * Pointers are aligned to their element.  numel may be 0 (nothing is touched).  No
 * array that is written may share memory with another array of the call (refused).
 * Any number of tensors from 1 to PB_ADAMW_MAX_TENSORS, 48 in a launch; results do not
 * depend on how tensors are divided over calls.  No workspace.
 * Errors: PB_ERR_INVALID_ARG for a bad config, pointer or decay, PB_ERR_UNSUPPORTED for
 * a tensor of more than 2^34 - 2^10 elements. */
#define PB_ADAMW_MAX_TENSORS 1024
#define PB_ADAMW_BLOCK 256
typedef enum { PB_ADAMW_F32 = 0, PB_ADAMW_E4M3 = 1 } pb_adamw_state;
typedef struct {
  float lr;            /* finite                                              */
  float beta1, beta2;  /* 0 <= beta < 1                                       */
  float eps;           /* > 0, finite                                         */
  float grad_scale;    /* finite                                              */
  int step;            /* t >= 1                                              */
  int bias_correction; /* 0 or 1                                              */
  int state;           /* pb_adamw_state                                      */
} pb_adamw_config;
typedef struct {
  float* param;        /* [numel] fp32                                        */
  const float* grad;   /* [numel] fp32                                        */
  void* exp_avg;       /* [numel] fp32, or e4m3 codes                         */
  void* exp_avg_sq;    /* [numel] fp32, or e4m3 codes of the root             */
  float* avg_scale;    /* [ceil(numel / PB_ADAMW_BLOCK)], PB_ADAMW_E4M3 only  */
  float* sq_scale;     /* the same                                            */
  void* param_copy;    /* NULL or [numel] in copy_dtype                       */
  size_t numel;
  uint64_t seed;       /* of the codes' rounding, PB_ADAMW_E4M3 only          */
  float weight_decay;  /* >= 0, finite                                        */
} pb_adamw_tensor;
pb_status pblock_adamw_step(const pb_adamw_config* cfg, int n_tensors,
                            const pb_adamw_tensor* tensors, pb_dtype copy_dtype,
                            hipStream_t stream);

/* Human-readable name of a status, and a description of the most recent
 * failed check on the calling thread ("" if none). */
const char* pblock_status_string(pb_status status);
const char* pblock_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* PBLOCK_H */
