/*
 * sparkattn -- block-sparse attention for long video-DiT token sequences on
 * NVIDIA B200 (sm_100a).  C ABI: plain pointers and sizes, no framework types.
 *
 * The library implements the sparse branch O_s = A_M(Q, K, V) of the paper's
 * compensated sparse attention (Sec. 2, "Block sparsity" and "Compensated
 * sparse attention"; Sec. 4.1): the attention matrix is cut into contiguous
 * query-block x key-block tiles, a selector keeps a fraction 1 - s of the key
 * blocks for every query block, and exact softmax attention
 * softmax(Q K^T / sqrt(d)) V is evaluated over the kept tiles only.
 *
 * Three device entry points make up the path:
 *   sparkattn_select     pooled block scores + top-k -> kept-block index lists
 *   sparkattn_quant_fp8  per-(head, token-block) absmax scale + E4M3 encode
 *   sparkattn_fwd        block-sparse flash-attention forward (bf16 or FP8)
 * plus one host-buffer convenience call that chains them with the copies, and
 * the low-rank compensation branch with the gate fusion that completes the
 * paper's attention module (sparkattn_comp_state, sparkattn_comp_apply).
 *
 * Conventions shared by all calls
 *   - Every data pointer is DEVICE memory owned by the caller unless a
 *     parameter name ends in `_host`.  The library allocates no device
 *     memory and keeps no pointer after the call returns.  What it does keep
 *     between calls, per device: two copy streams that
 *     sparkattn_attention_host creates on first use, the fixed scratch array
 *     of sparkattn_select_noalloc with its cached address, and the SM count.
 *   - Calls enqueue work on `cuda_stream` (a cudaStream_t passed as void*;
 *     NULL = the legacy default stream) and return without synchronising,
 *     except sparkattn_read_status and sparkattn_attention_host.
 *   - Tensors are [B, H, N, d] with d contiguous; strides are in elements.
 *   - Tokens are cut into nb = ceil(N / block) contiguous blocks; the last
 *     block may be ragged.  Rows >= N are never read as data or written.
 *   - Return value: SPARKATTN_OK (0) or a negative sparkattn_status code.
 *     Argument errors are detected on the host before anything is enqueued.
 *     Errors found on the device (a kept index outside [0, nb), a wait that
 *     ran out) are recorded in the first word of the caller's workspace and
 *     read back with sparkattn_read_status; the kernel skips the offending
 *     tile and still terminates.
 *   - Same inputs give bitwise identical outputs (no atomics on data, fixed
 *     reduction order).
 */
#ifndef SPARKATTN_H_
#define SPARKATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPARKATTN_VERSION 1

typedef enum {
  SPARKATTN_OK = 0,
  SPARKATTN_E_INVALID_ARG = -1,       /* NULL pointer, non-positive size, topk/kmax out of range      */
  SPARKATTN_E_UNSUPPORTED_SHAPE = -2, /* (d, block) not one of (64,64), (128,64), (128,128); nb too large */
  SPARKATTN_E_MISALIGNED = -3,        /* pointer not 16-byte aligned or stride * elem not 16-byte mult. */
  SPARKATTN_E_WORKSPACE_TOO_SMALL = -4,
  SPARKATTN_E_CUDA = -5,              /* launch or driver error; cudaGetLastError has the detail       */
  SPARKATTN_E_DEVICE_TIMEOUT = -6,    /* a bounded device-side wait expired (device status word)       */
  SPARKATTN_E_BAD_INDEX = -7,         /* a kept block index outside [0, nb) (device status word)       */
  SPARKATTN_E_NO_DEVICE = -8,         /* no CUDA device / driver entry point unavailable               */
  SPARKATTN_E_OUT_OF_PAGES = -9       /* fewer free pages than a reservation asks for (device status word) */
} sparkattn_status;

typedef enum { SPARKATTN_BF16 = 0, SPARKATTN_FP8_E4M3 = 1, SPARKATTN_FP32 = 2 /* weights of norms only */ } sparkattn_dtype;

/* Problem shape.  Caller fills it; the library reads it during the call only. */
typedef struct {
  uint32_t struct_size; /* sizeof(sparkattn_shape_t)                                   */
  uint32_t version;     /* SPARKATTN_VERSION                                           */
  int32_t B, H, N, d;   /* batch, heads (queries and keys share them), tokens, head dim */
  int32_t block;        /* tokens per query block = tokens per key block               */
  int32_t reserved;     /* must be 0                                                   */
  int64_t stride_b, stride_h, stride_n; /* element strides of [B,H,N,d]; d has stride 1 */
  float softmax_scale;  /* 0 selects 1/sqrt(d) (the paper's dense attention formula)   */
  uint32_t pad;         /* must be 0                                                   */
} sparkattn_shape_t;

int sparkattn_version(void);
const char* sparkattn_status_string(int status);

/* Bytes of device workspace a call needs.  which: 0 = sparkattn_select (pass
 * topk), 1 = sparkattn_fwd (pass kmax: for d = 128 the forward keeps a
 * range-checked copy of the kept lists (64-token blocks: the merged lists of
 * every pair of adjacent query blocks) and one scale per head behind the
 * status words, about 4 * B * H * nb * (kmax + 1) bytes either way; 256 bytes
 * for d = 64), 2 = sparkattn_gather_tokens (256).  Returns 0 for an invalid
 * shape or, for 0 and 1, a non-positive topk / kmax. */
size_t sparkattn_workspace_bytes(const sparkattn_shape_t* shape, int32_t which, int32_t topk_or_kmax);

/*
 * Block selection (the selector M_phi of Sec. 2 / Sec. 4.1; the paper lists
 * kinds of selectors, top-k over per-block scores among them, without fixing
 * a rule, so the rule is:)
 *   1. pooled sum over the valid tokens of a block, fp32, ascending token order
 *   2. pooled mean = sum / n_valid (IEEE fp32 divide)
 *   3. score(i, j) = fmaf chain over channels c ascending of pq[i,c] * pk[j,c]
 *   4. keep the `topk` key blocks first under (score descending, index ascending)
 *   5. write them in ascending index order.
 * Selection always reads the bf16 Q and K (Sec. 4.3 keeps mask selection in BF16).
 *
 * q_bf16, k_bf16 : in,  bf16 [B,H,N,d] with the strides of `shape`
 * topk           : in,  1 .. nb
 * kept_idx       : out, int32 [B,H,nb,topk] contiguous
 * kept_cnt       : out, int32 [B,H,nb] (every entry = topk); may be NULL
 * workspace      : scratch of >= sparkattn_workspace_bytes(shape, 0, topk) bytes,
 *                  256-byte aligned; its first word is the device status.
 */
int sparkattn_select(const sparkattn_shape_t* shape, const void* q_bf16, const void* k_bf16, int32_t topk,
                     int32_t* kept_idx, int32_t* kept_cnt, void* workspace, size_t workspace_bytes,
                     void* cuda_stream);

/*
 * Fused FP8 quantisation (Sec. 4.3: FP8 E4M3, scale and cast in one pass over
 * memory; the granularity here is one scale per (batch, head, token block)).
 *   amax = max |x| over the block's valid tokens x d ; amax = max(amax, 1e-12)
 *   scale = amax / 448 ; code = e4m3_rne_satfinite(x * (448 / amax))
 * x_bf16 : in,  bf16 [B,H,N,d] (strides of `shape`)
 * codes  : out, uint8 E4M3 codes, same element strides as x
 * scales : out, fp32 [B,H,nb] contiguous dequantisation scales (value = decode(code) * scale)
 * flags  : must be 0
 */
int sparkattn_quant_fp8(const sparkattn_shape_t* shape, const void* x_bf16, uint8_t* codes, float* scales,
                        uint32_t flags, void* cuda_stream);

/*
 * Quantisation and block pooling in one pass (Sec. 4.3 fuses scaling and
 * casting into a single pass over memory; here the selection's block pooling
 * rides on the same pass, so that in the FP8 configuration Q and K are read
 * from HBM once for selection and quantisation together).
 *
 * sparkattn_quant_fp8_pooled: sparkattn_quant_fp8 (same codes, same scales,
 *   bit for bit) that also writes the pooled fp32 block means of x -- steps 1
 *   and 2 of the selection rule above, same order of additions, same divide --
 *   into a selection workspace.  key_side: 0 = x is the query tensor, 1 = x is
 *   the key tensor.  select_workspace: the workspace a later
 *   sparkattn_select_pooled call takes (>= sparkattn_workspace_bytes(shape, 0,
 *   topk) bytes, 256-byte aligned); only its pooled-means region is written.
 * sparkattn_select_pooled: steps 3 to 5 of the selection rule on a workspace
 *   that one query-side and one key-side call above have filled (same shape,
 *   same stream order); outputs as sparkattn_select.  The three calls together
 *   give the same lists as sparkattn_select on the same Q and K.
 * Plain layout only (no causal window, no per-block token counts).
 */
int sparkattn_quant_fp8_pooled(const sparkattn_shape_t* shape, const void* x_bf16, uint8_t* codes, float* scales,
                               int32_t key_side, void* select_workspace, size_t workspace_bytes, void* cuda_stream);
int sparkattn_select_pooled(const sparkattn_shape_t* shape, int32_t topk, int32_t* kept_idx, int32_t* kept_cnt,
                            void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Per-token FP8 quantisation: the activation-quantisation kernel at the
 * paper's own granularity (Sec. 4.3: one dynamic scale per token row, scale
 * and cast in one pass).  Same arithmetic as sparkattn_quant_fp8 with the token
 * block replaced by one token row: amax over the row's d channels, clamped at
 * 1e-12; scale = amax / 448; code = e4m3_rne_satfinite(x * (448 / amax)).
 * Not consumed by sparkattn_fwd (which takes per-block scales); provided for
 * the activation path around it.  `shape->block` is ignored beyond validation.
 * x_bf16 : in,  bf16 [B,H,N,d] (strides of `shape`)
 * codes  : out, uint8 E4M3 codes, same element strides as x
 * scales : out, fp32 [B,H,N] contiguous
 */
int sparkattn_quant_fp8_per_token(const sparkattn_shape_t* shape, const void* x_bf16, uint8_t* codes,
                                  float* scales, void* cuda_stream);

/*
 * Block-sparse attention forward (Sec. 2 dense attention formula restricted
 * to the kept tiles; Sec. 4.1 sparse branch).  For query token i in query
 * block qb, over the keys j of the kept key blocks kept_idx[b,h,qb,0..cnt):
 *   out[i,:] = sum_j softmax_j(scale * q_i . k_j) v_j ,  lse[i] = ln sum_j exp(scale * q_i . k_j)
 * Keys >= N in a ragged last block are masked.  cnt = 0 gives out = 0, lse = -inf.
 *
 * dtype      : SPARKATTN_BF16: q,k,v bf16.  SPARKATTN_FP8_E4M3: q,k,v are E4M3
 *              codes from sparkattn_quant_fp8 with q_scale/k_scale/v_scale fp32
 *              [B,H,nb]; requires d = 128 (block 64 or 128).  Scales are NULL for bf16.
 * kept_idx   : in, int32 [B,H,nb,kmax]; entries distinct, each in [0, nb); kmax <= 2048
 *              (longer lists return SPARKATTN_E_UNSUPPORTED_SHAPE)
 * kept_cnt   : in, int32 [B,H,nb] with 0 <= cnt <= kmax; NULL means cnt = kmax everywhere
 * out_bf16   : out, bf16 [B,H,N,d], same strides as q
 * lse        : out, fp32 [B,H,N] contiguous (natural log); may be NULL
 * workspace  : >= sparkattn_workspace_bytes(shape, 1, kmax) bytes, 256-byte aligned
 * Accumulation, row maximum and row sum are fp32; P is rounded to the input
 * dtype for the second product.  The kept blocks of a list may come in any
 * order and are processed in an order of the library's choosing (the query
 * block's own key block first); the same inputs always give the same bits.
 * Out-of-range entries of a list are skipped and reported through the status
 * word of the workspace (SPARKATTN_E_BAD_INDEX).
 */
int sparkattn_fwd(const sparkattn_shape_t* shape, int32_t dtype, const void* q, const void* k, const void* v,
                  const float* q_scale, const float* k_scale, const float* v_scale, const int32_t* kept_idx,
                  const int32_t* kept_cnt, int32_t kmax, void* out_bf16, float* lse, void* workspace,
                  size_t workspace_bytes, void* cuda_stream);

/*
 * Causal frame window (Sec. 1, the auto-regressive extension: the paper says
 * the attention may be limited to a causal window and gives no formula, so
 * the reading is:)  tokens come in frames of
 * `frame_tokens` consecutive tokens; key token j counts for query token i iff
 *     i / frame_tokens - window_frames  <  j / frame_tokens  <=  i / frame_tokens.
 * sparkattn_select_window ranks only the key blocks that hold such a key for
 * some row of the query block (a contiguous run of blocks): kept_cnt =
 * min(topk, candidates) (kept_cnt must not be NULL) and the unused tail of a
 * list is -1.  sparkattn_fwd_window evaluates the same softmax attention as
 * sparkattn_fwd over the kept blocks with the token-exact window mask; a query
 * row without any admissible kept key gives a zero output row and lse = -inf.
 * All other arguments, layouts and errors are those of sparkattn_select /
 * sparkattn_fwd; frame_tokens < 1 or window_frames < 1 is SPARKATTN_E_INVALID_ARG.
 */
int sparkattn_select_window(const sparkattn_shape_t* shape, const void* q_bf16, const void* k_bf16, int32_t topk,
                            int32_t frame_tokens, int32_t window_frames, int32_t* kept_idx, int32_t* kept_cnt,
                            void* workspace, size_t workspace_bytes, void* cuda_stream);
int sparkattn_fwd_window(const sparkattn_shape_t* shape, int32_t dtype, const void* q, const void* k, const void* v,
                         const float* q_scale, const float* k_scale, const float* v_scale, const int32_t* kept_idx,
                         const int32_t* kept_cnt, int32_t kmax, int32_t frame_tokens, int32_t window_frames,
                         void* out_bf16, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Tokens stored brick by brick.  The paper partitions the sequence into
 * contiguous blocks (Sec. 2) and does not fix the order of the tokens; with
 * the raster order n = (t*Hg + y)*Wg + x a block is a strip of grid rows.
 * Here the (T, Hg, Wg) grid is cut into bricks of bt x bh x bw cells with
 * bt*bh*bw <= block (bricks at the far faces are cut to what the grid holds),
 * the bricks follow one another in raster order of the brick grid, the cells
 * of a brick in raster order inside it, and every brick takes one whole block
 * of the reordered tensors: its cells first, zero padding rows after them.
 * A block is then a compact box of the video; the reordered tensors have
 * N' = bricks * block tokens, and block_valid[b] says how many rows of block
 * b are real.  Padding rows are not keys, do not enter the pooled means of
 * the selection, and their output rows are to be ignored.
 *
 * sparkattn_brick_count : bricks of the layout (host arithmetic; 0 for invalid
 *                         arguments): the nb of the reordered tensors
 * sparkattn_brick_layout: grid_host, brick_host HOST int32[3]; block 64 or 128.
 *     gather_index  out, device int32 [bricks*block]: raster index of the token
 *                   at each padded position, -1 for padding (gather raster ->
 *                   bricks); may be NULL
 *     block_valid   out, device int32 [bricks]; may be NULL
 *     scatter_index out, device int32 [N]: padded position of raster token n
 *                   (gather bricks -> raster); may be NULL (not all three)
 * sparkattn_gather_tokens: out[b,h,i,:] = x[b,h,index[i],:] for i < N of
 *     dst_shape, one pass over memory; x bf16 with src_shape, out bf16 with
 *     dst_shape (same B, H, d; the two must not overlap); index device int32
 *     [dst N]: -1 leaves a zero row, any other value outside [0, src N) leaves
 *     a zero row and sets SPARKATTN_E_BAD_INDEX in the status word of
 *     `workspace` (>= sparkattn_workspace_bytes(shape, 2, 0) = 256 bytes,
 *     256-byte aligned; only the status header is used).
 * sparkattn_select_padded / sparkattn_fwd_padded: sparkattn_select /
 *     sparkattn_fwd on reordered tensors (N a multiple of the block size;
 *     d = 128 with 128- or 64-token blocks, else SPARKATTN_E_UNSUPPORTED_SHAPE) with
 *     block_valid device int32 [nb], every entry in [1, block]: pooled means
 *     over the real rows of a block, keys beyond block_valid[kb] of a kept
 *     block get weight 0.  Output rows of padding queries hold finite values
 *     without meaning.  All other arguments as in the plain calls.
 */
int64_t sparkattn_brick_count(const int32_t* grid_host, const int32_t* brick_host);
int sparkattn_brick_layout(const int32_t* grid_host, const int32_t* brick_host, int32_t block, int32_t* gather_index,
                           int32_t* block_valid, int32_t* scatter_index, void* cuda_stream);
int sparkattn_gather_tokens(const sparkattn_shape_t* src_shape, const void* x_bf16, const sparkattn_shape_t* dst_shape,
                            const int32_t* index, void* out_bf16, void* workspace, size_t workspace_bytes,
                            void* cuda_stream);
int sparkattn_select_padded(const sparkattn_shape_t* shape, const void* q_bf16, const void* k_bf16, int32_t topk,
                            const int32_t* block_valid, int32_t* kept_idx, int32_t* kept_cnt, void* workspace,
                            size_t workspace_bytes, void* cuda_stream);
int sparkattn_fwd_padded(const sparkattn_shape_t* shape, int32_t dtype, const void* q, const void* k, const void* v,
                         const float* q_scale, const float* k_scale, const float* v_scale, const int32_t* kept_idx,
                         const int32_t* kept_cnt, int32_t kmax, const int32_t* block_valid, void* out_bf16, float* lse,
                         void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Synchronises the stream and returns the device status word of a workspace
 * (SPARKATTN_OK, SPARKATTN_E_BAD_INDEX or SPARKATTN_E_DEVICE_TIMEOUT). */
int sparkattn_read_status(void* workspace, void* cuda_stream);

/*
 * Whole path on HOST buffers: copies Q, K, V to the device arena, runs
 * select (+ quant for FP8) + fwd, copies the output back and synchronises.
 * q_host, k_host, v_host, out_host: contiguous bf16 [B,H,N,d] in (preferably
 * pinned) host memory; kept_idx_host may be NULL or int32 [B,H,nb,topk] to
 * receive the selected lists.  arena: device scratch of at least
 * sparkattn_arena_bytes(shape, dtype, topk) bytes, 256-byte aligned.
 * The heads are independent, so the call runs as a pipeline over groups of
 * heads (about eight groups, at most 16; a group never spans two batch
 * entries, so B > 16 returns SPARKATTN_E_UNSUPPORTED_SHAPE): while one group is selected and
 * attended on `cuda_stream`, the next is copied in and the previous one's
 * output copied out on two copy streams that the library creates once per
 * device and keeps; both are ordered after work already queued on
 * `cuda_stream`, and `cuda_stream` ends after the last copy.  With pageable
 * host memory the copies are staged by the driver and the overlap is lost;
 * the result is the same.  Returns the first non-zero device status of any
 * group (SPARKATTN_E_BAD_INDEX, SPARKATTN_E_DEVICE_TIMEOUT), an argument or
 * CUDA error, or SPARKATTN_OK; on an error the output is undefined.
 */
size_t sparkattn_arena_bytes(const sparkattn_shape_t* shape, int32_t dtype, int32_t topk);
int sparkattn_attention_host(const sparkattn_shape_t* shape, int32_t dtype, const void* q_host,
                             const void* k_host, const void* v_host, int32_t topk, void* out_host,
                             int32_t* kept_idx_host, void* arena, size_t arena_bytes, void* cuda_stream);

/*
 * Low-rank compensation branch and gate fusion (Sec. 4.1, "low-rank
 * compensation branch" and the fused output O = O_s + g * r * O_lr).
 * With rank r = 64 projections P_q, P_k per head and the rank-truncated rotary
 * rotation R_r (adjacent feature pairs (2m, 2m+1) rotated by the angle
 * pos_axis[m] * freq[m], pos = the token's (t, y, x) coordinate on the latent
 * grid, raster token order n = (t * Hg + y) * Wg + x):
 *   q~_i = R_r(p_i) silu(P_q q_i)        k~_j = R_r(p_j) silu(P_k k_j)
 *   C    = sum_j k~_j v_j^T              (r x d per (batch, head): sparkattn_comp_state)
 *   y_i  = q~_i^T C ;  O_lr,i = y_i / sqrt(mean_c y_i[c]^2 + eps)      (RMSNorm, no weight)
 *   r_i  = sqrt(mean_c O_s,i[c]^2)  ;    O_i = O_s,i + g_i * r_i * O_lr,i   (sparkattn_comp_apply)
 * Linear in N.  Requires d = 128 and rank = 64; `shape->block` is validated but not used.
 *
 * Arithmetic: projections, C and y are tensor-core products of bf16 operands
 * with fp32 accumulation (q~, k~ and, in the apply pass, C are rounded to
 * bf16 first); silu, rotation, norms and the fusion are fp32; the state is
 * summed over fixed token chunks in a fixed order.
 *
 * k, v, q, o_sparse : in,  bf16 [B,H,N,d] with the strides of `shape`
 * pk, pq            : in,  bf16 [H, rank, d] contiguous, 16-byte aligned
 * grid_host         : in,  HOST int32[3] = (T, Hg, Wg), T*Hg*Wg = N
 * rope_axis_host    : in,  HOST int32[rank/2], entries 0 (t), 1 (y) or 2 (x)
 * rope_freq_host    : in,  HOST fp32[rank/2]
 * state             : comp_state out / comp_apply in, fp32 [B,H,rank,d] contiguous
 * gate              : in,  fp32 [B,H,N] contiguous (the token-wise gate g)
 * out_bf16          : out, bf16 [B,H,N,d], strides of `shape`; may alias o_sparse
 * eps               : RMSNorm epsilon (> 0)
 * workspace         : >= sparkattn_comp_workspace_bytes(shape, grid_host) bytes, 256-byte aligned
 *                     (sized for the state pass; the apply pass needs only its first
 *                     512 + 4 * rank * (T + Hg + Wg) bytes); first word = device status
 * The host arrays are read during the call only.
 */
size_t sparkattn_comp_workspace_bytes(const sparkattn_shape_t* shape, const int32_t* grid_host);
int sparkattn_comp_state(const sparkattn_shape_t* shape, const void* k_bf16, const void* v_bf16, const void* pk_bf16,
                         int32_t rank, const int32_t* grid_host, const int32_t* rope_axis_host,
                         const float* rope_freq_host, float* state, void* workspace, size_t workspace_bytes,
                         void* cuda_stream);
int sparkattn_comp_apply(const sparkattn_shape_t* shape, const void* q_bf16, const void* pq_bf16, int32_t rank,
                         const int32_t* grid_host, const int32_t* rope_axis_host, const float* rope_freq_host,
                         const float* state, const float* gate, const void* o_sparse_bf16, void* out_bf16, float eps,
                         void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Sparse forward and gate fusion in one kernel (Sec. 4.1: the module's output
 * O = O_s + g * r * O_lr, with O_s the block-sparse attention output).
 *
 * Equivalent to sparkattn_fwd (bf16) followed by sparkattn_comp_apply with
 * o_sparse = that call's output, without the round trip of O_s and the second
 * read of Q through device memory: the warpgroup that finishes a query block
 * keeps the normalised, bf16-rounded O_s rows in registers, forms
 * q~ = R_r(p) silu(P_q q) from the Q tile still in shared memory, y = q~^T C
 * on the tensor cores, and writes O_s + g * r * y / rms(y).  Every step is
 * taken in the arithmetic and order of the two separate calls, so the output
 * equals theirs bit for bit.  The state C comes from sparkattn_comp_state.
 *
 * Requires bf16 operands, d = 128, block = 128, rank = 64; no window mask and
 * no padded-brick layout (SPARKATTN_E_UNSUPPORTED_SHAPE otherwise).
 *
 * q, k, v           : in,  bf16 [B,H,N,d] with the strides of `shape`
 * kept_idx, kept_cnt, kmax, lse : as in sparkattn_fwd (lse is that of O_s)
 * pq, grid_host, rope_axis_host, rope_freq_host, state, gate, eps : as in sparkattn_comp_apply
 * out_bf16          : out, bf16 [B,H,N,d], strides of `shape`
 * workspace         : >= sparkattn_fwd_gated_workspace_bytes(shape, kmax, grid_host) bytes
 *                     (0 = unsupported arguments), 256-byte aligned; first word = device status
 * Errors as in sparkattn_fwd and sparkattn_comp_apply; on an error the output is undefined.
 */
size_t sparkattn_fwd_gated_workspace_bytes(const sparkattn_shape_t* shape, int32_t kmax, const int32_t* grid_host);
int sparkattn_fwd_gated(const sparkattn_shape_t* shape, const void* q_bf16, const void* k_bf16, const void* v_bf16,
                        const int32_t* kept_idx, const int32_t* kept_cnt, int32_t kmax, const void* pq_bf16,
                        int32_t rank, const int32_t* grid_host, const int32_t* rope_axis_host,
                        const float* rope_freq_host, const float* state, const float* gate, float eps, void* out_bf16,
                        float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Block selection without any allocation (the paper has no counterpart: this
 * is a packaging variant of sparkattn_select, same rule, same outputs).
 *
 * For callers that may not allocate device memory when they call: a serving
 * loop whose memory budget was fixed at start-up, a host application whose
 * allocator is frozen after initialisation, a plugin that only receives its
 * input and output buffers.  The scratch that sparkattn_select takes as a
 * workspace lives here in a fixed device array inside the library image, of
 * sparkattn_select_noalloc_max_bytes() bytes (32 MiB), which every GPU that
 * loads the library holds until the process exits.  The call itself performs
 * no cudaMalloc / cudaFree and calls no allocating library routine.
 *
 *   - Arguments as for sparkattn_select, minus the workspace.  q_bf16, k_bf16,
 *     kept_idx, kept_cnt are caller-owned device buffers.
 *   - A shape whose scratch need (sparkattn_workspace_bytes(shape, 0, topk))
 *     exceeds the array returns SPARKATTN_E_WORKSPACE_TOO_SMALL and enqueues
 *     nothing; the other argument errors are those of sparkattn_select.
 *   - The first call on each device looks up the array's device address (with
 *     that device current) and caches it; make that first call before starting
 *     any stream capture.
 *   - All calls on a device share the one array, which still holds the previous
 *     call's contents; the library clears what must start at zero.  Calls whose
 *     kernels can overlap on the GPU (different streams or threads) race on it:
 *     serialise them.
 *   - sparkattn_select_noalloc_status synchronises the stream and returns the
 *     device status word of the last call on the current device.
 */
size_t sparkattn_select_noalloc_max_bytes(void);
int sparkattn_select_noalloc(const sparkattn_shape_t* shape, const void* q_bf16, const void* k_bf16, int32_t topk,
                             int32_t* kept_idx, int32_t* kept_cnt, void* cuda_stream);
int sparkattn_select_noalloc_status(void* cuda_stream);

/*
 * Paged cache of keys and values (Sec. 1's auto-regressive extension: a generator that emits frames, or tokens, one after
 * another attends to what it has made so far.  The paper has no cache; layout and rules are this library's).
 *
 * The cache is a pool of pages; a page holds `page` consecutive tokens of one sequence, for every head that has keys of
 * its own.  K and V are two pools of the same strides, bf16 or E4M3 codes; with E4M3 every (page, head) has one positive
 * fp32 scale in k_scale and one in v_scale, [pages, H] contiguous (value = decode(code) * scale).
 * page_table[b][i] is the page of tokens i * page .. i * page + page - 1 of sequence b.
 *
 * A call works on a ragged batch: token rows q_start[b] .. q_start[b+1] - 1 of its row tensors ([T, heads, d], d
 * contiguous) are the newest tokens of sequence b, which has kv_len[b] tokens in the cache with them; their positions are
 * kv_len[b] - n_b .. kv_len[b] - 1.  Page table, lengths and starts are device memory and may change from call to call
 * under a captured graph; the sizes in the structs may not.
 *
 * Errors found on the device (SPARKATTN_E_BAD_INDEX in the status word): a page outside [0, pages) among those the call
 * reaches (its tokens are not stored, or not attended to), a length outside [0, max_pages * page], starts that are not
 * ascending within [0, T], more new tokens than max_new or than kv_len[b], a rotary position outside the table (the row is left unrotated).
 */
typedef struct {
  uint32_t struct_size; /* sizeof(sparkattn_cache_t)                                          */
  uint32_t version;     /* SPARKATTN_VERSION                                                  */
  int32_t dtype;        /* SPARKATTN_BF16 or SPARKATTN_FP8_E4M3                               */
  int32_t pages;        /* pages in the pool                                                  */
  int32_t H;            /* heads with keys and values of their own                            */
  int32_t page;         /* tokens per page: 16, 32, 64 or 128                                 */
  int32_t d;            /* head dim: 64 or 128                                                */
  int32_t reserved;     /* must be 0                                                          */
  int64_t stride_page, stride_h, stride_n; /* element strides of [pages, H, page, d]; d has stride 1; multiples of 16 bytes */
} sparkattn_cache_t;

typedef struct {
  uint32_t struct_size; /* sizeof(sparkattn_batch_t)                                          */
  uint32_t version;     /* SPARKATTN_VERSION                                                  */
  int32_t B;            /* sequences, at most 4096                                            */
  int32_t T;            /* token rows of the call                                             */
  int32_t max_new;      /* no sequence has more new tokens than this                          */
  int32_t max_pages;    /* columns of page_table                                              */
  const int32_t* page_table; /* [B, max_pages]                                                */
  const int32_t* kv_len;     /* [B] tokens of the sequence, the new ones included             */
  const int32_t* q_start;    /* [B + 1] first row of each sequence, or NULL: T / B rows each  */
} sparkattn_batch_t;

/* bf16 rows [T, heads, d], d contiguous; strides in elements, multiples of 8; 16-byte aligned */
typedef struct {
  void* data;
  int64_t stride_t, stride_h;
} sparkattn_rows_t;

/* Rotation of the first `rot` channels: pair m turns by the angle whose cosine and sine are cos[p][m], sin[p][m], with p
 * = positions[t][axis[m]], or the token's position in its sequence where positions is NULL.  Pairs are the channels
 * (2m, 2m+1) (interleaved) or (m, m + rot/2):  y1 = x1 cos - x2 sin,  y2 = x1 sin + x2 cos,  every product, sum and
 * difference rounded to fp32.  The table is the caller's: frequencies, scaling and long-context rules are in it. */
typedef struct {
  uint32_t struct_size;      /* sizeof(sparkattn_rotary_t)                                    */
  uint32_t version;          /* SPARKATTN_VERSION                                             */
  int32_t rot;               /* multiple of 16, at most d                                     */
  int32_t interleaved;       /* 0 or 1                                                        */
  int32_t rows;              /* rows of the tables                                            */
  int32_t axes;              /* columns of positions: 1 to 4; 1 without positions             */
  const float* cos;          /* [rows, rot/2], 16-byte aligned                                */
  const float* sin;
  const int32_t* positions;  /* [T, axes], or NULL                                            */
  const int32_t* axis;       /* [rot/2], entries in [0, axes); NULL: all 0                    */
} sparkattn_rotary_t;

/* RMS norm over the d channels of each head, in front of the rotation:  y_c = x_c / sqrt(mean(x^2) + eps) * weight_c.  The mean is a head's, with
 * weights of each head too: models whose norm takes one mean over all heads' channels (Wan2.1's, over 12 or 40 heads of 128) need theirs in front, and
 * norm = NULL here.  weight / sqrt(mean + eps) has to be a finite fp32 number.
 * fp32 throughout (squares, their sum, the root, the products); no rounding to 16 bits between norm and rotation, whose products and sums may be
 * fused here.  A row whose sum of squares passes
 * fp32's range, which takes entries of 1e18, comes out as zeros; one with an infinity or a NaN gives NaN there. */
typedef struct {
  uint32_t struct_size;   /* sizeof(sparkattn_norm_t)                                         */
  uint32_t version;       /* SPARKATTN_VERSION                                                */
  int32_t weight_dtype;   /* SPARKATTN_BF16 or SPARKATTN_FP32                                 */
  int32_t per_head;       /* 0: weights [d], shared by the heads; 1: [heads, d] contiguous    */
  float eps;              /* > 0, not a subnormal number                                      */
  uint32_t pad;           /* must be 0                                                        */
  const void* q_weight;   /* 16-byte aligned, or NULL: ones                                   */
  const void* k_weight;
} sparkattn_norm_t;

/* Bytes of device workspace that sparkattn_cache_fwd needs for H query heads (0: unsupported arguments);
 * sparkattn_cache_append needs 256. */
size_t sparkattn_cache_workspace_bytes(const sparkattn_cache_t* cache, const sparkattn_batch_t* batch, int32_t H);

/*
 * Rotates the new tokens' keys (and queries), and stores keys and values in the cache, in one launch.
 *   bf16 pages: the rotated keys and the values, rounded to nearest even.
 *   E4M3 pages: the scale of a (page, head) is the smallest power of two s with amax <= 448 s, amax the largest finite
 *     |x| of the page's tokens, at least 1e-12, and grows with the page: s = max(the page's scale, the new tokens'),
 *     unless the page's first token is among the new ones.  Where it grows, the codes of the tokens already there are
 *     encoded again (code * (old * (1/s))), which a power of two leaves exact but for values that fall below 2^-6 s, so
 *     that a page hardly depends on the steps in which it was filled.  New codes: e4m3_rne_satfinite(x * (1/s)).
 *     Infinities become the largest code, +-448 of the scale at that time, NaN stays NaN.
 * q, q_out : bf16 rows [T, H, d] and where they go rotated (may be the same memory), or both NULL (H is ignored)
 * k, v     : bf16 rows [T, cache->H, d]
 * rotary   : NULL: nothing is rotated
 * workspace: >= 256 bytes, 256-byte aligned; the status word
 * Two sequences of a call must not append to the same page.
 */
int sparkattn_cache_append(const sparkattn_cache_t* cache, const sparkattn_batch_t* batch, const sparkattn_rotary_t* rotary,
                           const sparkattn_rows_t* q, int32_t H, const sparkattn_rows_t* k, const sparkattn_rows_t* v,
                           void* k_cache, void* v_cache, float* k_scale, float* v_scale, const sparkattn_rows_t* q_out,
                           void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The same with the norm of keys and queries (not of values) in front of their rotation.  norm: NULL is sparkattn_cache_append. */
int sparkattn_cache_append_norm(const sparkattn_cache_t* cache, const sparkattn_batch_t* batch, const sparkattn_norm_t* norm,
                                const sparkattn_rotary_t* rotary, const sparkattn_rows_t* q, int32_t H, const sparkattn_rows_t* k,
                                const sparkattn_rows_t* v, void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                                const sparkattn_rows_t* q_out, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Norm and rotation of the queries and keys of whole sequences, in front of sparkattn_select, sparkattn_quant_fp8 and sparkattn_fwd,
 * which take them as the model's normalisation left them.  One launch; every row is read and written once.
 * q, k       : in,  bf16 [B, H, N, d]; B, N and d are the same, the heads may differ.  k_shape, k, k_out_shape, k_out NULL: queries alone
 * q_out, k_out : out, the same sizes with the strides of their own shape; may be q and k themselves with their strides, and overlap the inputs in
 *              no other way
 * norm, rotary : either may be NULL, not both.  Positions are [N, axes], the same for every sample; NULL: the token's index
 * workspace  : >= 256 bytes, 256-byte aligned; the status word: SPARKATTN_E_BAD_INDEX for a position or axis outside the tables, whose pairs
 *              are left unrotated
 * `block` and `softmax_scale` of the shapes are validated, not used.
 */
int sparkattn_norm_rotate(const sparkattn_shape_t* q_shape, const void* q, const sparkattn_shape_t* q_out_shape, void* q_out,
                          const sparkattn_shape_t* k_shape, const void* k, const sparkattn_shape_t* k_out_shape, void* k_out,
                          const sparkattn_norm_t* norm, const sparkattn_rotary_t* rotary, void* workspace, size_t workspace_bytes,
                          void* cuda_stream);

/*
 * Softmax attention of the new tokens over the cache.  For the token at position i of its sequence and query head h, over
 * the keys j of head h / (H / cache->H) with  lo(i) <= j < hi(i):
 *   out = sum_j softmax_j(softmax_scale * q . k_j) v_j ,   lse = ln sum_j exp(softmax_scale * q . k_j)
 *   frame_tokens = g >= 1 : hi = min(kv_len, (floor(i/g) + 1) g)   (causal by frames of g tokens; 1: by token)
 *                  lo = (floor(i/g) - window_frames + 1) g, at least 0; window_frames = 0: lo = 0
 *   frame_tokens = 0      : all of the sequence's keys (window_frames must be 0)
 * A row without a key (an empty sequence) gives out = 0, lse = -inf.  What lies in a page behind the sequence's last
 * token, or in a page that no row reaches, is not looked at, whatever it holds.
 *
 * H            : query heads, a multiple of cache->H
 * q, out       : bf16 rows [T, H, d]; rows that belong to no sequence are not written
 * softmax_scale: 0 selects 1/sqrt(d)
 * lse          : fp32 [T, H] contiguous (natural log), or NULL
 * workspace    : >= sparkattn_cache_workspace_bytes(cache, batch, H), 256-byte aligned; first word = device status
 * A key or value that is not finite reaches the rows that see its key, and no others.
 * Scores, maxima, sums and the output's accumulation are fp32.  The weights of the second product are rounded to fp16 over
 * E4M3 pages, where what lies below 2^-30 of a row's largest (weight times value scale) is lost to the output, not to lse; over bf16
 * pages to two bf16 parts (16 digits together) for up to 16 rows per key head (H / cache->H * max_new), to one for more.  A value
 * scale below 2^-64 counts as 2^-64.  Queries over E4M3 pages are used as bf16 holds them, but for entries below 2^-9 of their row's
 * largest, which are off by 2^-17 of that at most (d = 64 and more than 16 rows: below 2^-24, by 2^-32); a query row with
 * an infinity or a NaN in it gives NaN.  The same call gives the same bits.
 * Which kernel runs and how its work is split is chosen on the host, by max_new and by max_pages * page, the longest sequence that
 * the table allows, not by the lengths.  Both cost time where they are far above what the batch has: one token over 1000 keys, 32 heads
 * over 8, takes 6.2 us, under a table of 131,072 tokens 9.8; one token each of 64 sequences of 8000 keys, 40 heads over 8, 171 us, under
 * max_new = 2, 4 and 64 243, 311 and 457.
 * A batch whose structs allow more than 2^31 key tiles of 64 in all is SPARKATTN_E_UNSUPPORTED_SHAPE.
 */
int sparkattn_cache_fwd(const sparkattn_cache_t* cache, const sparkattn_batch_t* batch, const sparkattn_rows_t* q, int32_t H,
                        const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                        int32_t frame_tokens, int32_t window_frames, float softmax_scale, const sparkattn_rows_t* out,
                        float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The same through a window and with the sequence's first tokens, which stay visible however far it has gone on: the token at
 * position i sees the keys j < hi(i) with  lo(i) <= j  or  j < sink_tokens.
 * What a generator without end attends to: what has left the window is not read, its pages may be gone (any number, -1 among them, may
 * stand in the table there; sparkattn_pages_trim gives them back), and the first tokens or the first frame go on being seen.  Positions
 * are those of the sequence; keys keep the rotation they were stored with.
 * sink_tokens  : >= 0; without a window (window_frames = 0) and with 0 the call is sparkattn_cache_fwd
 * Everything else, the workspace among it, as in sparkattn_cache_fwd.
 */
int sparkattn_cache_fwd_sink(const sparkattn_cache_t* cache, const sparkattn_batch_t* batch, const sparkattn_rows_t* q, int32_t H,
                             const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                             int32_t frame_tokens, int32_t window_frames, int32_t sink_tokens, float softmax_scale,
                             const sparkattn_rows_t* out, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The book of a paged cache: which sequence holds which pages of the pool.  The tables name the pages, refs counts for every page how many entries
 * of tables name it (0: free); whoever keeps a page for another reason, a prompt that is asked for again for instance, adds 1 of its own.
 * Every layer has pools of its own; the book is one for all, and the calls that move pages leave (from, to) pairs that
 * sparkattn_cache_copy_pages takes once for each layer.  Nothing here waits for the host: a captured graph can reserve, append,
 * attend and trim step after step, by the lengths that sparkattn_pages_reserve_len leaves, which stop a step whose pages do not suffice.
 *
 * An entry of a table is a page, or -1 where a sequence has none.  The calls write table, counts and lengths to where they are told, which
 * may be where they come from (but for sparkattn_pages_fork's tables and lengths); entries that name no page of the pool count as none.
 * Free pages are handed out in ascending order, in the order of the sequences: the same call gives the same book.
 */
typedef struct {
  uint32_t struct_size; /* sizeof(sparkattn_book_t)                                           */
  uint32_t version;     /* SPARKATTN_VERSION                                                  */
  int32_t B;            /* sequences, at most 4096                                            */
  int32_t max_pages;    /* columns of page_table; B * max_pages at most 2^31 - 256            */
  int32_t pages;        /* pages in the pool, at most 2^30                                    */
  int32_t page;         /* tokens per page: 16, 32, 64 or 128                                 */
  const int32_t* page_table; /* [B, max_pages]                                                */
  const int32_t* refs;       /* [pages]                                                       */
} sparkattn_book_t;

/* Bytes of device workspace, 256-byte aligned, that each of the four calls needs (0: unsupported arguments); first word = device status. */
size_t sparkattn_pages_workspace_bytes(const sparkattn_book_t* book);

/*
 * Sequence b of the new batch goes on from sequence parent[b] of the old one: fork (the same parent several times), reorder, and drop (a sequence
 * that is nobody's parent gives its pages back).  Children share their parent's pages, the partly filled last one and those reserved ahead too,
 * until sparkattn_pages_reserve finds that both go on in them.
 * kv_len     : in,  int32 [B]
 * parent     : in,  int32 [B_out], entries in [-1, B); -1: an empty sequence (so does any other number, which is reported)
 * B_out      : sequences of the new batch, at most 4096
 * table_out  : out, int32 [B_out, max_pages];  kv_len_out : out, int32 [B_out];  refs_out : out, int32 [pages], may be refs
 * Device errors (SPARKATTN_E_BAD_INDEX): a parent outside [-1, B); in rows whose number of users changes, an entry outside [-1, pages) or a page
 * whose count falls below 0.
 */
int sparkattn_pages_fork(const sparkattn_book_t* book, const int32_t* kv_len, const int32_t* parent, int32_t B_out, int32_t* table_out,
                         int32_t* kv_len_out, int32_t* refs_out, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Pages for the tokens kv_len[b] .. kv_new[b] - 1 of every sequence, in front of sparkattn_cache_append: the columns that these tokens begin get
 * free pages.  Those that have one, reserved ahead, keep it if nobody else holds it; if others do, since the sequence was forked behind that,
 * the column gets another one.  Where the token kv_len[b] falls into a partly filled page that others hold as well, it is replaced
 * by a free one, and the pair (src, dst) says what has to be copied; of the sequences that go on in one such page the first keeps it if nobody
 * else holds it.  So no token of the call lies in a page that another sequence has.  All or nothing: where the pool has fewer free pages than that, the book stays as it was, and the status is
 * SPARKATTN_E_OUT_OF_PAGES, its detail the number of pages that are missing, whatever else was found.  Nothing may be appended then: sequences
 * still share the page that they go on in.  Who does not read the status before the append takes sparkattn_pages_reserve_len.
 * kv_len, kv_new : in,  int32 [B], 0 <= kv_len <= kv_new <= max_pages * page
 * src, dst   : out, int32 [B]: pages to copy for sequence b, or -1 and -1
 * table_out, refs_out : out, may be page_table and refs
 * Device errors (SPARKATTN_E_BAD_INDEX): lengths that are not so (the sequence is left out), a partly filled page that is none or
 * that nobody holds, a page that stands in a column that is asked for and that nobody holds (it stays there).
 */
int sparkattn_pages_reserve(const sparkattn_book_t* book, const int32_t* kv_len, const int32_t* kv_new, int32_t* table_out, int32_t* refs_out,
                            int32_t* src, int32_t* dst, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The same, and the lengths for the calls of the step behind it, so that the host need not learn first how it went.
 * kv_len_out : out, int32 [B], neither kv_len nor kv_new: kv_new[b]; -1 where sequence b has not got what it asked for, whether its own numbers
 *              make no sense or the pages do not suffice (then every b with kv_new[b] > kv_len[b]).  By a length of -1 sparkattn_cache_append stores
 *              nothing, sparkattn_cache_fwd gives rows of a sequence without keys, and sparkattn_pages_trim gives nothing back; all three
 *              report it, and so does a reservation that takes it as kv_len.
 */
int sparkattn_pages_reserve_len(const sparkattn_book_t* book, const int32_t* kv_len, const int32_t* kv_new, int32_t* kv_len_out, int32_t* table_out,
                                int32_t* refs_out, int32_t* src, int32_t* dst, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Gives back the pages that no token from position kv_len[b] on reads, under the rules of sparkattn_cache_fwd_sink: those that lie
 * between the first sink_tokens tokens and the window of the next token, and those behind the sequence's length (tokens that were
 * drafted and not taken; kv_len 0: all of the sequence's).  Their entries become -1.
 * kv_len     : in,  int32 [B]
 * frame_tokens, window_frames, sink_tokens : as in that call; window_frames 0: every token reads all earlier ones
 * Device errors (SPARKATTN_E_BAD_INDEX): a length outside [0, max_pages * page] (the sequence stays as it is), an entry among those given back that
 * names no page, a page whose count falls below 0.
 */
int sparkattn_pages_trim(const sparkattn_book_t* book, const int32_t* kv_len, int32_t frame_tokens, int32_t window_frames, int32_t sink_tokens,
                         int32_t* table_out, int32_t* refs_out, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Moves the pages in use to the front of the pool: with n of them, the pages from n on go, in ascending order, to the free ones below n.
 * The book has to hold every table that names pages of the pool.  The pages themselves move with sparkattn_cache_copy_pages, which has to
 * come before anything reads or appends by the new table.
 * src, dst   : out, int32 [pages / 2]: the pairs, then -1
 * Device errors (SPARKATTN_E_BAD_INDEX): an entry that names no page, or one that nobody holds (it becomes -1).
 */
int sparkattn_pages_compact(const sparkattn_book_t* book, int32_t* table_out, int32_t* refs_out, int32_t* src, int32_t* dst, void* workspace,
                            size_t workspace_bytes, void* cuda_stream);

/*
 * Pages src[i] of one pool to pages dst[i] of another, or of the same (the same pointers and the same struct): keys, values and scales.
 * from, to   : dtype, H, page and d alike; pages and strides of their own
 * src, dst   : in,  int32 [n], n >= 0; pairs of -1 and -1 are passed over
 * workspace  : >= 256 bytes, 256-byte aligned; the status word
 * Device errors (SPARKATTN_E_BAD_INDEX): a number outside its pool (that pair is passed over); a page that is written twice, or written and
 * read (what such a page then holds is undefined).
 */
int sparkattn_cache_copy_pages(const sparkattn_cache_t* from, const void* k_from, const void* v_from, const float* k_scale_from,
                               const float* v_scale_from, const sparkattn_cache_t* to, void* k_to, void* v_to, float* k_scale_to,
                               float* v_scale_to, const int32_t* src, const int32_t* dst, int32_t n, void* workspace, size_t workspace_bytes,
                               void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* SPARKATTN_H_ */
