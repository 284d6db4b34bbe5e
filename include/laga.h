/*
 * laga.h — C ABI of one rank's share of LAGA (Latent All-Gather Attention).
 *
 * After the latent all-gather (Alg. 1 step 3) a rank holds, for the whole
 * gathered sequence, the compressed latent c_kv [B,S,d_c] and the shared RoPE
 * key k_pe [B,S,d_rope]; after the head-scatter (Alg. 1 step 2) it holds the
 * queries q [B,S,H,d_nope+d_rope] of its H heads, and it owns the head shard
 * W_kv_b [d_c, H*(d_nope+d_v)] of the up-projection. This library computes:
 *
 *   laga_reconstruct_kv : Alg. 1 step 4 — kv = c_kv @ W_kv_b (per-head K_nope, V)
 *   laga_attn_fwd       : Alg. 1 step 5 — causal softmax attention with
 *                         K_h = [K_nope,h || k_pe] (k_pe broadcast to all heads,
 *                         property P2 of Section 2.1) and V_h; also returns the
 *                         per-row log-sum-exp that the backward reuses
 *   laga_attn_bwd       : the per-rank backward (Section 5.2 covers the
 *                         collectives around it): dq, the head-shard partials
 *                         dc_kv and dk_pe, and the W_kv_b shard gradient dW
 *   laga_out_proj_fwd/_bwd : Alg. 1 step 7, the output projection W_o after the
 *                         out all-to-all, and its backward
 *   laga_page_plan/_release, laga_cache_append, laga_paged_attn : serving the trained
 *                         block, new tokens against a paged cache of [c_kv || k_pe]
 *
 * Layouts (all row-major, contiguous, device memory, 16-byte aligned):
 *   c_kv   [B, S, d_c]                     element dtype
 *   k_pe   [B, S, d_rope]                  element dtype
 *   q      [B, S, H, d_nope + d_rope]      element dtype; q_nope first, then q_rope
 *   w_kv_b [d_c, H * (d_nope + d_v)]       element dtype; head h owns the column
 *                                          block [h*(d_nope+d_v), (h+1)*(d_nope+d_v)),
 *                                          K_nope columns first, then V
 *   kv     [B, S, H, d_nope + d_v]         element dtype (= [B*S, H*(d_nope+d_v)])
 *   out    [B, S, H, d_v]                  element dtype
 *   lse    [B, H, S]                       fp32, natural-log log-sum-exp of each row
 *   dout   [B, S, H, d_v]                  element dtype
 *   dq     [B, S, H, d_nope + d_rope]      element dtype
 *   dc_kv  [B, S, d_c]                     fp32 (partial sum over this head shard)
 *   dk_pe  [B, S, d_rope]                  fp32 (partial sum over this head shard)
 *   dw_kv_b[d_c, H * (d_nope + d_v)]       fp32 (the full gradient of this shard)
 *
 * Conventions:
 *   - Ownership: the caller owns every buffer, including the workspace; the
 *     library allocates and frees nothing and keeps no state between calls.
 *   - Asynchrony: work is enqueued on `stream` (a hipStream_t passed as void*,
 *     NULL = the default stream); calls return without synchronising.
 *   - Validation happens on the host before any launch; on error nothing is
 *     launched and no output is touched. Asynchronous device faults surface at
 *     the caller's next synchronisation. No exception crosses the ABI.
 *   - Every output is overwritten, never accumulated into.
 *   - dc_kv and dk_pe are partial sums over this rank's heads; across ranks
 *     they are completed by the reduce-scatter that is the backward of the
 *     latent all-gather (Section 5.2), so they are returned in fp32 to be summed
 *     before any rounding to the element dtype.
 *   - Causal means key j is visible to query i iff j <= i (0-based positions in
 *     the gathered sequence, S_q == S_k). Non-causal attends to every key.
 *   - Supported head dims: (d_nope, d_rope, d_v) = (128, 64, 128) — DeepSeek-V3 —,
 *     (64, 32, 64) and (32, 16, 32); d_c a multiple of 32 up to 1024; S >= 1;
 *     B >= 1; H >= 1. Anything else returns LAGA_ERR_UNSUPPORTED. Each width is a
 *     compile-time kernel instance (the tile shapes follow from it); the
 *     DeepSeek-V3 widths have the tuned bf16 kernels, the others the generic ones.
 *   - Kernels index inside a tensor with 32-bit element offsets: B*S*H*W, with
 *     W = d_nope + max(d_rope, d_v) + max(d_nope, d_v), B*S*d_c, B*S, and
 *     16*d_c*H*(d_nope + d_v) must each stay below 2^31, else
 *     LAGA_ERR_UNSUPPORTED (and laga_workspace_bytes() returns 0). Memory,
 *     not this limit, bounds S first for the backward with dq_mode FROM_STORE:
 *     its dS^T store holds B*H*S*S/2 bf16 values (dq_mode RECOMPUTE has none).
 *   - Results do not depend on H: every per-head output (kv columns, out, lse,
 *     dq, dw_kv_b columns) of a head is bit-identical whichever head shard it is
 *     computed in; repeated calls are bit-identical.
 */
#ifndef LAGA_H_
#define LAGA_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__) || defined(__clang__)
#define LAGA_API __attribute__((visibility("default")))
#else
#define LAGA_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

#define LAGA_ABI_VERSION 3

typedef enum {
  LAGA_OK = 0,
  LAGA_ERR_NULL = 1,        /* a required pointer (or the problem) is NULL */
  LAGA_ERR_SHAPE = 2,       /* a dimension is <= 0 or sizes are inconsistent */
  LAGA_ERR_UNSUPPORTED = 3, /* dims/dtype/mode/size the library has no kernel for */
  LAGA_ERR_ALIGN = 4,       /* a pointer is not 16-byte aligned */
  LAGA_ERR_WORKSPACE = 5,   /* workspace smaller than laga_workspace_bytes() */
  LAGA_ERR_DEVICE = 6,      /* the HIP runtime reported an error at launch */
  LAGA_ERR_SCRATCH = 7      /* laga_attn_bwd_noalloc: workspace need above its fixed array */
} laga_status_t;

typedef enum { LAGA_DTYPE_BF16 = 0, LAGA_DTYPE_FP32 = 1 } laga_dtype_t;

/* Where attention gets its per-head K_nope/V from.
 * MATERIALIZED: from `kv`, written beforehand by laga_reconstruct_kv.
 * FUSED: rebuilt tile by tile on chip from c_kv and w_kv_b; no per-head K/V
 *        tensor is ever written to HBM by the forward. */
typedef enum { LAGA_KV_MATERIALIZED = 0, LAGA_KV_FUSED = 1 } laga_kv_mode_t;

typedef enum { LAGA_OP_FWD = 0, LAGA_OP_BWD = 1, LAGA_OP_PROLOGUE_BWD = 2 } laga_op_t;

/* How the backward gets dq = scale * dZ K (dZ = P * (dP - delta), the score gradient).
 * FROM_STORE: the key-stationary pass that forms dZ for dK also writes it (bf16) to a
 *        store in the workspace, and the dq pass is a product over that store. This
 *        is the fastest path, but the store holds B*H*S*S/2 values (about 4.3 GB at
 *        S = 16384, H = 16). Only bf16 with 192/128-wide heads has it; other problems
 *        recompute (below) whatever this field says.
 * RECOMPUTE: no buffer of S*S size anywhere (workspace linear in S): the dq pass is
 *        query-stationary and recomputes the scores and dP for its queries, which costs
 *        the Q K^T and dO V^T products a second time. Every output equals FROM_STORE's
 *        exactly for bf16 with 192/128-wide heads (the same products, exp2 arguments,
 *        roundings and key order); elsewhere dq may differ in fp32 summation order. */
typedef enum { LAGA_DQ_FROM_STORE = 0, LAGA_DQ_RECOMPUTE = 1 } laga_dq_mode_t;

typedef struct {
  int64_t batch;       /* B */
  int64_t seq_len;     /* S: gathered sequence length */
  int64_t n_heads;     /* H: heads of THIS rank's shard */
  int64_t d_c;         /* latent width (d_kv) */
  int64_t d_nope;      /* per-head no-RoPE q/k width */
  int64_t d_rope;      /* shared RoPE band width */
  int64_t d_v;         /* per-head value width */
  float softmax_scale; /* multiplies q.k; the paper's 1/sqrt(d) with d = d_nope + d_rope */
  int32_t causal;      /* 1: causal mask, 0: none */
  int32_t dtype;       /* laga_dtype_t: element type of all non-fp32 tensors */
  int32_t kv_mode;     /* laga_kv_mode_t */
  int32_t deterministic; /* 1: asks for bitwise-reproducible results. Every kernel of
                            this library is deterministic (no floating-point atomics),
                            so 0 is accepted and changes nothing */
  int32_t dq_mode;     /* laga_dq_mode_t */
} laga_problem_t;

/* Alg. 1 step 4: kv[b,t,:] = c_kv[b,t,:] @ w_kv_b, stored [B,S,H,d_nope+d_v].
 * Accumulates in fp32 over d_c in ascending order; bf16 outputs are rounded to
 * nearest-even. */
LAGA_API laga_status_t laga_reconstruct_kv(const laga_problem_t* p, const void* c_kv,
                                  const void* w_kv_b, void* kv, void* stream);

/* Alg. 1 step 5 for the H heads of the shard: out and lse.
 * kv is required (non-NULL) for MATERIALIZED and ignored for FUSED, which
 * instead reads c_kv and w_kv_b. k_pe is shared by all heads. The workspace
 * must hold laga_workspace_bytes(p, LAGA_OP_FWD) bytes (may be 0 / NULL). */
LAGA_API laga_status_t laga_attn_fwd(const laga_problem_t* p, const void* q,
                            const void* c_kv, const void* k_pe,
                            const void* w_kv_b, const void* kv, void* out,
                            float* lse, void* workspace, size_t workspace_bytes,
                            void* stream);

/* Backward of laga_reconstruct_kv + laga_attn_fwd given dout:
 *   dq = dL/dq (element dtype); dc_kv = dL/dc_kv and dk_pe = dL/dk_pe summed
 *   over this shard's heads (fp32); dw_kv_b = dL/dW_kv_b (fp32). All overwritten.
 *   Deterministic: no floating-point atomics are used.
 * out and lse are the forward's outputs. kv is required for MATERIALIZED; for
 * FUSED it may be NULL and K/V are rebuilt into the workspace. */
LAGA_API laga_status_t laga_attn_bwd(const laga_problem_t* p, const void* q,
                            const void* c_kv, const void* k_pe,
                            const void* w_kv_b, const void* kv, const void* out,
                            const float* lse, const void* dout, void* dq,
                            float* dc_kv, float* dk_pe, float* dw_kv_b,
                            void* workspace, size_t workspace_bytes,
                            void* stream);

/* The backward in its stages; laga_attn_bwd runs all four in this order on one
 * stream. A caller may run them itself (same arguments and workspace for every
 * stage) to put other work between them or to time them one by one:
 *   LAGA_BWD_PREPARE  per-row delta = sum(dout * out) (and the K/V rebuild of
 *                     the FUSED mode when kv is NULL)
 *   LAGA_BWD_DKDV     key-stationary attention backward: dK, dV of every key
 *                     (bf16 with 192/128-wide heads and dq_mode FROM_STORE: also
 *                     stores dS^T of every causal pair, bf16, in the workspace)
 *   LAGA_BWD_DQ       attention backward for dq (with the store: the product
 *                     K^T dS^T over it; otherwise a query-stationary pass that
 *                     recomputes the scores)
 *   LAGA_BWD_FINISH   dk_pe head sum, dc_kv and dw_kv_b up-projection GEMMs
 * Each stage reads what the previous ones left in the workspace. */
typedef enum {
  LAGA_BWD_PREPARE = 0,
  LAGA_BWD_DKDV = 1,
  LAGA_BWD_DQ = 2,
  LAGA_BWD_FINISH = 3
} laga_bwd_stage_t;

LAGA_API laga_status_t laga_attn_bwd_stage(int stage, const laga_problem_t* p,
                                           const void* q, const void* c_kv,
                                           const void* k_pe, const void* w_kv_b,
                                           const void* kv, const void* out,
                                           const float* lse, const void* dout,
                                           void* dq, float* dc_kv, float* dk_pe,
                                           float* dw_kv_b, void* workspace,
                                           size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid allocation): laga_attn_bwd without a workspace
 * argument. Same arguments, results and stream semantics as laga_attn_bwd; its
 * workspace is a static device array of LAGA_NOALLOC_SCRATCH_BYTES that the library
 * holds on each GPU it runs on until the process ends (the entry point itself calls no
 * allocator). Limits and behaviour:
 *   - a problem whose laga_workspace_bytes(p, LAGA_OP_BWD) exceeds the array returns
 *     LAGA_ERR_SCRATCH before any launch (e.g. bf16 V3 heads, H = 16: S up to 2048
 *     with dq_mode RECOMPUTE, up to 1024 with FROM_STORE);
 *   - the array belongs to the current device; `stream` (NULL: the default stream) must
 *     be a stream of that device, else LAGA_ERR_DEVICE;
 *   - every call on one GPU uses the same array, and a call leaves its contents behind:
 *     calls that can overlap on one GPU (on different streams, or from different host
 *     threads without ordering) race and must not be issued. */
#define LAGA_NOALLOC_SCRATCH_BYTES ((size_t)128 << 20)
LAGA_API laga_status_t laga_attn_bwd_noalloc(const laga_problem_t* p, const void* q,
                                             const void* c_kv, const void* k_pe,
                                             const void* w_kv_b, const void* kv, const void* out,
                                             const float* lse, const void* dout, void* dq,
                                             float* dc_kv, float* dk_pe, float* dw_kv_b,
                                             void* stream);

/* ---- Producers around the latent all-gather ---------------------------------
 * The per-token steps that make this block's inputs and consume its gradients
 * (Alg. 1 step 1's latent normalisation; the decoupled RoPE of Section 2.1,
 * property P2, and Section 5.3). Token t of the sequence axis sits at position
 * p = position_offset + t (0 for the gathered sequence; a rank's chunk of S/P
 * tokens starts at r*S/P). R(p) rotates each pair (2i, 2i+1) of a d_rope-wide
 * band counter-clockwise by p * rope_base^(-2i/d_rope):
 * (x0, x1) -> (x0 cos - x1 sin, x0 sin + x1 cos). The problem must be valid as
 * for the attention calls; its softmax_scale, causal and kv_mode are not used. */
typedef struct {
  float eps;               /* added to the mean square, >= 0 (e.g. 1e-6) */
  float rope_base;         /* rotary base, > 1 (e.g. 10000) */
  int64_t position_offset; /* position of token 0, 0 <= offset, offset + S < 2^53 */
} laga_prologue_t;

/* Forward, per token (b, t):
 *   rstd[b,t]  = 1 / sqrt(mean_j latent_raw[b,t,j]^2 + eps)               fp32 [B,S]
 *   c_kv[b,t,j] = latent_raw[b,t,j] * rstd[b,t] * gamma[j]  (gamma NULL: 1) [B,S,d_c]
 *   k_pe[b,t,:] = R(p) kpe_raw[b,t,:]                                      [B,S,d_rope]
 *   q[b,t,h,d_nope:] = R(p) q[b,t,h,d_nope:] for every head, IN PLACE; the
 *                      q_nope columns are left untouched; q may be NULL.
 * latent_raw [B,S,d_c], gamma [d_c], kpe_raw [B,S,d_rope] and q [B,S,H,d_nope+
 * d_rope] are in the element dtype, as are c_kv and k_pe. Statistics in fp32.
 * No workspace. Errors: LAGA_ERR_NULL (problem, cfg or a required pointer),
 * LAGA_ERR_SHAPE (eps < 0, rope_base <= 1, offset out of range, or the problem),
 * LAGA_ERR_ALIGN, LAGA_ERR_UNSUPPORTED (dims as for the attention calls). */
LAGA_API laga_status_t laga_prologue_fwd(const laga_problem_t* p, const laga_prologue_t* cfg,
                                         const void* latent_raw, const void* gamma,
                                         const void* kpe_raw, void* q, void* c_kv,
                                         void* k_pe, float* rstd, void* stream);

/* Backward of laga_prologue_fwd, given the complete fp32 gradients dc_kv [B,S,d_c]
 * and dk_pe [B,S,d_rope] (on one rank with every head: laga_attn_bwd's; across
 * ranks: after the reduce-scatter of Section 5.2) and dq:
 *   d_latent_raw = rstd * (g - y * mean_j(g y)),  y = rstd * latent_raw,
 *                  g = gamma * dc_kv (gamma NULL: dc_kv)                 fp32 [B,S,d_c]
 *   d_gamma[j]   = sum over (b, t) of dc_kv[b,t,j] * y[b,t,j], in a fixed order
 *                  (bitwise repeatable)           fp32 [d_c]; required iff gamma given
 *   d_kpe_raw    = R(p)^T dk_pe                                        fp32 [B,S,d_rope]
 *   dq[b,t,h,d_nope:] = R(p)^T dq[b,t,h,d_nope:], IN PLACE (element dtype); may be NULL.
 * rstd is the forward's. With gamma the workspace must hold
 * laga_workspace_bytes(p, LAGA_OP_PROLOGUE_BWD) bytes (partial sums of d_gamma);
 * without, it may be NULL. Errors as for the forward, plus LAGA_ERR_WORKSPACE. */
LAGA_API laga_status_t laga_prologue_bwd(const laga_problem_t* p, const laga_prologue_t* cfg,
                                         const void* latent_raw, const void* gamma,
                                         const float* rstd, const float* dc_kv,
                                         const float* dk_pe, void* dq, float* d_latent_raw,
                                         float* d_kpe_raw, float* d_gamma, void* workspace,
                                         size_t workspace_bytes, void* stream);

/* ---- Consumer of the block: the output projection (Alg. 1 step 7) -------------
 * After the out all-to-all (Alg. 1 step 6) a rank holds the attention output of every
 * head for its tokens; step 7 returns W_o(reshape(out)):
 *   out  [T, n_heads, d_v]    element dtype (head-major: feature f = h * d_v + e)
 *   w_o  [F, d_model]         element dtype, F = n_heads * d_v (in x out)
 *   y    [T, d_model]         element dtype:  y = reshape(out) @ w_o
 * and its backward given dy [T, d_model] (element dtype):
 *   d_out [T, n_heads, d_v]   element dtype:  d_out = dy @ w_o^T
 *   dw_o  [F, d_model]        fp32:           dw_o = reshape(out)^T @ dy (over all T tokens,
 *                             in a fixed order: bitwise repeatable)
 * fp32 accumulation throughout. T is whatever rows the caller has: a rank's S/P tokens
 * after the all-to-all, or B*S on one rank. Validation as for the attention calls: NULL
 * problem or pointer -> LAGA_ERR_NULL; a non-positive size -> LAGA_ERR_SHAPE; F or d_model
 * not a multiple of 16, an unknown dtype, reserved != 0, or T*F, T*d_model or F*d_model
 * not below 2^31 -> LAGA_ERR_UNSUPPORTED; misaligned -> LAGA_ERR_ALIGN; workspace smaller
 * than laga_out_proj_workspace_bytes() -> LAGA_ERR_WORKSPACE. */
typedef struct {
  int64_t tokens;  /* T */
  int64_t n_heads; /* every head of the layer */
  int64_t d_v;
  int64_t d_model; /* D */
  int32_t dtype;   /* laga_dtype_t */
  int32_t reserved; /* must be 0 */
} laga_out_proj_t;

LAGA_API laga_status_t laga_out_proj_fwd(const laga_out_proj_t* p, const void* out, const void* w_o,
                                         void* y, void* stream);
LAGA_API laga_status_t laga_out_proj_bwd(const laga_out_proj_t* p, const void* out, const void* w_o,
                                         const void* dy, void* d_out, float* dw_o, void* workspace,
                                         size_t workspace_bytes, void* stream);
/* Workspace of laga_out_proj_bwd (partial sums of dw_o over token ranges); 0 if none is
 * needed or p is invalid. */
LAGA_API size_t laga_out_proj_workspace_bytes(const laga_out_proj_t* p);

/* ---- Serving: new tokens against a paged cache of latents ----------------------
 * A model that this block trained answers one token per request and step. What a step
 * reads of the past is a cached position's row [c_kv || k_pe] (the normalised latent and
 * the shared rotated key, which every head reads), held in pages of a pool:
 *   cache       [n_pages][page_size, d_c + d_rope]  element dtype, rows contiguous, pages
 *                                    page_stride elements apart (page offsets are 64-bit)
 *   block_table [requests, table_width]  int32: position j of request r is in page
 *                                    block_table[r][j / page_size], row j % page_size
 *   lengths     [requests]           int32: cached positions of each request
 *   free_pages  [n_pages]            int32: a stack, its free_count[0] first entries free
 *   row_request, position, slot [rows] int32: of each of the step's new tokens its
 *                                    request, its position in it, and page * page_size +
 *                                    row where it is cached; -1 in rows of padding
 * all on the device; a decoding step is laga_page_plan, laga_cache_append,
 * laga_paged_attn (and laga_out_proj_fwd), none of which reads a length on the host, so a
 * captured step serves every later one. Conventions as above, and:
 *   - an index that the device finds out of range is never followed: a slot outside the
 *     pool stores nothing; a row whose request or position lies outside the table, or one
 *     of whose visible pages lies outside the pool, gets NaN in every output element;
 *   - cached rows past a row's position, and table entries past a request's pages, are
 *     never read: they may hold anything;
 *   - repeated calls are bit-identical; the attention's sums over a row's keys are grouped
 *     by how the call's tiles are shared out, so a row's last bits (of fp32 sums) may depend on the
 *     other rows' lengths and on n_heads, its precision does not.
 * Limits: head dims and d_c as for the attention calls; page_size >= 1; page_stride 0 (read
 * as page_size * (d_c + d_rope)) or at least that and a multiple of 8; n_pages * page_size,
 * requests * table_width, rows * n_heads, rows * (table_width * page_size / 32 + 10) and
 * 16 * d_c * n_heads * (d_nope + d_v) below 2^31;
 * table_width * page_size at most 2^30; rows below 2^22, rows * ceil(n_heads / 8) below 2^24;
 * else LAGA_ERR_UNSUPPORTED. A size <= 0 is LAGA_ERR_SHAPE. */
typedef struct {
  int64_t rows;        /* T: new tokens of the step, rows of padding included */
  int64_t requests;    /* R */
  int64_t table_width; /* entries of a request in block_table */
  int64_t n_pages, page_size;
  int64_t page_stride; /* elements between pages; 0: page_size * (d_c + d_rope) */
  int64_t n_heads, d_c, d_nope, d_rope, d_v; /* as in laga_problem_t */
  float softmax_scale;
  int32_t dtype;       /* laga_dtype_t */
  int32_t reserved;    /* must be 0 */
} laga_paged_t;

/* Bits of the status[0] that laga_page_plan and laga_page_release write (0: done). */
enum {
  LAGA_PLAN_ROWS = 1,    /* more new tokens than rows */
  LAGA_PLAN_TABLE = 2,   /* a request would not fit in table_width pages */
  LAGA_PLAN_PAGES = 4,   /* fewer free pages than needed; release: more than the stack holds */
  LAGA_PLAN_INVALID = 8  /* a negative length or count, or free_count outside [0, n_pages] */
};

typedef enum { LAGA_OP_PAGE_PLAN = 3, LAGA_OP_PAGED_ATTN = 4, LAGA_OP_PAGED_ATTN_Q8 = 5 } laga_paged_op_t;

/* Pages, slots and positions of a step that adds fresh[r] >= 0 tokens to request r:
 *   request r's ceil((lengths[r] + fresh[r]) / page_size) - ceil(lengths[r] / page_size) new
 *   pages are popped from the stack's end, requests in order, into block_table (its other
 *   entries stay); lengths_out = lengths + fresh; free_count_out[0] = free_count[0] - pages;
 *   row_begin [requests + 1]: the requests' first rows (exclusive sums of fresh); rows
 *   row_begin[r] .. are request r's new tokens in order, rows from row_begin[requests] on are
 *   padding (-1).
 * lengths_out may be lengths and free_count_out free_count (in place). All or nothing: if
 * the step does not fit, status[0] says why (LAGA_PLAN_*), lengths_out and free_count_out are
 * the inputs, block_table stays, row_begin is 0 and every row padding (so the calls after it
 * store nothing and return empty rows). Workspace: laga_paged_workspace_bytes(p,
 * LAGA_OP_PAGE_PLAN). */
LAGA_API laga_status_t laga_page_plan(const laga_paged_t* p, const int32_t* lengths,
                                      const int32_t* fresh, int32_t* block_table,
                                      const int32_t* free_pages, const int32_t* free_count,
                                      int32_t* lengths_out, int32_t* free_count_out,
                                      int32_t* row_begin, int32_t* row_request, int32_t* position,
                                      int32_t* slot, int32_t* status, void* workspace,
                                      size_t workspace_bytes, void* stream);

/* The pages of every request with drop[r] != 0 go back on the stack, requests and their
 * pages in order; its lengths_out is 0 (its table entries stay and mean nothing). In place
 * as above; all or nothing as above. Same workspace. */
LAGA_API laga_status_t laga_page_release(const laga_paged_t* p, const int32_t* lengths,
                                         const int32_t* drop, const int32_t* block_table,
                                         int32_t* free_pages, const int32_t* free_count,
                                         int32_t* lengths_out, int32_t* free_count_out,
                                         int32_t* status, void* workspace, size_t workspace_bytes,
                                         void* stream);

/* The cache rows of a step's tokens: with the producers' arithmetic (laga_prologue_fwd),
 *   cache row slot[t] = [ gamma * x * rsqrt(mean(x^2) + eps) || R(position_offset + position[t]) k ]
 * of x = latent_raw[t], k = kpe_raw[t] (element dtype; rows latent_stride and kpe_stride
 * elements apart, multiples of 8 and at least d_c and d_rope: both may be columns of one
 * projection's output). Rows whose slot lies outside the pool store nothing. Slots of one
 * call must differ (of two tokens with one slot, either's elements may be stored).
 * gamma may be NULL. */
LAGA_API laga_status_t laga_cache_append(const laga_paged_t* p, const laga_prologue_t* cfg,
                                         const void* latent_raw, int64_t latent_stride,
                                         const void* gamma, const void* kpe_raw, int64_t kpe_stride,
                                         const int32_t* position, const int32_t* slot, void* cache,
                                         void* stream);

/* Attention of rows over their requests' cached positions 0 .. position[t] (the row's own
 * among them, appended before): laga_attn_fwd's result at that row, from the cache alone,
 *   out [rows, n_heads, d_v] element dtype, lse [rows, n_heads] fp32 (may be NULL)
 * for q [rows, n_heads, d_nope + d_rope]. With cfg, q's rope band is turned by the row's
 * position_offset + position[t] first (q is not written; cfg's eps is not used); NULL: it
 * has been. row_request NULL: row t is request t. A row at a negative position sees nothing:
 * out 0, lse -infinity. Any number of rows may belong to one request.
 * The product with W_kv_b's K columns is taken on the query's side and the one with its V
 * columns after the softmax. Statistics, sums and joins of a row's parts are fp32. In bf16 the
 * values in between keep 16 bits of mantissa or more, so out is the exact result rounded once, to
 * little more than that, for scores of any spread. Workspace: laga_paged_workspace_bytes(p, LAGA_OP_PAGED_ATTN). */
LAGA_API laga_status_t laga_paged_attn(const laga_paged_t* p, const laga_prologue_t* cfg,
                                       const void* q, const void* w_kv_b, const void* cache,
                                       const int32_t* block_table, const int32_t* row_request,
                                       const int32_t* position, void* out, float* lse,
                                       void* workspace, size_t workspace_bytes, void* stream);

/* ---- The same from a cache held in 8 bits ---------------------------------------
 * About half the bytes of a bf16 cache, kept and read. A cached position is d_c + d_rope
 * numbers of 8 bits, and one scale for each of its two parts, the latent and the shared key:
 *   cache   [n_pages][page_size, d_c + d_rope]  e4m3 (finite, 448 the largest; one byte), rows
 *                      contiguous, pages page_stride BYTES apart (a multiple of 16; 0:
 *                      page_size * (d_c + d_rope), which is one)
 *   scales  [n_pages][page_size][2]  uint8, contiguous: byte x stands for 2^(x - 127), 255 for NaN;
 *                      [0] is the latent's, [1] the key's
 * so element j of the latent is cache[j] * 2^(scales[0] - 127). laga_paged_t and the conventions
 * of the calls above hold as they are (dtype: of q, W_kv_b, out and the tokens), pages are planned
 * and released by the same calls, and the limits are theirs (rows * (table_width * page_size / 32 + 15) below 2^31).
 *
 * laga_cache_append_q8: laga_cache_append, its row quantised as it is written. With a the
 * largest finite magnitude of a part's elements, the part's scale is 2^e, e the least whole
 * number with a <= 448 * 2^e, -100 at least and 119 at most, and each element the e4m3 number
 * nearest to x / 2^e (ties to even), +-448 beyond them, NaN where x is not finite. The row is formed
 * in double precision, so the byte is that of the exact value. Slots of one call must differ (of
 * two tokens with one slot, either's bytes and scales may be stored).
 *
 * laga_cache_read_q8: cached positions back as numbers, row t the position[t] of request
 * row_request[t] (NULL: of request t):
 *   c_kv [rows, d_c], k_pe [rows, d_rope]  element dtype
 * to export or inspect a request, to write it to a cache in other bits, or to compute over its whole
 * sequence again (laga_reconstruct_kv, laga_attn_fwd: as many queries as keys). A chunk of a prompt over
 * its cached prefix goes through laga_paged_attn_q8, a row per new token. Exact in both element types (in bf16 and fp32 an e4m3
 * number times a power of two that the append writes has all its bits). A row at a negative position is 0; one
 * outside the table, or whose page lies outside the pool, NaN.
 *
 * laga_paged_attn_q8: laga_paged_attn on the numbers that the cache stands for. A NaN
 * among the visible ones makes the rows that see it NaN, as would an infinity's product with zero. Statistics, sums and
 * joins are fp32, the products take a query's number with 22 bits down to 2^-17 of its
 * part's largest (q_rope, or q_nope times W_k) and within 2^-39 of that below, and a probability times its key's
 * power with 22 bits or within 2^-29 of the largest so far. */
LAGA_API laga_status_t laga_cache_append_q8(const laga_paged_t* p, const laga_prologue_t* cfg,
                                            const void* latent_raw, int64_t latent_stride,
                                            const void* gamma, const void* kpe_raw, int64_t kpe_stride,
                                            const int32_t* position, const int32_t* slot, void* cache,
                                            uint8_t* scales, void* stream);
LAGA_API laga_status_t laga_cache_read_q8(const laga_paged_t* p, const void* cache, const uint8_t* scales,
                                          const int32_t* block_table, const int32_t* row_request,
                                          const int32_t* position, void* c_kv, void* k_pe, void* stream);
LAGA_API laga_status_t laga_paged_attn_q8(const laga_paged_t* p, const laga_prologue_t* cfg,
                                          const void* q, const void* w_kv_b, const void* cache,
                                          const uint8_t* scales, const int32_t* block_table,
                                          const int32_t* row_request, const int32_t* position, void* out,
                                          float* lse, void* workspace, size_t workspace_bytes,
                                          void* stream);

/* Workspace bytes of op (laga_paged_op_t); 0 if p is invalid. */
LAGA_API size_t laga_paged_workspace_bytes(const laga_paged_t* p, int op);

/* Workspace bytes that op (laga_op_t) needs for problem p; 0 if none or if p
 * is invalid (check with the entry point itself for the error code). For the
 * backward in bf16 with 192/128-wide heads and dq_mode FROM_STORE this includes the
 * dS^T store: 2 * B * H * 512 * T * (T + 1) bytes with the causal mask
 * (2 * B * H * 1024 * T^2 without), T = ceil(S / 32) -- about 4.3 GB at S = 16384,
 * H = 16. With dq_mode RECOMPUTE the backward workspace is linear in S. */
LAGA_API size_t laga_workspace_bytes(const laga_problem_t* p, int op);

/* Static, never-NULL description of a status code. */
LAGA_API const char* laga_status_string(laga_status_t s);

/* LAGA_ABI_VERSION of the built library. */
LAGA_API int laga_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LAGA_H_ */
