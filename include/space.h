/* libspace - one auto-correct decoding step of SPACE (arXiv 2402.11809) on
 * NVIDIA B200 (sm_100a).
 *
 * One step is the single model invocation of Algorithm 1: the block of
 * (k+1)^2 query rows (last verified token, k candidates, k+1 groups of k mask
 * tokens, Eq. 4) attends over the verified KV cache under the mask of Eq. 5,
 * the resulting logits verify the candidates and propose the next ones
 * (Algorithm 1, Sec. 3.2), and the accepted rows are compacted into the cache.
 *
 * Conventions
 *  - Every pointer named "device" must be device memory of the context's GPU;
 *    "host" pointers are ordinary host memory.  The library never takes
 *    ownership of a caller buffer; it borrows it until the work enqueued on
 *    the given stream has finished.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the legacy default
 *    stream).  All entry points except space_step_host are asynchronous and
 *    perform no allocation and no synchronisation after space_create.
 *  - Every entry point that takes a context makes the context's device the
 *    calling thread's current device (cudaSetDevice) and leaves it current.
 *  - Return value: SPACE_OK or a negative SPACE_E_* code; nothing aborts.
 *    Conditions only the GPU can see are reported per sequence in the
 *    `status` array (bit set of SPACE_ST_*).
 *  - Block row order: row g*(k+1)+o, g = 0..k sub-block, o = 0 the real token
 *    (root for g = 0, candidate c_g otherwise), o = 1..k the o-th mask token.
 */
#ifndef SPACE_H
#define SPACE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPACE_MAX_K     7      /* (k+1)^2 <= 64 block rows                    */
#define SPACE_MAX_ROWS  64
#define SPACE_PAGE_SIZE 128    /* key rows per page of a paged cache (the kernels' key tile) */

enum {
  SPACE_OK            =  0,
  SPACE_E_INVALID_ARG = -1,    /* NULL pointer, size out of range             */
  SPACE_E_UNSUPPORTED = -2,    /* shape outside what the kernels implement    */
  SPACE_E_ALIGNMENT   = -3,    /* base pointer / stride not 16-byte aligned   */
  SPACE_E_WORKSPACE   = -4,    /* request exceeds what space_create reserved  */
  SPACE_E_CUDA        = -5,    /* a CUDA runtime or driver call failed        */
  SPACE_E_NO_DEVICE   = -6,    /* no usable sm_100 device                     */
  SPACE_E_STATIC_LIMIT = -7    /* size beyond the fixed scratch of space_verify_greedy_noalloc */
};

enum { SPACE_MASK_SAME_GROUP = 0, SPACE_MASK_EQ5_LITERAL = 1 };
enum { SPACE_MODE_GREEDY = 0, SPACE_MODE_SAMPLE = 1 };
enum { SPACE_RESAMPLE_RESIDUAL_POINTMASS = 0, SPACE_RESAMPLE_PAPER_LITERAL = 1, SPACE_RESAMPLE_RESIDUAL_DRAFT = 2 };
enum { SPACE_DTYPE_BF16 = 0, SPACE_DTYPE_F32 = 1 };
enum { SPACE_ATTN_TENSOR = 0, SPACE_ATTN_SIMT = 1, SPACE_ATTN_TENSOR_ROWS = 2 };

/* per-sequence device status bits */
enum {
  SPACE_ST_CAPACITY      = 1,  /* kv_len + (k+1)^2 exceeds the cache capacity */
  SPACE_ST_BAD_CANDIDATE = 2,  /* a candidate id outside [0, vocab): rejected */
  SPACE_ST_TIMEOUT       = 4,  /* a bounded on-chip wait expired              */
  SPACE_ST_BAD_PAGE      = 8,  /* a page-table entry outside [0, n_pages): that page is not
                                  touched (attention reads zeros in its place, the commit skips
                                  the row)                                     */
  SPACE_ST_NONFINITE     = 16, /* a row handed to the 4-bit or 8-bit cache (space_kvq_*, space_kvb_*) held a
                                  NaN, counted as 0, or an infinity, counted as the largest finite bf16 */
  SPACE_ST_BAD_POSITION  = 32, /* a position outside the rotation table: the nearest one in it was used */
  SPACE_ST_BAD_MASK      = 64  /* space_logits_adjust: a mask number from n_masks on (the row counts as one
                                  without a mask), or a mask that leaves a row no token          */
};

typedef struct space_ctx space_ctx;   /* opaque; owns only its own workspace */

typedef struct {
  int32_t device;        /* CUDA device ordinal                                */
  int32_t max_batch;     /* largest batch any call will pass                   */
  int32_t n_q_heads;     /* H_q                                                */
  int32_t n_kv_heads;    /* H_kv, divides H_q; H_q/H_kv in {1,2,4,8,16}        */
  int32_t head_dim;      /* d in {64, 128}                                     */
  int32_t k_max;         /* largest k any call will pass, 1..SPACE_MAX_K       */
  int32_t vocab;         /* largest vocabulary any verify call will pass       */
  int32_t host_staging;  /* != 0: also reserve device staging for space_step_host */
  int64_t s_cap;         /* cache capacity (rows) per sequence and KV head     */
} space_config;

/* Block layout of Eq. 4 with the visibility rule of Eq. 5 and the position
 * rule of Sec. 3.2 (position = number of visible keys - 1). */
typedef struct {
  int32_t  k;
  int32_t  n_q;                          /* (k+1)^2                            */
  uint8_t  kind[SPACE_MAX_ROWS];         /* 0 real token, 1 mask token         */
  uint8_t  group[SPACE_MAX_ROWS];        /* sub-block g                        */
  uint8_t  offset[SPACE_MAX_ROWS];       /* o                                  */
  int32_t  relpos[SPACE_MAX_ROWS];       /* position id minus kv_len           */
  uint64_t mask[SPACE_MAX_ROWS];         /* bit j: row attends to block row j  */
  int32_t  target_rows[SPACE_MAX_K + 1]; /* row of the real token of sub-block t */
} space_layout_t;

/* Attention of the block over cache + block (Algorithm 1 model call restricted
 * to the attention operator; Eq. 5).  The caller has already written the
 * block's K/V rows at cache positions kv_len[b] .. kv_len[b]+n_q-1. */
typedef struct {
  int32_t batch;            /* B <= max_batch                                  */
  int32_t k;                /* candidates per sequence                         */
  int32_t mask_variant;     /* SPACE_MASK_*                                    */
  int32_t out_dtype;        /* SPACE_DTYPE_F32 or SPACE_DTYPE_BF16             */
  int32_t impl;             /* SPACE_ATTN_TENSOR (default: keys on the MMA M extent),
                               SPACE_ATTN_TENSOR_ROWS (query rows on M) or SPACE_ATTN_SIMT */
  float   scale;            /* softmax scale, normally 1/sqrt(d)               */
  const void*    q;         /* device bf16 [B, n_q, H_q, d], contiguous        */
  const void*    k_cache;   /* device bf16, element (b,h,s,:) at               */
  const void*    v_cache;   /*   b*stride_b + h*stride_h + s*stride_s (elements), d contiguous */
  int64_t kv_stride_b, kv_stride_h, kv_stride_s;  /* multiples of 8 elements   */
  const int32_t* kv_len;    /* device [B] verified lengths L_b                 */
  void*          out;       /* device [B, n_q, H_q, d] of out_dtype            */
  float*         lse;       /* device [B, H_q, n_q] natural-log sum-exp, or NULL */
  int32_t*       status;    /* device [B], OR-ed with SPACE_ST_*, or NULL      */
  /* Paged cache (the serving setting of Sec. 4.3: continuous batching over a pool of pages).
     page_table == NULL: the contiguous cache described above.  Otherwise k_cache / v_cache are
     pools of pages of SPACE_PAGE_SIZE key rows, element (page, h, r, :) at
     page*kv_stride_b + h*kv_stride_h + r*kv_stride_s, and key position s of sequence b (cache
     rows and the block's own rows L_b .. L_b+n_q-1 alike) is row s % SPACE_PAGE_SIZE of page
     page_table[b*pages_per_seq + s / SPACE_PAGE_SIZE].  A sequence's capacity is
     pages_per_seq * SPACE_PAGE_SIZE rows (it replaces s_cap in the SPACE_ST_CAPACITY check, and
     must not exceed the context's s_cap).  Entries past the pages a sequence needs are
     ignored.  Rows of its last page beyond L_b+n_q may hold anything, NaN included.            */
  const int32_t* page_table;   /* device [B, pages_per_seq] or NULL                            */
  int32_t pages_per_seq;
  int32_t n_pages;             /* pages in the pool                                            */
} space_attn_args;

/* Verification and emission (Algorithm 1 after the model call; Sec. 3.2). */
typedef struct {
  int32_t batch, k, vocab;
  int32_t logits_dtype;        /* SPACE_DTYPE_BF16 or SPACE_DTYPE_F32          */
  int32_t mode;                /* SPACE_MODE_*                                 */
  int32_t resample;            /* SPACE_RESAMPLE_* (sampling mode only)        */
  int32_t eos_id;              /* -1: no end-of-sequence handling              */
  float   temperature;         /* > 0 (sampling mode)                          */
  uint64_t seed;               /* Philox key                                   */
  const void*     logits;      /* device [B, n_q, V]; row stride below         */
  int64_t         logits_row_stride;   /* elements between rows; batch stride = n_q * row stride */
  const int32_t*  cand;        /* device [B, k]  L_c                           */
  const float*    cand_prob;   /* device [B, k]  P_c: probability the candidate was drafted with
                                  (sampling mode; ignored in greedy mode).  +inf is Algorithm 1's
                                  initial state and is always rejected; a candidate is accepted only
                                  if its id is in range, P_c > 0 and r * P_c <= Q(c) (NaN, zero and
                                  negative values are rejected).  With SPACE_RESAMPLE_RESIDUAL_POINTMASS
                                  a rejected candidate is removed from the extra token's distribution
                                  only when its P_c is exactly 1 (a point-mass draft); after the
                                  rejection of any other P_c the extra token is drawn from Q itself */
  const uint32_t* seq_id;      /* device [B] or NULL (= batch index)           */
  const int32_t*  kv_len;      /* device [B]: positions for the random counters */
  int32_t* n_accept;           /* device [B]       i*                          */
  int32_t* out_tokens;         /* device [B, k+1]  emitted tokens, -1 padded   */
  int32_t* n_out;              /* device [B]       emitted count               */
  int32_t* next_cand;          /* device [B, k]                                */
  float*   next_cand_prob;     /* device [B, k]                                */
  uint8_t* finished;           /* device [B]       1 once <EOS> was emitted    */
  int32_t* status;             /* device [B] or NULL                           */
  int32_t top_k;               /* sampling mode: 0 = unfiltered; 1..32 = every distribution that is tested
                                  against or sampled from is softmax(z/T) over its top_k largest logits
                                  (lowest token first on ties), cut to the shortest prefix, in descending
                                  order, whose probability reaches top_p, and renormalised (App. A.4 runs
                                  sampling with top-k = 10, top-p = 0.95); ignored in greedy mode        */
  float   top_p;               /* in (0, 1] when top_k > 0 (1 = no nucleus cut)                         */
  /* SPACE_RESAMPLE_RESIDUAL_DRAFT (sampling mode with top_k > 0 through space_verify / space_verify_commit;
     ignored otherwise): sampled candidates whose rejection keeps the output distribution unchanged
     (Sec. 3.2).  Candidate o of the next step is drawn from the filtered distribution D_o of its mask row,
     P_c = D_o(candidate), and D_o is handed on as a list of top_k (token, probability) pairs in descending
     order, dropped entries as (-1, 0).  After rejecting candidate i the extra token is drawn from
     norm(max(0, Q - D_i)) (from Q if that has no mass), after k acceptances from Q.                      */
  const int32_t* draft_tok;    /* device [B, k, top_k] lists the candidates were drawn from, or NULL together
                                  with draft_prob (no lists: Algorithm 1's initial state, a ~ Q)          */
  const float*   draft_prob;   /* device [B, k, top_k]; entries with a token outside [0, vocab) or a
                                  probability that is not positive and finite do not count              */
  int32_t* next_draft_tok;     /* device [B, k, top_k]: lists of the next candidates (required)          */
  float*   next_draft_prob;    /* device [B, k, top_k]                                                   */
} space_verify_args;

/* Output projection fused with verification: the end of the model call P = M(I) of
 * Algorithm 1 (logits[r, x] = <h_r, W_x> for every block row r and vocabulary token
 * x; the rows of P are softmax(logits / T)) and the loop after it (acceptance of the
 * candidates -- against the arg-max chain in greedy mode, by r <= Q/P_c with Philox
 * draws in sampling mode --, extra token, <EOS>, next candidates from the mask rows of
 * group i*; Sec. 3.2).  The logits are never written: only per-row statistics
 * (maximum, lowest arg-max, sum of exponentials, best noisy score) leave the chip. */
#define SPACE_LMHEAD_MAX_ROWS 256   /* block rows one kernel launch covers; a larger batch is
                                       split into groups of sequences, one launch (and one pass
                                       over the output embedding) per group                   */
typedef struct {
  int32_t batch, k, vocab;
  int32_t hidden_dim;          /* D, a multiple of 8                           */
  int32_t eos_id;              /* -1: no end-of-sequence handling              */
  int32_t mode;                /* SPACE_MODE_GREEDY or SPACE_MODE_SAMPLE       */
  int32_t resample;            /* SPACE_RESAMPLE_* (sampling mode)             */
  float   temperature;         /* > 0 (sampling mode)                          */
  uint64_t seed;               /* Philox key (sampling mode), keyed as in space_verify */
  const void* hidden;          /* device bf16 [B * n_q, D]: final hidden state of every block row,
                                  sequence-major, block row order               */
  int64_t hidden_row_stride;   /* elements between rows, a multiple of 8       */
  const void* weight;          /* device bf16 [V, D]: output embedding, one row per token */
  int64_t weight_row_stride;   /* elements between rows, a multiple of 8       */
  const int32_t* cand;         /* device [B, k]  L_c                           */
  const float*   cand_prob;    /* device [B, k]  P_c (sampling mode; may be NULL in greedy mode);
                                  same rules as space_verify_args.cand_prob    */
  const uint32_t* seq_id;      /* device [B] or NULL (= batch index): sequence ids of the random counters */
  const int32_t*  kv_len;      /* device [B] or NULL (= 0): positions of the random counters */
  int32_t* n_accept;           /* device [B]       i*                          */
  int32_t* out_tokens;         /* device [B, k+1]  emitted tokens, -1 padded   */
  int32_t* n_out;              /* device [B]                                   */
  int32_t* next_cand;          /* device [B, k]                                */
  float*   next_cand_prob;     /* device [B, k]  greedy: softmax (T = 1) of the token's own row;
                                  sampling: as space_verify                    */
  uint8_t* finished;           /* device [B]                                   */
  int32_t* status;             /* device [B] or NULL                           */
  float*   row_max;            /* device [B * n_q] or NULL: largest logit of every block row */
  int32_t* row_argmax;         /* device [B * n_q] or NULL: its token (lowest on ties) */
} space_lmhead_args;

/* Compaction of the accepted rows (no counterpart in Algorithm 1, which
 * re-runs the model on the whole sequence; needed by any cached forward). */
typedef struct {
  int32_t batch, k;
  void*   k_cache;             /* device bf16, same addressing as space_attn_args */
  void*   v_cache;
  int64_t kv_stride_b, kv_stride_h, kv_stride_s;
  const int32_t* n_accept;     /* device [B] from space_verify                 */
  const int32_t* kv_len;       /* device [B] lengths before the step           */
  int32_t* kv_len_out;         /* device [B] lengths after, may alias kv_len, or NULL */
  int32_t* commit_src;         /* device [B, k+1] or NULL, -1 padded           */
  int32_t* commit_dst;         /* device [B, k+1] or NULL                      */
  int32_t* status;             /* device [B] or NULL                           */
  const int32_t* page_table;   /* paged cache as in space_attn_args, or NULL (contiguous)      */
  int32_t pages_per_seq;
  int32_t n_pages;
} space_commit_args;

/* Whole step from host memory (copies in, the three stages, copies out). */
typedef struct {
  int32_t batch, k, vocab, logits_dtype, mode, resample, eos_id, mask_variant;
  float   scale, temperature;
  uint64_t seed;
  const void*    q;            /* host bf16 [B, n_q, H_q, d]                   */
  void*          k_cache;      /* host bf16 [B, H_kv, s_cap, d]; committed rows are written back */
  void*          v_cache;
  const void*    logits;       /* host [B, n_q, V] contiguous                  */
  const int32_t* cand;         /* host [B, k]                                  */
  const float*   cand_prob;    /* host [B, k]                                  */
  int32_t*       kv_len;       /* host [B]; updated in place                   */
  float*    out;               /* host f32 [B, n_q, H_q, d]                    */
  int32_t*  n_accept;          /* host [B]                                     */
  int32_t*  out_tokens;        /* host [B, k+1]                                */
  int32_t*  n_out;             /* host [B]                                     */
  int32_t*  next_cand;         /* host [B, k]                                  */
  float*    next_cand_prob;    /* host [B, k]                                  */
  uint8_t*  finished;          /* host [B]                                     */
  int32_t*  status;            /* host [B]                                     */
  int64_t*  h2d_bytes;         /* host, optional: bytes of input the device is handed (all rows of logits, though
                                  from pinned buffers only those the step decides on travel) */
  int64_t*  d2h_bytes;         /* host, optional: bytes handed back            */
  int32_t   cache_resident;    /* 0: upload rows 0 .. kv_len+n_q-1 of every sequence's K and V.
                                  1: the KV cache is the decoder's state and already sits in the context's
                                  staging copy from an earlier call (rows 0 .. kv_len-1 of every sequence,
                                  as that call's commit left them); only the block's own rows
                                  kv_len .. kv_len+n_q-1 are uploaded                               */
  int32_t   reserved;          /* 0                                                              */
} space_host_step_args;

/* Create a context on cfg->device: validates the shape, reserves the
 * workspace (split partials, reduction scratch, counters, optional staging).
 * Errors: INVALID_ARG, UNSUPPORTED, NO_DEVICE, CUDA. */
int space_create(space_ctx** out, const space_config* cfg);
void space_destroy(space_ctx* ctx);

/* Device bytes space_create reserves for cfg (0 on invalid cfg). */
size_t space_workspace_bytes(const space_config* cfg);

/* Host only.  Eq. 4 row kinds, Eq. 5 visibility (mask_variant picks the
 * same-group reading of Sec. 3.2 / App. A.3 or Eq. 5 as printed), Sec. 3.2
 * position ids.  Errors: INVALID_ARG for k outside 1..SPACE_MAX_K. */
int space_layout(int k, int mask_variant, space_layout_t* out);

/* Eq. 5 attention of the (k+1)^2 block rows over cache + block. */
int space_attn_step(space_ctx* ctx, const space_attn_args* args, void* stream);

/* Algorithm 1 verification loop, extra token and next candidates. */
int space_verify(space_ctx* ctx, const space_verify_args* args, void* stream);

/* space_verify followed by space_kv_commit with one kernel launch less: the
 * verification kernels also move the accepted cache rows (Algorithm 1's loop
 * body after the model call, then the compaction any cached forward needs).
 * Results are those of the two separate calls, with one freedom: cache rows
 * L+i*+1 .. L+k, which lie beyond the new length and held mask-token rows of
 * the step's block that nothing reads again, are left with unspecified block
 * rows (the single-launch greedy path moves all k candidate rows while the
 * logits still stream, before i* is known).  Rows below the new length and
 * rows from L+k+1 on are exactly as space_kv_commit leaves them.
 * commit->n_accept must be
 * verify->n_accept, and batch and k must agree (INVALID_ARG otherwise); every
 * other rule of the two calls applies.  The attention that reads the cache rows
 * of this step must have been enqueued on `stream` before this call. */
int space_verify_commit(space_ctx* ctx, const space_verify_args* verify, const space_commit_args* commit,
                        void* stream);

/* Greedy verification without any allocation.  (The paper has no counterpart:
 * this entry point exists for how the library is embedded, not for the method.)
 *
 * Some hosts of this library may not allocate device memory once they are
 * running: a serving process that hands all of the GPU's memory to its own pool
 * at start-up leaves nothing for cudaMalloc, and a latency-critical decode loop
 * cannot afford the implicit device-wide synchronisation an allocation can
 * cause.  Such callers cannot use space_create, which reserves a workspace.
 * This call needs no context: its scratch (chunk results and per-sequence
 * arrival counters, SPACE_NOALLOC_MAX_BATCH * 32 KiB + 256 bytes) is a fixed
 * array inside the library image, resident on every GPU that loads the library
 * until the process exits.  It calls no cudaMalloc / cudaFree and no allocating
 * library routine.
 *
 * Same arguments, outputs and results as space_verify in SPACE_MODE_GREEDY
 * (args->mode must be SPACE_MODE_GREEDY; temperature, seed, resample ignored);
 * all (k+1)^2 logits rows are read in one kernel.  Runs on the current device.
 * Limits: batch <= SPACE_NOALLOC_MAX_BATCH, else SPACE_E_STATIC_LIMIT; k in
 * 1..SPACE_MAX_K.
 * The first call on a device is a set-up call: it looks up the array's device
 * address (cudaGetSymbolAddress) and makes the CUDA runtime load the library's
 * device code, which is when the array and the kernels take their (fixed) share
 * of device memory.  Make that call once at start-up as a warm-up - before the
 * host's own pool takes the rest of the memory, and outside any stream capture.
 * Later calls on that device load nothing and reserve nothing.
 * All calls share the one array, which keeps the last call's contents: the
 * arrival counters are cleared at the start of every call, and two calls whose
 * kernels overlap on the GPU (different streams, or several host threads) race
 * on it - serialise them. */
#define SPACE_NOALLOC_MAX_BATCH 8
int space_verify_greedy_noalloc(const space_verify_args* args, void* stream);

/* One step from hidden states (see space_lmhead_args): the output embedding is read
 * once per group of at most SPACE_LMHEAD_MAX_ROWS block rows, products on the tensor cores
 * in bf16 with fp32 accumulation, every decision taken on the fp32 accumulators (arg-max:
 * lowest token on exact ties; sampling: the same tests and Gumbel arg-maxes as
 * space_verify, with the same Philox counters).  Same outputs as space_verify on the
 * logits the projection defines.  Asynchronous on `stream`, no allocation.  One call at
 * a time per context (the calls share the context's reduction scratch).
 * Errors: INVALID_ARG (NULL pointer, sizes, mode, temperature), WORKSPACE (batch or k
 * beyond the context's), ALIGNMENT (16-byte base, strides and D multiples of 8),
 * UNSUPPORTED (one sequence alone exceeds the rows of a launch: cannot happen for k <= 7), CUDA. */
int space_lmhead_verify(space_ctx* ctx, const space_lmhead_args* args, void* stream);

/* Move accepted rows L+g(k+1) -> L+g, g = 1..i*; lengths grow by i*+1. */
int space_kv_commit(space_ctx* ctx, const space_commit_args* args, void* stream);

/* The three stages from host buffers; synchronises `stream` before returning.
 * (The logits go up, or are verified, on a second stream of the context, ordered against
 * `stream` by events, beside the attention; when the call returns everything it enqueued on
 * either stream has finished.  With cache_resident and pinned, 16-byte aligned q, caches,
 * logits and out, kernels move the pieces, the attention stores its output into host memory and
 * verification reads the rows of logits it needs where they lie.)
 * Needs cfg.host_staging.  Only sequence prefixes in use are copied (with
 * cache_resident: only the block's rows, see the field).  The call stages the
 * small per-sequence arrays in a pinned buffer of the context: one call at a
 * time per context.  Errors: INVALID_ARG (NULL pointer, or a value that
 * space_attn_step or space_verify_commit refuses), WORKSPACE (no staging, or sizes
 * beyond cfg), both before anything is launched; CUDA, after which nothing that the
 * call launched is still running and the outputs are undefined. */
int space_step_host(space_ctx* ctx, const space_host_step_args* args, void* stream);

/* Device-resident state of the decoding loop (Algorithm 1 in full): the generated
 * tokens O, the candidates L_c with their probabilities P_c, the verified length, the
 * <EOS> latch, and the token and position ids of the block rows the next model call
 * evaluates (Eq. 4: the last verified token, then every candidate followed by k mask
 * tokens; Sec. 3.2: position = visible keys - 1).  All arrays are device memory owned
 * by the caller; the library only reads and writes them in the two calls below. */
typedef struct {
  int32_t batch, k;
  int32_t max_tokens;       /* capacity of `tokens` per sequence; a full buffer ends the sequence */
  int32_t mask_token_id;    /* id of the mask token [M]                                       */
  int32_t mask_variant;     /* SPACE_MASK_*: the reading of Eq. 5 the position ids follow     */
  int32_t reserved;         /* 0                                                              */
  int32_t* tokens;          /* [B, max_tokens] generated tokens (the prompt is not stored)    */
  int32_t* n_tokens;        /* [B]   how many of them                                         */
  int32_t* last_token;      /* [B]   x_l: the last verified token, whose KV is not cached yet */
  int32_t* cand;            /* [B, k] L_c                                                     */
  float*   cand_prob;       /* [B, k] P_c                                                     */
  int32_t* kv_len;          /* [B]   verified cache length L_b (set by the caller's prefill)  */
  uint8_t* finished;        /* [B]   1 once <EOS> was met or the token buffer is full; latched */
  int32_t* block_tokens;    /* [B, (k+1)^2] token ids of the next call's block rows           */
  int32_t* block_pos;       /* [B, (k+1)^2] their position ids                                */
} space_decode_state;

/* Initial state of Algorithm 1: no generated token, L_c = [0]*k, P_c = [+inf]*k (so
 * that the first step accepts nothing in sampling mode), finished = 0, and the block
 * rows of the first step.  last_prompt_token: device [B], the last token of every
 * prompt (the cache already holds the tokens before it and state->kv_len says how many).
 * Asynchronous on `stream`.  Errors: INVALID_ARG, WORKSPACE (batch beyond the context's), CUDA. */
int space_decode_begin(space_ctx* ctx, const space_decode_state* state, const int32_t* last_prompt_token,
                       void* stream);

/* End of one loop iteration of Algorithm 1, after space_verify (+ space_kv_commit) of
 * the step: appends the step's out_tokens[b, 0 .. n_out[b]-1] to O, latches finished
 * when the step met <EOS> (step_finished, from space_verify) or the buffer is full,
 * and otherwise carries next_cand / next_cand_prob into L_c / P_c, takes kv_len_next
 * (the commit's kv_len_out; must not alias state->kv_len) as the new length and writes
 * the next call's block rows.  A sequence that is already finished is left untouched:
 * the step's results for it are dropped and its length no longer grows.  All pointers
 * device memory, shapes as in space_verify_args / space_commit_args.
 * Asynchronous on `stream`, no host synchronisation: model, attention, verification,
 * commit and this call can be enqueued step after step, or captured in one CUDA graph. */
int space_decode_advance(space_ctx* ctx, const space_decode_state* state, const int32_t* out_tokens,
                         const int32_t* n_out, const int32_t* next_cand, const float* next_cand_prob,
                         const uint8_t* step_finished, const int32_t* kv_len_next, void* stream);

/* Data-loader transform of semi-autoregressive fine-tuning (Sec. 3.1, App. A.1) on a
 * padded batch of training samples, in place.  A sample (prompt of prompt_len tokens, then
 * an answer y_1..y_N of answer_len tokens, in the first slots of its row) stays as it is
 * with probability p_ar; otherwise a position m is drawn from {0..N-k}, the k answer tokens
 * from there on become mask_token_id in input_ids (labels keep their tokens), and both rows
 * are cut after the first m+k answer tokens (input_ids padded with pad_token_id, labels set
 * to ignore_index).  An answer shorter than k stays autoregressive.
 * Randomness is the caller's: two 32-bit words per sample; the sample stays autoregressive
 * when the first is below ar_threshold (= p_ar * 2^32), and m = (second * (N-k+1)) >> 32.
 * Needs no context; runs on the current device, asynchronous on `stream`.
 * Errors: INVALID_ARG (NULL pointer, sizes), CUDA. */
typedef struct {
  int32_t batch, seq_cap, k;
  int32_t mask_token_id, pad_token_id, ignore_index;
  uint32_t ar_threshold;
  int32_t reserved;            /* 0                                                   */
  int32_t* input_ids;          /* device [B, seq_cap], in place                       */
  int32_t* labels;             /* device [B, seq_cap], in place                       */
  const int32_t* prompt_len;   /* device [B]                                          */
  const int32_t* answer_len;   /* device [B]  N                                       */
  const uint32_t* rand_words;  /* device [B, 2]                                       */
  int32_t* new_len;            /* device [B] or NULL: tokens kept (prompt + answer part) */
  int32_t* mask_start;         /* device [B] or NULL: m, or -1 for an unchanged sample */
} space_sar_args;
int space_sar_sft_transform(const space_sar_args* args, void* stream);

/* ---- KV cache in 4 bits ------------------------------------------------------------------------
 * (No counterpart in the paper: a cache in 4 bits is about a quarter of the bf16 one, so that a server holds
 * more or longer sequences.)  Paged like the bf16 cache: a pool of pages of
 * SPACE_PAGE_SIZE rows behind a page table, row s of sequence b in row s % SPACE_PAGE_SIZE of page
 * page_table[b * pages_per_seq + s / SPACE_PAGE_SIZE], K and V of a row in the same page.
 *
 * A row of d channels x is held as 4-bit codes u with one step and one lowest value, both bf16:
 *   lo = min x,   step = bf16(max((max x - lo) / 15, max|x| / 4096, 2^-100)),
 *   u = min(round((x - lo) / step), 15) (ties to even),   and stands for lo + step * u.
 * NaN counts as 0 and an infinity as the largest finite bf16 (SPACE_ST_NONFINITE).
 *
 * Bytes of a page, per kv head (head_stride apart): 4 blocks of 32 rows, each
 *   K codes  [32][d/2]: byte i of a row holds channels 2i (low four bits) and 2i + 1
 *   V codes  [32 d / 2]: channel c = 32w + 8q + n of row r = 16a + 8e + 2t + h in byte
 *            512w + 64n + 16t + 8a + 4e + 2h + q/2, low four bits for even q
 *   K steps  [32] {bf16 step, bf16 lo}, V steps [32] {bf16 step, bf16 lo}
 * i.e. 32 d + 256 bytes a block: the order in which the attention's tensor-core operands are unpacked. */
typedef struct {
  void*   pool;                /* device, 16-byte aligned                                          */
  int64_t page_stride;         /* bytes, multiples of 16; several layers may share one allocation  */
  int64_t head_stride;         /* bytes, at least 4 * (32 d + 256)                                 */
  const int32_t* page_table;   /* device [B, pages_per_seq]                                        */
  int32_t pages_per_seq;
  int32_t n_pages;             /* pages in the pool                                                */
} space_kvq_cache;

/* Bytes of one page of a contiguous pool: n_kv_heads * 4 * (32 head_dim + 256); 0 for a head_dim other
 * than 64 and 128.  Host only. */
int64_t space_kvq_page_bytes(int32_t n_kv_heads, int32_t head_dim);

/* Puts rows behind the cached ones: row g * row_step of k_new / v_new becomes cache row kv_len[b] + g for
 * g < count[b] + count_bias (at least 0, at most what `rows` holds).  A prompt's rows or one new token:
 * row_step = 1; the accepted rows of a step out of its block rows: row_step = k + 1, count = n_accept,
 * count_bias = 1.  A sequence with kv_len < 0, or whose rows would not fit pages_per_seq pages, is left as
 * it is (SPACE_ST_CAPACITY); rows of a page outside the pool are skipped (SPACE_ST_BAD_PAGE).
 * Asynchronous on `stream`.  Errors: INVALID_ARG, ALIGNMENT, WORKSPACE (batch beyond the context's), CUDA. */
typedef struct {
  int32_t batch;
  int32_t rows;                /* rows per sequence in k_new / v_new                               */
  int32_t row_step;            /* >= 1                                                             */
  int32_t count_bias;
  const void* k_new;           /* device bf16, element (b, r, h, :) at b*stride_b + r*stride_r + h*stride_h */
  const void* v_new;           /*   (elements, multiples of 8; base 16-byte aligned), d contiguous  */
  int64_t new_stride_b, new_stride_r, new_stride_h;
  space_kvq_cache cache;
  const int32_t* kv_len;       /* device [B] lengths before the call                               */
  const int32_t* count;        /* device [B], or NULL: all of `rows` (every row_step-th)           */
  int32_t* kv_len_out;         /* device [B] lengths after, or NULL; must not be kv_len            */
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
} space_kvq_append_args;
int space_kvq_append(space_ctx* ctx, const space_kvq_append_args* args, void* stream);

/* Reads cache rows first[b] .. first[b] + rows - 1 back as the bf16 values nearest to what they stand for;
 * rows below 0, at kv_len[b] and beyond, or of a page outside the pool (SPACE_ST_BAD_PAGE) are written as
 * zeros.  Asynchronous on `stream`.  Errors: as space_kvq_append. */
typedef struct {
  int32_t batch;
  int32_t rows;
  space_kvq_cache cache;
  const int32_t* kv_len;       /* device [B]                                                       */
  const int32_t* first;        /* device [B], or NULL (0)                                          */
  void* k_out;                 /* device bf16, element (b, r, h, :) at b*stride_b + r*stride_r + h*stride_h */
  void* v_out;                 /*   (elements, multiples of 8; base 16-byte aligned), d contiguous  */
  int64_t out_stride_b, out_stride_r, out_stride_h;
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
} space_kvq_read_args;
int space_kvq_read(space_ctx* ctx, const space_kvq_read_args* args, void* stream);

/* Attention of a step's block rows over a 4-bit cache: softmax(scale q k^T) v over cache rows
 * 0 .. kv_len[b]-1 and, with k_new / v_new, over the block's own rows (bf16, not in the cache yet) as Eq. 5
 * shows them.  k = 0 is one row per sequence, plain token-by-token decoding.  Without k_new / v_new every
 * row sees the cache alone (a token whose row has been appended before); a row that sees nothing at all
 * (an empty cache) gives zeros and lse = -inf, and so does every row of a sequence with kv_len outside
 * 0 .. pages_per_seq * SPACE_PAGE_SIZE (SPACE_ST_CAPACITY).  Keys of a page outside the pool are left out
 * (SPACE_ST_BAD_PAGE).  Hidden rows have no influence, whatever they hold; non-finite elements of k_new /
 * v_new count as they do in space_kvq_append (without the status bit).
 * The output is bf16: scores and sums are fp32, the weights of the second product are rounded to 11 bits.  A call whose
 * kv heads have 49 to 64 or most numbers above 96 of query rows may run in another form, if pages_per_seq gives every SM
 * work: it rounds the cache's V values, in steps, and the block's K and V rows to 11 bits too.  (So a wider table can
 * change last bits.)
 * The products take query rows as f16, scaled by one power of two for up to 64 rows of a kv head together: elements
 * more than 2^21 times smaller than the largest of those rows are rounded, by at most 2^-29 of it; all others are exact
 * below 2^109.  Scores are held to +-6.9e37 (1e38 in units of log2): of keys beyond that none is preferred.  A weight below
 * 2^-118 of a row's largest counts as nothing; outputs below 2^-110 may be rounded to multiples of 2^-117.
 * Asynchronous on `stream`, no allocation; one call at a time per context (scratch of the context).
 * Errors: INVALID_ARG, ALIGNMENT, WORKSPACE (batch or k beyond the context's), UNSUPPORTED (batch * n_kv_heads *
 * ceil(query rows of a kv head / 8) * (pages_per_seq + 4) above 2e9), CUDA. */
typedef struct {
  int32_t batch;
  int32_t k;                   /* 0 .. k_max; (k+1)^2 query rows                                   */
  int32_t mask_variant;        /* SPACE_MASK_*                                                     */
  float   scale;               /* > 0, normally 1/sqrt(d)                                          */
  const void* q;               /* device bf16, element (b, i, h, :) at b*stride_b + i*stride_r + h*stride_h */
  int64_t q_stride_b, q_stride_r, q_stride_h;          /* elements, multiples of 8                 */
  const void* k_new;           /* device bf16 [B, n_q, H_kv, d] by strides, or NULL together with v_new */
  const void* v_new;
  int64_t new_stride_b, new_stride_r, new_stride_h;
  space_kvq_cache cache;
  const int32_t* kv_len;       /* device [B] rows cached                                           */
  void*    out;                /* device bf16 [B, n_q, H_q, d]                                     */
  float*   lse;                /* device [B, H_q, n_q] natural-log sum-exp, or NULL                */
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
} space_kvq_attn_args;
int space_kvq_attn_step(space_ctx* ctx, const space_kvq_attn_args* args, void* stream);

/* ---- Positions by rotation ---------------------------------------------------------------------
 * (No counterpart in the paper, whose models bring it along; its block has positions of its own, Sec. 3.2.)
 * Channel pairs (x1, x2) of a query or key row at position p turn by the p-th row of a table:
 *   x1' = x1 cos - x2 sin,   x2' = x2 cos + x1 sin,
 * in fp32, each product and the sum rounded, then to the output's type.  Channels from rot_dim on stay as they are. */
typedef struct {
  const float* table;          /* device [n_pos, rot_dim], 16-byte aligned: cosines of a position's rot_dim/2
                                  angles, then their sines                                            */
  int32_t n_pos;
  int32_t rot_dim;             /* a multiple of 16, at most head_dim                               */
  int32_t interleaved;         /* 0: channel i turns with i + rot_dim/2; 1: channel 2i with 2i + 1 */
  int32_t reserved;            /* 0                                                                */
  const int32_t* pos;          /* device [B, rows] (row r of the call), or NULL: the cache row that r becomes */
} space_rope;

/* The rows that attention is about to see: queries and keys of row r < count[b] are rotated, the keys and the values
 * go to cache row kv_len[b] + r (bf16, contiguous or paged as in space_attn_args; without `pos` that is the position
 * too).  With k_cache == NULL the rotated keys go to k_out instead, for a cache that takes its rows after the step
 * (space_kvq_*, space_kvb_*).  q_out may be q and k_out may be k, with their strides; q may be NULL.  Rows from count[b] on stay
 * untouched, and so does all of a sequence whose rows would not fit its capacity (SPACE_ST_CAPACITY); K and V of a page
 * outside the pool are skipped (SPACE_ST_BAD_PAGE).  Asynchronous on `stream`, no allocation.
 * Errors: INVALID_ARG, ALIGNMENT, WORKSPACE (batch beyond the context's), UNSUPPORTED (rot_dim), CUDA. */
typedef struct {
  int32_t batch;
  int32_t rows;                /* rows per sequence in q, k and v                                  */
  space_rope rope;
  const void* q;               /* device bf16, element (b, r, h, :) at b*stride_b + r*stride_r + h*stride_h */
  int64_t q_stride_b, q_stride_r, q_stride_h;          /* elements, multiples of 8; bases 16-byte aligned */
  void* q_out;
  int64_t q_out_stride_b, q_out_stride_r, q_out_stride_h;
  const void* k;               /* device bf16 [B, rows, H_kv, d] by strides                        */
  const void* v;               /* the same strides; NULL without a cache                           */
  int64_t new_stride_b, new_stride_r, new_stride_h;
  void* k_out;                 /* device bf16 [B, rows, H_kv, d] by strides, or NULL with a cache  */
  int64_t k_out_stride_b, k_out_stride_r, k_out_stride_h;
  void* k_cache;               /* device bf16, addressing as in space_attn_args                    */
  void* v_cache;
  int64_t kv_stride_b, kv_stride_h, kv_stride_s;
  const int32_t* page_table;   /* device [B, pages_per_seq] or NULL (contiguous)                   */
  int32_t pages_per_seq;
  int32_t n_pages;
  const int32_t* kv_len;       /* device [B] lengths before the call                               */
  const int32_t* count;        /* device [B], or NULL: all of `rows` (less than 0 counts as 0, more than `rows` as `rows`) */
  int32_t* kv_len_out;         /* device [B] lengths after, or NULL; must not be kv_len            */
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
} space_rope_args;
int space_rope_append(space_ctx* ctx, const space_rope_args* args, void* stream);

/* ---- KV cache in 8 bits ------------------------------------------------------------------------
 * (No counterpart in the paper: half the bf16 cache.)  Paged as the 4-bit one: row s of sequence b in row
 * s % SPACE_PAGE_SIZE of page page_table[b * pages_per_seq + s / SPACE_PAGE_SIZE], K and V of a row in the same page.
 *
 * Elements are e4m3 numbers (four bits of significance, up to 448); the 32 rows of a block (rows 0..31, 32..63, ..
 * of a page) share a power of two 2^e per kv head, one for K and one for V, and an element stands for code * 2^e:
 *   e = the least whole number with max|x| <= 448 2^e, -100 at least;   code = x / 2^e to the nearest, ties to even.
 * (At e = 120, where 256 2^e is no bf16 number any more, codes are held to 240.)
 * NaN counts as 0 and an infinity as the largest finite bf16 (SPACE_ST_NONFINITE).  Rows come one after another: e covers
 * the rows that a block has had since its first row was last written, and where a later row raises it the block's earlier
 * codes are rounded once more, to multiples of 2^(e - 9) (all others stay exactly what they were).
 * (So a page that sequences share is copied before one of them writes into it, space_pager_make_writable: the block's earlier
 * rows are the others' too.)
 *
 * Bytes of a page, per kv head (head_stride apart), the order of the attention's tensor-core operands:
 *   K codes [d/16][128][16]: channel c of row r in byte (c/16) 2048 + 16 r + c%16
 *   V codes [8][d][16]:      channel c of row r in byte 128 d + (r/16) 16 d + 16 c + r%16
 *   scales  [4] {f32 K 2^e, f32 V 2^e} */
typedef space_kvq_cache space_kvb_cache;   /* (head_stride: at least 256 d + 32 bytes) */

/* Bytes of one page of a contiguous pool: n_kv_heads * (256 head_dim + 32); 0 for a head_dim other than 64 and 128. */
int64_t space_kvb_page_bytes(int32_t n_kv_heads, int32_t head_dim);

/* Puts rows behind the cached ones, as space_kvq_append does: row g * row_step of k_new / v_new becomes cache row
 * kv_len[b] + g for g < count[b] + count_bias.  With rope.table the keys are rotated on the way (rope.pos [B, rows]) and, where q is
 * given, the same source rows of q into q_out.  Whether a sequence fits, bad pages, errors and the rest: as space_kvq_append;
 * UNSUPPORTED (rot_dim; more than 2^31 - 1 blocks of 32 rows and heads).  A sequence that does not fit keeps its q_out too. */
typedef struct {
  int32_t batch;
  int32_t rows;                /* rows per sequence in k_new / v_new                               */
  int32_t row_step;            /* >= 1                                                             */
  int32_t count_bias;
  const void* k_new;           /* device bf16, element (b, r, h, :) at b*stride_b + r*stride_r + h*stride_h */
  const void* v_new;           /*   (elements, multiples of 8; base 16-byte aligned), d contiguous  */
  int64_t new_stride_b, new_stride_r, new_stride_h;
  space_kvb_cache cache;
  const int32_t* kv_len;       /* device [B] lengths before the call                               */
  const int32_t* count;        /* device [B], or NULL: all of `rows` (every row_step-th)           */
  int32_t* kv_len_out;         /* device [B] lengths after, or NULL; must not be kv_len            */
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
  space_rope rope;             /* table == NULL: the rows as they are                              */
  const void* q;               /* device bf16 [B, rows, H_q, d] by strides, or NULL                */
  int64_t q_stride_b, q_stride_r, q_stride_h;
  void* q_out;                 /* may be q, with its strides                                       */
  int64_t q_out_stride_b, q_out_stride_r, q_out_stride_h;
} space_kvb_append_args;
int space_kvb_append(space_ctx* ctx, const space_kvb_append_args* args, void* stream);

/* Reads cache rows first[b] .. first[b] + rows - 1 back: arguments, zeros and errors as space_kvq_read.  The bf16 values
 * are exactly what the codes stand for. */
typedef struct {
  int32_t batch;
  int32_t rows;
  space_kvb_cache cache;
  const int32_t* kv_len;       /* device [B]                                                       */
  const int32_t* first;        /* device [B], or NULL (0)                                          */
  void* k_out;                 /* device bf16, element (b, r, h, :) at b*stride_b + r*stride_r + h*stride_h */
  void* v_out;                 /*   (elements, multiples of 8; base 16-byte aligned), d contiguous  */
  int64_t out_stride_b, out_stride_r, out_stride_h;
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
} space_kvb_read_args;
int space_kvb_read(space_ctx* ctx, const space_kvb_read_args* args, void* stream);

/* Attention of a step's block rows over an 8-bit cache: softmax(scale q k^T) v over cache rows 0 .. kv_len[b]-1 and, with
 * k_new / v_new, over the block's own rows (bf16, not in the cache yet) as Eq. 5 shows them.  k = 0 is one row per
 * sequence.  Rows that see nothing, sequences that do not fit, bad pages, hidden rows and non-finite elements of
 * k_new / v_new: as space_kvq_attn_step.  A query row that holds a NaN or an infinity gives NaN.
 * The output is bf16, the sums are fp32.  Query rows are taken as two e4m3 numbers an element with a power of two per row: bf16
 * exactly, but elements more than 2^8 times smaller than the largest of their row are rounded, by at most 2^-17 of it; so are
 * the block's own rows where a kv head has more than sixteen query rows (else they are bf16 as they are).  Weights are rounded likewise:
 * each to eight bits, and by at most 2^-18 of the largest among the keys that it goes with (32 or 128 of them; there times
 * their V scales).  Scores, in units of log2, are good up to +-2^29: the largest of 32
 * neighbouring cached keys, and each of the block's own, is held to that (the others of those 32 in proportion), so that keys beyond it
 * are not told apart for what they are.
 * Asynchronous on `stream`, no allocation; one call at a time per context (scratch of the context).
 * Errors: INVALID_ARG, ALIGNMENT, WORKSPACE (batch or k beyond the context's), UNSUPPORTED (batch * n_kv_heads *
 * ceil(query rows of a kv head / 8) * (pages_per_seq + 4) above 2e9), CUDA. */
typedef struct {
  int32_t batch;
  int32_t k;                   /* 0 .. k_max; (k+1)^2 query rows                                   */
  int32_t mask_variant;        /* SPACE_MASK_*                                                     */
  float   scale;               /* > 0, normally 1/sqrt(d)                                          */
  const void* q;               /* device bf16, element (b, i, h, :) at b*stride_b + i*stride_r + h*stride_h */
  int64_t q_stride_b, q_stride_r, q_stride_h;          /* elements, multiples of 8                 */
  const void* k_new;           /* device bf16 [B, n_q, H_kv, d] by strides, or NULL together with v_new */
  const void* v_new;
  int64_t new_stride_b, new_stride_r, new_stride_h;
  space_kvb_cache cache;
  const int32_t* kv_len;       /* device [B] rows cached                                           */
  void*    out;                /* device bf16 [B, n_q, H_q, d]                                     */
  float*   lse;                /* device [B, H_q, n_q] natural-log sum-exp, or NULL                */
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
} space_kvb_attn_args;
int space_kvb_attn_step(space_ctx* ctx, const space_kvb_attn_args* args, void* stream);

/* ---- Logits before verification ----------------------------------------------------------------
 * (No counterpart in the paper, which decodes unpenalised.)  Changes a step's logits [B, (k+1)^2, vocab] (k = 0: one row
 * per sequence) before space_verify.  Row (g, o) stands behind the generated tokens and candidates 1 .. g: with n the times that
 * a token occurs among them, and z its logit, in fp32, each operation rounded, then to the logits' type:
 *   z > 0 ? z / repetition : z * repetition      where n > 0 or the token occurs in the prompt
 *   z - frequency * n,   then z - presence       where n > 0
 *   z + bias                                     for a token of the list (named twice: the sum, in order)
 *   -infinity                                    where the row's mask has a 0 bit
 * A row that its mask leaves no token is -infinity throughout (SPACE_ST_BAD_MASK): no token can be taken from it.
 * `out` may be `logits` with its row stride: then only what changes is written.  Asynchronous on `stream`, no
 * allocation; one call at a time per context.  Errors: INVALID_ARG, ALIGNMENT, WORKSPACE (batch, k or vocab beyond the
 * context's), CUDA. */
#define SPACE_COUNT_PROMPT    (1 << 30)   /* bit of a count: the token occurs in the prompt; below it, how often it was generated
                                             (from 2^24 - 1 on counts as 2^24 - 1)                         */
#define SPACE_LOGITS_MAX_BIAS 1024
typedef struct {
  int32_t batch, k, vocab;
  int32_t dtype;               /* SPACE_DTYPE_* of logits and out                                  */
  const void* logits;          /* device [B, (k+1)^2, vocab]; batch stride = (k+1)^2 * row stride  */
  int64_t logits_row_stride;   /* elements                                                         */
  void* out;                   /* the same shape                                                   */
  int64_t out_row_stride;
  const int32_t* counts;       /* device [B, vocab] (space_token_counts), or NULL: no token so far */
  const int32_t* cand;         /* device [B, k], or NULL: candidates do not count; ids outside [0, vocab) never do */
  const float* repetition;     /* device [B], > 0, or NULL (1)                                     */
  const float* presence;       /* device [B], or NULL (0)                                          */
  const float* frequency;      /* device [B], or NULL (0)                                          */
  int32_t n_bias;              /* 0 .. SPACE_LOGITS_MAX_BIAS                                       */
  int32_t n_masks;
  const int32_t* bias_tok;     /* device [B, n_bias]; ids outside [0, vocab) are skipped           */
  const float* bias_val;       /* device [B, n_bias]                                               */
  const uint32_t* mask_bits;   /* device [n_masks, ceil(vocab / 32)]: bit t % 32 of word t / 32 allows token t; or NULL */
  const int32_t* mask_row;     /* device [B, (k+1)^2]: mask of every row, below 0: none; with mask_bits */
  int32_t* status;             /* device [B], OR-ed, or NULL                                       */
} space_logits_args;
int space_logits_adjust(space_ctx* ctx, const space_logits_args* args, void* stream);

/* Counts tokens [B, n] for space_logits_adjust: the first n_tokens[b] of a sequence are added to its counts, or, with `prompt`, marked
 * as occurring in the prompt.  After a step: the emitted ones (out_tokens, n_out of space_verify).  Ids outside
 * [0, vocab) are skipped.  With `reset` the counts are 0 before.  Asynchronous on `stream`, no allocation.
 * Errors: INVALID_ARG, WORKSPACE (batch or vocab beyond the context's), CUDA. */
typedef struct {
  int32_t batch, vocab, n;
  int32_t prompt, reset;
  int32_t reserved;            /* 0                                                                */
  const int32_t* tokens;       /* device, n of a sequence stride_b elements apart                  */
  int64_t tokens_stride_b;
  const int32_t* n_tokens;     /* device [B], or NULL: all n (less than 0 counts as 0, more than n as n) */
  int32_t* counts;             /* device [B, vocab]                                                */
} space_counts_args;
int space_token_counts(space_ctx* ctx, const space_counts_args* args, void* stream);

/* ---- Moving pages ------------------------------------------------------------------------------
 * Rows 0 .. rows-1 of page src become those of page dst, for every move and in every pool (the pools of all
 * layers, K and V, share their page numbers), in one launch per SPACE_PAGES_MAX_MOVES moves: what a fork's
 * copy-on-write and a compaction (space_pager_make_writable, space_pager_compact) hand out.
 * A page is `parts` pieces, part_stride apart, of rows in groups of group_rows, group_bytes each; of a
 * group that `rows` ends in all is copied.  bf16 pool [n_pages, H_kv, 128, d]: one pool for K, one for V,
 * parts = H_kv, group_rows = 1, group_bytes = 2 d.  4-bit pool: parts = H_kv, group_rows = 32,
 * group_bytes = 32 d + 256.  8-bit pool: parts = H_kv, group_rows = 128, group_bytes = 256 d + 32.  No page may be written twice in a call, or both read and written.
 * Both lists are host memory, read before the call returns; no context, current device, asynchronous on
 * `stream`, no allocation on the device.
 * Errors: INVALID_ARG (sizes, pages, overlap), ALIGNMENT (base, strides and group_bytes not multiples of 16), CUDA. */
#define SPACE_PAGES_MAX_POOLS 256
#define SPACE_PAGES_MAX_MOVES 1024
typedef struct {
  void*   base;                /* device                                                           */
  int64_t page_stride;         /* bytes                                                            */
  int64_t part_stride;         /* bytes                                                            */
  int32_t parts;
  int32_t group_rows;          /* divides SPACE_PAGE_SIZE                                          */
  int32_t group_bytes;
  int32_t n_pages;
} space_page_pool;
typedef struct { int32_t src, dst, rows; } space_page_move;
int space_pages_copy(const space_page_pool* pools, int32_t n_pools, const space_page_move* moves, int32_t n_moves,
                     void* stream);

/* Number of kernels this context has launched so far. */
int64_t space_launch_count(const space_ctx* ctx);

/* Per-kernel timing with CUDA events recorded on the launching stream around
 * every kernel (attention, merge, verify target rows, verify emit, commit,
 * projection + verify).
 * space_profile_enable(ctx, 1) starts a fresh recording (at most
 * SPACE_PROFILE_MAX_STEPS steps are kept; later ones are not recorded);
 * space_profile_enable(ctx, 0) stops it.  Do not enable during stream capture.
 * space_profile_read waits for the recorded events, writes the summed
 * milliseconds per kernel into ms[SPACE_K_COUNT] and the number of recorded launches
 * per kernel into n[SPACE_K_COUNT], and clears the recording. */
#define SPACE_PROFILE_MAX_STEPS 4096
enum { SPACE_K_ATTN = 0, SPACE_K_MERGE = 1, SPACE_K_VERIFY_TARGET = 2, SPACE_K_VERIFY_EMIT = 3,
       SPACE_K_COMMIT = 4, SPACE_K_LMHEAD = 5, SPACE_K_COUNT = 6 };
int space_profile_enable(space_ctx* ctx, int on);
int space_profile_read(space_ctx* ctx, float* ms, int64_t* n);

/* Test hook: n Philox4x32-10 blocks (Salmon et al., SC'11) for counters
 * (c0[i], c1[i], c2[i], c3[i]) and key `seed`; out receives 4 words each.
 * All pointers device memory. */
int space_debug_philox(space_ctx* ctx, uint64_t seed, int64_t n, const uint32_t* c0,
                       const uint32_t* c1, const uint32_t* c2, const uint32_t* c3,
                       uint32_t* out, void* stream);

/* Test hook for the bounded on-chip waits (every mbarrier wait of the tensor-core
 * kernels gives up after one second, sets SPACE_ST_TIMEOUT and lets the block drain;
 * no wait in the library is unbounded).  Launches one small kernel that waits, with that
 * same wait routine and a limit of limit_ns (1 .. 10^8 ns), on a barrier nothing ever
 * arrives on.  The kernel returns normally; the context stays usable.
 * out4: device int32[4], written as {status bits: SPACE_ST_TIMEOUT when the wait expired,
 * 8 if a later wait did not also give up, 16 when the block's abort flag was set;
 * the recorded site (77); microseconds the expired wait took; microseconds a second
 * wait took (about 0: a block that has given up never blocks again)}.
 * Errors: INVALID_ARG (NULL, limit out of range), CUDA. */
int space_debug_wait_timeout(space_ctx* ctx, uint64_t limit_ns, int32_t* out4, void* stream);

/* Page bookkeeping for a paged cache shared by sequences that come and go between steps (the
 * serving setting of Sec. 4.3: continuous batching).  Host-side only: it hands out pages of a pool
 * and keeps every sequence's page list; the pool's memory and the device copy of a table belong to
 * the caller.  A sequence occupies a slot from space_pager_admit to space_pager_release; a step's
 * batch is any list of slots, and space_pager_batch_table writes the table rows of those slots in
 * that order, the page_table that space_attn_args / space_commit_args take for that batch.
 * Not thread-safe.  Errors: INVALID_ARG (NULL, slot not in use, sizes out of range), WORKSPACE (no
 * free slot; not enough free pages, in which case nothing has changed). */
typedef struct space_pager space_pager;
int  space_pager_create(int32_t n_pages, int32_t pages_per_seq, int32_t max_slots, space_pager** out);
void space_pager_destroy(space_pager* p);
int  space_pager_admit(space_pager* p, int32_t* slot);          /* a free slot, holding no page yet     */
int  space_pager_reserve(space_pager* p, int32_t slot, int32_t n_rows);
                             /* pages so that cache rows 0 .. n_rows-1 of the slot exist (a sequence
                                of length L needs L + (k+1)^2 rows before its next step); pages a
                                slot already holds stay where they are                                */
int  space_pager_release(space_pager* p, int32_t slot);         /* its pages return to the pool         */
int32_t space_pager_free_pages(const space_pager* p);
int32_t space_pager_rows(const space_pager* p, int32_t slot);   /* rows reserved for the slot, -1 if unused */
int  space_pager_batch_table(const space_pager* p, const int32_t* slots, int32_t n,
                             int32_t* table_out);               /* host [n, pages_per_seq]; -1 = no page */

/* Sequences that share pages.  A fork holds the pages of its parent's first n_rows rows and no copy of them;
 * a page returns to the pool when the last slot that holds it gives it up (release, truncate).  Before a slot's rows
 * from first_row on are written (they, and whatever the same pages hold behind them, are not kept),
 * space_pager_make_writable gives it pages of its own for rows first_row .. first_row + n_rows - 1 where it
 * shares them, and lists the moves that carry the rows before first_row over; the caller runs them
 * (space_pages_copy) before the write.  The rows must have been reserved.
 * space_pager_compact renumbers pages so that those in use come to stand at the pool's start: it takes the
 * highest page in use to the lowest free one, at most max_moves times (*n_moves = 0: nothing left to move); batch
 * tables have to be written anew, and the moves run before the next call on the cache.
 * Errors: INVALID_ARG, WORKSPACE (no free slot, not enough free pages or room for the moves: nothing has changed). */
int  space_pager_fork(space_pager* p, int32_t parent, int32_t n_rows, int32_t* slot);
int  space_pager_make_writable(space_pager* p, int32_t slot, int32_t first_row, int32_t n_rows,
                               space_page_move* moves, int32_t max_moves, int32_t* n_moves);
int  space_pager_truncate(space_pager* p, int32_t slot, int32_t n_rows);  /* pages past n_rows rows are given up */
int  space_pager_compact(space_pager* p, space_page_move* moves, int32_t max_moves, int32_t* n_moves);
int32_t space_pager_page_refs(const space_pager* p, int32_t page);        /* slots that hold it; -1: no such page */

const char* space_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SPACE_H */
