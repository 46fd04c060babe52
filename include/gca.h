/*
 * libgca -- Grouped Cross Attention (GCA) hot path for AMD Instinct MI355X (gfx950).
 *
 * Method: "Efficient Length-Generalizable Attention via Causal Retrieval for
 * Long-Context Language Modeling" (arXiv 2410.01651), Methodology / Model
 * Architecture: causal relevance scores and top-k retrieval (Eq. 1), grouped
 * cross attention fused by the softmaxed scores (Eq. 2 and Eq. 3), and the
 * hardware-aware forward and backward passes of Appendix B (Algorithms 1-2).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - All tensor pointers are DEVICE pointers, row-major and densely packed, in the
 *   layouts stated per argument.  The caller owns every buffer; the library never
 *   allocates, frees or retains memory.  Temporary storage comes from a caller
 *   workspace sized by gca_workspace_size().
 * - Chunks are numbered from 0.  In CAUSAL mode a sequence of L = n_chunks * S
 *   tokens has n_chunks chunks; landmark row t retrieves among chunks [0, t)
 *   (Eq. 1 ranges over strictly earlier chunks) and its retrieved set feeds the
 *   tokens of chunk t+1 (Eq. 2 applies C_t to chunk t+1).  In DECODE mode one new
 *   chunk of S tokens has one landmark query, scored against all n_chunks past
 *   chunks; that set feeds the new chunk's own tokens.
 * - nQ (landmark query rows) = n_chunks in CAUSAL mode and 1 in DECODE mode;
 *   Lq (query tokens) = nQ * Sq with Sq = S (S + 1 under GCA_FLAG_LMK_ROW);
 *   Lkv (key/value tokens) = n_chunks * S.  Query chunk c is rows
 *   [c * Sq, (c + 1) * Sq) of the query-side tensors.
 * - Retrieval heads: Hr = 1 shares one score per chunk pair across all H heads
 *   (Eq. 1 yields one scalar per pair); Hr = H gives every head its own landmarks.
 *   Head h uses retrieval head (Hr == 1 ? 0 : h).
 * - Retrieved sets are written in ascending chunk order, padded with index -1
 *   and score -inf.  Membership is decided by (score descending, chunk index
 *   ascending): ties go to the lower chunk index.
 * - Every element of every non-NULL output is written (zeros where the method
 *   gives nothing, e.g. the outputs of chunks 0 and 1 in CAUSAL mode).
 * - Arguments are validated before anything is launched; on error nothing is
 *   launched and a status != GCA_OK is returned, with detail in gca_last_error().
 *   Launch failures return GCA_ERR_HIP.  Kernel faults surface at the caller's
 *   next synchronisation.
 * - All work is enqueued on `stream`; no call synchronises (unless the
 *   environment variable GCA_DEBUG_SYNC is set to a value other than 0 when the
 *   library first launches: then every kernel launch is followed by a
 *   synchronisation of `stream` and an error check that names the kernel in
 *   gca_last_error(), for debugging).  Calls are
 *   re-entrant (no global mutable state besides the thread-local error string
 *   and the thread-local profiling hook below).
 * - Supported in this version: d == 64, S == 64, 1 <= topk <= 32, Hr in {1, H},
 *   D a positive multiple of 64 up to 8192, dtype FP32 or BF16 (all tensor
 *   inputs of a call share the dtype; scores, sel, w, lse, dsel and landmark
 *   gradients are always fp32).  Device pointers must be 16-byte aligned.
 */
#ifndef LIBGCA_GCA_H
#define LIBGCA_GCA_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  GCA_OK = 0,
  GCA_ERR_INVALID = 1,      /* malformed problem or NULL required pointer */
  GCA_ERR_UNSUPPORTED = 2,  /* well-formed but outside the supported shapes */
  GCA_ERR_WORKSPACE = 3,    /* workspace pointer NULL or smaller than required */
  GCA_ERR_HIP = 4           /* a HIP launch failed; see gca_last_error() */
} gca_status;

typedef enum { GCA_FP32 = 0, GCA_BF16 = 1 } gca_dtype;
typedef enum { GCA_CAUSAL = 0, GCA_DECODE = 1 } gca_mode;

/* Problem flags (gca_problem.flags). */
#define GCA_FLAG_FUSED_TOPK 1u   /* gca_forward, CAUSAL: score and select in one pass (no score matrix) */
#define GCA_FLAG_MATERIALIZE 2u  /* gca_forward, CAUSAL: always write the score matrix, then select */
#define GCA_FLAG_HOST_KV 8u      /* DECODE: k and v are pinned host allocations (hipHostMalloc),
                                  * the past chunks offloaded to CPU memory (Training &
                                  * Inference, "Memory Offloading"); landmarks, q and every
                                  * output stay in device memory.  The decode attention reads
                                  * the k retrieved chunks straight from host memory over the
                                  * host link (their device mapping, hipHostGetDevicePointer).
                                  * GCA_ERR_INVALID if k or v has no device mapping, or in
                                  * CAUSAL mode. */
#define GCA_FLAG_LMK_ROW 16u     /* CAUSAL: every query chunk has S + 1 rows, its S tokens followed
                                  * by its landmark (LMK) token (Methodology, Model Architecture:
                                  * the LMK token is inserted at the end of each chunk, and the
                                  * grouped cross attention of chunk t+1 takes its S + 1 hidden
                                  * states as queries against S-row retrieved chunks).  q, out,
                                  * lse, dout and dq then hold Lq = nQ * (S + 1) rows, row
                                  * c * (S + 1) + S being chunk c's LMK row; k, v, dk and dv keep
                                  * n_chunks * S rows.  The LMK row attends to and is fused over
                                  * the same retrieved set as its chunk's tokens.
                                  * GCA_ERR_UNSUPPORTED in DECODE mode. */
#define GCA_FLAG_GUMBEL 4u       /* Gumbel top-k selection (Training & Inference, "Gumbel Top-k
                                  * sampling"): every selection (gca_topk, gca_forward in both
                                  * modes) ranks score + g, g = -ln(-ln u) with u from the
                                  * Philox4x32-10 generator (Salmon et al., SC 2011) keyed by
                                  * gumbel_seed, counter (j / 4, t, b * Hr + hr, 0), word j mod 4,
                                  * u = (top 24 bits + 1/2) / 2^24 for candidate chunk j of
                                  * landmark row t (DECODE: t = 0).  sel, w and everything after
                                  * use the raw scores. */

/* Workspace queries (gca_workspace_size op argument). */
#define GCA_OP_FORWARD 0
#define GCA_OP_BACKWARD 1

/* The problem statement of Eq. 1-3: tokens per chunk S, top-k, heads H, head
 * dimension d, and the landmark representation width D. */
typedef struct {
  int32_t B;            /* batch */
  int32_t H;            /* attention heads */
  int32_t d;            /* head dimension (64) */
  int32_t S;            /* tokens per chunk (64) */
  int64_t n_chunks;     /* CAUSAL: chunks in the sequence; DECODE: past chunks */
  int32_t topk;         /* retrieved chunks per landmark row, 1..32 */
  int32_t Hr;           /* retrieval heads: 1 or H */
  int32_t D;            /* landmark vector width */
  float score_scale;    /* multiplies <landmark query, landmark key> (Eq. 1 uses 1/sqrt(D)) */
  float attn_scale;     /* multiplies <q, k> inside each chunk's attention (Eq. 3: 1/sqrt(d)) */
  int32_t off_by_one;   /* 0: plain softmax per chunk (Algorithm 1); 1: softmax-off-by-one (Eq. 3) */
  int32_t dtype;        /* gca_dtype of q, k, v, dout, dq, dk, dv, out, lmk_q, lmk_k */
  int32_t mode;         /* gca_mode */
  uint32_t flags;       /* GCA_FLAG_* */
  uint64_t gumbel_seed; /* generator seed for GCA_FLAG_GUMBEL (ignored otherwise) */
} gca_problem;

/* Causal relevance scores (Eq. 1):
 *   scores[b,hr,t,j] = score_scale * <lmk_q[b,hr,t,:], lmk_k[b,hr,j,:]>
 * for every j < t (CAUSAL) or every j (DECODE); -inf elsewhere.
 *   lmk_q  [B, Hr, nQ, D]        dtype      landmark queries (one per query chunk)
 *   lmk_k  [B, Hr, n_chunks, D]  dtype      landmark keys (one per chunk)
 *   scores [B, Hr, nQ, n_chunks] fp32       output
 */
gca_status gca_chunk_scores(const gca_problem* p, const void* lmk_q, const void* lmk_k,
                            float* scores, hipStream_t stream);

/* Top-k retrieval (Eq. 1): for each landmark row, the min(topk, #candidates)
 * best chunks, where candidates are the finite entries with j < t (CAUSAL) or
 * all finite entries (DECODE).
 *   scores [B, Hr, nQ, n_chunks] fp32   input (e.g. from gca_chunk_scores)
 *   idx    [B, Hr, nQ, topk]     int32  output: chunk indices ascending, -1 padded
 *   sel    [B, Hr, nQ, topk]     fp32   output: scores of the chosen chunks, -inf padded
 */
gca_status gca_topk(const gca_problem* p, const float* scores, int32_t* idx, float* sel,
                    hipStream_t stream);

/* Grouped cross attention forward (Eq. 2-3; Algorithm 1).  For every head h and
 * query chunk c with retrieval row t (CAUSAL: t = c-1; DECODE: t = 0) and every
 * valid slot s (idx >= 0) of that row:
 *   w[t,s]   = softmax over valid slots of sel[t,:]            (Eq. 2)
 *   P_s      = rowsoftmax(attn_scale * Q_c K_{j_s}^T)           (Eq. 3, per chunk)
 *   out_c    = sum_s w[t,s] * P_s V_{j_s}                       (Eq. 2)
 *   lse[., s]= log of slot s's softmax denominator (natural log, max included)
 * Rows whose retrieval row has no valid slot (CAUSAL chunks 0 and 1) get out = 0
 * and lse = -inf; pad slots get lse = -inf.  Slots with idx outside
 * [0, n_chunks) are treated as pads.
 *   q   [B, H, Lq, d]        dtype
 *   k,v [B, H, Lkv, d]       dtype
 *   idx [B, Hr, nQ, topk]    int32   (from gca_topk)
 *   sel [B, Hr, nQ, topk]    fp32    (from gca_topk; finite on valid slots)
 *   out [B, H, Lq, d]        dtype   output
 *   lse [B, H, Lq, topk]     fp32    output, may be NULL
 *   w   [B, Hr, nQ, topk]    fp32    output fusion weights, may be NULL
 */
gca_status gca_grouped_xattn_fwd(const gca_problem* p, const void* q, const void* k,
                                 const void* v, const int32_t* idx, const float* sel,
                                 void* out, float* lse, float* w, hipStream_t stream);

/* Backward of gca_grouped_xattn_fwd and of the score path (Algorithm 2, with the
 * gradient carried into the relevance scores through Eq. 2 and into the landmark
 * vectors through Eq. 1).  With dout the gradient of the loss w.r.t. out:
 *   dq, dk, dv [same shapes as q, k, v] dtype  gradients (dk/dv summed over every
 *                                             retrieval of each chunk)
 *   dsel   [B, Hr, nQ, topk] fp32  gradient w.r.t. the retrieved scores sel
 *                                  (0 on pad slots; the indices carry no gradient)
 *   dlmk_q [B, Hr, nQ, D]    fp32  gradient w.r.t. lmk_q (may be NULL)
 *   dlmk_k [B, Hr, n_chunks, D] fp32 gradient w.r.t. lmk_k (may be NULL)
 * lmk_q/lmk_k are needed only when dlmk_q/dlmk_k are requested (all four NULL
 * skips the landmark gradients; dlmk_q needs lmk_k, dlmk_k needs lmk_q).
 * lse must be the one written by gca_grouped_xattn_fwd for the same inputs.
 * The result is deterministic (no floating-point atomics).
 * Workspace: gca_workspace_size(p, GCA_OP_BACKWARD) bytes, 256-byte aligned.
 * GCA_ERR_UNSUPPORTED when nQ * topk exceeds INT32_MAX or nQ >= 2^26.
 */
gca_status gca_grouped_xattn_bwd(const gca_problem* p, const void* q, const void* k,
                                 const void* v, const int32_t* idx, const float* sel,
                                 const float* lse, const void* dout, void* dq, void* dk,
                                 void* dv, float* dsel, const void* lmk_q,
                                 const void* lmk_k, float* dlmk_q, float* dlmk_k,
                                 void* workspace, size_t ws_bytes, hipStream_t stream);

/* The whole forward path: scores (Eq. 1) -> top-k (Eq. 1) -> weights (Eq. 2) ->
 * grouped cross attention (Eq. 2-3).  Outputs as for the calls above; idx and sel
 * are required (the backward needs them), lse and w may be NULL.  In CAUSAL mode
 * the score matrix is written to the workspace and then selected, or, for long
 * sequences or with GCA_FLAG_FUSED_TOPK, scored and selected without it (landmarks
 * wider than 512 columns, 256 in fp32, may then use `out` as scratch until the attention
 * writes it, unless it overlaps another argument).  In DECODE mode the past landmark keys are scanned in parallel ranges that
 * each leave their best k in the workspace; the attention kernel merges them
 * into idx/sel (the exact top-k) before attending.
 * Workspace: gca_workspace_size(p, GCA_OP_FORWARD) bytes, 256-byte aligned.
 */
gca_status gca_forward(const gca_problem* p, const void* lmk_q, const void* lmk_k,
                       const void* q, const void* k, const void* v, void* out,
                       int32_t* idx, float* sel, float* lse, float* w, void* workspace,
                       size_t ws_bytes, hipStream_t stream);

/* gca_forward for callers that cannot allocate memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * path and results as gca_forward on the same arguments, with the workspace
 * taken from a device array of GCA_NOALLOC_SCRATCH_BYTES that the library
 * holds on every device it runs on until the process ends.  The caller still
 * passes every input and output.  No memory is allocated or freed.
 * - GCA_ERR_UNSUPPORTED if gca_workspace_size(p, GCA_OP_FORWARD) exceeds
 *   GCA_NOALLOC_SCRATCH_BYTES (nothing is launched);
 * - all calls on one device share that device's array: calls that overlap in
 *   time on one device (different streams, or different threads without
 *   ordering) race on it and must not be issued.  Calls ordered on one stream
 *   are safe: no part of the array needs to start at any value, every byte a
 *   call reads was written earlier in the same call.
 * - GCA_ERR_HIP if the array's device address cannot be looked up (once per
 *   device, on the first call there). */
#define GCA_NOALLOC_SCRATCH_BYTES (16u << 20)
gca_status gca_forward_noalloc(const gca_problem* p, const void* lmk_q, const void* lmk_k,
                               const void* q, const void* k, const void* v, void* out,
                               int32_t* idx, float* sel, float* lse, float* w,
                               hipStream_t stream);

/* ---------------------------------------------------------------- chunk cache ----
 *
 * A bounded cache of past chunks in 8 bits, for serving: every sequence has `capacity`
 * slots of one chunk (up to S tokens).  The calls below store chunks into slots, select
 * the slots to attend to by landmark, attend to them, and evict the chunks that were
 * attended to least.  All state is the caller's device memory, named in gca_cache; every
 * call reads lengths, slots and counters on the device, so a serving loop needs no
 * synchronisation and can be captured into a HIP graph.  Calls on one cache are ordered by the
 * caller (one stream, or events), as are calls that share a workspace.
 *
 * GCA has no positions between chunks (Methodology: retrieved chunks are attended to one
 * by one), so a chunk may sit in any slot; ties between scores go to the lower slot.
 *
 * Numbers.  A cached number stands for itself times its tile's scale; a tile is the keys
 * or the values of one chunk of one cached head.
 *   GCA_E4M3  8-bit floats (OCP e4m3, 4 exponent and 3 mantissa bits, largest 448); the
 *             scale is the least power of two (at least 2^-126) that brings the tile's largest
 *             finite magnitude to at most 448.  Infinities are stored as +-448, NaN as NaN.
 *   GCA_INT8  integers -127 .. 127; the scale is the largest finite magnitude (at least
 *             2^-100) over 127.  Infinities are stored as +-127; a tile with a NaN gets the
 *             scale NaN.
 * Values are stored transposed, so that both products of the attention read their operand
 * from memory in the order in which the matrix cores take it.
 */
typedef enum { GCA_E4M3 = 0, GCA_INT8 = 1 } gca_format;

/* B sequences; H query heads share Hkv cached heads (query head h reads cached head
 * h / (H / Hkv)); Hr = 1 list of slots per sequence, or Hr = Hkv, one per cached head.
 * Supported: d == 64, S == 64, H a multiple of Hkv, 1 <= capacity <= 262144, 1 <= topk
 * <= 32, D a positive multiple of 64 up to 8192.  A call requires the members it names. */
typedef struct {
  int32_t B, H, Hkv, Hr;
  int32_t d, S;
  int64_t capacity;     /* slots per sequence */
  int32_t topk;         /* entries of a list of slots, 1..32 */
  int32_t D;            /* landmark vector width */
  float score_scale;    /* multiplies <landmark query, landmark key> */
  float attn_scale;     /* multiplies <q, k> */
  int32_t off_by_one;   /* as in gca_problem */
  int32_t dtype;        /* gca_dtype of q, k, v, out, lmk and landmark queries */
  int32_t format;       /* gca_format of the cached numbers */
  uint32_t flags;       /* 0 */
  void* k;              /* [B, Hkv, capacity, S, d] 8-bit keys */
  void* v;              /* [B, Hkv, capacity, d, S] 8-bit values, transposed per chunk */
  float* k_scale;       /* [B, Hkv, capacity] */
  float* v_scale;       /* [B, Hkv, capacity] */
  void* lmk;            /* [B, Hr, capacity, D] dtype: landmark keys */
  int32_t* tokens;      /* [B, capacity] tokens of the chunk in each slot; <= 0: the slot is free */
  float* mass;          /* [B, capacity] attention weight that the chunk has gathered */
  int32_t* number;      /* [B, capacity] the chunk's number in its sequence */
  int32_t* next;        /* [B] number of the sequence's next chunk */
} gca_cache;

/* Store chunk i of sequence b, tokens 64 i .. 64 i + 63 of the new keys and values, into
 * slot slots[b, i]: quantised tiles and scales, its length into `tokens`, its landmark key
 * into `lmk`.  Rows behind a chunk's last token are stored as zeros.  Entries outside
 * [0, capacity) and chunks without tokens are skipped, and nothing of any other slot is
 * written.  Where a sequence names a slot twice, its last chunk with tokens is stored.
 *   k, v    [B, Hkv, n * S, d] dtype
 *   lmk     [B, Hr, n, D]      dtype    landmark keys; NULL: c->lmk is left as it is
 *   slots   [B, n]             int32    (e.g. from gca_cache_evict)
 *   lengths [B]                int32    new tokens of each sequence, at most n * S of which
 *                                       count; NULL: n * S
 * Requires c->k, v, k_scale, v_scale, tokens, and lmk if the argument is given. */
gca_status gca_cache_store(const gca_cache* c, const void* k, const void* v, const void* lmk,
                           const int32_t* slots, const int32_t* lengths, int64_t n, hipStream_t stream);

/* Retrieval among the slots in use (Eq. 1, as DECODE mode): for each retrieval row the
 * min(topk, #candidates) best scores score_scale * <lmk_q, lmk[slot]>, where candidates
 * are the slots with tokens > 0 whose score is finite; ties go to the lower slot.
 *   lmk_q [B, Hr, 1, D]    dtype
 *   idx   [B, Hr, 1, topk] int32  output: slots ascending, -1 padded
 *   sel   [B, Hr, 1, topk] fp32   output: their scores, -inf padded
 *   w     [B, Hr, 1, topk] fp32   output: softmax of sel (Eq. 2), 0 on pads; may be NULL
 * Requires c->lmk and tokens.  Workspace: gca_cache_workspace_size(c,
 * GCA_OP_CACHE_SELECT, 0) bytes, 256-byte aligned. */
gca_status gca_cache_select(const gca_cache* c, const void* lmk_q, int32_t* idx, float* sel, float* w,
                            void* workspace, size_t ws_bytes, hipStream_t stream);

/* Grouped cross attention over the cache (Eq. 2-3; as gca_grouped_xattn_fwd).  The query
 * rows come in nQ groups of `rows` rows (one token, a few, a chunk, or any number), and
 * group t attends to the chunks of list t - lag: lag = 0 gives every group the list of its
 * own number, lag = 1 the one before (CAUSAL lists; group 0 then has none).  Entries that
 * name no slot in use (outside [0, capacity), or tokens <= 0) are pads; a slot's softmax
 * is over its first `tokens` keys.  Rows without a valid entry get out = 0.  NaN in a query
 * row, or in the keys, values or scales of an entry's tokens, comes out as NaN; what lies
 * behind a slot's tokens or in free slots has no effect, whatever it is.
 *   q   [B, H, nQ * rows, d]    dtype
 *   idx [B, Hr, nQ, topk]       int32
 *   sel [B, Hr, nQ, topk]       fp32   finite on valid entries
 *   out [B, H, nQ * rows, d]    dtype  output
 *   lse [B, H, nQ * rows, topk] fp32   output: log of each entry's softmax denominator
 *                                      (-inf on pads), may be NULL
 *   w   [B, Hr, nQ, topk]       fp32   output: fusion weights of every list, may be NULL
 * Products of q with the cached numbers are exact and summed in fp32.  Probabilities, with
 * their entry's fusion weight and value scale in them, are rounded to fp16 (fp32 tensors: to
 * two fp16 terms), but not finer than to a 2^-40th of the list's largest product of weight
 * and value scale, before they meet the values.
 * Requires c->k, v, k_scale, v_scale, tokens. */
gca_status gca_cache_xattn(const gca_cache* c, const void* q, const int32_t* idx, const float* sel, void* out,
                           float* lse, float* w, int64_t nQ, int64_t rows, int32_t lag, hipStream_t stream);

/* Make room for the n next chunks of every sequence by evicting the chunks that gathered
 * the least attention weight.  In this order, for each sequence b:
 *   1. mass[b, j] = decay * mass[b, j] + the weights w of the entries of its lists that name
 *      slot j, for slots in use (each weight counted to the nearest 2^-48, or where a
 *      sequence has 2^16 entries or more, of less than 2^e to the nearest 2^(e - 64), so that
 *      the sum does not depend on its order; negative and NaN ones as 0, ones above 1 as 1);
 *      0 for free slots;
 *   2. m = want[b] slots (n if want is NULL; between 0 and n) are asked for: free slots first,
 *      lowest first, then the chunks in order of (mass, slot), except those numbered below
 *      keep_first or not below next[b] - keep_last, so that fewer than m may be taken.  A
 *      negative or NaN mass ranks as 0;
 *   3. the slots taken are written to slots[b, 0 ..], ascending, padded with -1 up to n; tokens
 *      and mass of each become 0 and number[b, slots[b, i]] = next[b] + i; then next[b] += m
 *      (chunks that found no slot keep their numbers).
 * m is to be the number of chunks that the sequence will store: a slot that nothing is stored
 * in was emptied for nothing, and a number that no chunk has counts towards keep_last.
 * gca_cache_store then fills them.  With n = 0 only the masses change.
 *   idx, w [B, Hr, nQ, topk] int32, fp32  lists and fusion weights since the last call; both
 *                                         NULL (and nQ ignored): none
 *   want   [B]               int32        may be NULL
 *   slots  [B, n]            int32        output
 * Requires c->tokens, mass, number, next.  Workspace: gca_cache_workspace_size(c,
 * GCA_OP_CACHE_EVICT, n) bytes (0 for small caches), 256-byte aligned. */
gca_status gca_cache_evict(const gca_cache* c, const int32_t* idx, const float* w, int64_t nQ, float decay,
                           int32_t keep_first, int32_t keep_last, const int32_t* want, int32_t* slots, int64_t n,
                           void* workspace, size_t ws_bytes, hipStream_t stream);

#define GCA_OP_CACHE_SELECT 2
#define GCA_OP_CACHE_EVICT 3
/* Bytes of workspace that `op` (GCA_OP_CACHE_SELECT, or GCA_OP_CACHE_EVICT of n chunks) asks
 * for; 0 if c is invalid or none is asked for.  It depends on c's sizes alone and never falls as
 * n grows.  A selection asks for what the scan in two launches needs, also where the cache
 * is small enough for the form in one launch, which leaves it unused. */
size_t gca_cache_workspace_size(const gca_cache* c, int op, int64_t n);

/* --------------------------------------------------------------- token window ----
 *
 * The tokens that a layer's self-attention looks back at (the sliding window, with linear biases, of
 * Methodology / Model Architecture, beside the retrieved chunks), in 8 bits, for serving: every
 * sequence has `capacity` rows.  The calls below append new tokens (one, a tree of drafted ones, or
 * a prompt), attend with their queries, verify drafts against the target's probabilities, and
 * keep the accepted ones.  As with the chunk cache all state is the caller's device memory, every
 * count is read on the device, and calls on one window are ordered by the caller.
 *
 * length[b] counts the tokens of sequence b, the newest included; position p is in row
 * p mod capacity (window > 0: a ring), or in row p if p < capacity (window = 0: all tokens are
 * seen; those past the capacity are counted but neither kept nor seen).  Sequences of up to 2^30
 * tokens.
 *
 * Numbers.  As in the chunk cache, but with one scale per token and cached head for its 64
 * keys, and one for its 64 values: the least power of two (at least 2^-126) that brings the largest
 * finite magnitude to at most 448 (GCA_E4M3), or that magnitude (at least 2^-100) over 127
 * (GCA_INT8; an entry is multiplied in fp32 by 127 times the magnitude's reciprocal, and rounded to the nearest, ties
 * to even).  Infinities are stored as the largest number; a token with a NaN among its keys
 * (values) has the scale NaN for its keys (values).
 *
 * B sequences; H query heads share Hkv cached heads, as in gca_cache.  Supported: d == 64, H a
 * multiple of Hkv, B H < 2^19, capacity a multiple of 64 up to 2^24, window 0 .. capacity, and
 * calls of T tokens with T up to 16 floor((2^23 - 8) / (B H)), so B H T up to 2^26 at least. */
typedef struct {
  int32_t B, H, Hkv;
  int32_t d;
  int64_t capacity;     /* rows per sequence */
  int32_t window;       /* tokens that a row sees, itself included; 0: all */
  float attn_scale;     /* multiplies <q, k>; 0, or at least 2^-64 in magnitude */
  int32_t off_by_one;   /* 1: the softmax's denominator is 1 + its sum, as in gca_problem */
  int32_t dtype;        /* gca_dtype of q, k, v, out */
  int32_t format;       /* gca_format of the kept numbers */
  uint32_t flags;       /* 0 */
  void* k;              /* [B, Hkv, capacity, d] 8-bit keys */
  void* v;              /* [B, Hkv, capacity / 64, d, 64] 8-bit values, transposed per 64 rows */
  float* k_scale;       /* [B, Hkv, capacity]; GCA_E4M3: powers of two */
  float* v_scale;       /* [B, Hkv, capacity] */
  int32_t* length;      /* [B] tokens of each sequence so far */
  int32_t* ticket;      /* [B, 2 H] zeros before the first call; every call leaves them so */
} gca_window;

/* Append T new tokens to every sequence: token i of sequence b becomes position length[b] + i, and
 * length[b] grows by their number.  Where that exceeds a ring's capacity, the last `capacity` of
 * them are kept.  No row of another position is written.
 *   k, v    [B, Hkv, T, d] dtype
 *   lengths [B]            int32  new tokens of each sequence, 0 .. T of which count; NULL: T
 * Requires w->k, v, k_scale, v_scale, length, ticket. */
gca_status gca_window_append(const gca_window* w, const void* k, const void* v, const int32_t* lengths, int64_t T,
                             hipStream_t stream);

/* Attention of the newest tokens (those of the last append), n_b = lengths[b] (NULL: T) of them, over the
 * window.  With base = length[b] - n_b, row i is at position base + depth(i), its depth being i in a
 * chain (parents NULL) and in a tree of drafted tokens its number of ancestors; it sees
 *   - the positions p < base with p > base + depth(i) - window,
 *   - itself and its ancestors (a chain: the new tokens before it) less than `window` levels above,
 * with scores  attn_scale <q, k> + slopes[h] (position of the key - position of the row),
 * one softmax over all of them, and out = softmax V.  Rows from n_b on, rows that see nothing and rows whose scores
 * are all -inf get out = 0 and lse = -inf.  NaN in a row's query or in the scales of a token that it sees comes
 * out as NaN, and so does an infinity in its query that leaves a score above -inf.  What a row does not see has no effect on it, whatever it is (a value's number that is NaN,
 * which gca_window_append never stores, in a row that others see aside), but for the roundings below: they go by
 * value scales that other rows of its block see.
 *   q       [B, H, T, d] dtype
 *   parents [B, T]       int32  of each node; entries outside 0 .. i - 1 make node i a root.  Needs
 *                               T <= 64.  NULL: a chain, of any T
 *   lengths [B]          int32  as for the append; may be NULL
 *   slopes  [H]          fp32   may be NULL: 0
 *   out     [B, H, T, d] dtype  output
 *   lse     [B, H, T]    fp32   output: log of each row's softmax denominator; may be NULL
 * In a ring, a row's window has to outlast the new tokens: window + T - 1 <= capacity (a
 * longer prompt comes in pieces; GCA_ERR_INVALID).  Products of q with the kept numbers are exact (GCA_E4M3: with
 * scales from 2^-117 up, below which keys times their scale are bf16 numbers without all their bits) and summed
 * in fp32.  Probabilities relative to the row's largest so far, with their value scale in them, are rounded to
 * fp16 (fp32 tensors: to two fp16 terms): by 2^-11 (2^-22) of themselves, or, where they are so small, by up to a
 * 2^-39th of the largest value scale that a row of the row's block sees.  (Blocks of 64 rows, for
 * GCA_E4M3 and bf16 where there are enough to fill the chip, round the probabilities alone, by 2^-11 or 2^-40, and
 * hold values in fp16, exactly, or, where they are so small, to a 2^-30th of that scale.)  The same call on the same
 * state gives the same bits.  How the work is cut, and with it the order of sums, goes by the call's sizes and, with
 * window = 0, by all sequences' lengths: a sequence in another batch keeps to these roundings, but not to the bit.
 * Requires w->k, v, k_scale, v_scale, length, ticket.  Workspace: gca_window_workspace_size(w, T)
 * bytes, 256-byte aligned. */
gca_status gca_window_attn(const gca_window* w, const void* q, const int32_t* parents, const int32_t* lengths,
                           const float* slopes, void* out, float* lse, int64_t T, void* workspace, size_t ws_bytes,
                           hipStream_t stream);

/* Of the newest n_b = lengths[b] (NULL: T) tokens keep those that path names, in its order, and drop the
 * others: token path[b, i] moves to position base + i, base = length[b] - n_b, and length[b] becomes
 * base + m.  The path's m entries end at the first that is not larger than the one before, is
 * outside 0 .. n_b - 1 (-1 padding), or (window = 0) would bring a token from past the capacity, which was
 * not kept, below it.
 *   path    [B, n] int32, 0 <= n <= 64 (e.g. from gca_verify)
 *   lengths [B]    int32, as for the append; may be NULL
 * Requires w->k, v, k_scale, v_scale, length, ticket.  T >= 1; in a ring window + T - 1 <= capacity, as for the
 * attention: the rows of dropped tokens then held none that the next ones see. */
gca_status gca_window_keep(const gca_window* w, const int32_t* path, int64_t n, const int32_t* lengths, int64_t T,
                           hipStream_t stream);

/* Bytes of workspace that gca_window_attn of up to T tokens asks for; 0 if w is invalid or none is
 * asked for.  It depends on w's sizes alone and never falls as T grows. */
size_t gca_window_workspace_size(const gca_window* w, int64_t T);

/* Verification of drafted tokens by rejection sampling, so that what is kept is distributed as the target's
 * own samples.  Node 0 of sequence b's tree is its newest token, nodes 1 .. n_b - 1 are drafts; p[b, i] are
 * the target's probabilities of the token behind node i, and q[b, i] those that node i's children
 * were drawn from, independently (q NULL: the children were chosen, not drawn).  From node a = 0, with
 * r = p[a] and z = 1, the children of a are tested in ascending order: child c, of token x, has
 *   s = z q[a, x] (NULL: z)   and is accepted if u[c] s < r[x]:  then a = c, r = p[a], z = 1, and its
 * children follow; otherwise
 *   r = max(r - z q[a], 0), z = sum r   (NULL: z = max(z - r[x], 0), r[x] = 0).
 * When no child is left, the next token is drawn from r: the first x whose partial sum r[0] + .. + r[x]
 * exceeds u[0] sum r.  If r is zero everywhere, from p[a]; if that is too, next = -1.  Probabilities count
 * as 0 where they are negative or NaN and as 1 above 1.  Products and differences are in fp64, and sums are of
 * r to the nearest 2^-44, exactly: they do not depend on their order.  (With q, the R-th rejected child of a node that
 * has a sibling left takes a pass over p[a] and q[a] of about R steps per entry: trees of a few siblings are meant.)
 *   p, q    [B, T, V] fp32 (q may be NULL)
 *   tokens  [B, T]    int32  drafted tokens; one outside 0 .. V - 1 is rejected, leaving r as it is
 *   parents [B, T]    int32  as for the attention, but a node without a parent is never reached (but node
 *                            0).  NULL: a chain
 *   u       [B, T]    fp32   random numbers in [0, 1)  (NaN and below: 0; above: the largest below 1)
 *   lengths [B]       int32  nodes n_b, at most T of which count; NULL: T.  0: path is empty, next = -1
 *   path    [B, T]    int32  output: node 0 and the accepted nodes, ascending, -1 padded
 *   count   [B]       int32  output: their number
 *   next    [B]       int32  output: the token that follows
 * Supported: 1 <= T <= 64, 1 <= V <= 2^19.  Workspace: gca_verify_workspace_size(B, T, V) bytes,
 * 256-byte aligned. */
gca_status gca_verify(int64_t B, int64_t T, int64_t V, const float* p, const float* q, const int32_t* tokens,
                      const int32_t* parents, const float* u, const int32_t* lengths, int32_t* path, int32_t* count,
                      int32_t* next, void* workspace, size_t ws_bytes, hipStream_t stream);

/* Bytes of gca_verify's workspace; 0 if the sizes are invalid. */
size_t gca_verify_workspace_size(int64_t B, int64_t T, int64_t V);

/* Profiling aid (outside the method).  While armed, the i-th kernel that libgca
 * launches from the calling thread (i = 0, 1, ... while 2 (i + 1) <= capacity,
 * capacity <= 4096) is dispatched with events[2 i] and events[2 i + 1] as its
 * start and stop events (hipExtLaunchKernel), so a caller can time each kernel
 * alone without adding work to the stream.  The events are created and owned
 * by the caller.  gca_profile_arm(NULL, 0) disarms; arming resets the count.
 * gca_profile_count() is the number of kernels timed since arming and
 * gca_profile_name(i) the name of kernel i (NULL if out of range). */
void gca_profile_arm(hipEvent_t* events, int capacity);
int gca_profile_count(void);
const char* gca_profile_name(int i);

/* Bytes of workspace `op` (GCA_OP_FORWARD or GCA_OP_BACKWARD) needs for problem p;
 * 0 if p is invalid or needs none.  In DECODE mode the forward's size never falls as
 * n_chunks grows: a workspace sized for the longest past serves every shorter one. */
size_t gca_workspace_size(const gca_problem* p, int op);

/* Static description of a status code. */
const char* gca_status_string(gca_status s);

/* Detail of the last error raised on the calling thread ("" if none). */
const char* gca_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* LIBGCA_GCA_H */
