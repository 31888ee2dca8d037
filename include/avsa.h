/*
 * avsa -- protected sparse video attention for joint audio-video diffusion transformers, sm_100a.
 *
 * C ABI of libavsa.so.  Three calls make one layer-step of the path:
 *
 *   avsa_cross_attn_scores   audio->video cross-attention (Eq. 1) that also emits the per-video-token
 *                            cross-modal response scores (Eq. 2, with the blend of Eq. 4 folded in)
 *   avsa_build_block_mask    protected token set (Eq. 3 / Eq. 8), block-importance top-k, and the
 *                            protected block mask (Eq. 9) as ascending per-row column lists
 *   avsa_sparse_self_attn    video self-attention under that mask (Eq. 10 / Eq. 11)
 *
 * A generation that continues a clip keeps keys and values in a paged cache (avsa_cache_*), which the candidates of a
 * continuation share as far as they begin alike, and attends to it with avsa_prefix_attn.  The cache may be held in 4 bits
 * (avsa_cache_write_q4, avsa_cache_read_q4, avsa_prefix_attn_q4).  avsa_rope turns queries and keys by their places.
 *
 * Conventions for every call
 *   - All data pointers are DEVICE pointers unless a parameter says "host".  The caller owns every
 *     buffer.  The library allocates no device memory, never synchronises the stream (except
 *     avsa_read_status) and enqueues work on the given stream only.
 *   - Tensors are bf16 with the head dimension contiguous, described by element strides (avsa_bf16_4d),
 *     so both [B,H,N,d] and [B,N,H,d] storage work.  Base pointers must be 16-byte aligned and strides
 *     multiples of 8 elements.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).  No call reads device
 *     data on the host, so the calls may be recorded into a CUDA graph by stream capture (not on the legacy
 *     default stream) and replayed; pointers, sizes and counts are fixed at capture time.
 *   - `ws` is scratch of at least the matching *_workspace_bytes(), which depends on the shape and on the number of SMs
 *     of the current device (148 are assumed where there is none) and makes no context.  Its first AVSA_STATUS_BYTES (256) bytes
 *     are reserved for a 24-byte status record of six int32: code (avsa_status), where, item, aux -- filled
 *     when a device-side check fails (a wait that ran out of time, or a malformed column list) -- then at
 *     byte 16 a count of work items or query tiles (see below) and at byte 20 the head of the persistent
 *     kernels' work queue.  Calls on the same workspace must not overlap on the GPU.
 *   - Alignment of `ws`: 32 bytes are enough for every call, 16 for the changes of a paged cache, 4 for sparse self-attention, for
 *     cross-attention against at most 256 keys and for a mask under given block scores.  With less than a call's kernels need
 *     (16 or 32 bytes, by shape) it returns AVSA_ERR_INVALID_ARG and enqueues nothing.
 *   - The attention calls (cross-attention against more than 256 keys that is not short, sparse self-attention, protected rows) run
 *     a kernel that normalises each row by the maximum of its first key tile instead of a running maximum
 *     (softmax is invariant to that shift), and recompute with exact rescaling the work items whose rows outgrew
 *     that reference (a row whose sum of exp(logit - reference) ends above 2^64 or not finite): in the same kernel
 *     in short calls, in one behind it in long ones (with 64 channels and many blocks, where two query blocks are run
 *     at a time, also those with an output that is not finite).  Results do not depend on which way produced them
 *     beyond rounding; the int32 at byte 16 of ws counts the recomputed items (diagnostic).  Cross-attention in short calls
 *     against at most 4096 keys recomputes nothing (every part of a row takes its own maximum), nor does it
 *     against at most 256 keys: there a row whose keys from 128 on outgrow the maximum of the first 128 by more
 *     than 2^57 (as factors of exp) takes a larger reference on the way, and the int32 counts the tiles of 128
 *     queries in which one did so by more than 2^64.  Values of v are assumed to stay below 2^60 in magnitude.
 *   - Errors detectable on the host return at once with nothing enqueued.  Return values are
 *     avsa_status codes.
 *   - Supported shapes: (blk, d) in {(128,128), (64,64)}; B and H up to 65535, B*H below 2^31 (mask: up to
 *     65535); any N >= 1 (the last block may be partial: pooled means divide by the valid count, invalid
 *     keys are masked, rows >= N are not written).  Those of the paged cache and of rope stand at their calls, (6) to (9).
 */
#ifndef AVSA_H_
#define AVSA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define AVSA_API __attribute__((visibility("default")))
#else
#define AVSA_API
#endif

typedef enum {
  AVSA_OK = 0,
  AVSA_ERR_INVALID_ARG = 1,  /* null pointer, bad size, bad stride or alignment (of a tensor or of ws) */
  AVSA_ERR_UNSUPPORTED = 2,  /* (blk, d) combination or device not supported */
  AVSA_ERR_WORKSPACE = 3,    /* ws is NULL or smaller than *_workspace_bytes() */
  AVSA_ERR_CUDA = 4,         /* a CUDA runtime / driver call failed */
  AVSA_ERR_TIMEOUT = 5,      /* device: a bounded wait expired (read with avsa_read_status) */
  AVSA_ERR_BAD_MASK = 6,     /* device: a column list entry was out of range or not ascending */
  AVSA_ERR_BAD_TABLE = 7,    /* device: a sequence, a page of a sequence or a length of a paged cache is out of range */
  AVSA_ERR_NO_PAGES = 8      /* device: a paged cache has too few free pages, or a sequence's row of the table is full */
} avsa_status;

/* Size of the status record area at the start of every workspace. */
#define AVSA_STATUS_BYTES 256

/* bf16 tensor [B,H,N,d], d contiguous; strides in elements. */
typedef struct {
  const void* ptr;
  int64_t stride_b, stride_h, stride_n;
} avsa_bf16_4d;

/*
 * Paged K/V cache of a generation.  The keys and values of `seqs` sequences live in `pages` pages of `page` tokens;
 * token t of sequence s is in page table[s*width + t / page] at place t % page.  A page may belong to several
 * sequences that begin alike (avsa_cache_fork).  All arrays are contiguous device memory:
 *   table   int32 [seqs,width]  pages of each sequence in order, -1 behind its last one
 *   length  int32 [seqs]        tokens of each sequence, 0 = an empty place
 *   ref     int32 [pages]       sequences that hold the page, 0 = free
 * A call reads table, length and ref and writes the state behind it to table_out, length_out and ref_out: the same
 * pointers (in place) or arrays that overlap none of those read.  `page` is 16, 32, 64 or 128 tokens.
 */
typedef struct {
  const int32_t* table;
  const int32_t* length;
  const int32_t* ref;
  int32_t* table_out;
  int32_t* length_out;
  int32_t* ref_out;
  int seqs, width, pages, page;
} avsa_cache;

/* The memory of the pages, `planes` times over (2 x layers: keys and values of each): page p of plane i is page_bytes
 * bytes at ptr + i*stride_plane + p*stride_page.  All of them multiples of 16 bytes. */
typedef struct {
  void* ptr;
  int planes;
  int64_t page_bytes, stride_plane, stride_page;
} avsa_pages;

/*
 * Pages of keys, or of values, held in 4 bits.  A page of a key/value head is one piece of page * (d/2 + d/16) bytes; pages are stride_page bytes apart and
 * heads stride_head, multiples of 16, as is ptr.  For each 16 tokens there are 16 x d/2 bytes of codes, then 16 x d/32 scales (bf16).  32 channels
 * of a token share a scale, the nearest number of five significant bits to their largest magnitude over 7 (halfway: the larger one), and each has a code,
 * the nearest whole number of scales (halfway: the even one), -7 .. 7, so that every value that a page stands for is a bf16 number.  A token's codes are little-endian words
 * of eight channels, code + 8 of channel 2i at bits 4i, of channel 2i + 1 at bits 16 + 4i.
 * A group of channels whose largest magnitude is below 2^-100 is held as zeros; one with an infinity, a NaN or a magnitude of 2^125 and more reads as NaN.
 */
typedef struct {
  void* ptr;
  int64_t stride_page, stride_head;
} avsa_q4_pool;

/* flags of avsa_rope */
#define AVSA_ROPE_HALVES 1u    /* the pairs are channels (i, i + d/2), not (2i, 2i + 1) */
#define AVSA_ROPE_INVERSE 2u   /* turns back: the inverse, and the gradient */
#define AVSA_ROPE_AXES 4       /* at most */

/* flags of avsa_build_block_mask */
#define AVSA_PROTECT_ROWS 1u            /* Eq. 9: a protected query block keeps every key block */
#define AVSA_PROTECT_COLS 2u            /* opt-in superset: protected key blocks visible to all rows */
#define AVSA_USE_GIVEN_BLOCK_SCORES 4u  /* block_scores is an input; q and k are not read */
#define AVSA_PROTECT_TOKENS 8u          /* lists carry the base pattern only (no block is made dense); the
                                           protected rows are restored by avsa_protected_rows_attn */

#define AVSA_PROTECT_BLOCK_SUM 16u      /* not in the paper: n_protect counts BLOCKS (0..NB); the protected blocks are
                                           those with the largest summed response (fp64 sum of the block's scores
                                           rounded to fp32, ties to the lowest block index); prot_tok flags every
                                           token of a protected block.  Combines with ROWS / COLS / TOKENS. */

/* Optional, ORed into flags: a block counts as protected only if it holds at least n (1..blk) protected tokens.
 * Not in the paper: in raster order a compact region straddles many blocks, and n > 1 trades the protection of
 * stray tokens for fewer dense blocks.  n = 0 or 1 is the block lift of Eq. 9 (any protected token). */
#define AVSA_MIN_TOKENS_PER_BLOCK(n) (((unsigned)(n) & 0xffu) << 8)

/*
 * (1) Cross-attention with response scores -- Eq. 1, Eq. 2 (and the running blend of Eq. 4).
 *
 *   A[b,h,j,i] = softmax_i(q[b,h,j,:] . k[b,h,i,:] * softmax_scale)            (queries j, keys i)
 *   o[b,h,j,:] = sum_i A[b,h,j,i] v[b,h,i,:]                  -> o   bf16, same strides as q's tensor
 *   lse[b,h,j] = natural-log log-sum-exp of row j              -> lse fp32 [B,H,Nq]
 *   scores[b,i] = score_beta * scores[b,i] + score_gamma * sum_h sum_j A[b,h,j,i]   fp32 [B,Nk]
 *
 * For the audio->video direction q holds the audio queries and k, v the video keys/values.  The
 * paper's Norm is any scalar: score_gamma = 1/(H*Nq*layers) makes the scores sum to 1; score_beta = 1
 * accumulates layers; score_beta = alpha with score_gamma = (1-alpha)/(H*Nq) is Eq. 4.
 * With score_beta == 0 the previous contents of scores are ignored (may be uninitialised).
 * o, lse and scores may each be NULL to skip that output (scores == NULL skips the second pass).
 * softmax_scale == 0 means 1/sqrt(d).  When scores are requested min(Nq, Nk) <= 512 (the score pass keeps the
 * shorter axis of a head on chip: the audio queries, or, in the reverse video->audio direction of the
 * bidirectional pair, the audio keys); without scores any Nq and Nk.  The head sum is taken in a fixed order, so
 * results reproduce bit for bit, and o and lse are the same bits with scores and without.  `o` has strides
 * (o_stride_b, o_stride_h, o_stride_n) = q's.
 */
AVSA_API int avsa_cross_attn_scores(int B, int H, int Nq, int Nk, int d, avsa_bf16_4d q, avsa_bf16_4d k, avsa_bf16_4d v,
                           void* o_bf16, float* lse, float* scores, float score_beta, float score_gamma,
                           float softmax_scale, void* ws, size_t ws_bytes, void* stream);
AVSA_API size_t avsa_cross_attn_scores_workspace_bytes(int B, int H, int Nq, int Nk, int d);

/*
 * (2) Mask construction -- Eq. 3 / Eq. 8 (protected set), Eq. 9 (protected mask), and the base
 * sparse pattern the paper leaves open, here: block mean-pooling of q and k, block scores
 * Bs[b,h,qb,kb] = mean(q block qb) . mean(k block kb) * softmax_scale, per (head, query block)
 * top-k_keep over kb.
 *
 *   scores       fp32 [B,N] token saliency; may be NULL iff n_protect == 0
 *   n_protect    size of the protected token set, 0 <= n_protect <= N (= ceil(rho N), host integer)
 *   k_keep       kept key blocks per unprotected row, 1 <= k_keep <= NB, NB = ceil(N / blk)
 *   block_scores fp32 [B,H,NB,NB]: output, or input with AVSA_USE_GIVEN_BLOCK_SCORES (never NULL)
 *   col_idx      int32 [B,H,NB,NB]: kept key blocks of each row, ascending, unused slots = -1
 *   col_cnt      int32 [B,H,NB]
 *   prot_tok     uint8 [B,N]  1 = token in the protected set (optional, may be NULL)
 *   prot_blk     uint8 [B,NB] 1 = block holds a protected token (optional, may be NULL)
 *
 * Every top-k orders by (value larger, then index smaller); NaN ranks as -inf; -0 equals +0.
 * Given the same fp32 scores / block_scores the outputs are exactly determined (integer results).
 * Without any AVSA_PROTECT_* flag AVSA_PROTECT_ROWS is assumed.  NB <= 2048.
 */
AVSA_API int avsa_build_block_mask(int B, int H, int N, int d, int blk, avsa_bf16_4d q, avsa_bf16_4d k, const float* scores,
                          int n_protect, int k_keep, unsigned flags, float softmax_scale, float* block_scores,
                          int32_t* col_idx, int32_t* col_cnt, uint8_t* prot_tok, uint8_t* prot_blk, void* ws,
                          size_t ws_bytes, void* stream);
AVSA_API size_t avsa_build_block_mask_workspace_bytes(int B, int H, int N, int d, int blk);

/*
 * (3) Block-sparse self-attention -- Eq. 10 (Eq. 5 when every list is full).
 *
 *   o[b,h,i,:] = softmax_j(q_i . k_j * softmax_scale  restricted to keys j of the listed blocks) v
 *
 * For query block qb of head h the kept key blocks are col_idx[b,h,qb,0 .. col_cnt[b,h,qb]-1]
 * (row stride NB, ascending, each in [0,NB)).  Every list needs at least one entry; a malformed
 * entry sets AVSA_ERR_BAD_MASK in the status record and that block is skipped without any
 * out-of-range access.  o is bf16 with the strides of q; lse (optional) is fp32 [B,H,N] natural log.
 *
 * After the call the int32 at byte 16 of ws is the number of work items the exact kernel recomputed (see
 * the conventions above), and their indices ((b*H + h)*NB + query block, in no particular order) follow
 * as int32 behind the first AVSA_STATUS_BYTES bytes (diagnostic; results do not depend on it).
 */
AVSA_API int avsa_sparse_self_attn(int B, int H, int N, int d, int blk, avsa_bf16_4d q, avsa_bf16_4d k, avsa_bf16_4d v,
                          const int32_t* col_idx, const int32_t* col_cnt, void* o_bf16, float* lse,
                          float softmax_scale, void* ws, size_t ws_bytes, void* stream);
AVSA_API size_t avsa_sparse_self_attn_workspace_bytes(int B, int H, int N, int d, int blk);

/*
 * (4) Token-exact protection -- Eq. 9 applied to tokens, i.e. the row-wise form of Eq. 11: the rows of
 * the protected tokens are dense attention rows ("dense-row recomputation" in the paper's notes).
 *
 * Use with lists built under AVSA_PROTECT_TOKENS: run avsa_sparse_self_attn first, then this call, which
 * recomputes o[b,h,i,:] (and lse[b,h,i], if given) for every token i with prot_tok[b,i] != 0 as dense
 * attention over all N keys and overwrites those rows in place.  The cost is n_protect * N per head
 * (Eq. 16's rho N^2 term) instead of a whole block row per touched block.
 *   prot_tok   uint8 [B,N] as written by avsa_build_block_mask; exactly n_protect flags per batch item,
 *              otherwise AVSA_ERR_BAD_MASK is recorded and that batch item is left untouched
 *   o_bf16     in/out, bf16 with the strides of q;  lse in/out fp32 [B,H,N] or NULL
 * n_protect == 0 is a no-op.  The workspace also depends on n_protect.
 */
AVSA_API int avsa_protected_rows_attn(int B, int H, int N, int d, int blk, avsa_bf16_4d q, avsa_bf16_4d k,
                                      avsa_bf16_4d v, const uint8_t* prot_tok, int n_protect, void* o_bf16,
                                      float* lse, float softmax_scale, void* ws, size_t ws_bytes, void* stream);
AVSA_API size_t avsa_protected_rows_attn_workspace_bytes(int B, int H, int N, int d, int blk, int n_protect);

/*
 * (5) Cache-reuse indicators -- Eq. 12 (stream-wise feature change), Eq. 13 (change over the protected video
 * tokens), Eq. 14 (saliency drift) and Eq. 15 (their maximum against the threshold).
 *
 *   y_v, yhat_v  bf16 [B,Nv,C] contiguous: current and cached block outputs of the video stream
 *   y_a, yhat_a  bf16 [B,Na,C] contiguous: the same for the audio stream
 *   prot_tok     uint8 [B,Nv] protected-token flags (NULL: no protected set, dp = 0)
 *   s_cur, s_anchor  fp32 [B,Nv] current and anchor saliency maps (both NULL: ds = 0)
 *   out          fp32 [B,8]: dv, da, dp, ds, dsync = max(dv, da, lambda_p*dp, lambda_s*ds), reuse (1.0 iff
 *                dsync < tau), two unused slots
 *   dv = sum|y - yhat| / (sum|y| + eps), likewise da and dp; ds = 1 - <s,s^>/(|s||s^| + eps).
 * C must be a multiple of 8.  Sums are taken in a fixed order (bit-reproducible).  The paper's settings are
 * lambda_p = 0.5, lambda_s = 0.1, tau = 0.2.
 */
AVSA_API int avsa_cache_indicators(int B, int Nv, int Na, int C, const void* y_v, const void* yhat_v, const void* y_a,
                                   const void* yhat_a, const uint8_t* prot_tok, const float* s_cur,
                                   const float* s_anchor, float lambda_p, float lambda_s, float tau, float eps,
                                   float* out, void* ws, size_t ws_bytes, void* stream);
AVSA_API size_t avsa_cache_indicators_workspace_bytes(int B, int Nv, int Na, int C);

/*
 * Allocation-free variant of avsa_build_block_mask.  The paper has no counterpart; this is a
 * convenience of the library for callers that have no device allocator to draw a workspace from:
 * code that runs after its host application has frozen its memory budget, extensions loaded into
 * a runtime that owns all device memory and hands none out, and latency-critical loops in which a
 * synchronising allocation is not acceptable.
 *
 * Same arguments and results as avsa_build_block_mask, without `ws`: the scratch (pooled block means,
 * fallback flag buffers and the status record) lives in a fixed array of AVSA_STATIC_SCRATCH_BYTES
 * inside the library, which every GPU that loads libavsa.so holds until the process exits.
 *   - Shapes whose avsa_build_block_mask_workspace_bytes() exceeds AVSA_STATIC_SCRATCH_BYTES are
 *     refused with AVSA_ERR_WORKSPACE and nothing is enqueued.
 *   - The first call on each device looks up the array's device address (with that device current).
 *     Make that first call before starting any stream capture.
 *   - The call allocates nothing: no cudaMalloc/cudaFree, no allocating library routine.
 *   - All calls on a device share the one array, and it keeps the previous call's contents; what must
 *     start from zero (the status record) is cleared by the call itself.  Two such calls that overlap
 *     on the GPU (different streams) race on the array: serialise them.
 *   - The mask kernels have no device-side failure mode (no waits, no list input), so there is no
 *     status record to read after this call.
 *   - Call it from one host thread at a time per device.  The looked-up address belongs to the current
 *     context: after cudaDeviceReset() it is stale, and the library must be reloaded before the next call.
 */
#define AVSA_STATIC_SCRATCH_BYTES (16u << 20)
AVSA_API int avsa_build_block_mask_static(int B, int H, int N, int d, int blk, avsa_bf16_4d q, avsa_bf16_4d k,
                                          const float* scores, int n_protect, int k_keep, unsigned flags,
                                          float softmax_scale, float* block_scores, int32_t* col_idx,
                                          int32_t* col_cnt, uint8_t* prot_tok, uint8_t* prot_blk, void* stream);

/*
 * (6) Attention of a batch that shares a long beginning, over a paged cache.
 *
 *   o[b,h,i,:] = sum_{t < lim} softmax_t(q[b,h,i,:] . k_t * softmax_scale) v_t          -> o bf16, strides of q
 *   lse[b,h,i] = natural-log log-sum-exp of the row                                      -> lse fp32 [B,H,L], optional
 *
 * for the keys k_t and values v_t of sequence s = seq[b] (seq NULL: s = b), key/value head h / (H/Hkv), with
 * lim = length[s], or with AVSA_CAUSAL lim = length[s] - L + i + 1: the L queries are the last L tokens of the
 * sequence.  Rows with lim <= 0, and all rows of a batch entry with seq[b] < 0, are empty: o = 0, lse = -inf.
 *
 * avsa_prefix_attn_step  the same for a step in which the sequences got different numbers of tokens: with AVSA_CAUSAL the first count[b] (int32 [B],
 *                   0..L; NULL: L) of the L queries are the last count[b] tokens of their sequence, lim = length[s] - count[b] + i + 1, and the rows
 *                   behind them are empty.  Without AVSA_CAUSAL all L queries see all tokens.  A count out of range sets AVSA_ERR_BAD_TABLE
 *                   and is cut; it says that not all tokens of the step were written.  `log` as in (7).
 *
 *   k_pool, v_pool  [pages,Hkv,page,d]: stride_b is the distance of pages, stride_h of heads, stride_n of tokens
 *   prefix_pages    the first prefix_pages pages of all sequences of the batch are the same ones (of a shorter
 *                   sequence: all it has).  Where it costs less they are read once for the whole batch, all its queries stacked on
 *                   each other; the longest sequence's row of the table (of several the first batch entry's) then says which pages they are.  0: nothing is
 *                   shared.
 *
 * What pages hold behind the last token of the longest sequence that has them is never used (it may be anything, NaN too).  Values of tokens that some rows
 * of a call see and others must not have to be finite (their weight is 0, and 0 times an infinity is no number): those behind a causal row's limit, and those in
 * the shared pages that a sequence of the batch ends in front of.  A page of the table out of range reads as zeros and sets AVSA_ERR_BAD_TABLE, a
 * length beyond the table's width is cut there and sets it as well.
 * d is 64 or 128, H a multiple of Hkv, H/Hkv at most 128.  table has `seqs` rows of `width` entries.  o overlaps no input.  Rows that outgrow the maximum of
 * their first key tile, or that see keys there but none with a logit above -inf, are run again as in the other attention calls (up to 32 query rows a key head
 * take a running maximum instead).  Same bits on every run.
 * There is no backward pass: a cache is read by generation alone.
 */
#define AVSA_CAUSAL 1u
AVSA_API int avsa_prefix_attn(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q,
                              avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table, const int32_t* length,
                              const int32_t* seq, int prefix_pages, unsigned flags, float softmax_scale, void* o_bf16, float* lse,
                              void* ws, size_t ws_bytes, void* stream);
AVSA_API int avsa_prefix_attn_step(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q,
                                   avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table, const int32_t* length,
                                   const int32_t* seq, const int32_t* count, int prefix_pages, unsigned flags, float softmax_scale,
                                   void* o_bf16, float* lse, int32_t* log, void* ws, size_t ws_bytes, void* stream);
AVSA_API size_t avsa_prefix_attn_workspace_bytes(int B, int H, int Hkv, int L, int d, int page, int width, int prefix_pages);

/*
 * (7) Changes of a paged cache.  Lists are device int32 [n]; a negative entry is left out, a list names no sequence twice
 * (a second time is left out and sets AVSA_ERR_BAD_TABLE; for avsa_cache_free it is empty by then).  Free pages are taken from the lowest on, in the order of the list, and
 * what cannot be had leaves its sequence as it was and sets AVSA_ERR_NO_PAGES.  Every call sees the state before it.
 *
 * avsa_cache_extend   room for count[k] more tokens (>= 0) in sequence seq[k]: new pages where its last one does not
 *                     hold them, length += count[k].
 * avsa_cache_extend_step  the same, and granted[k] (int32 [n], apart from all other arrays; NULL: not wanted) becomes what entry k got: count[k], or 0
                     where it was refused or left out.
 * avsa_cache_write    the last count[k] tokens of sequence seq[k] (seq NULL: k, count NULL: L) from k_new and v_new
 *                     [n,Hkv,L,d], of which they are the first count[k] (0..L), into the pages.  Tokens whose page is missing are left out.
 *                   `count` is what avsa_cache_extend_step granted, wherever it may have refused something: a sequence that was refused has its old
 *                   length, and the count that was asked for would replace its last tokens, which it may share with others.
 * avsa_cache_fork     sequence child[k], which has to be empty, becomes a copy of parent[k]: it shares the pages that are full, and the
 *                     contents of the one that is not are copied to a page of its own, in all planes of `pool`.
 * avsa_cache_free     sequence seq[k] gives its pages back and is empty (all that its row of the table names; `page` is not looked at).
 * avsa_cache_compact  the pages in use become the first n_live[0] ones: the k-th of those behind moves to the k-th free place among them.
 *
 * avsa_cache_fork_step, avsa_cache_free_step, avsa_cache_compact_step  the same with a log.
 *
 * All need the workspace but avsa_cache_write, which has none and no status record.
 *
 * `log` of the *_step calls (int32 [4], apart from all other arrays; NULL: none) is a record that no call clears: code, where, item and aux of the first error since
 * the caller set its code to 0.  A status record holds the last call's alone; a log may be one for many calls, replays of a graph among them.
 */
AVSA_API int avsa_cache_extend(avsa_cache c, const int32_t* seq, const int32_t* count, int n, void* ws, size_t ws_bytes, void* stream);
AVSA_API int avsa_cache_extend_step(avsa_cache c, const int32_t* seq, const int32_t* count, int n, int32_t* granted, int32_t* log, void* ws,
                                    size_t ws_bytes, void* stream);
AVSA_API int avsa_cache_write(int n, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d k_new,
                              avsa_bf16_4d v_new, avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table,
                              const int32_t* length, const int32_t* seq, const int32_t* count, void* stream);
AVSA_API int avsa_cache_fork(avsa_cache c, avsa_pages pool, const int32_t* parent, const int32_t* child, int n, void* ws, size_t ws_bytes,
                             void* stream);
AVSA_API int avsa_cache_free(avsa_cache c, const int32_t* seq, int n, void* ws, size_t ws_bytes, void* stream);
AVSA_API int avsa_cache_compact(avsa_cache c, avsa_pages pool, int32_t* n_live, void* ws, size_t ws_bytes, void* stream);
AVSA_API int avsa_cache_fork_step(avsa_cache c, avsa_pages pool, const int32_t* parent, const int32_t* child, int n, int32_t* log, void* ws,
                                  size_t ws_bytes, void* stream);
AVSA_API int avsa_cache_free_step(avsa_cache c, const int32_t* seq, int n, int32_t* log, void* ws, size_t ws_bytes, void* stream);
AVSA_API int avsa_cache_compact_step(avsa_cache c, avsa_pages pool, int32_t* n_live, int32_t* log, void* ws, size_t ws_bytes, void* stream);
AVSA_API size_t avsa_cache_workspace_bytes(int seqs, int pages, int n);

/*
 * (8) A paged cache held in 4 bits: the same table, length, ref and list calls (avsa_cache_extend, _fork, _free, _compact with page_bytes of such pages), and these
 * in the places of avsa_cache_write and avsa_prefix_attn_step.  Arguments that have their names mean what they mean there.
 *
 * avsa_cache_write_q4 quantises the new tokens into the pages.  A list names no sequence twice.
 * avsa_cache_read_q4  the last count[k] tokens of sequence seq[k] (count NULL: T of them) become the first count[k] (0..T) tokens of k and v [n,Hkv,T,d], exactly.
 *                     Tokens that there are not (behind count[k], in front of the sequence's first, without a page) are zeros.
 * avsa_prefix_attn_q4 attention on the values that the pages stand for.  Where many query rows read the same keys (more than 6 x 128 of a sequence and key head, or
 *                     stacked ones) the pages that the batch reads are first made bf16 in the workspace, which then has room for these: as many as the
 *                     rows can name, N = prefix_pages + B * (width - prefix_pages), or all that the pool has where these are fewer (2 * Hkv * page * d of bf16 each).
 *                     The query's answer grows with its `pages`; a call needs no more than for min(pages, N) of them.  It may be the same workspace for all layers.
 *                     The shared pages are then read by the longest sequence's row, as where they are stacked.
 *
 * Neither a write nor a read needs a workspace or leaves a status.
 */
AVSA_API int avsa_cache_write_q4(int n, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d k_new, avsa_bf16_4d v_new,
                                 avsa_q4_pool k_pool, avsa_q4_pool v_pool, const int32_t* table, const int32_t* length, const int32_t* seq,
                                 const int32_t* count, void* stream);
AVSA_API int avsa_cache_read_q4(int n, int Hkv, int T, int d, int page, int pages, int seqs, int width, avsa_q4_pool k_pool, avsa_q4_pool v_pool,
                                const int32_t* table, const int32_t* length, const int32_t* seq, const int32_t* count, avsa_bf16_4d k, avsa_bf16_4d v,
                                void* stream);
AVSA_API int avsa_prefix_attn_q4(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q, avsa_q4_pool k_pool,
                                 avsa_q4_pool v_pool, const int32_t* table, const int32_t* length, const int32_t* seq, const int32_t* count,
                                 int prefix_pages, unsigned flags, float softmax_scale, void* o_bf16, float* lse, int32_t* log, void* ws,
                                 size_t ws_bytes, void* stream);
AVSA_API size_t avsa_prefix_attn_q4_workspace_bytes(int B, int H, int Hkv, int L, int d, int page, int pages, int width, int prefix_pages);

/*
 * (9) Rotary positions with several axes (time, height, width): pair i of a head's channels turns by the angle 2 pi * pos[b,n,axis] * freq[i],
 *
 *   (y_a, y_b) = (x_a cos - x_b sin, x_a sin + x_b cos)
 *
 * for the queries q [B,H,N,d] and keys k [B,Hk,N,d] of the same tokens in one call (H or Hk 0: not there, its pointers are not looked at).
 *   pos       int32 [B,N,axes], contiguous but for the distance pos_stride_b of batch entries (in elements; 0: all have the same)
 *   sections  host int [axes]: channel pairs of each axis, d/2 in all; pair i belongs to the axis whose section it falls in
 *   freq      fp64 [d/2], 8-byte aligned: turns of each pair for a step along its axis (base^(-2i/n) / (2 pi) for the i-th of an axis of n channels; 0: never turned)
 * An output is its input (in place, same strides) or overlaps none.  d is 64 or 128, and neither needs a workspace or leaves a status.
 */
AVSA_API int avsa_rope(int B, int H, int Hk, int N, int d, avsa_bf16_4d q, avsa_bf16_4d k, avsa_bf16_4d q_out, avsa_bf16_4d k_out, const int32_t* pos,
                       int64_t pos_stride_b, int axes, const int* sections, const double* freq, unsigned flags, void* stream);

/* Host integer ceil(pct/100 * n): the count forms of rho and kappa (Eq. 8's ceiling). */
AVSA_API int avsa_count_from_percent(int pct, int n);

/* Synchronises `stream`, copies the status record of `ws` to the host and returns its code
 * (AVSA_OK, AVSA_ERR_TIMEOUT, AVSA_ERR_BAD_MASK, AVSA_ERR_BAD_TABLE or AVSA_ERR_NO_PAGES).  detail (host, optional) receives 3 ints that
 * say where the check failed.  For tests and debugging; the hot path never calls it. */
AVSA_API int avsa_read_status(const void* ws, void* stream, int* detail);

/* Self-test of the device-side time limit (tests only): enqueues one warp that waits on a barrier nothing
 * ever signals, gives up after `limit_cycles` SM clock cycles (0 .. 2e9, i.e. about a second at most), records
 * AVSA_ERR_TIMEOUT in the status record at `ws` (>= AVSA_STATUS_BYTES; detail = {99, 0, cycles waited / 1024})
 * and returns; the context stays usable.  The tile kernels bound every one of their waits the same way. */
AVSA_API int avsa_selftest_bounded_wait(void* ws, size_t ws_bytes, long long limit_cycles, void* stream);

AVSA_API const char* avsa_status_string(int status);
AVSA_API int avsa_version(void);

#ifdef __cplusplus
}
#endif
#endif /* AVSA_H_ */
