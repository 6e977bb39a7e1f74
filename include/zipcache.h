/*
 * zipcache.h - C ABI of the MI355X (gfx950) implementation of ZipCache's
 * data-parallel hot path (arXiv 2405.14256).
 *
 * Four operations, in the order Algorithm 2 (prefill) and Algorithm 3 (decode)
 * use them (and, beside them, the prefill attention of Algorithm 2 itself,
 * zc_prefill_attention, whose row normalisers feed the first):
 *
 *   zc_probe_saliency    Eq. 9 + Eq. 8: normalized attention score of every
 *                        key token from a probe subset of query rows.
 *   zc_select_salient    Algorithm 2 "Split": the k most salient tokens.
 *   zc_quantize_pack     Eq. 5, Eq. 6, Algorithm 1: channelwise or
 *                        channel-separable tokenwise quantization of the
 *                        salient subset at bits_hi and of the rest at bits_lo,
 *                        bit-packed into the cache arenas as a new chunk.
 *   zc_decode_attention  Eq. 4 over the packed cache (de-quantized on the
 *                        fly) plus a full-precision tail of recent tokens.
 *
 * General rules
 *   - Every pointer marked "device" is GPU memory owned by the caller; every
 *     other pointer is host memory.  The library allocates nothing, keeps no
 *     pointer after a call returns and has no global mutable state (apart from
 *     a cached copy of the device's compute-unit count and, for
 *     zc_decode_attention_static, its per-device scratch buffer).
 *   - All work is enqueued on the given HIP stream (`stream` is a hipStream_t
 *     passed as void*; NULL is the default stream).  Calls never synchronise
 *     with the host and never read results back.
 *   - A call may be several launches.  Calls that share a workspace (or the buffer of
 *     zc_decode_attention_static) on one stream must therefore be issued one after the other:
 *     host threads that share a stream need a lock around them, or workspaces of their own.
 *   - Every function returns a zc_status.  Arguments are validated on the host
 *     before anything is launched; a failed validation launches nothing and
 *     leaves outputs untouched.  A launch failure returns ZC_ERR_HIP.
 *   - Device pointers must be 16-byte aligned; tensors must have unit stride
 *     along the last (channel) axis and all other strides multiples of 8
 *     elements.
 *   - Supported: head dimension D in {64, 128}; dtypes f32, f16, bf16;
 *     code widths in {2, 4, 8}; Hq a multiple of Hkv with Hq/Hkv <= 8.
 *   - HIP graph capture.  Every call may be captured (nothing synchronises or
 *     allocates).  The state of a zc_packed on the host - slots in use, number of
 *     chunks, the mirror of the chunk table - is read when a call is *issued* and
 *     travels in the kernel arguments: a captured zc_decode_attention replays over the
 *     chunks the cache had at capture time, a captured zc_quantize_pack appends at the
 *     slots it was captured for.  A graph therefore has to be captured in the order its
 *     calls will run and replayed as a whole sequence from the same starting state
 *     (after the host fields have been reset to what they were when capture began);
 *     the library cannot check this.
 *   - Value ranges (not checked: the data lives on the device).  All inputs must be
 *     finite - no NaN, no infinity (the quantizer takes minima and maxima without
 *     regard to NaN; a channel of nothing but NaN has NaN for its channelwise parameters).  zc_decode_attention feeds the matrix cores fp16 operands:
 *     every |q[c] * chan_scale[c] * sm_scale| of the keys' channel scales must stay
 *     below 700 and every token scale of the values below 1000 (an fp16 overflow
 *     there turns the output into NaN); activations of the models the paper
 *     compresses are orders of magnitude inside these bounds.
 *   - Size limits (beyond them a call returns ZC_ERR_UNSUPPORTED and launches
 *     nothing): B <= 65535 and heads <= 65535; a token row of a cache tensor at
 *     most 8192 channels (W = H*D) in zc_quantize_pack; the kernels address one
 *     (batch, head) slab with 32-bit byte offsets, so the span of such a slab -
 *     L * sL elements of q, (L + 128) * sL of k in the probe calls, tail_len * sL
 *     of the tail, cap * D * bits / 8 bytes of a code arena in the decode call -
 *     must stay below 4 GiB - 4 KiB.
 */
#ifndef ZIPCACHE_H
#define ZIPCACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ZC_OK = 0,
  ZC_ERR_INVALID_ARG = -1, /* null / misaligned pointer, bad size or stride  */
  ZC_ERR_UNSUPPORTED = -2, /* dtype, head dim, bit width, scheme, size limit  */
  ZC_ERR_WORKSPACE = -3,   /* workspace smaller than the call needs: never one of *_workspace() bytes */
  ZC_ERR_CAPACITY = -4,    /* arena or chunk table of a zc_packed is full    */
  ZC_ERR_HIP = -5,         /* the HIP runtime refused a launch               */
  ZC_ERR_STATIC_LIMIT = -6 /* needs more scratch than ZC_STATIC_SCRATCH_BYTES */
} zc_status;

typedef enum { ZC_F32 = 0, ZC_F16 = 1, ZC_BF16 = 2 } zc_dtype;

/* Quantization granularity of one cache tensor.
 *   CHANNEL: one (s, z) of Eq. 5 per channel over the tokens of the subset
 *            (the paper's choice for keys, Section 4.1).
 *   CST:     Algorithm 1 - c_i = sqrt(max|X_i|) per channel (Eq. 6), then one
 *            (s, z) per token over the W = H*D normalized values of its row
 *            (the paper's choice for values).
 *   TOKEN:   CST with c = 1 (plain tokenwise quantization, Table 1 row 3).
 * In every scheme
 *   x_hat[t, w] = chan_scale[w] * tok_scale[t] * (code[t, w] - tok_zero[t] - chan_zero[w])
 * with tok_scale = 1, tok_zero = 0 for CHANNEL and chan_zero = 0 otherwise. */
typedef enum { ZC_SCHEME_CHANNEL = 0, ZC_SCHEME_CST = 1, ZC_SCHEME_TOKEN = 2 } zc_scheme;

/* Bit layout of the codes of one (batch, head) inside an arena.
 *   ROW    (keys): slot-major rows of D codes; code of channel c sits at bit
 *          offset c*bits of its row, little-endian (for 4 bits: channel 2j in
 *          the low nibble of byte j).
 *   TGROUP (values): 32-bit words indexed [block][kg][c], kg in 0..3, c the
 *          channel, each word holding E = 32/bits codes of one channel for E
 *          different slots; a block covers 4*E consecutive slots.  Field e
 *          (bits e*bits .. (e+1)*bits-1) of word [blk][kg][c] belongs to slot
 *             blk*4*E + 16*j(e) + 4*kg + e%4,
 *          j(e) = e/4 for bits in {4, 8};  for bits == 2, j(e) = 0,2,1,3 for
 *          e/4 = 0,1,2,3.
 *          (Keys are contracted over channels and values over tokens, so each
 *          tensor packs along the axis its matrix-core operand runs over.)
 * Both layouts take B*H*cap*D*bits/8 bytes per arena. */
typedef enum { ZC_LAYOUT_ROW = 0, ZC_LAYOUT_TGROUP = 1 } zc_layout;

#define ZC_SLOT_ALIGN 64 /* every chunk starts at a multiple of this many slots */
#define ZC_MAX_GROUP 8   /* largest supported Hq / Hkv                          */

/* A strided 4-D view [B, H, L, D] of device memory; strides in elements,
 * the D axis is contiguous. */
typedef struct zc_tensor4 {
  void* ptr; /* device */
  int32_t dtype; /* zc_dtype */
  int32_t reserved;
  int64_t B, H, L, D;
  int64_t sB, sH, sL;
} zc_tensor4;

/* One tensor (K or V) of the compressed cache.  The struct lives on the host;
 * all arrays are caller-allocated.  Salient tokens go to the "hi" arena at
 * bits_hi, the others to the "lo" arena at bits_lo.  Each zc_quantize_pack
 * call appends one chunk: chunk_table row i = {begin_hi, len_hi, begin_lo,
 * len_lo} in slots.  A chunk has its own channel parameters (one set per
 * subset); slot r of the hi part of chunk i is slot begin_hi + r of the hi
 * arena for the codes, the token parameters and the positions alike.  The K
 * and V structs of one cache must be filled by the same sequence of calls so
 * that their chunk tables agree. */
typedef struct zc_packed {
  int32_t layout;  /* zc_layout */
  int32_t scheme;  /* zc_scheme */
  int32_t bits_hi, bits_lo;
  int64_t B, H, D;          /* W = H*D channels per token row */
  int64_t cap_hi, cap_lo;   /* slots per arena, multiples of ZC_SLOT_ALIGN */
  int64_t n_hi, n_lo;       /* slots in use (aligned end of the last chunk) */
  uint8_t* codes_hi;        /* device, B*H*cap_hi*D*bits_hi/8 bytes */
  uint8_t* codes_lo;        /* device */
  float* tok_scale_hi;      /* device [B, cap_hi]; unused for CHANNEL (may be NULL) */
  float* tok_zero_hi;
  float* tok_scale_lo;      /* device [B, cap_lo] */
  float* tok_zero_lo;
  int32_t* pos_hi;          /* device [B, cap_hi] original token positions, or NULL */
  int32_t* pos_lo;          /* device [B, cap_lo], or NULL */
  float* chan_scale;        /* device [max_chunks, 2 (hi, lo), B, W] */
  float* chan_zero;         /* device [max_chunks, 2, B, W] */
  int32_t* chunk_table;     /* device [max_chunks, 4] */
  int32_t* chunk_table_host; /* host   [max_chunks, 4], kept equal to the above */
  int32_t n_chunks, max_chunks;
} zc_packed;

/* ---- Eq. 9 + Eq. 8 ------------------------------------------------------
 * q [B, Hq, Lq, D], k [B, Hkv, Lk, D], same dtype.  Probe p uses query row
 * probe_rows[p] of q (probe_pos[p] when probe_rows is NULL) and attends key
 * columns i <= probe_pos[p]; probe_pos must be ascending (device int32 [P],
 * values in [0, Lk)).  Logits are q.k * sm_scale (sm_scale == 0 means
 * 1/sqrt(D)); query head h reads KV head h / (Hq/Hkv).
 * With lse_ext == NULL each probe row is soft-maxed over its visible columns.
 * With lse_ext (device float [B, Hq, P], natural log) the probabilities are
 * exp(logit - lse_ext): decode-time probes whose softmax also covered tokens
 * outside k.
 * Output scores (device float [B, Lk]): mean over query heads of
 *   sum_{p : probe_pos[p] >= i} A[p, i] / #{p : probe_pos[p] >= i}
 * (0 where no probe sees column i).  scores_per_head (device float
 * [B, Hq, Lk]) receives the per-head values when not NULL.
 * The result is deterministic: no floating-point atomics are used.
 * A workspace of zc_probe_saliency_workspace() bytes suffices for any call of these sizes.  For
 * P > 64 one that lacks up to 32 * min(B * Hq, 1024) * min(P, 512) of them (rounded up to 256) is
 * taken as well; without lse_ext the partial sums of a row may then be added in another order,
 * so scores are the same bits only for workspaces on the same side of the full size. */
size_t zc_probe_saliency_workspace(int64_t B, int64_t Hq, int64_t Lk, int64_t P);
int zc_probe_saliency(const zc_tensor4* q, const zc_tensor4* k,
                      const int32_t* probe_rows, const int32_t* probe_pos, int32_t P,
                      float sm_scale, const float* lse_ext,
                      float* scores, float* scores_per_head,
                      void* ws, size_t ws_bytes, void* stream);

/* ---- Eq. 7 (the accumulated attention score the paper argues against) ------
 * Same arguments, workspace and error behaviour as zc_probe_saliency; the
 * column sums are NOT divided by the number of probes that see the column:
 *   scores[b, i] = mean over query heads of sum_{p : probe_pos[p] >= i} A[p, i].
 * With all rows as probes this is Eq. 7 itself (earlier tokens accumulate more
 * terms: the bias of Section 4.2); serves as the comparison metric. */
int zc_probe_accumulated(const zc_tensor4* q, const zc_tensor4* k,
                         const int32_t* probe_rows, const int32_t* probe_pos, int32_t P,
                         float sm_scale, const float* lse_ext,
                         float* scores, float* scores_per_head,
                         void* ws, size_t ws_bytes, void* stream);

/* ---- Algorithm 2, the attention line (Eq. 2 applied to V; Appendix B, prefill) -------
 * The attention output of all prompt tokens at once, with the causal mask:
 *   out[b, h, p, :] = sum_{i <= p} softmax_i(q[b,h,p] . k[b,h/G,i] * sm_scale) v[b,h/G,i, :]
 * q, out [B, Hq, L, D]; k, v [B, Hkv, L, D]; all four of one dtype (out may have strides of
 * its own); sm_scale == 0 means 1/sqrt(D).  lse (device float [B, Hq, L], optional)
 * receives the natural-log normaliser of every row.  With P > 0 the normalisers of the
 * rows probe_pos[0..P) (device int32, values in [0, L)) are also gathered into lse_probe
 * (device float [B, Hq, P]; needs lse): exactly the lse_ext argument with which
 * zc_probe_saliency scores the same probe rows in one sweep instead of two.
 * fp32 tensors are multiplied on the fp32 matrix pipes, never rounded to 16 bits; the
 * probabilities of 16-bit tensors enter the second product rounded to the tensors' type.
 * Where heads and rows leave the chip idle a row's keys are shared by waves and their parts
 * joined in fp32: the last bits of a row's output and normaliser may depend on how many
 * heads and rows the call has.  A row has a number for its result whatever its first keys' logits, -inf included, unless all are -inf.
 * Needs no workspace; enqueued on `stream`.
 * Errors: ZC_ERR_INVALID_ARG for mismatching shapes or types, ZC_ERR_UNSUPPORTED for a
 * (batch, head) slab of 4 GiB or more. */
int zc_prefill_attention(const zc_tensor4* q, const zc_tensor4* k, const zc_tensor4* v, float sm_scale,
                         const zc_tensor4* out, float* lse,
                         const int32_t* probe_pos, int32_t P, float* lse_probe, void* stream);

/* ---- Algorithm 2, Split(., p~, r%) ------------------------------------------
 * scores: device float [B, L] (must not contain NaN).  For every batch row
 * the k largest scores are salient; among equal scores the lower index wins.
 * salient_idx (device int32 [B, k]) and regular_idx (device int32 [B, L-k])
 * are both ascending; mask (device uint8 [B, L], optional) is 1 for salient.
 * 0 <= k <= L.  Exact and deterministic. */
size_t zc_select_salient_workspace(int64_t B, int64_t L);
int zc_select_salient(const float* scores, int64_t B, int64_t L, int64_t k,
                      int32_t* salient_idx, int32_t* regular_idx, uint8_t* mask,
                      void* ws, size_t ws_bytes, void* stream);

/* ---- Eq. 5, Eq. 6, Algorithm 1; the four quantizer calls of Algorithm 2 -----
 * x [B, H, L, D] is one cache tensor.  Tokens salient_idx[b, 0..k) are
 * quantized at out->bits_hi, tokens regular_idx[b, 0..n_reg) at out->bits_lo,
 * each subset with its own channel statistics, by out->scheme, rounding half
 * to even; s := 1 when max == min, c := 1 when the channel is all zero.  An
 * empty subset gets chan_scale = 1, chan_zero = 0.  The codes are appended as
 * chunk out->n_chunks in out->layout; positions idx + pos_offset are stored
 * when pos arrays are present.  On success the host fields n_hi, n_lo,
 * n_chunks and chunk_table_host are updated (the device copy is written by
 * the enqueued work).  Index lists must hold distinct values in [0, L). */
size_t zc_quantize_pack_workspace(int64_t B, int64_t H, int64_t L /* tokens per call, k + n_reg */, int64_t D);
int zc_quantize_pack(const zc_tensor4* x, const int32_t* salient_idx, int64_t k,
                     const int32_t* regular_idx, int64_t n_reg, int64_t pos_offset,
                     zc_packed* out, void* ws, size_t ws_bytes, void* stream);

/* ---- the four quantizer calls of Algorithm 2 at once ------------------------------------
 * Keys and values of one cache compressed by the same launches: exactly what two
 * zc_quantize_pack calls (xk into outK, then xv into outV, same index lists and offset)
 * leave behind, bit for bit, in half the launches or fewer (two, when outK is CHANNEL / ROW, outV is
 * CST / TGROUP and a token row has at most 2048 channels or the keys' tokens fit the registers of
 * one sweep; three at most otherwise; one more where long subsets of few channels go by token
 * ranges).  xk and xv
 * must agree in shape and dtype; outK and outV are two different descriptors.  Workspace:
 * zc_quantize_pack_kv_workspace(B, H, k + n_reg, D).  Errors as for zc_quantize_pack; when
 * one is returned neither descriptor has been changed. */
size_t zc_quantize_pack_kv_workspace(int64_t B, int64_t H, int64_t L, int64_t D);
int zc_quantize_pack_kv(const zc_tensor4* xk, const zc_tensor4* xv, const int32_t* salient_idx, int64_t k,
                        const int32_t* regular_idx, int64_t n_reg, int64_t pos_offset,
                        zc_packed* outK, zc_packed* outV, void* ws, size_t ws_bytes, void* stream);

/* ---- Eq. 4 over the packed cache (Algorithm 3, attention line) -------------------
 * q [B, Hq, 1, D]; Kp (ROW layout) and Vp (TGROUP layout) hold the same
 * chunks; tail_k / tail_v [B, Hkv, >=tail_len, D] are the full-precision
 * recent tokens (same dtype as q; may be NULL when tail_len == 0).
 * out (device, q's dtype, [B, Hq, D]) = softmax(q.K^T * sm_scale) V over all
 * packed tokens and the first tail_len tail tokens; lse_out (device float
 * [B, Hq], optional) receives the natural-log normaliser of each row.
 * Deterministic for fixed shapes.  Calls that share a workspace must not run
 * concurrently. */
size_t zc_decode_attention_workspace(int64_t B, int64_t Hq, int64_t D);
int zc_decode_attention(const zc_tensor4* q, const zc_packed* Kp, const zc_packed* Vp,
                        const zc_tensor4* tail_k, const zc_tensor4* tail_v, int64_t tail_len,
                        float sm_scale, void* out, float* lse_out,
                        void* ws, size_t ws_bytes, void* stream);

/* ---- groupwise quantization: the baseline granularity of Table 1 / Appendix A (Eq. A) -----
 * Every `group` (8, 16, 32, 64 or 128; the paper's n = 32) consecutive channels of a token
 * row w = h*D + c share one (s, z) of Eq. 5 (s := 1 when the group is constant; round half to
 * even).  x [B, H, L, D]; the n token rows idx[b, 0..n) (device int32, or NULL for rows 0..n-1)
 * are quantized at `bits` (2, 4 or 8).  A comparator, not a cache format: outputs are
 * token-major and unpacked, each optional - codes_out device uint8 [B, n, W], scale_out /
 * zero_out device float [B, n, W / group], dequant_out device float [B, n, W] =
 * (code - z) * s.  Needs no workspace. */
int zc_group_quantize(const zc_tensor4* x, const int32_t* idx, int64_t n, int32_t bits, int32_t group,
                      uint8_t* codes_out, float* scale_out, float* zero_out, float* dequant_out, void* stream);

/* ---- Algorithm 3 with its re-compression branch taken at its word ----------------------
 * ("Extract K[:-100] and V[:-100] and adaptively compress them with A_probe": every 100
 * steps everything but the newest 100 tokens is compressed again as a whole, ranked by the
 * explicit attention rows of the window's probe steps.)  Three building blocks; together
 * with zc_select_salient and zc_quantize_pack into a fresh zc_packed they make that branch.
 *
 * zc_decode_probs: the attention row a of one decode step (Eq. 4's probabilities; the
 * "Compute attention scores a of current token" line), in token order:
 *   probs_out[b, h, pos] = exp(q[b,h] . k_hat[b, h/G, pos] * sm_scale - lse[b, h])
 * over every token of Kp (at its stored position: Kp needs its pos arrays) and the first
 * tail_len rows of tail_k (token tail_pos0 + t).  lse (device float [B, Hq]) is the
 * normaliser zc_decode_attention returned for the same step; probs_out is device float
 * [B, Hq, N], N >= tail_pos0 + tail_len, and entries of positions the cache does not hold
 * are left untouched.  Arguments as for zc_decode_attention otherwise.
 *
 * zc_rows_saliency: Eq. 8 on explicit rows.  rows is device float [P, B, Hq, row_stride]
 * (row j valid for tokens i < row_len[j]; row_len device int32 [P]):
 *   scores[b, i] = mean over heads of sum_{j : row_len[j] > i} rows[j, b, h, i] / #{j : row_len[j] > i}
 * for i < n_out (scores: device float [B, n_out]; 0 where no row sees the token; without the
 * division when normalize == 0: Eq. 7).  Deterministic (fixed summation order).
 *
 * zc_dequantize_cache: out[b, h, pos, :] = x_hat of every token of p (all chunks), rounded to
 * out's dtype, at its stored position (p needs its pos arrays; positions >= out->L are
 * skipped).  out [B, H, L', D] is typically the caller's full-precision token buffer, whose
 * rows pos >= (tokens in p) already hold the tokens not compressed yet. */
int zc_decode_probs(const zc_tensor4* q, const zc_packed* Kp, const zc_tensor4* tail_k, int64_t tail_len,
                    int64_t tail_pos0, float sm_scale, const float* lse, float* probs_out, int64_t N, void* stream);
int zc_rows_saliency(const float* rows, const int32_t* row_len, int32_t P, int64_t B, int64_t Hq,
                     int64_t row_stride, int64_t n_out, int32_t normalize, float* scores, void* stream);
int zc_dequantize_cache(const zc_packed* p, const zc_tensor4* out, void* stream);

/* ---- zc_decode_attention for callers that cannot allocate ----------------------------
 * For code under HIP graph capture, tight serving loops and harnesses that forbid
 * hipMalloc: the same operation, arguments, kernels and results as zc_decode_attention,
 * without a workspace argument.  The partial results of the split-K workgroups go to a
 * buffer of ZC_STATIC_SCRATCH_BYTES that lives in the library's own device image (one
 * copy per GPU, held until the process ends); the call allocates and frees nothing.
 * Limit: zc_decode_attention_workspace(B, Hq, D) must not exceed ZC_STATIC_SCRATCH_BYTES
 * (B*Hq <= 1790 query heads at D = 128 is always within it), else the call returns
 * ZC_ERR_STATIC_LIMIT and launches nothing.  All calls on one GPU share that buffer: two
 * calls that may overlap on the same GPU (different streams) race; calls on one stream,
 * or ordered by events, are safe.  Nothing in the buffer has to start at zero: every
 * partial a call reads was written by that call. */
#define ZC_STATIC_SCRATCH_BYTES (8u << 20)
int zc_decode_attention_static(const zc_tensor4* q, const zc_packed* Kp, const zc_packed* Vp,
                               const zc_tensor4* tail_k, const zc_tensor4* tail_v, int64_t tail_len,
                               float sm_scale, void* out, float* lse_out, void* stream);

/* ---- a paged full-precision cache: requests before (or without) their compression -----------
 * Keys and values of many requests lie in pages of two pools (one for keys, one for values):
 * k_pages, v_pages [N, Hkv, page, D], `page` token rows to a page, a power of two from
 * ZC_PAGE_MIN to ZC_PAGE_MAX, any strides (a page may hold its heads one after the other or its
 * tokens; a head's rows of one page span less than 2 GB, pages lie less than 4 GB apart).
 * N * page must stay below 2^31, the heads below 65536.  Request r's block table is row r
 * of block_table (device int32 [R, max_blocks], rows row_stride elements apart): entry c is the page
 * of its tokens c * page .. c * page + page - 1.  A step's new tokens lie request after request in
 * tensors of T rows, q_start[r] .. q_start[r + 1] - 1 (device int32 [R + 1]) those of request r;
 * kv_len[r] (device int32 [R]) counts all its tokens, the new ones, its last, included.  T may be
 * larger than q_start[R] (calls captured for the largest step): rows behind the last request are
 * neither read nor written.  R and T may be 0.  What is written must not overlap itself - out, the tensors
 * that zc_paged_load fills, the pools that zc_paged_store fills: the stride of an axis of more than one
 * element is at least what the axes of smaller strides span; what is only read may have any.  Unlike elsewhere, memory that no token of a call
 * lies in or sees - slots past kv_len, pages behind every window, rows behind the last request -
 * may hold anything, NaN included; the values of a request's tokens must be finite.
 *
 * zc_paged_tables: one step's bookkeeping from the requests' lengths.  Request r has kv_len[r] tokens
 * of which q_len[r] are new (0 <= q_len <= kv_len; values outside are taken for the nearest inside), so
 * it holds ceil((kv_len - q_len) / page) pages, whose entries are read, and needs ceil(kv_len / page):
 * the missing ones are taken from the end of free_pages (device int32 [n_list], of which the first
 * *n_free are free; n_free is device memory, NULL for all) - in the order of the requests, a request's in
 * the order of its blocks, the first is free_pages[*n_free - 1] - and written to block_table.
 * Outputs: q_start; slot_map (device int32 [T]), page * page_rows + row of every new token, -1 for rows
 * behind the last request; *n_taken, the number of pages the requests needed: where it is more than
 * *n_free, the entries without a page are -1 and so are their tokens' slots, and the caller has to find pages
 * and repeat the step.  Entries a request does not need are left as they are.  Tokens past T, and
 * blocks past max_blocks, get no slot and no entry.  free_pages and n_free are not changed: subtract
 * *n_taken from *n_free before the next step, on the device if need be.  The new tokens of all
 * requests and the pages they need must number less than 2^31 each.
 * A finished request's pages go back by writing its row's first ceil(kv_len / page) entries to free_pages behind the
 * first *n_free and adding their number to *n_free (n_list must have room), in the order of the stream with the calls that read the pages.
 *
 * zc_paged_store: k, v [1, Hkv, T, D] (any strides) to the slots of their tokens; a token whose slot is
 * outside [0, N * page) is left out.  Of tokens with one slot every 16 bytes of the
 * slot's rows are one token's, and not of all the same token's: zc_paged_tables gives no slot twice.
 *
 * zc_paged_load: k[r, h, i, :] and v[r, h, i, :] = token i of request r, for i < min(kv_len[r], k->L,
 * max_blocks * page); other rows are left as they are.  k, v [R, Hkv, L, D]: what zc_probe_saliency and
 * zc_quantize_pack_kv take.  R <= 32767, L <= 2^28 (fp32 of 128 channels: 16 fewer).
 *
 * A block-table entry that is no page (negative, N or more) reads as rows of zeros.  Nothing here needs a workspace.  Errors as elsewhere; a page size that is not
 * supported is ZC_ERR_UNSUPPORTED. */
#define ZC_PAGE_MIN 16
#define ZC_PAGE_MAX 65536
int zc_paged_tables(const int32_t* q_len, const int32_t* kv_len, int64_t R, int32_t* block_table, int64_t row_stride,
                    int64_t max_blocks, const int32_t* free_pages, int64_t n_list, const int32_t* n_free, int64_t page,
                    int32_t* q_start, int32_t* slot_map, int64_t T, int32_t* n_taken, void* stream);
int zc_paged_store(const zc_tensor4* k, const zc_tensor4* v, const int32_t* slot_map, const zc_tensor4* k_pages,
                   const zc_tensor4* v_pages, void* stream);
int zc_paged_load(const zc_tensor4* k_pages, const zc_tensor4* v_pages, const int32_t* block_table, int64_t row_stride,
                  int64_t max_blocks, const int32_t* kv_len, const zc_tensor4* k, const zc_tensor4* v, void* stream);

/* ---- Eq. 2 / Eq. 4 over the pages: a step's new tokens, one a request or many ------------------
 * Row j of request r's nq = q_start[r + 1] - q_start[r] new tokens stands at position
 * pos = kv_len[r] - nq + j (its keys and values are in the pages already) and sees the tokens i <= pos,
 * with window > 0 only those with i > pos - window or i < sinks:
 *   out[h, t, :] = sum_i softmax_i(q[h, t] . k[h/G, i] * sm_scale) v[h/G, i, :]
 * q, out [1, Hq, T, D] of the pools' type, Hq / Hkv whole and at most 4096; sm_scale == 0 means
 * 1/sqrt(D); a negative one is refused, and one above 2.35e38 (its product with log2(e) is no finite float).  lse (device float [Hq, T], optional) receives the natural-log
 * normalisers (for zc_probe_saliency's lse_ext).  A row that sees no token (kv_len < nq), or only logits of
 * -inf, has zeros for its output and -inf for its normaliser.  A request may have no new tokens.
 * fp32 tensors are multiplied on the fp32 matrix pipes; the probabilities of 16-bit tensors enter the
 * second product rounded to the tensors' type.  Deterministic for equal lengths and shapes; a row's last bits may
 * depend on the other requests (long rows are split by what the whole call has to do, and joined in fp32).
 * Workspace: zc_paged_attention_workspace() bytes, 16-byte aligned, with any contents; calls that share one
 * must not run concurrently.  It is what the finest split of R requests and T rows takes, whether this call is split or not: up to
 * 280 MB of 128 channels (32 heads over 8: one token 9 MB, 64 requests of one 90, a chunk of 2048 206), none where R or T are too large
 * for a split.  q_start must ascend within [0, T], kv_len be 0 to max_blocks * page (values outside are
 * taken for the nearest).
 * The host knows neither q_start nor kv_len; how rows are split, and whether at all, follows from R, T, the heads, the window and the room
 * of a table's row, max_blocks * page.  So a table much wider than its requests costs time (one token each of 12 requests of 1024
 * tokens 12.5 us in 16 columns of 64 tokens, 16.0 in 64 or 256): pass as many columns as the longest request needs, where the caller knows
 * it, with the row stride of the whole table.  A step of so many rows that their blocks fill the chip is not split, whatever its
 * lengths: of single tokens with 32 heads over 8 from 113 requests on (109 of 500 tokens and one of 32768 76 us, 113 and one 315); and
 * where T * Hq / Hkv is more than 64 R it is T that counts, not q_start[R]: one token over 32768 in a step captured for T = 1000
 * 29 us, for T = 5120 251.
 * Limits: R < 2^24, T * Hq < 2^31; a step has at most 2^24 - 1 blocks of all heads, units of split ones among them: T * Hq / 128 (fp32: / 32) + 2 min(R, T) Hkv
 * + Hkv + 2560 below 2^24 is always enough. */
size_t zc_paged_attention_workspace(int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int64_t D);
int zc_paged_attention(const zc_tensor4* q, const zc_tensor4* k_pages, const zc_tensor4* v_pages, const int32_t* block_table,
                       int64_t row_stride, int64_t max_blocks, const int32_t* q_start, const int32_t* kv_len, int64_t R,
                       int32_t window, int32_t sinks, float sm_scale, const zc_tensor4* out, float* lse,
                       void* ws, size_t ws_bytes, void* stream);

/* ---- attention of a step's new tokens where groups of requests share a prefix ---------------------
 * Prefix g's prefix_len[g] tokens (device int32 [P]) lie in the pages of row g of prefix_table (device int32 [P, prefix_max_blocks], rows
 * prefix_row_stride elements apart), in the same pools and stored once.  Requests group_start[g] .. group_start[g + 1] - 1 (device int32 [P + 1],
 * ascending within [0, R]) begin with it; those in front of group_start[0] and from group_start[P] on have none.  block_table, kv_len and q_start are, as in
 * zc_paged_attention, of the requests' own tokens, which follow the prefix: a new token sees its whole prefix and its request's own tokens
 * up to itself,
 *   out[h, t, :] = sum_i softmax_i(q[h, t] . k[h/G, i] * sm_scale) v[h/G, i, :]   over i in both,
 * and lse is the normaliser of both (zc_paged_scores takes it for the own tokens as it is).  The rows of requests with up to 64 of them
 * (new tokens times Hq / Hkv) go through their prefix together, so that a key of it is read and multiplied once for all; a longer chunk fills
 * blocks of its own.  There is no sliding window here: where one is wanted, put the prefix's pages into every request's own row.
 * prefix_len outside [0, prefix_max_blocks * page] is taken for the nearest; pages that are none read as zeros.  A row that sees nothing has zeros for its
 * output and -inf for its normaliser.  Types, shapes, strides, sm_scale and rounding as in zc_paged_attention; deterministic for equal lengths and
 * shapes; a row's last bits may depend on the other requests.  P, R and T may be 0; P <= 1024, R < 2^24, T * Hq < 2^31; T * Hq / 64 (fp32: / 16) +
 * 6 min(R, T) Hkv + 512 below 2^24 is always enough for the blocks of a step.  Workspace: zc_paged_shared_attention_workspace() bytes, 16-byte aligned, with any contents; calls that share one must
 * not run concurrently. */
size_t zc_paged_shared_attention_workspace(int64_t P, int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int64_t D);
int zc_paged_shared_attention(const zc_tensor4* q, const zc_tensor4* k_pages, const zc_tensor4* v_pages, const int32_t* prefix_table,
                              int64_t prefix_row_stride, int64_t prefix_max_blocks, const int32_t* prefix_len, const int32_t* group_start, int64_t P,
                              const int32_t* block_table, int64_t row_stride, int64_t max_blocks, const int32_t* q_start, const int32_t* kv_len,
                              int64_t R, float sm_scale, const zc_tensor4* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* ---- the weight that cached tokens gather (Eq. 7 over the pages, step by step) --------------------
 * For every request with new tokens, every KV head h and every token i < kv_len[r] of it
 *   scores[h, i] = (i < kv_len[r] - nq ? decay * scores[h, i] : 0) + sum over rows (new token, query head of h) that see i of exp(logit - lse[row])
 * at the token's place in the pages: scores is device float [N, Hkv, page], 16-byte aligned.  A step's new tokens start from 0,
 * whatever their places held, so nothing has to be cleared when a page is taken.  Other places are left as they are, a request's without new tokens too.
 * q, q_start, kv_len, window, sinks, sm_scale and the rows' positions as in zc_paged_attention, lse (device float [Hq, T]) as it returns
 * it, or zc_paged_shared_attention, whose softmax also went over a prefix (whose own tokens gather nothing here: they are in no row of
 * block_table).  A row of lse = -inf weighs nothing (if its logits are below infinity).  decay is 0 (what was there is not read) to 1: without one, tokens that more
 * rows saw have gathered more.  fp32 tensors are multiplied on the fp32 matrix pipes; weights and sums are fp32.  A token's score is
 * of its own request's rows only.  Deterministic for equal lengths and shapes; its last bits may depend on the step's other requests, R and
 * T, by which the work is divided, so of nearly equal scores another batch may rank others first.  A request's pages must be
 * its own (not another's, not twice in its row); a token without a page has no score.
 * T and R may be 0.  Needs no workspace.  R < 2^24, T * Hq < 2^31, Hq / Hkv <= 4096. */
int zc_paged_scores(const zc_tensor4* q, const zc_tensor4* k_pages, const int32_t* block_table, int64_t row_stride, int64_t max_blocks,
                    const int32_t* q_start, const int32_t* kv_len, int64_t R, int32_t window, int32_t sinks, float sm_scale,
                    const float* lse, float decay, float* scores, void* stream);

/* ---- eviction by gathered weight -----------------------------------------------------------------
 * Request r keeps min(kv_len[r], keep[r], most) of its kv_len[r] tokens (keep: device int32 [R], negative: 0; most: what the
 * host knows of it): the `recent` newest; of what is left the `sinks` first; of the others those of the largest scores,
 * every KV head its own, and of equal ones the first.  Where recent is more than a request keeps its newest tokens stay, and where sinks
 * is more than what is then left the first of them.  scores (device float [N, Hkv, page], 16-byte aligned) has a token's score at its
 * place in the pages; of NaN any may stay.  With `together` (not 0) all heads keep the same tokens, by the sum of their scores
 * (of 64 bits, rounded once).
 * What stays moves, in its order, to the first places of the request's pages: keys, values and scores; what lies behind it is left as it
 * was.  A place is not the token's position any more: windows and sinks of later calls count what is left.  new_len (device int32 [R], no memory of kv_len or keep) receives the numbers, kept (device int32 [R, Hkv, most], [R, 1, most]
 * with `together`) the places that the tokens had, ascending; entries behind them are left as they were.
 * Pages that a request then does not need, entries ceil(new_len / page) to ceil(kv_len / page) - 1 of its row, are written to free_pages
 * (device int32 [n_list]) from *n_free on (device int32), request after request, what passes the list's end left out; *n_freed
 * (device int32, may be NULL, not n_free itself) is their number.  As in zc_paged_tables *n_free is not changed: add *n_freed to it, in the order of the stream.  block_table is
 * not changed.  free_pages may be NULL.
 * A request's pages must be its own: not another's, not twice in its row.  A token whose entry is no page has a score of 0 and zeros for
 * its rows, a place without a page takes nothing, and among the pages that are left such an entry is written like any other: evict with the lengths
 * that zc_paged_tables found pages for.  kv_len outside [0, max_blocks * page] is taken for the nearest.
 * Deterministic.  R may be 0; R and 3 Hkv <= 65535.  Workspace: zc_paged_evict_workspace() bytes, 16-byte aligned, with any contents (4 for every
 * list, with `together` 4 for every place of every row of the table too); calls that share one must not run concurrently. */
size_t zc_paged_evict_workspace(int64_t R, int64_t Hkv, int64_t max_blocks, int64_t page, int32_t together);
int zc_paged_evict(const zc_tensor4* k_pages, const zc_tensor4* v_pages, float* scores, const int32_t* block_table, int64_t row_stride,
                   int64_t max_blocks, const int32_t* kv_len, const int32_t* keep, int64_t R, int64_t most, int32_t sinks, int32_t recent,
                   int32_t together, int32_t* new_len, int32_t* kept, int32_t* free_pages, int64_t n_list, const int32_t* n_free,
                   int32_t* n_freed, void* ws, size_t ws_bytes, void* stream);

/* ---- helpers ------------------------------------------------------------------ */
/* Bytes of one code arena of `cap` slots. */
size_t zc_arena_bytes(int64_t B, int64_t H, int64_t D, int64_t cap, int32_t bits);
/* Smallest legal capacity that holds `n_chunks` chunks totalling n tokens. */
int64_t zc_arena_slots(int64_t n_tokens, int64_t n_chunks);
/* ---- inverse of the packing (Eq. 5's de-quantization; the bit layouts above) ----
 * Unpacks subset `which` (0: hi / salient, 1: lo / regular) of chunk `chunk` of
 * a packed tensor into canonical token-major arrays: element [b, r, w] belongs
 * to slot r of that chunk's subset (ascending original position) and channel
 * w = h*D + c.  codes_out (device uint8 [B, len, W], one byte per code) and
 * dequant_out (device float [B, len, W], x_hat of the formula at zc_scheme) may
 * each be NULL.  len is the subset's length in the chunk table (host mirror).
 * Nothing is allocated; the work is enqueued on `stream`.
 * Errors: ZC_ERR_INVALID_ARG for a bad descriptor, chunk or subset index. */
int zc_unpack(const zc_packed* p, int32_t which, int32_t chunk, uint8_t* codes_out, float* dequant_out,
              void* stream);

const char* zc_status_string(int status);
int zc_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ZIPCACHE_H */
