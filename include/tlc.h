/*
 * tlc.h -- C ABI of the MI355X (gfx950) 3LC compression library.
 *
 * 3LC compresses one fp32 state-change tensor (a gradient push or a model
 * delta pull) per call, as described in the paper "3LC: Lightweight and
 * Effective Traffic Compression for Distributed Machine Learning":
 *
 *   encode (Section 3.1, Fig. 3; Sections 3.2 and 3.3)
 *     acc = tensor + residual                        error accumulation
 *     M   = max|acc| * s,  1 <= s < 2                Eq. 1
 *     q   = round(acc / M) in {-1, 0, 1}             Eq. 2 (half to even)
 *     residual = acc - M*q                           steps a and b
 *     Q   = quartic encoding of q + 1                Section 3.2
 *     C   = zero-run encoding of Q                   Section 3.3
 *   decode
 *     Q = zero-run expansion of C; q = quartic decoding of Q;
 *     out = M*q (Eq. 3)  or  out += M*q (aggregation at a server).
 *
 * The payload of one call is the byte string C plus the fp32 scalar M.
 *
 * Layout conventions (bit-exact contract):
 *   - m = ceil(n/5) quartic bytes.  The n values are padded with trit 0 to
 *     5m and split into five CONTIGUOUS partitions p_k = [k*m, (k+1)*m);
 *     byte j = 81*t(j) + 27*t(m+j) + 9*t(2m+j) + 3*t(3m+j) + t(4m+j).
 *   - A run of L bytes equal to 121 becomes floor(L/14) bytes 255, then
 *     243 + (L mod 14) - 2 if L mod 14 >= 2, or 121 if L mod 14 == 1.
 *   - Division is IEEE fp32 and rounding is half-to-even, so results are
 *     bit-identical to a sequential fp32 implementation.
 *
 * Memory: every tensor / byte pointer passed to tlc_compress and
 * tlc_decompress is DEVICE memory owned by the caller (for example a torch
 * tensor's data_ptr()).  The context owns its device workspace and a small
 * pinned host buffer; nothing is allocated per call.
 *
 * Streams: a context is bound to one HIP stream (passed as void*; NULL is
 * the default stream).  All work of a context is ordered on that stream.  A
 * context must not be used by two host threads at once.
 *
 * Errors: functions return TLC_OK (0) or a negative TLC_E_* code; no C++
 * exception crosses this boundary.  tlc_last_error_string() describes the
 * most recent failure of the calling thread.
 */
#ifndef TLC_H
#define TLC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TLC_OK 0
#define TLC_E_INVALID (-1)   /* bad argument: NULL pointer, s not in [1,2), n > max_n, scale not finite */
#define TLC_E_CAPACITY (-2)  /* bytes_cap < tlc_max_compressed_bytes(n) */
#define TLC_E_NONFINITE (-3) /* NaN/Inf in tensor+residual, or max*s overflows */
#define TLC_E_CORRUPT (-4)   /* compressed stream does not expand to ceil(n/5) bytes */
#define TLC_E_DEVICE (-5)    /* HIP runtime error, or the context is unusable */
#define TLC_E_INDEX (-6)     /* a token id outside the embedding table or the vocabulary */

/* Largest number of values one call accepts, summed over a batch (the
 * quartic byte counts must fit the 30-bit counters of the zero-run scans). */
#define TLC_MAX_N ((size_t)4294967295u)

/* Largest number of tensors (or streams) one batched call accepts. */
#define TLC_MAX_TENSORS 65536

typedef struct tlc_ctx tlc_ctx;

/* Upper bound of the compressed length for n values: ceil(n/5).  Zero-run
 * encoding (Section 3.3) never lengthens the quartic byte string. */
size_t tlc_max_compressed_bytes(size_t n);

/* Create a context for tensors of up to max_n values (1 <= max_n <=
 * TLC_MAX_N) whose work is issued on `hip_stream` (a hipStream_t, or NULL).
 * Allocates one device workspace of about 0.52 * max_n bytes (140 MB for
 * max_n = 2^28): partial maxima, look-back status words, the decoder's
 * start index, and for the single-tensor encoder per-tile slots and records,
 * a byte per four values (trits) and two per 32 (bounds).  No later call allocates device memory.  On success
 * *ctx receives the context; on failure *ctx is NULL.  Same as
 * tlc_ctx_create_batch(ctx, max_n, 1, hip_stream). */
int tlc_ctx_create(tlc_ctx** ctx, size_t max_n, void* hip_stream);

/* Create a context for batched calls: at most max_tensors tensors (or
 * streams) per call, 1 <= max_tensors <= TLC_MAX_TENSORS, and at most max_n
 * values per call summed over the batch (for tlc_decompress_sum: count * n).
 * Each tensor of a batch is still compressed on its own, with its own scale
 * and error buffer (Section 3: one compression context per tensor); the
 * batch only shares launches and the host synchronisation. */
int tlc_ctx_create_batch(tlc_ctx** ctx, size_t max_n, size_t max_tensors,
                         void* hip_stream);

/* Wait for the context's outstanding work and free it.  NULL is a no-op. */
int tlc_ctx_destroy(tlc_ctx* ctx);

/* Encode one tensor (Sections 3.1-3.3).
 *   tensor    device fp32[n], read only (the new state change).
 *   residual  device fp32[n], in/out: the error-accumulation buffer
 *             (Section 3.1, Fig. 3); on success it holds acc - M*q with
 *             acc = tensor + residual.  Must not overlap tensor.
 *   n         value count, 0 <= n <= max_n of the context.
 *   s         sparsity multiplier, 1 <= s < 2.
 *   bytes     device uint8[bytes_cap] receiving the zero-run encoded stream.
 *   bytes_cap must be >= tlc_max_compressed_bytes(n).
 *   bytes_len host out: stream length (0 on error).
 *   scale     host out: M (0 when n == 0).
 * Synchronous: returns after the stream length is known, which the encode
 * hands to the host a little before its last kernels end: the stream bytes
 * and the residual are complete in the order of the context's stream (work
 * issued there afterwards sees them; the host or another stream waits for
 * that stream, e.g. with tlc_sync, before reading them).  On
 * TLC_E_NONFINITE the residual and the bytes are left unchanged (with
 * TLC_OPT_IN_PLACE_FEEDBACK the residual holds acc instead). */
int tlc_compress(tlc_ctx* ctx, const float* tensor, float* residual, size_t n,
                 float s, uint8_t* bytes, size_t bytes_cap, size_t* bytes_len,
                 float* scale);

/* Decode one stream (inverse of Section 3.3, Section 3.2 decoding, Eq. 3).
 *   bytes       device uint8[bytes_len] from tlc_compress.
 *   scale       M from tlc_compress: finite and >= 0.
 *   n           value count of the encoded tensor, <= max_n.
 *   out         device fp32[n]: out = M*q (accumulate == 0) or
 *               out = out + M*q (accumulate != 0), for every element
 *               (-0.0 + M*0 gives +0.0; a value whose sum has the bits it
 *               already holds is not stored again).  Must not overlap
 *               bytes (TLC_E_INVALID).
 * Asynchronous on the context's stream; returns only errors detectable on
 * the host.  If the stream does not expand to exactly ceil(n/5) bytes, out
 * is left unchanged and the next tlc_sync() returns TLC_E_CORRUPT. */
int tlc_decompress(tlc_ctx* ctx, const uint8_t* bytes, size_t bytes_len,
                   float scale, size_t n, float* out, int accumulate);

/* ---- comparison encodings (decoded by tlc_decompress like any stream) --- */

#define TLC_MODE_3LC 0        /* Sections 3.1-3.3: same as tlc_compress */
#define TLC_MODE_NO_ZRE 1     /* 3-value quantization with error feedback and
                                 quartic encoding, no zero-run encoding
                                 (Table 2, row "No ZRE"): ceil(n/5) bytes */
#define TLC_MODE_STOCHASTIC 2 /* stochastic 3-value quantization + quartic
                                 encoding, no error feedback (the "Stoch
                                 3-value + QE" design of Section 5.1, TernGrad
                                 without clipping; Section 3.1) */
#define TLC_MODE_INT8 3       /* 8-bit integer quantization, codes -127..127
                                 (the "8-bit int" design of Section 5.1): n
                                 bytes, decoded by tlc_decompress_ex */

/* Encode with a comparison mode.  TLC_MODE_3LC forwards to tlc_compress
 * (seed and step unused).  TLC_MODE_NO_ZRE: as tlc_compress but the payload
 * is the ceil(n/5) quartic bytes.  TLC_MODE_STOCHASTIC: M = max|tensor| * s;
 * value i becomes sign(tensor[i]) with probability |tensor[i]|/M, else 0,
 * decided by u < |tensor[i]|/M with u = (w >> 8) * 2^-24 and w word (i mod
 * 4) of Philox4x32-10 (Salmon et al., SC 2011) at counter (i/4 low, i/4
 * high, step low, step high) and key (seed low, seed high); residual is not
 * used (may be NULL).  Both return *bytes_len = ceil(n/5); the bytes are
 * 0..242, so tlc_decompress decodes them unchanged.
 * TLC_MODE_INT8: acc = tensor + residual (error feedback, residual
 * rewritten) or, with residual == NULL, acc = tensor; M = max|acc| * s
 * (Eq. 1), step D = fl(M / 127); byte i is the two's-complement int8 code
 * rint(fl(acc_i / D)) clamped to [-127, 127] (0 when D == 0) and the
 * residual becomes fl(acc_i - fl(code * D)).  bytes_cap >= n; *bytes_len =
 * n.  Synchronous; on TLC_E_NONFINITE the residual and bytes are unchanged
 * (with TLC_OPT_IN_PLACE_FEEDBACK a non-NULL residual holds acc), as for
 * tlc_compress; the same holds for TLC_MODE_NO_ZRE. */
int tlc_compress_ex(tlc_ctx* ctx, int mode, const float* tensor, float* residual, size_t n,
                    float s, uint64_t seed, uint64_t step, uint8_t* bytes, size_t bytes_cap,
                    size_t* bytes_len, float* scale);

/* Decode a stream of any mode.  TLC_MODE_3LC, TLC_MODE_NO_ZRE and
 * TLC_MODE_STOCHASTIC forward to tlc_decompress.  TLC_MODE_INT8: bytes is
 * device uint8[n] of int8 codes (every code accepted), out = fl(code * D)
 * or out + fl(code * D) with D = fl(scale / 127); bytes_len != n returns
 * TLC_E_CORRUPT at once with out unchanged.  Asynchronous on the context's
 * stream. */
int tlc_decompress_ex(tlc_ctx* ctx, int mode, const uint8_t* bytes, size_t bytes_len,
                      float scale, size_t n, float* out, int accumulate);

/* Encode `count` tensors (in one launch; those of more than 1,310,720 values
 * in four launches of their own, together, or five each above 41,943,040; one
 * synchronisation): for every t, exactly tlc_compress(ctx, tensors[t], residuals[t], ns[t],
 * s[t], bytes[t], caps[t], &bytes_len[t], &scales[t]).  All arrays are host
 * arrays of `count` entries; the pointers in them are device pointers, and
 * buffers of different tensors must not overlap.  Argument errors reject the
 * whole call before any work.  status[t] receives TLC_OK or
 * TLC_E_NONFINITE (that tensor's residual and bytes unchanged, or its
 * residual holding acc with TLC_OPT_IN_PLACE_FEEDBACK; bytes_len[t] = 0);
 * the call returns TLC_E_NONFINITE if any tensor was refused. */
int tlc_compress_batch(tlc_ctx* ctx, size_t count, const float* const* tensors,
                       float* const* residuals, const size_t* ns, const float* s,
                       uint8_t* const* bytes, const size_t* caps, size_t* bytes_len,
                       float* scales, int* status);

/* Decode `count` streams into `count` outputs in two launches: for every t,
 * tlc_decompress(ctx, bytes[t], bytes_len[t], scales[t], ns[t], outs[t],
 * accumulate).  Host arrays of device pointers; outputs must not overlap.
 * Asynchronous; if any stream is corrupt no output is written and the next
 * tlc_sync() returns TLC_E_CORRUPT. */
int tlc_decompress_batch(tlc_ctx* ctx, size_t count, const uint8_t* const* bytes,
                         const size_t* bytes_len, const float* scales, const size_t* ns,
                         float* const* outs, int accumulate);

/* Server-side aggregation (Section 2, Fig. 1; Section 3, Fig. 2): decode
 * `count` streams of the same n-value tensor and add them into one fp32
 * output in stream order, element by element:
 *   out = (((accumulate ? out : 0) + v_0) + v_1) + ... + v_{count-1}
 * (with accumulate == 0 the first term is v_0 itself), bit-identical to
 * tlc_decompress(stream 0, accumulate) followed by tlc_decompress(stream
 * t, accumulate = 1) for t = 1 .. count-1, but reading and writing out only
 * once.  Asynchronous; if any stream is corrupt out is left unchanged and
 * the next tlc_sync() returns TLC_E_CORRUPT.  count * n must not exceed the
 * context's max_n. */
int tlc_decompress_sum(tlc_ctx* ctx, size_t count, const uint8_t* const* bytes,
                       const size_t* bytes_len, const float* scales, size_t n, float* out,
                       int accumulate);

/* ---- encoding without a context (no allocation) ------------------------ */

/* Result of tlc_compress_noalloc, written to device memory by the call's
 * last kernel: status is TLC_OK, TLC_E_NONFINITE (residual and bytes left
 * unchanged, as for tlc_compress) or TLC_E_DEVICE (a look-back wait gave
 * up; the residual may then already hold its new values and no stream was
 * written); bytes_len and scale are those tlc_compress returns (0 unless
 * status is TLC_OK). */
typedef struct tlc_result {
  int32_t status;
  uint32_t bytes_len;
  float scale;
  uint32_t reserved; /* 0 */
} tlc_result;

/* Largest n tlc_compress_noalloc accepts: 2^23 values (the scratch, 16 KiB of
 * device memory, holds a status word for each of their encoder tiles). */
#define TLC_NOALLOC_MAX_N ((size_t)8388608u)

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * tlc_compress without a context.  Same encoding, bit for bit, with the
 * default error policy (the check pass leaves residual and bytes unchanged
 * on NaN/Inf), for n <= TLC_NOALLOC_MAX_N (larger n: TLC_E_INVALID, nothing
 * runs).
 *   tensor, residual, n, s, bytes, bytes_cap   as for tlc_compress.
 *   result      device pointer to one tlc_result (16 bytes), written last.
 *   hip_stream  a hipStream_t of the calling thread's current device (or
 *               NULL, the default stream); every pointer belongs to that
 *               device.
 * Asynchronous: returns after queueing its kernels (argument errors are
 * returned at once, and nothing runs); read *result after the stream has
 * reached it.  No device or pinned memory is allocated, and no library
 * routine that allocates is called: the scratch (a control block, partial
 * maxima, look-back status words) is a static device array of 16 KiB per
 * device, located once per device on the first call there.  Every call on
 * a device shares that array and clears it first, so calls that may
 * overlap on one device (other streams, other host threads) race and must
 * be ordered by the caller. */
int tlc_compress_noalloc(const float* tensor, float* residual, size_t n, float s,
                         uint8_t* bytes, size_t bytes_cap, tlc_result* result,
                         void* hip_stream);

/* ---- before the codec: embedding tables, gradient norm and clipping ------
 *
 * What a training step of a language model runs around tlc_compress: the
 * lookup of its tokens' embedding rows, the gradient of the embedding table
 * (fp32, dense, rows without a token exactly zero: a tensor that zero-run
 * encoding shortens well), and the clipping of all gradients by their global
 * norm, written as the fp32 tensors that tlc_compress reads.
 *
 * They run on a context of their own, bound to one HIP stream like a tlc_ctx:
 * asynchronous on that stream, no device memory allocated per call, tensors
 * device memory owned by the caller, the same rules for host threads and
 * errors.  Their calls may be captured into a graph (lists of tensors: up to
 * TLC_CAPTURE_TENSORS; longer ones are handed over in host memory that later
 * calls use again, and refused; tlc_adamw's of any length).  A replay uses the
 * context's workspace like the calls that it holds: it runs on the context's
 * stream or is ordered with the context's other work by the caller, and before
 * tlc_train_destroy().
 * tlc_profile_* does not time them. */
typedef struct tlc_train tlc_train;

#define TLC_CAPTURE_TENSORS 128

/* Types of values and of token ids. */
#define TLC_F32 0
#define TLC_BF16 1
#define TLC_F16 2
#define TLC_I32 0
#define TLC_I64 1

/* Largest table height and row length. */
#define TLC_MAX_ROWS 2147483646
#define TLC_MAX_DIM 16777216

/* Create a context on `hip_stream` for embedding gradients of up to
 * max_tokens tokens (below 2^31) into tables of up to max_rows rows of up to
 * max_dim values, and for lists of up to max_tensors tensors (at most
 * TLC_MAX_TENSORS).  Any of them may be 0: that call is then refused
 * (tlc_embedding needs none of them).  Allocates one device workspace of about
 * 1.1 MB + (24 + max_dim / 8) * max_tokens + max_rows bytes and, for more than 64
 * tensors, which do not all travel with a launch's arguments, 24 * (4096 +
 * max_tensors) bytes of it and 512 * (4096 + max_tensors) of pinned host memory
 * (eight places for the pieces of a list: 2.1 MB for 65 tensors, 36 for 65536). */
int tlc_train_create(tlc_train** ctx, size_t max_tokens, size_t max_rows, size_t max_dim,
                     size_t max_tensors, void* hip_stream);

/* Wait for the context's outstanding work and free it.  NULL is a no-op. */
int tlc_train_destroy(tlc_train* ctx);

/* Wait for all work of the context and return (then clear) the sticky
 * status of its lookups, embedding gradients and token log probabilities: TLC_OK or
 * TLC_E_INDEX. */
int tlc_train_sync(tlc_train* ctx);

/* Embedding lookup with scaling: for every token t
 *   out[t, k] = round(scale * table[ids[t], k]),  0 <= k < dim,
 * the product in fp32, rounded once (half to even) to out's type.
 *   table       device, `rows` rows of dim values of table_type, the first
 *               values of two rows table_stride values apart (any stride).
 *   ids         device int32 or int64 [count] (ids_type).
 *   out         device, count rows of dim values of out_type, out_stride >=
 *               dim values apart; must not overlap table or ids.
 *   scale       finite.
 * An id outside [0, rows) gives a row of zeros, and the next
 * tlc_train_sync() returns TLC_E_INDEX. */
int tlc_embedding(tlc_train* ctx, const void* table, int table_type, size_t rows, size_t dim,
                  size_t table_stride, const void* ids, int ids_type, size_t count, float scale,
                  void* out, int out_type, size_t out_stride);

/* The gradient of an embedding table: for every row v
 *   out[v, k] = (accumulate ? out[v, k] : 0) + scale * sum grad[t, k]
 * over the tokens t with ids[t] == v.  fp32 sums; the order in which they
 * are formed is fixed by the sizes, types and ids, so that the same call gives the
 * same bits.  A row without a token becomes 0, or with accumulate stays as it
 * is, bit for bit.
 *   grad        device, count rows of dim values of grad_type, grad_stride
 *               values apart (0: one row for all tokens).
 *   padding_id  tokens with this id add nothing (negative: there are none).
 *   out         device fp32, `rows` rows of dim values out_stride >= dim
 *               values apart; values between rows are left alone.  Must not
 *               overlap grad or ids.
 * An id outside [0, rows) adds nothing, and the next tlc_train_sync()
 * returns TLC_E_INDEX.  The rows of grad of tokens that add nothing are not
 * part of any sum, whatever they hold. */
int tlc_embedding_grad(tlc_train* ctx, const void* grad, int grad_type, size_t grad_stride,
                       const void* ids, int ids_type, size_t count, size_t rows, size_t dim,
                       float scale, int64_t padding_id, float* out, size_t out_stride,
                       int accumulate);

/* Result of the calls on lists of tensors, in device memory. */
typedef struct tlc_norm_result {
  double sumsq;      /* sum of the squares of all values, in 64 bits */
  float norm;        /* sqrt(sumsq), rounded to fp32 */
  float coef;        /* the factor of the values: 1 where norm <= max_norm, else max_norm / norm */
  int32_t status;    /* TLC_OK, or TLC_E_NONFINITE: NaN/Inf among the values (coef is NaN) */
  uint32_t reserved; /* 0 */
} tlc_norm_result;

/* The global norm of `count` tensors: result->sumsq, norm and status (coef is
 * 1).  Host arrays of device pointers, of types and of value counts (each at
 * most TLC_MAX_N, 2^40 in all); a tensor of no values may be NULL.  Squares and sums are
 * in 64 bits: no value of any type overflows them.  The order of the sums is fixed by
 * the sizes: the same call gives the same bits.  The same values cut into other
 * tensors are added in another order, which can change the last bits of sumsq and,
 * where its root lies that close between two fp32 values, norm by one unit in the
 * last place. */
int tlc_grad_norm(tlc_train* ctx, size_t count, const void* const* tensors, const int* types,
                  const size_t* ns, tlc_norm_result* result);

/* Clip `count` tensors by a norm that is known: with norm =
 * sqrt(result->sumsq) and coef = norm > max_norm ? max_norm / norm : 1 (64
 * bits, rounded to fp32),
 *   outs[i][k] = coef * tensors[i][k]   (one fp32 product)
 * for every tensor; also writes result's norm, coef and status.  A program
 * whose gradients are spread over ranks adds up the sumsq of tlc_grad_norm
 * (of its shards) between the two calls.
 *   max_norm    finite, >= 0.
 *   outs        fp32 buffers; outs[i] may be tensors[i] itself where that is
 *               fp32.  NULL: in place in the tensors' own types (rounded half
 *               to even; with coef 1 nothing is written).
 * No buffer may overlap another one that is written.  If sumsq is not finite
 * no buffer is written. */
int tlc_clip(tlc_train* ctx, size_t count, const void* const* tensors, const int* types,
             const size_t* ns, float max_norm, tlc_norm_result* result, float* const* outs);

/* tlc_grad_norm followed by tlc_clip. */
int tlc_clip_grad_norm(tlc_train* ctx, size_t count, const void* const* tensors,
                       const int* types, const size_t* ns, float max_norm,
                       tlc_norm_result* result, float* const* outs);

/* ---- the loss, and the server's step --------------------------------------
 *
 * The ends of the same training step, on the same contexts: the log
 * probabilities of given tokens (their negative mean is a language model's
 * loss) with their gradient, and the optimizer's step that turns the gradients
 * which tlc_decompress_sum has added up into new weights and into the change
 * that tlc_compress encodes for the workers' pulls. */

/* Most alternatives of a token, and the values that share a scale of the
 * optimizer's states in 8 bits. */
#define TLC_MAX_TOP 64
#define TLC_STATE_BLOCK 256

/* Of one row of logits x with scale s, in device memory. */
typedef struct tlc_token_result {
  float logprob; /* s * (x[target] - max) - log_sum; 0 without a target */
  float entropy; /* -sum p ln p, p = exp(s * (x - max) - log_sum) */
  float max;     /* the largest logit, as it is in the row */
  float log_sum; /* ln sum exp(s * (x - max)) */
} tlc_token_result;

/* Log probabilities of given tokens, the entropy of every row and its most
 * likely alternatives, from logits that are read once.
 *   logits        device, count rows of vocab values of type (vocab in [1,
 *                 TLC_MAX_DIM], count below 2^31), stride values apart (any).
 *   scale         of the logits, in (0, 1e18]: the inverse temperature.
 *   targets       device int32 or int64 [count] (ids_type), or NULL: none.
 *   ignore_id     rows with this target (any value) are left out: not read,
 *                 all their outputs 0 and their top_ids -1.  So are rows
 *                 whose target is outside [0, vocab); the next
 *                 tlc_train_sync() then returns TLC_E_INDEX.
 *   results       device [count].
 *   top           alternatives of a row, at most TLC_MAX_TOP and vocab:
 *                 top_logprobs and top_ids (device, count rows of top, NULL
 *                 for none) hold the largest logits' log probabilities and
 *                 columns, the largest first, the lowest column first among
 *                 equal logits.
 * Sums are in fp32 in an order that the sizes alone fix.  log_sum is the logarithm
 * of a sum that holds the largest logit's own 1, which each addition may round by
 * 2^-24: where a token is nearly certain, the error of log_sum, logprob and the
 * target's gradient is absolute (a logit 20 above 99 others: 1 - p of 2.0e-7 may come
 * out as 2.4e-7, one below 2^-24 as 0).
 * Entries of -inf have probability 0.  A row with no other entry has max, log_sum and
 * log probabilities -inf and entropy 0; its top_ids are its first columns.  A row that
 * holds NaN or +inf has NaN in its place, and top_ids -1.  No output may overlap
 * another argument. */
int tlc_token_logprobs(tlc_train* ctx, const void* logits, int type, size_t count, size_t vocab,
                       size_t stride, float scale, const void* targets, int ids_type,
                       int64_t ignore_id, tlc_token_result* results, size_t top,
                       float* top_logprobs, int32_t* top_ids);

/* The gradient of logits from those of the log probabilities and entropies
 * that tlc_token_logprobs gave:
 *   out[t, j] = round(scale * (a (1[j = target] - p_j) - b p_j (ln p_j + entropy)))
 * with a = grad_logprob[t] and b = grad_entropy[t] (device fp32 [count]; NULL:
 * zeroes) and p from results.  Rows that are left out (see there) and rows of
 * -inf alone get zeroes and are not read; a row of NaN gets NaN.
 *   out           device, count rows of vocab values of out_type, out_stride >=
 *                 vocab values apart; values between rows are left alone.
 *                 It may be logits itself (the same address, type and
 *                 stride); apart from that it must not overlap another argument.
 * Without targets grad_logprob must be NULL. */
int tlc_token_logprobs_grad(tlc_train* ctx, const void* logits, int type, size_t count,
                            size_t vocab, size_t stride, float scale, const void* targets,
                            int ids_type, int64_t ignore_id, const tlc_token_result* results,
                            const float* grad_logprob, const float* grad_entropy, void* out,
                            int out_type, size_t out_stride);

/* How an optimizer's states are held. */
#define TLC_STATE_F32 0
#define TLC_STATE_8BIT 1

/* Steps done, in device memory: {0, 1.0f, 0} before the first one. */
typedef struct tlc_adamw_clock {
  int64_t step;      /* of steps done; tlc_adamw counts it up */
  float lr_scale;    /* factor of lr: a schedule that a graph's replays follow */
  uint32_t reserved; /* 0 */
} tlc_adamw_clock;

typedef struct tlc_adamw_options {
  double lr;           /* finite, >= 0 */
  double beta1, beta2; /* in [0, 1) */
  double eps;          /* finite, above 0 in fp32 */
  double weight_decay; /* finite, >= 0 */
  float max_norm;      /* >= 0, may be infinite; read where there is a result */
} tlc_adamw_options;

/* One step of AdamW over `count` tensors (at most the context's max_tensors).
 * With t = clock->step + 1, lr = options->lr * clock->lr_scale and the factors
 * rounded to fp32 from 64 bits
 *   c1 = 1 - beta1, c2 = 1 - beta2, d = lr * weight_decay,
 *   a = lr / (1 - beta1^t),  r = 1 / sqrt(1 - beta2^t),
 * every value takes, each operation rounded to fp32,
 *   g = coef * grad
 *   m = m + (g - m) * c1
 *   v = v + (g * g - v) * c2
 *   new = param - (a * (m / (sqrt(v) * r + eps)) + d * param)
 * and new is rounded half to even to the parameter's type.
 *   params, types, grads, grad_types, ns
 *                 host arrays of device pointers, types and value counts
 *                 (each at most TLC_MAX_N, 2^40 in all); a tensor of no
 *                 values may be NULL.
 *   exp_avgs, exp_avg_sqs
 *                 the states m and v, device buffers of ns[i] values: fp32,
 *                 or with state_type TLC_STATE_8BIT bytes (below).  Zeroes
 *                 before the first step.
 *   scales        TLC_STATE_8BIT: device buffers of two floats (of m and of v)
 *                 for every TLC_STATE_BLOCK values; else NULL.
 *   deltas        NULL, or device fp32 buffers that get new - param, as stored
 *                 and rounded once; deltas[i] may be grads[i] itself where
 *                 that is fp32.
 *   clock         device; its step becomes t.
 *   result        NULL: coef is 1.  Else the norm of the gradients as
 *                 tlc_grad_norm left it: coef and the result's fields are
 *                 those of tlc_clip with options->max_norm, without the
 *                 clipped gradients' being written anywhere.  Where sumsq is not
 *                 finite the step is left out: nothing is written but
 *                 zeroes in deltas and the result, and the clock stays.
 * A state in 8 bits is an OCP E4M3 (m) or E5M2 (v) number times its block's
 * scale: after a step, scale = max(largest |m| * (1 / 448), 2^-126) (v: 1 / 57344;
 * the constant rounded to fp32), 0 where all are 0.  |m| / scale lies between two
 * codes (0 being one, the largest 448 or 57344) and goes to the upper one where its
 * share of the way there plus a dither reaches 1: with
 *   h = (k * 0xC13FA9A9 + t * 0x91E10DA5) mod 2^32
 * of value k of its tensor, the top 20 bits of h (m) or the top 21 of h xor
 * 2^31 (v) as a fraction.  Over steps and neighbours these are spread evenly,
 * so that a slow mean is followed where rounding to nearest would hold still.
 * v > 0 never gets the code 0.  A block in which a value of m (v) is NaN or infinite
 * has the scale NaN.
 * No buffer may overlap another one that is written. */
int tlc_adamw(tlc_train* ctx, size_t count, void* const* params, const int* types,
              const size_t* ns, const void* const* grads, const int* grad_types, int state_type,
              void* const* exp_avgs, void* const* exp_avg_sqs, float* const* scales,
              float* const* deltas, const tlc_adamw_options* options, tlc_adamw_clock* clock,
              tlc_norm_result* result);

/* ---- options ------------------------------------------------------------ */

/* TLC_OPT_IN_PLACE_FEEDBACK: take step 1 of error accumulation (Section
 * 3.1, Fig. 3: the tensor is added into the buffer) as done in the
 * residual itself before Eq. 1 is known.  The encoders of large tensors then
 * read tensor and residual once instead of twice (12 instead of 20 bytes per
 * value for the 3-value modes); every result is the same, except that after
 * TLC_E_NONFINITE the residual holds tensor + residual instead of being
 * left unchanged.  For callers that check their tensors for NaN/Inf
 * themselves, or reset the residual after such an error. */
#define TLC_OPT_IN_PLACE_FEEDBACK 1u

/* Set the context's options (a combination of TLC_OPT_*; 0, the default,
 * is the behaviour documented above).  Takes effect from the next call. */
int tlc_ctx_set_options(tlc_ctx* ctx, uint32_t options);

/* Wait for all work of the context and return (then clear) the sticky
 * status of asynchronous decodes: TLC_OK or TLC_E_CORRUPT. */
int tlc_sync(tlc_ctx* ctx);

/* Look-back epochs.  Every launch of a chained or batched encode and every
 * decode tags the status words of its scan with the next value of a
 * per-context counter (encode 1 .. TLC_ENC_EPOCH_MAX, decode 1 ..
 * TLC_DEC_EPOCH_MAX), so the words need no clearing between launches;
 * when a counter wraps, its status words are cleared first (and for the
 * decode counter the range starts, the verdict and the mark that flags a
 * corrupt stream's launch). */
#define TLC_ENC_EPOCH_MAX 8388607  /* 2^23 - 1 */
#define TLC_DEC_EPOCH_MAX 67108863 /* 2^26 - 1 */

/* For tests of the wrap: wait for the context's work, clear the
 * epoch-tagged words of both scans (status words, the decoder's range
 * starts and its verdict: no word of an earlier launch can then carry a
 * future epoch) and set the counters to the last epochs used, enc_epoch
 * <= TLC_ENC_EPOCH_MAX and dec_epoch <= TLC_DEC_EPOCH_MAX (else
 * TLC_E_INVALID).  The corrupt-stream mark is left as it is: only the wrap
 * clears it. */
int tlc_ctx_set_epochs(tlc_ctx* ctx, uint32_t enc_epoch, uint32_t dec_epoch);

/* Text of the calling thread's most recent error (never NULL). */
const char* tlc_last_error_string(void);

/* ---- per-kernel timing (HIP events on the context's stream) ----------- */

#define TLC_KERNEL_ABSMAX 0         /* in place: step 1 into the residual, partial max (Eq. 1);
                                       without a residual: partial max */
#define TLC_KERNEL_QUANT_ENCODE 1   /* large tensors: quartic pack from trits, each tile's own
                                       zero-run encoding */
#define TLC_KERNEL_ZRE_INDEX 2      /* zero-run scan: where each output range starts
                                       (a small stream's scan runs in the next kernel) */
#define TLC_KERNEL_EXPAND_DEQUANT 3 /* zero-run expansion, quartic unpack, Eq. 3 (for a
                                       small stream, with the scan in its first blocks) */
#define TLC_KERNEL_ABSMAX_BATCH 4
#define TLC_KERNEL_QUANT_ENCODE_BATCH 5
#define TLC_KERNEL_ZRE_INDEX_BATCH 6
#define TLC_KERNEL_EXPAND_DEQUANT_BATCH 7
#define TLC_KERNEL_EXPAND_SUM 8     /* multi-stream expansion + summed dequantization */
#define TLC_KERNEL_QUANT_PACK 9     /* comparison modes: (stochastic trits and) quartic pack */
#define TLC_KERNEL_INT8_QUANT 10    /* 8-bit comparator: codes and residual */
#define TLC_KERNEL_INT8_DEQUANT 11  /* 8-bit comparator: decode */
#define TLC_KERNEL_ZRE_CHUNKS 12    /* zero-run encoding: summaries of tile chunks */
#define TLC_KERNEL_ZRE_COMPACT 13   /* zero-run encoding: tiles compacted into the stream */
#define TLC_KERNEL_QUANT_ENCODE_CHAINED 14 /* a small tensor's whole encode */
#define TLC_KERNEL_ABSMAX_CHECK 15  /* partial max of |tensor + residual|, nothing written */
#define TLC_KERNEL_ABSMAX_CHECK_BATCH 16
#define TLC_KERNEL_ACCUM_QUANTIZE 17 /* large tensors: Eq. 2, the residuals and 2-bit trits
                                        (after the check pass, with step 1) */
#define TLC_KERNEL_COUNT 18

/* Enable (on != 0) or disable recording of a start/stop event pair around
 * every kernel launch of the tlc_ctx (of the kernels selected by
 * tlc_profile_mask; all of them by default). */
int tlc_profile_enable(tlc_ctx* ctx, int on);

/* Select which kernels are timed while profiling is enabled: bit k of mask
 * selects kernel id k (TLC_KERNEL_*).  Each timed launch adds an event pair
 * to the stream, whose ordering costs some microseconds of device time, so
 * a caller measuring throughput may time only the kernel it needs. */
int tlc_profile_mask(tlc_ctx* ctx, uint32_t mask);

/* Synchronize, then report the summed device time (ms) and the number of
 * timed launches of kernel `kernel` since the last reset. */
int tlc_profile_get(tlc_ctx* ctx, int kernel, double* total_ms,
                    uint64_t* launches);

/* Zero the accumulated timings. */
int tlc_profile_reset(tlc_ctx* ctx);

/* Name of a kernel id (the __global__ function's name), or NULL. */
const char* tlc_kernel_name(int kernel);

#ifdef __cplusplus
}
#endif

#endif /* TLC_H */
