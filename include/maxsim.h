/*
 * maxsim.h -- C ABI of the fused MaxSim library for AMD MI355X (gfx950).
 *
 * The operator is the late-interaction score of the "Flash-MaxSim" paper,
 *     score(Q, D) = sum_i max_j <Q_i, D_j>                      (Eq. 1),
 * computed tile by tile so that the [N_q, B, L_q, L_d] similarity tensor is
 * never written to memory (Alg. 1), its training backward through the stored
 * argmax (Eqs. 2-3, Alg. 2), and int8 scoring with per-token scales applied
 * once per similarity cell (Sec. "Quantised Scoring", Alg. 4).
 *
 * Conventions shared by every entry point
 *   - Every pointer is a DEVICE pointer owned by the caller (the one exception, the host
 *     corpus of the *_streamed entry points, is marked HOST).  The library never allocates,
 *     frees or keeps device memory.
 *   - `stream` is a hipStream_t passed as void*.  Calls only enqueue work on it
 *     and return; they never synchronise.  NULL means the default stream.
 *   - Tensors are row-major with the innermost stride 1 and no gaps.  Base
 *     pointers of Q, D and the int8 tensors must be 16-byte aligned, all other
 *     pointers 4-byte aligned.
 *   - d (embedding width).  The paper's setting is 128 (Tab. "shapes"); its "fat embedding" extension
 *     (App. "split-d") goes to 2048.  Here:
 *       float forward (maxsim_forward, _ragged, _streamed): any width whose rows are a multiple of 64 bytes, from
 *         d = 32 up to rows of 16 KB: d = 32, 64, 96, ... , 8192 for fp16/bf16 and d = 32, 48, 64, ... , 4096 for
 *         fp32.  Rows of 128, 256 and 512 bytes can keep the queries in registers; every other width streams both
 *         operands in slabs of the embedding dimension (the paper's inner loop over d).
 *       backward (maxsim_backward, _ragged, _csr, _csr_static): any multiple of 8 from 8 to 8192; Q must stay
 *         below 4 GiB and D below 64 GiB.
 *       int8 entry points and the quantiser: any multiple of 32 from 32 to 8192.  d = 128 takes the tuned kernels
 *         (queries resident in LDS or registers); other multiples of 64 stream both operands in slabs like the
 *         float forward; the remaining widths take a plain inner loop over d at a fraction of the speed.  The same
 *         arithmetic and the same bits everywhere.
 *     Other widths must be zero-padded by the caller; anything else returns MAXSIM_ERR_UNSUPPORTED.
 *   - Five kernel families use more than 64 KB of LDS, which HIP wants allowed per kernel and device before the
 *     first launch.  maxsim_init() does that (and all other per-device set-up) for the current device; an entry
 *     point whose device has not been set up does it itself first, which is not possible while `stream` is being
 *     captured into a HIP graph: call maxsim_init() once per device before capturing anything.
 *   - L_q and L_d are arbitrary positive integers (no tile multiples needed).
 *   - Inputs must be finite; the result for NaN/Inf inputs is unspecified.
 *   - Return value: MAXSIM_OK (0) or a negative error code.  MAXSIM_ERR_INVALID, _UNSUPPORTED and _SCRATCH
 *     are found before anything is enqueued.  MAXSIM_ERR_LAUNCH means the HIP runtime refused a step of the
 *     call: earlier steps of the same call (kernels, copies, waits between streams) may already be queued and the
 *     outputs are then undefined.  No exceptions, no abort, nothing printed.
 */
#ifndef MAXSIM_H
#define MAXSIM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MAXSIM_OK 0
#define MAXSIM_ERR_INVALID (-1)     /* null pointer, non-positive size, misaligned pointer, bad enum */
#define MAXSIM_ERR_UNSUPPORTED (-2) /* an embedding width or a size that the kernels are not built for */
#define MAXSIM_ERR_LAUNCH (-3)      /* the HIP runtime reported an error at launch */
#define MAXSIM_ERR_SCRATCH (-4)     /* sizes beyond the library's static scratch buffer (maxsim_backward_csr_static) or a workspace */

typedef enum { MAXSIM_F32 = 0, MAXSIM_F16 = 1, MAXSIM_BF16 = 2 } maxsim_dtype;

/* Human-readable text for a return code (static storage, never NULL). */
const char *maxsim_strerror(int code);

/*
 * Per-device set-up for the CURRENT device: raises the LDS limit of the kernels that need it and looks up
 * the library's static scratch array.  Allocates nothing, enqueues nothing, may be called any number of times
 * and from several host threads.  Optional unless entry points are to be captured into HIP graphs (see above).
 * Returns MAXSIM_OK or MAXSIM_ERR_LAUNCH (the HIP runtime refused).
 */
int maxsim_init(void);

/*
 * Fused forward over a uniform corpus (Eq. 1; Alg. 1; Prop. 1).
 *   Q       [n_q, l_q, d]  dtype          query token embeddings
 *   D       [b,   l_d, d]  dtype          document token embeddings
 *   scores  [n_q, b]       float32        fully overwritten
 *   argmax  [n_q, b, l_q]  int32 or NULL  winning document-token index, local to
 *                                         the document (Sec. "Closed-Form Gradients");
 *                                         ties go to the lowest index ("Tied maxima")
 * Products are formed in the input dtype's exact values and accumulated in fp32.
 * With fp16/bf16 inputs and argmax requested, similarities below 512 in magnitude that differ by less than
 * 2^-19 relative count as tied (the lower index wins) and the maxima that enter the score may be truncated by
 * that much; without argmax, and for fp32 inputs, the maxima are the exact fp32 sums.
 */
int maxsim_forward(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d,
                   maxsim_dtype dtype, float *scores, int32_t *argmax, void *stream);

/*
 * Out-of-core forward (Sec. "Corpus-scale scoring": a corpus that does not fit in device memory is
 * streamed through a fixed buffer while the kernel runs).
 *   D_host      [b, l_d, d] dtype in HOST memory (page-locked memory makes the copies asynchronous;
 *               pageable memory works but serialises them)
 *   block_docs  documents per block (clamped to b); block_docs * l_d must be < 2^31
 *   staging     DEVICE buffer of 2 * block_docs * l_d * d * sizeof(dtype) bytes owned by the caller;
 *               its contents are overwritten
 *   scores      [n_q, b] float32 (device), fully overwritten; no argmax
 * Block k + 1 is copied (on a copy stream the library creates once per device, default priority)
 * while block k is scored on `stream`; all work is ordered after what `stream` already holds and
 * the call returns without synchronising.  D_host and staging must stay valid until `stream`
 * has run the last kernel.  Same arithmetic as maxsim_forward (identical bits).
 */
int maxsim_forward_streamed(const void *Q, int n_q, int l_q, const void *D_host, int64_t b, int l_d,
                            int d, maxsim_dtype dtype, int64_t block_docs, void *staging,
                            float *scores, void *stream);

/*
 * Fused forward over a packed ragged corpus (Sec. "Ragged corpora and kernel family";
 * the cu_seqlens variant).  No padding is read or computed.
 *   D_packed     [total_tokens, d] dtype   documents back to back
 *   doc_offsets  [b + 1] int32 (device)    non-decreasing, doc_offsets[0] = 0,
 *                                          doc_offsets[b] = total_tokens
 *   total_tokens host copy of doc_offsets[b]; must be < 2^31
 * A document of length 0 gets score -inf and argmax -1.
 * Other arguments as in maxsim_forward.
 */
int maxsim_forward_ragged(const void *Q, int n_q, int l_q, const void *D_packed,
                          const int32_t *doc_offsets, int64_t b, int64_t total_tokens, int d,
                          maxsim_dtype dtype, float *scores, int32_t *argmax, void *stream);

/*
 * Backward through the stored argmax (Eqs. 2-3; Alg. 2), uniform corpus.
 *   argmax  [n_q, b, l_q] int32   as written by maxsim_forward; negative entries are skipped,
 *                                 entries >= l_d are a caller error (skipped, never dereferenced)
 *   dscore  [n_q, b]      float32 upstream gradient of the scores
 *   dQ      [n_q, l_q, d] float32 fully overwritten:  dQ[q,i,:] = sum_b dscore[q,b] D[b, A[q,b,i], :]
 *   dD      [b,  l_d, d]  float32 fully overwritten:  dD[b,t,:] = sum_{(q,i): A[q,b,i]=t} dscore[q,b] Q[q,i,:]
 * Accumulation is fp32 in a fixed order: results are bitwise reproducible from run to run
 * (no atomics; every dD row has one owner, a wavefront, which adds the row's edges by increasing edge id
 * (q * b + j) * l_q + i: the role of the paper's inverse-grid CSR, without building it in global memory;
 * dQ adds the documents of each of up to eight contiguous partitions in order and then the partitions in order).
 * dD doubles as work space during the call: it holds partial sums of dQ until its own rows are written.
 */
int maxsim_backward(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d,
                    maxsim_dtype dtype, const int32_t *argmax, const float *dscore, float *dQ,
                    float *dD, void *stream);

/*
 * Backward over a packed ragged corpus (Eqs. 2-3 with the ragged layout of Sec. "Ragged corpora
 * and kernel family").
 *   D_packed, doc_offsets, total_tokens as in maxsim_forward_ragged
 *   argmax  [n_q, b, l_q] int32   document-local indices as written by maxsim_forward_ragged;
 *                                 negative entries (empty documents) are skipped
 *   dQ      [n_q, l_q, d] float32 fully overwritten
 *   dD_packed [total_tokens, d] float32 fully overwritten, packed like D_packed
 * Same arithmetic and reproducibility as maxsim_backward.
 */
int maxsim_backward_ragged(const void *Q, int n_q, int l_q, const void *D_packed,
                           const int32_t *doc_offsets, int64_t b, int64_t total_tokens, int d,
                           maxsim_dtype dtype, const int32_t *argmax, const float *dscore,
                           float *dQ, float *dD_packed, void *stream);

/*
 * The inverse-grid CSR of the deterministic backward, built on the device (Alg. 2; Sec.
 * "Closed-Form Gradients"): the map destination row -> source edges that bincount, cumsum and
 * a stable argsort by destination define.  Uniform corpus.
 *   argmax   [n_q, b, l_q] int32 (device)   an entry t with 0 <= t < l_d is an edge with id
 *                                           e = (i * b + j) * l_q + s and destination row
 *                                           j * l_d + t; other entries are not edges
 *   row_ptr  [b * l_d + 1] int32 (device)   output: row r's edges are col_idx[row_ptr[r] ..
 *                                           row_ptr[r + 1]); row_ptr[b * l_d] = number of edges
 *   col_idx  [n_q * b * l_q] int32 (device) output: edge ids, by destination row and by
 *                                           increasing id within a row; only the first
 *                                           row_ptr[b * l_d] entries are written
 * Limits: l_d <= 4096 and n_q * b * l_q < 2^31 (MAXSIM_ERR_UNSUPPORTED beyond).  The result is
 * the same on every run.  argmax must not change while the call is in flight.
 */
int maxsim_csr_build(const int32_t *argmax, int n_q, int64_t b, int l_q, int l_d, int32_t *row_ptr,
                     int32_t *col_idx, void *stream);

/*
 * maxsim_backward with dD taken through the explicit CSR (Alg. 2 as stated: build the CSR from
 * argmax, then one owner per dD row walks that row's edge list).  row_ptr and col_idx are
 * caller-provided device buffers of the sizes maxsim_csr_build states; they are overwritten
 * and hold the CSR afterwards.  dQ, dD, the skipping of negative entries and the fp32
 * accumulation order (a row's edges by increasing id) are those of maxsim_backward, so the two
 * give the same bits.  Limits of maxsim_csr_build and of maxsim_backward apply.
 */
int maxsim_backward_csr(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d,
                        maxsim_dtype dtype, const int32_t *argmax, const float *dscore,
                        int32_t *row_ptr, int32_t *col_idx, float *dQ, float *dD, void *stream);

/*
 * maxsim_backward_csr for callers that cannot allocate device memory at all (code that runs under HIP graph
 * capture, tight serving loops, harnesses that forbid it): the same kernels, with row_ptr and col_idx in a
 * device array that is part of the library's image (9.4 MB, one copy on every GPU the library runs on, held
 * until the process ends) instead of caller buffers.  The call allocates and frees nothing.
 *   Limits: b * l_d <= 262144 rows and n_q * b * l_q <= 2097152 argmax entries (config 4 exactly); larger
 *   sizes return MAXSIM_ERR_SCRATCH and enqueue nothing.  Other arguments, limits, arithmetic and results
 *   as maxsim_backward_csr (identical bits); the CSR itself is not returned.
 *   All calls on one GPU share that GPU's array: two calls whose work overlaps in time on one GPU (different
 *   streams, different host threads) race; calls on one stream are ordered and safe.  Nothing has to be
 *   cleared between calls.  The array's address is looked up by the per-device set-up (maxsim_init, or the first
 *   call of any entry point on the device): no allocation there either.
 */
int maxsim_backward_csr_static(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d,
                               maxsim_dtype dtype, const int32_t *argmax, const float *dscore, float *dQ,
                               float *dD, void *stream);

/*
 * Per-token symmetric absmax quantiser (Sec. "Quantised Scoring").
 *   X      [rows, d] dtype
 *   X_i8   [rows, d] int8    round_half_even(x / scale), clamped to [-127, 127]
 *   scale  [rows]    float32 absmax / 127 (IEEE fp32 division); an all-zero row gets scale 0, codes 0
 */
int maxsim_quantize_rows_i8(const void *X, int64_t rows, int d, maxsim_dtype dtype, int8_t *X_i8,
                            float *scale, void *stream);

/*
 * int8 x int8 scoring with deferred dequantisation (Alg. 4; App. "INT8 Kernel").
 *   Q_i8 [n_q, l_q, d] int8, q_scale [n_q, l_q] float32
 *   D_i8 [b,   l_d, d] int8, d_scale [b,   l_d] float32   (scales must be >= 0; a nonzero
 *        scale below 2^-100 may cost the last bit of a negative score)
 *   scores [n_q, b] float32;  l_q <= 1024, b * l_d < 2^31
 * Per cell: n = exact int32 dot product; v = fl32(n * d_scale[j]); m_i = max_j v;
 * r_i = fl32(q_scale[i] * m_i); score = sum_i r_i carried in fp64 and rounded once to fp32.
 * The result is a pure function of the inputs (bitwise reproducible).
 */
int maxsim_forward_i8(const int8_t *Q_i8, const float *q_scale, int n_q, int l_q,
                      const int8_t *D_i8, const float *d_scale, int64_t b, int l_d, int d,
                      float *scores, void *stream);

/*
 * int8 scoring of a packed ragged corpus (Sec. "Ragged corpora and kernel family" applied to Alg. 4).
 *   D_i8_packed    [total_tokens, d] int8, d_scale_packed [total_tokens] float32
 *   doc_offsets    [b + 1] int32 (device), as in maxsim_forward_ragged; total_tokens < 2^31
 * A document of length 0 gets score -inf.  Arithmetic and other arguments as in maxsim_forward_i8.
 */
int maxsim_forward_i8_ragged(const int8_t *Q_i8, const float *q_scale, int n_q, int l_q,
                             const int8_t *D_i8_packed, const float *d_scale_packed,
                             const int32_t *doc_offsets, int64_t b, int64_t total_tokens, int d,
                             float *scores, void *stream);

/*
 * Out-of-core int8 scoring: maxsim_forward_i8 with codes and scales in HOST memory, streamed like
 * maxsim_forward_streamed.
 *   D_i8_host [b, l_d, d] int8 and d_scale_host [b, l_d] float32 in HOST memory
 *   staging_codes  DEVICE, 2 * block_docs * l_d * d bytes;  staging_scales  DEVICE, 2 * block_docs * l_d floats
 * Other arguments, limits and arithmetic as in maxsim_forward_i8 (identical bits).
 */
int maxsim_forward_i8_streamed(const int8_t *Q_i8, const float *q_scale, int n_q, int l_q,
                               const int8_t *D_i8_host, const float *d_scale_host, int64_t b, int l_d,
                               int d, int64_t block_docs, int8_t *staging_codes, float *staging_scales,
                               float *scores, void *stream);

/*
 * Gradient of the in-batch-negatives cross-entropy on a score matrix (helper for the
 * contrastive training step; the paper leaves the loss open, this is softmax
 * cross-entropy with temperature tau, label of query i = document i, mean over queries).
 *   scores [n, b] float32 (b >= n);  g [n, b] float32 = (softmax_j(s_i/tau) - [i==j]) / (tau n)
 *   (g may be scores itself: the gradient then takes the scores' place)
 *   loss   [1] float32 or NULL
 */
int maxsim_ce_grad(const float *scores, int n, int b, float tau, float *g, float *loss,
                   void *stream);

/*
 * Operators of the model that makes the embeddings: rotary positions, attention over packed sequences with its
 * gradient, and the clipping of gradients by their global norm.  The sequences are laid out as the packed corpus
 * of maxsim_forward_ragged is: token rows back to back, with int32 offsets on the device.
 *
 * Packed tensors [tokens, heads, d] of these entry points may be views (slices of a fused projection, transposed
 * heads): strides are counted in elements, the innermost one is 1.  Rows of an output lie apart: a token's heads
 * before the next token or a head's tokens before the next head; other strides are refused.
 */

/*
 * Rotary positions.  For token t at position p(t), and i = 0 .. rot / 2 - 1, the pair (x_i, x_j) of every head becomes
 *     y_i = scale (x_i cos a - x_j sin a),  y_j = scale (x_i sin a + x_j cos a),  a = p(t) * freqs[i],
 * with j = i + rot / 2 or, with `neighbours`, the pair (2 i, 2 i + 1).  Entries from rot on are copied.  With
 * `inverse` the angle's sign is turned: the transposed map, hence the gradient of the forward one.
 *   X, Y       [tokens, heads, d] dtype    Y may be X, with X's strides (and is otherwise apart from it)
 *   freqs      [rot / 2] float32           angle per position; 2 <= rot <= d, even, rot <= 4096
 *   positions  [tokens] int32 or NULL      p(t); NULL: the place of t in its sequence
 *   offsets    [b + 1] int32 or NULL       the sequences (not looked at where positions are given); NULL: one sequence
 *   scale      the factor that long-context scalings apply beside their frequencies, 1 otherwise
 * Angles are reduced in 64 bits, the rotation is computed in fp32 and rounded once.  Rows whose addresses and strides are
 * multiples of 16 bytes are moved in such pieces; others are taken entry by entry.
 */
int maxsim_rope(const void *X, int64_t tokens, int heads, int d, int64_t x_token_stride, int64_t x_head_stride,
                maxsim_dtype dtype, const float *freqs, int rot, const int32_t *positions, const int32_t *offsets,
                int64_t b, float scale, int neighbours, int inverse, void *Y, int64_t y_token_stride,
                int64_t y_head_stride, void *stream);

/*
 * Attention over b packed sequences: of sequence i, queries q_offsets[i] .. q_offsets[i + 1] see keys
 * k_offsets[i] .. k_offsets[i + 1] (the same offsets for a whole prompt; few queries against many kept keys and
 * values when serving).
 *     O = softmax(scale Q K^T + mask) V,   lse = log sum exp of the masked scores
 *   Q, O  [q_tokens, hq, d],  K, V [k_tokens, hkv, d]   fp16 or bf16; query head h reads key head h / (hq / hkv)
 *   strides  HOST int64 [8]: token and head stride of Q, K, V, O in this order, multiples of 8 and token strides below
 *         2^24; NULL: all without gaps.  Base pointers are multiples of 16 bytes.
 *   q_offsets, k_offsets [b + 1] int32 (device), as doc_offsets in maxsim_forward_ragged (they may be the same array); sequences may be
 *         empty.  A sequence's keys end where the next one's begin: kept keys cannot grow in place.
 *   hq    a multiple of hkv;  d  a multiple of 8 up to 256;  10^-30 < scale < 10^30
 *   causal  nonzero: the last query sees all keys, the one before it all but the last, and so on
 *           (query t of lq sees keys j <= t + lk - lq).  Zero: all queries see all keys of their sequence.
 *   lse   [q_tokens, hq] float32 or NULL
 *   workspace  maxsim_attention_workspace(...) bytes (device, 16-byte aligned); may be NULL where that is 0
 * A query that sees no key gets O = 0 and lse = -inf.  Scores, the softmax's maximum and sum and the sums over keys are
 * fp32; probabilities are rounded to the inputs' type before they multiply V (in fp16 to 2^-32 of the largest at
 * the finest).  The result is the same on every run.  O lies apart from the inputs.
 * Inputs are finite, as everywhere here.  What is not stays in its sequence: another sequence's results are what they were, and
 * a NaN among the keys that a query sees makes its lse NaN.  Within the sequence a key behind the causal mask does not
 * reach a query, but a value behind it has weight 0 in the products, which an infinity or a NaN does not survive.
 */
int64_t maxsim_attention_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d);
int maxsim_attention(const void *Q, const void *K, const void *V, const int64_t *strides, const int32_t *q_offsets,
                     const int32_t *k_offsets, int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d,
                     maxsim_dtype dtype, int causal, float scale, void *O, float *lse, void *workspace,
                     int64_t workspace_bytes, void *stream);

/*
 * Gradient of maxsim_attention: with P the probabilities and delta = sum_d dO O,
 *     dV = P^T dO,   dS = P (dO V^T - delta),   dQ = scale dS K,   dK = scale dS^T Q  (summed over a key head's queries)
 *   O, lse  as maxsim_attention left them;  dO [q_tokens, hq, d] the upstream gradient
 *   dQ [q_tokens, hq, d], dK, dV [k_tokens, hkv, d]  in the inputs' type, every row fully overwritten (zeros where there is nothing)
 *   strides  HOST int64 [16]: token and head stride of Q, K, V, O, dO, dQ, dK, dV, as above; NULL: all without gaps
 *   workspace  maxsim_attention_backward_workspace(...) bytes (device, 16-byte aligned)
 * Sums are fp32 in a fixed order (no atomics): the same bits on every run.  P and dS are rounded to the inputs' type
 * before they enter the last products (dS in two parts for dQ, except in causal rows of more than 512 keys whose sequence begins
 * with its first query), so that fp16 gradients want the usual loss scale: what is below 3e-8 in P or dS is lost.  P is computed
 * again from the scores and lse: it is as exact as fp32 is at the size of the scores (2^-24 of them, in the exponent).  The
 * gradients lie apart from the inputs and from each other.
 */
int64_t maxsim_attention_backward_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d);
int maxsim_attention_backward(const void *Q, const void *K, const void *V, const void *O, const float *lse,
                              const void *dO, const int64_t *strides, const int32_t *q_offsets,
                              const int32_t *k_offsets, int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv,
                              int d, maxsim_dtype dtype, int causal, float scale, void *dQ, void *dK, void *dV,
                              void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Clipping by the global norm:  norm = sqrt(sum of all gradients' squares),  out_i = min(1, max_norm / (norm + 1e-6)) g_i.
 *   grads, out  HOST arrays of n device pointers (out[i] may be grads[i]: in place); tensors without gaps, aligned to their elements,
 *               which otherwise lie apart from each other
 *   numel       HOST int64 [n], may be 0;  dtypes  HOST int32 [n], maxsim_dtype of grads[i] and out[i]
 *   norm        [1] float32 (device); inf where the norm is beyond fp32 (the factor is right all the same)
 *   workspace   maxsim_clip_workspace(n) bytes (device, 16-byte aligned)
 * The arrays on the host may be reused when the call returns.  Squares are added in fp64 in a fixed order.  A gradient that
 * is not finite shows in the norm and, as in the formula, in every product with the factor 0 or NaN that it makes.
 */
int64_t maxsim_clip_workspace(int n);
int maxsim_clip_grad_norm(const void *const *grads, void *const *out, const int64_t *numel, const int32_t *dtypes,
                          int n, float max_norm, float *norm, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MAXSIM_H */
