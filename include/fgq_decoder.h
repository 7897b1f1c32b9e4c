/*
 * fgq_decoder.h -- C ABI of libfgq's operators for decoders served from quantized state: a paged
 * cache of keys and values held in 4 bits, the attention that reads it, and linear layers on
 * 8-bit integers with a scale for each token and each output channel.
 *
 * The conventions of fgq.h hold: device pointers owned by the caller, calls asynchronous on the
 * given stream, host-detected errors returned, kernel-detected errors in the device error word
 * that fgq_stream_status() reads, per-call temporaries from the library's stream-ordered pool.
 * Empty problems (B, T, P or M equal to 0) are valid and launch nothing.
 *
 * The cache
 *   Each group of `group` consecutive values of one token and kv head is held as 4-bit codes c
 *   with two bf16 parameters; code c stands for lo + s c:
 *     lo = the group's minimum rounded down to bf16,
 *     s  = fp32((maximum - lo) / 15) rounded up to bf16,
 *     c  = fp32((x - lo) / s) rounded half to even, at most 15 (0 where s = 0),
 *   so that the sixteen values span the group and |x - (lo + s c)| <= s / 2 up to fp32 rounding.
 *   bf16 parameters keep fp32's range at 4 bytes a group; rounding outwards keeps the bound.
 *   k_codes, v_codes    uint8 [pages][kv_heads][page_size][head_dim / 2]
 *   k_params, v_params  uint32 [pages][kv_heads][page_size][head_dim / group], lo in the high
 *                       16 bits and s in the low 16 bits
 *   Codes of a row interleave its nb = head_dim / 32 blocks of 32 values, so that one aligned
 *   piece of a row holds what one thread of a matrix instruction multiplies:
 *     keys    32-bit word t nb + j (t = 0..3, j < nb) holds values 32 j + 8 t + i, i = 0..7, in
 *             nibbles 0 4 1 5 2 6 3 7 (i = 0 in nibble 0, i = 1 in nibble 4, ...);
 *     values  16-bit unit g nb + j (g = 0..7) holds values 32 j + 4 g + i in nibble i.
 *   Position p of sequence b lies in slot p % page_size of page page_table[b][p / page_size];
 *   page_table is int32 [B][max_pages], and entries that no call needs may hold anything.  A
 *   needed entry outside [0, pages), or a position outside [0, max_pages page_size), records
 *   FGQ_ERR_ARG; such positions are not written, and what is read for them is unspecified.
 *   head_dim 64, 128 or 256; group 32, 64 or 128, dividing head_dim; page_size a multiple of 16.
 */
#ifndef FGQ_DECODER_H_
#define FGQ_DECODER_H_

#include "fgq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FGQ_F32 = 0, FGQ_BF16 = 1, FGQ_F16 = 2 } fgq_float_type;

typedef struct {
  void* k_codes;   /* the four arrays 16-byte aligned */
  void* k_params;
  void* v_codes;
  void* v_params;
  int pages;
  int page_size;
  int kv_heads;
  int head_dim;
  int group;
} fgq_kv_cache;

/*
 * Quantizes new keys and values into the cache: k[b][i], v[b][i] go to position starts[b] + i of
 * sequence b, for i < lens[b] (lens NULL: i < T).
 *   k, v     elements of `type`, [B][T][kv_heads][head_dim], the last two axes contiguous;
 *            batch_stride and token_stride are in elements and multiples of 16 bytes.
 *   starts   int32 [B];  lens int32 [B] or NULL (entries above T count as T).
 * A group that holds NaN or Inf gets codes and parameters 0, and FGQ_ERR_NONFINITE is recorded.
 * No two positions of one call may share a slot.
 * Errors: FGQ_ERR_ARG (null pointer, negative size, bad cache or type), FGQ_ERR_ALIGN (k, v or a
 * cache array not 16-byte aligned, a stride not a multiple of 16 bytes, an int32 array not 4-byte
 * aligned), FGQ_ERR_UNSUPPORTED (T kv_heads above 2^31 - 1, T above 2^31 - 2^16), FGQ_ERR_CUDA.
 */
fgq_status fgq_kv_append(const fgq_kv_cache* cache, const void* k, const void* v, fgq_float_type type,
                         int B, int T, int64_t k_batch_stride, int64_t k_token_stride,
                         int64_t v_batch_stride, int64_t v_token_stride, const int32_t* page_table,
                         int max_pages, const int32_t* starts, const int32_t* lens,
                         cudaStream_t stream);

/*
 * Reads positions starts[b] + i, i < lens[b] (NULL: i < T), back as the values that their codes
 * stand for: k, v out, elements of `type`, [B][T][kv_heads][head_dim] contiguous, fully written
 * (zeros for i >= lens[b] and for positions that a bad page table entry hides).
 * Errors as fgq_kv_append.
 */
fgq_status fgq_kv_read(const fgq_kv_cache* cache, void* k, void* v, fgq_float_type type, int B, int T,
                       const int32_t* page_table, int max_pages, const int32_t* starts,
                       const int32_t* lens, cudaStream_t stream);

/*
 * Attention of T queries per sequence over the cache, softmax(scale q k^T) v per query head, the
 * q_heads / kv_heads query heads h of kv head h / (q_heads / kv_heads) sharing its keys.
 *   q        elements of `type`, [B][T][q_heads][head_dim], the last two axes contiguous;
 *            strides in elements, multiples of 16 bytes.
 *   seq_lens int32 [B], tokens of each sequence in the cache, the queries' own among them.
 *   q_lens   int32 [B] or NULL (T for every sequence): the queries that sequence b really has
 *            (entries above T count as T).  Query i < q_lens[b] stands at position
 *            seq_lens[b] - q_lens[b] + i.
 *   max_len  an upper bound of seq_lens known on the host (0: max_pages page_size).  It shapes
 *            the launch (and so the order of fp32 sums) only; longer sequences are still read whole.
 *   causal   1: a query sees positions up to its own; 0: all seq_lens[b] positions.
 *   window   with causal, > 0: a query sees at most the last `window` positions, its own among
 *            them; 0: no limit.
 *   out      elements of `type`, [B][T][q_heads][head_dim] contiguous, fully written.  A query
 *            that sees nothing, and i >= q_lens[b], give zeros (whatever they hold).  A head of a
 *            query that holds NaN or Inf and sees something gives NaN.
 * Scores, softmax statistics and sums are held in fp32.  The products take fp16 operands: codes
 * are exact; queries are scaled by a power of two per row and are exact for bf16 and fp16 (fp32:
 * two fp16 parts, about 22 bits); probability times value scale is rounded to fp16 (fp32: two
 * parts).  More than eight rows (queries times query heads of a kv head) of bf16 or fp16 queries may
 * run on a second kernel, where that is the faster; it takes keys, values and probabilities as fp16
 * (fp16 queries: two parts of a probability).
 * Queries may have any magnitude, keys up to 1e30; values from 1e-18 to 1e30 that lie within 1e25 of one
 * another in a sequence, or are 0.  Smaller values lose precision (an error of at most 1e-25).
 * Errors: FGQ_ERR_ARG (null pointer, negative size, bad cache or type, kv_heads not dividing
 * q_heads, causal neither 0 nor 1, window < 0, a window without causal, max_len < 0, a scale that is not
 * finite or not above 0), FGQ_ERR_ALIGN as fgq_kv_append (q, out too), FGQ_ERR_UNSUPPORTED (more than
 * 2^31 - 1 blocks of work, rows of the output B T q_heads or positions max_pages page_size, or T
 * q_heads / kv_heads above 2^30), FGQ_ERR_CUDA (also where a temporary cannot be had).
 */
fgq_status fgq_kv_attention(const fgq_kv_cache* cache, const void* q, fgq_float_type type, int B, int T,
                            int q_heads, int64_t q_batch_stride, int64_t q_token_stride,
                            const int32_t* page_table, int max_pages, const int32_t* seq_lens,
                            const int32_t* q_lens, int max_len, int causal, int window, float scale,
                            void* out, cudaStream_t stream);

/*
 * Symmetric 8-bit quantization with one scale per token: x [P][K] of `type`, rows ldx elements
 * apart (ldx >= K), gives q[p][k] = round half to even of fp32(127 x / amax_p) in [-127, 127] and
 * scale[p] = amax_p / 127, amax_p = max_k |x[p][k]|; a row of zeros gives codes and scale 0.  A row
 * that holds NaN or Inf gets codes and scale 0, and FGQ_ERR_NONFINITE is recorded.
 *   q  out, int8 [P][K] contiguous;  scale  out, fp32 [P].  No alignment beyond the element's.
 * Errors: FGQ_ERR_ARG, FGQ_ERR_ALIGN (x or scale not aligned to their elements), FGQ_ERR_UNSUPPORTED
 * (P or K above 2^31 - 2^16), FGQ_ERR_CUDA.
 */
fgq_status fgq_quantize_tokens(const void* x, fgq_float_type type, int P, int K, int64_t ldx, int8_t* q,
                               float* scale, cudaStream_t stream);

/*
 * 8-bit integer matrix product with a scale per token and per output channel:
 *   y[p][m] = scale[p] wscale[m] sum_k q[p][k] wq[m][k] + bias[m]
 *   q int8 [P][K], scale fp32 [P] (as from fgq_quantize_tokens); wq int8 [M][K], wscale fp32 [M]
 *   (as from fgq_quantize_weights_w8); bias fp32 [M] or NULL; y out, `ytype` [P][M] contiguous.
 * The integer sums are exact below 2^24 in magnitude (always for K <= 1040); past that they are cut off
 * to fp32 once in 16 products, an error of at most K 2^-27 sum_k |q wq|.  No alignment beyond the elements'; rows of q and wq that
 * start on 16-byte boundaries (K a multiple of 16) are read fastest.
 * Errors: FGQ_ERR_ARG (null pointer, negative size, bad type), FGQ_ERR_ALIGN (scale, wscale, bias
 * or y not aligned to their elements), FGQ_ERR_UNSUPPORTED (P, K or M above 2^31 - 2^16),
 * FGQ_ERR_CUDA (also where a temporary cannot be had).
 */
fgq_status fgq_gemm_w8a8(const int8_t* q, const float* scale, int P, int K, const int8_t* wq,
                         const float* wscale, int M, const float* bias, void* y, fgq_float_type ytype,
                         cudaStream_t stream);

/*
 * A linear layer: fgq_quantize_tokens of x, then fgq_gemm_w8a8 with y of x's type, the quantized
 * tokens in temporaries of the library.  Results are those of the two calls, also where y takes the place of
 * x.  (No other output of this header may overlap what its call reads.)
 */
fgq_status fgq_linear_w8a8(const void* x, fgq_float_type type, int P, int K, int64_t ldx, const int8_t* wq,
                           const float* wscale, int M, const float* bias, void* y, cudaStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FGQ_DECODER_H_ */
