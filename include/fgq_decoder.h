/*
 * fgq_decoder.h -- C ABI of libfgq's operators for decoders served from quantized state: a paged
 * cache of keys and values held in 4 bits, the attention that reads it, linear layers on
 * 8-bit integers with a scale for each token and each output channel, linear layers and mixtures of
 * experts on 4-bit weights with a scale for each group, rotary positions, and the norms between blocks.
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

/*
 * Rotary positions.  A head's first `rot` values are rot / 2 pairs, (j, j + rot / 2) with
 * FGQ_ROPE_HALF and (2 j, 2 j + 1) with FGQ_ROPE_INTERLEAVED; pair j at position p turns by
 * p freq_j radians, freq_j = base^(-2 j / rot) changed for long contexts as `scaling` says:
 *   FGQ_ROPE_PLAIN    as it is;
 *   FGQ_ROPE_LINEAR   freq_j / factor;
 *   FGQ_ROPE_BASE     base factor^(rot / (rot - 2)) in the place of base, which divides the slowest pair by factor and
 *                     leaves the fastest (rot = 2: as it is);
 *   FGQ_ROPE_RAMP     with n_j = length freq_j / (2 pi), the turns over the context of `length` that a model was trained
 *                     with, and k = (n_j - low) / (high - low) cut to [0, 1]: k freq_j + (1 - k) freq_j / factor.
 * The table holds rint(2^64 freq_j / (2 pi)), so that the fraction of a turn at any position is an integer product modulo
 * 2^64 and far positions lose nothing (freq_j to 2^-65 of a turn a position).
 */
typedef enum { FGQ_ROPE_HALF = 0, FGQ_ROPE_INTERLEAVED = 1 } fgq_rope_layout;
typedef enum { FGQ_ROPE_PLAIN = 0, FGQ_ROPE_LINEAR = 1, FGQ_ROPE_BASE = 2, FGQ_ROPE_RAMP = 3 } fgq_rope_scaling;

/*
 * Writes the table of rot / 2 entries to HOST memory (no GPU is needed); copy it to the device for fgq_rope.
 * Errors: FGQ_ERR_ARG (null table, rot not even or below 2, base not finite or not above 1, factor not finite or below 1,
 * an unknown scaling; FGQ_ROPE_RAMP: length not above 0, high not above low or either not finite).  factor, length, low and high
 * are looked at where the scaling uses them.
 */
fgq_status fgq_rope_table(int rot, double base, fgq_rope_scaling scaling, double factor, double length, double low,
                          double high, uint64_t* table);

/*
 * Turns the heads of T tokens per sequence: token i < lens[b] (NULL: i < T) of sequence b stands at position starts[b] + i
 * (any int32, and past it; negative ones turn backwards).  x, y: elements of `type`, [B][T][heads][head_dim], the last two axes
 * contiguous, other strides in elements.  Each pair (a, b) becomes magnitude (a cos - b sin, b cos + a sin); inverse
 * 1: the angle is negated (what gradients of the outputs turn by, and the way back where magnitude is 1).
 * Values past rot, and tokens i >= lens[b], are those of x.  y may be x (with its strides), or must not overlap it.
 * Products and sums are fp32, angles within 2^-24 of half a turn, y is rounded once.
 * Errors: FGQ_ERR_ARG (null pointer, negative size, rot not even, below 2 or above head_dim, a bad type, layout or inverse, a
 * magnitude that is not finite, y at x with other strides, strides with which y's tokens overlap), FGQ_ERR_ALIGN (x or y not aligned to their elements,
 * table not 8-byte, starts or lens not 4-byte aligned), FGQ_ERR_UNSUPPORTED (B T heads above 2^31 - 1, head_dim above 65536),
 * FGQ_ERR_CUDA.
 */
fgq_status fgq_rope(const void* x, void* y, fgq_float_type type, int B, int T, int heads, int head_dim,
                    int64_t x_batch_stride, int64_t x_token_stride, int64_t y_batch_stride, int64_t y_token_stride, int rot,
                    fgq_rope_layout layout, const uint64_t* table, float magnitude, int inverse, const int32_t* starts,
                    const int32_t* lens, cudaStream_t stream);

/*
 * What stands between two blocks of a decoder.  For each token, with x a block's output and r the residual stream:
 *   u = post(x)                    a norm of the block's output, or x (post NULL)
 *   s = r + scale gate u           element by element; gate NULL: 1; r NULL: 0
 *   y = pre(s)                     the norm that the next block reads (pre NULL: none, y NULL)
 * norm(z) = z' / sqrt(mean(z'^2) + eps) weight + bias, with z' = z (FGQ_NORM_RMS) or z - mean(z) (FGQ_NORM_LAYER); weight
 * NULL: 1, bias NULL: 0; fp32 [K] both.
 *   x      elements of `type`, [P][K], rows ldx elements apart (ldx >= K).
 *   gate   elements of `type`, rows ldg elements apart; token p takes row p / tokens_per_gate.
 *   r      elements of `rtype`, which is `type` or FGQ_F32, rows ldr apart.
 *   s      out, elements of `rtype`, rows lds apart, or NULL (not written).  May be r, with its stride.
 *   y      out, elements of `type`, [P][K] contiguous.  May be x where that is contiguous.
 * Everything between is fp32 and y is formed from s before it is rounded.  Sums of squares are fp32, of values up to 1e18 in rows of any length.
 * A token that holds NaN gives NaN, one that holds Inf what fp32 gives; other tokens are as without it.
 * Errors: FGQ_ERR_ARG (null pointer, negative size, K = 0, bad types or kind, eps not above 0 or not finite, a scale that is not
 * finite, tokens_per_gate < 1 with a gate, a stride below K, y without pre or pre without y, neither s nor y, y at x or s at r with
 * other strides),
 * FGQ_ERR_ALIGN (not aligned to the elements), FGQ_ERR_UNSUPPORTED (P or K above 2^31 - 2^16), FGQ_ERR_CUDA.
 */
typedef enum { FGQ_NORM_RMS = 0, FGQ_NORM_LAYER = 1 } fgq_norm_kind;
typedef struct {
  const float* weight;
  const float* bias;
  float eps;
  int kind; /* fgq_norm_kind */
} fgq_norm;

fgq_status fgq_add_norm(const void* x, fgq_float_type type, int P, int K, int64_t ldx, const fgq_norm* post, const void* gate,
                        int64_t ldg, int tokens_per_gate, float scale, const void* r, fgq_float_type rtype, int64_t ldr,
                        void* s, int64_t lds, const fgq_norm* pre, void* y, cudaStream_t stream);

/*
 * Weights in 4 bits: `experts` matrices [rows][cols] (1 for a linear layer), a bf16 scale for each group of `group` (32, 64
 * or 128) consecutive columns of a row; nibble n stands for (n - 8) scale.  Both arrays are laid out in tiles of 16 rows and 128
 * columns, RT = ceil(rows / 16) by CT = ceil(cols / 128) of them:
 *   codes   uint8 [experts][RT][CT][1024]: row g + 8 r (g < 8, r < 2), column 32 j + 8 t + i (j, t < 4, i < 8) of the tile is
 *           nibble (0 4 1 5 2 6 3 7)[i] of little-endian 32-bit word ((8 r + g) 4 + t) 4 + j;
 *   scales  bf16 [experts][RT][CT][16][128 / group].
 * So a warp reads a tile as two runs of 512 bytes, and 16 bytes hold what one of its threads multiplies.  What stands for rows and
 * columns past the matrix may be any finite values.  Both arrays 16-byte aligned.
 */
typedef struct {
  const void* codes;
  const void* scales;
  int experts;
  int rows;
  int cols;
  int group;
} fgq_w4;

/* Bytes of codes and of scales of one matrix (0 for sizes below 0 and a bad group). */
size_t fgq_w4_code_bytes(int rows, int cols);
size_t fgq_w4_scale_bytes(int rows, int cols, int group);

/*
 * w fp32 [experts][rows][cols] contiguous to codes -7 .. 7 in the arrays of `out` (written through its pointers): with amax
 * a group's largest magnitude, scale = fp32(amax / 7) rounded up to bf16, code = fp32(w / scale) rounded half to even
 * (0 where the scale is 0).  A group that holds NaN or Inf gets codes and scale 0, and FGQ_ERR_NONFINITE is recorded.
 * Rows and columns past the matrix get codes and scales 0.
 * fgq_read_weights_w4 gives back what codes and scales stand for, fp32, exactly.
 * Errors: FGQ_ERR_ARG (null pointer, a size below 0, a bad group), FGQ_ERR_ALIGN (w not 4-byte, codes or scales not 16-byte
 * aligned), FGQ_ERR_UNSUPPORTED (rows or cols above 2^31 - 2^16, more than 2^31 - 1 tiles in all), FGQ_ERR_CUDA.
 */
fgq_status fgq_quantize_weights_w4(const float* w, const fgq_w4* out, cudaStream_t stream);
fgq_status fgq_read_weights_w4(const fgq_w4* w, float* out, cudaStream_t stream);

/*
 * A linear layer: y[p][m] = sum_k x[p][k] W[m][k] + bias[m].
 *   x    elements of `type`, [P][K] with K = w->cols, rows ldx elements apart (ldx >= K); bias fp32 [M] or NULL.
 *   y    out, elements of `type`, [P][M] contiguous, M = w->rows; may overlap x.
 * Few tokens: codes and 16-bit tokens are exact operands of the products (fp32 tokens: three bf16 parts, exactly), a group's sum
 * takes its scale in fp32, y is rounded once.  More than 16 tokens (fp32: 8) whose product with the
 * number of weights is above about 2^30 (2^27) run on fp16 operands on tcgen05: weights are exact there too within 2^26 of their row's largest scale, bf16 tokens within 2^26 of their largest
 * value (smaller ones are off by at most 2^-39 of it), fp32 tokens within 2^-22 of each value (or 2^-39 of the largest).  Sums
 * of 16 products are cut off at 2^-23 of the sum so far, fp32 tokens' over runs of 256 columns that are added in fp32.  Scales
 * 2^-100 to 2^100 there, and outputs below 2^-100 may be 0.  A token that holds NaN or Inf gives values that are not finite; other
 * tokens are as without it.
 * Errors: FGQ_ERR_ARG (null pointer, negative size, bad type, bad weights, more than one matrix, ldx < K), FGQ_ERR_ALIGN (x or y
 * not aligned to their elements, codes or scales not 16-byte, bias not 4-byte aligned), FGQ_ERR_UNSUPPORTED (P, K or M above
 * 2^31 - 2^16, more than 2^30 - 2^15 fp32 tokens, more than 2^31 - 1 tiles), FGQ_ERR_CUDA (also where a temporary cannot be had).
 */
fgq_status fgq_linear_w4(const void* x, fgq_float_type type, int P, int64_t ldx, const fgq_w4* w, const float* bias, void* y,
                         cudaStream_t stream);

/*
 * The experts that a router picks for each token: logits l[p][e] = sum_k x[p][k] router[e][k], the `top` largest first (equal
 * ones, and NaN, which counts as the smallest: lowest index first), and their weights
 *   FGQ_SCORE_SOFTMAX   exp(l_e) / sum over all experts of exp(l), or over the chosen ones where renormalize is 1;
 *   FGQ_SCORE_SIGMOID   1 / (1 + exp(-l_e)), divided by the chosen ones' sum where renormalize is 1;
 * times scale.  A logit's terms are added in fp32 by runs of eight, and the runs as pairs of fp32, unrounded: it is within 2^-21 of the sum
 * of its terms' magnitudes (terms of random signs: about an fp32 rounding of itself), and is compared so.
 *   router   elements of `rtype`, which is `type` or FGQ_F32, [E][K] contiguous.
 *   ids      out, int32 [P][top];  weights  out, fp32 [P][top].
 * A token that holds NaN gives weights NaN; one that holds Inf what its infinite logits give (softmax: NaN).
 * Errors: FGQ_ERR_ARG (null pointer, negative size, K or E below 1, bad types or score, top outside 1 .. E, renormalize neither 0
 * nor 1, a scale that is not finite, ldx < K), FGQ_ERR_ALIGN, FGQ_ERR_UNSUPPORTED (E above 1024, top above 32, P above 2^29, K above
 * 2^31 - 2^16), FGQ_ERR_CUDA.
 */
typedef enum { FGQ_SCORE_SOFTMAX = 0, FGQ_SCORE_SIGMOID = 1 } fgq_score;

fgq_status fgq_route_tokens(const void* x, fgq_float_type type, int P, int K, int64_t ldx, const void* router,
                            fgq_float_type rtype, int E, int top, fgq_score score, int renormalize, float scale,
                            int32_t* ids, float* weights, cudaStream_t stream);

/*
 * The sum of chosen experts' gated feed-forward layers:
 *   y[p] = sum_j weights[p][j] down_e (silu(gate_e x[p]) * (up_e x[p])),  e = ids[p][j],  silu(a) = a / (1 + exp(-a)).
 *   gate, up   E matrices [F][K], of one group size;  down  E matrices [K][F].
 *   ids        int32 [P][top], entries outside [0, E) are left out (a token without any gives zeros); an expert may be there
 *              twice.  weights  fp32 [P][top].
 *   y          out, elements of `type`, [P][K] contiguous; may be x where that is contiguous.
 * Between the layers values are held to 2^-22, or 2^-39 of a choice's largest (16-bit tokens), or exactly (fp32).  Sums are
 * fp32, in an order that depends on the sizes and on the tokens that share an expert.  Up to 4096 choices are taken at a time; with more
 * than 16 of them for an expert on average (8 of fp32; fewer where rows of more than 4096 leave room for fewer tokens) products run on
 * fp16 operands as those of a linear layer of many tokens, with what is said there, and values between the layers are held as those of 16-bit tokens.
 * Errors: FGQ_ERR_ARG (null pointer, negative size, bad type or weights, sizes that do not fit, top outside 1 .. 32, ldx < K),
 * FGQ_ERR_ALIGN, FGQ_ERR_UNSUPPORTED (E above 1024, K or F above 2^31 - 2^16, more than 2^31 - 1 tiles), FGQ_ERR_CUDA (also
 * where a temporary cannot be had).
 */
fgq_status fgq_experts_w4(const void* x, fgq_float_type type, int P, int64_t ldx, const int32_t* ids, const float* weights,
                          int top, const fgq_w4* gate, const fgq_w4* up, const fgq_w4* down, void* y, cudaStream_t stream);

/*
 * A mixture-of-experts layer: fgq_route_tokens, then fgq_experts_w4, the choice in temporaries of the library.  Results and errors
 * are those of the two calls.
 */
fgq_status fgq_moe_w4(const void* x, fgq_float_type type, int P, int64_t ldx, const void* router, fgq_float_type rtype, int top,
                      fgq_score score, int renormalize, float scale, const fgq_w4* gate, const fgq_w4* up, const fgq_w4* down,
                      void* y, cudaStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FGQ_DECODER_H_ */
