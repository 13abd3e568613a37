/* SQuant weight-quantization solver for AMD MI355X (gfx950) -- C ABI.
 *
 * Implements the progressive CASE-flipping solver of "SQuant: On-the-Fly Data-Free
 * Quantization via Diagonal Hessian Approximation" (ICLR 2022), Section 3.3-3.4:
 * Algorithm 1 (progressive SQuant), Algorithm 2 (SQuantFlip) and Algorithm 3
 * (perturbation update, Appendix B.3), preceded by the per-output-channel
 * quantization range of Section 4 (symmetric absmax scale) and the
 * scale/clip/round formula of Section 2.2.
 *
 * A weight tensor is W[cout][cin][kh][kw], contiguous, row-major, binary32
 * (Section 2.1: M = cout output channels, N = cin "kernels" per output channel,
 * K = kh*kw elements per kernel; a fully connected layer is kh = kw = 1; for a
 * grouped / depthwise convolution cin is the per-group input channel count).
 *
 * For every output channel m:
 *   scales[m] = max|W[m]| / qmax,  qmax = 2^(bits-1) - 1   (1.0f if the channel is all zero)
 *   x = W / scales[m] (one IEEE division), clamped to [-qmax, qmax]
 *   SQuant-E : code = round-half-even(x), perturbation p = code - x      (Eq. 5)
 *   SQuant-K : per kernel, flip the k = round(|sum p|) same-sign elements with
 *              the largest |p| one step against the sum                 (Eq. 6, Alg. 2)
 *   update   : per kernel, keep one flip candidate                      (Alg. 3)
 *   SQuant-C : per channel, flip the candidate of the k_c = round(|sum p|)
 *              same-sign kernels with the largest candidate |p|         (Eq. 7, Alg. 2)
 * Perturbations are held in Q23 fixed point (steps of 2^-23) and summed as integers, an exact half
 * in round(|sum|) takes the fewer flips, and ties in a top-k go to the lowest
 * index, so the result does not depend on launch geometry and is reproducible
 * bit for bit.
 *
 * Conventions for every entry point
 *   - pointers named d_* are DEVICE pointers (HIP), h_* are HOST pointers;
 *   - the caller owns every buffer; the library allocates no device memory and keeps
 *     no state between calls;
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream); calls
 *     enqueue work and return; outputs are valid once the stream has been synchronised;
 *     the calls only launch kernels (no allocation, no memset, no host synchronisation),
 *     so they may be captured into a HIP graph;
 *   - codes must not alias the weights; inputs must be finite (NaN/Inf: memory
 *     safe, result unspecified);
 *   - arguments are checked on the host before anything is launched and an
 *     integer status is returned (never an exception or abort).
 */
#ifndef SQUANT_H_
#define SQUANT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Which stages run (Section 4.3 ablation names E, E&K, E&K&C, E&C). */
typedef enum {
  SQUANT_MODE_E = 0,   /* rounding only */
  SQUANT_MODE_EK = 1,  /* + kernel-wise flip */
  SQUANT_MODE_EKC = 2, /* + output-channel-wise flip (the full method) */
  SQUANT_MODE_EC = 3   /* channel-wise flip on the rounded weights, no kernel-wise flip */
} squant_mode_t;

typedef enum {
  SQUANT_OK = 0,
  SQUANT_ERR_NULL = 1,      /* a required pointer is NULL */
  SQUANT_ERR_SHAPE = 2,     /* a dimension is <= 0, or the sizes overflow */
  SQUANT_ERR_BITS = 3,      /* bits outside [2, 8] */
  SQUANT_ERR_MODE = 4,      /* unknown mode, activation or kept form, or a pair of them that does not go together */
  SQUANT_ERR_WORKSPACE = 5, /* a workspace size without a workspace pointer, or too small or misaligned a workspace */
  SQUANT_ERR_DEVICE = 6,    /* a HIP call failed */
  SQUANT_ERR_UNSUPPORTED = 7, /* not returned by this version: every channel within the shape limits is taken */
  SQUANT_ERR_FORMAT = 8     /* unknown weight or output type, or a buffer misaligned for its element type */
} squant_status_t;

/* What the solver writes for each weight (squant_quantize_ex).  Section 2.2 defines the
 * quantised weight as an integer code times the scale and Algorithm 1 returns that
 * product; a deployment stores the codes, and at 4 bits and below two of them fit a byte.
 *   INT8  one int8 code per weight, the tensor's own layout.
 *   INT4  bits <= 4 only.  Output channel m occupies bytes [m*R, (m+1)*R) with
 *         R = (cin*kh*kw + 1) / 2; byte j of a row holds element 2j in its low nibble and
 *         element 2j+1 in its high nibble, each the code's 4-bit two's complement; the
 *         unused high nibble of an odd row's last byte is 0.
 *   F32   the dequantised weight (float)code * scales[m] (one binary32 multiply), the
 *         tensor's own layout.
 *   BF16  that binary32 product rounded to bfloat16 (round to nearest, ties to even),
 *         2 bytes per weight, the tensor's own layout. */
typedef enum {
  SQUANT_OUT_INT8 = 0,
  SQUANT_OUT_INT4 = 1,
  SQUANT_OUT_F32 = 2,
  SQUANT_OUT_BF16 = 3
} squant_output_t;

/* Element type of the weights handed in.  The solver's arithmetic is binary32 whatever the
 * type: binary16 and bfloat16 weights are widened exactly first. */
typedef enum {
  SQUANT_W_F32 = 0,
  SQUANT_W_F16 = 1,  /* IEEE binary16 */
  SQUANT_W_BF16 = 2  /* bfloat16: the upper 16 bits of a binary32 */
} squant_wtype_t;

/* One weight tensor of a batched call. */
typedef struct {
  const void* w;             /* in : device, cout*cin*kh*kw weights (binary32 unless the call says otherwise) */
  void* codes;               /* out: device; int8 codes in [-qmax, qmax], same count and layout as w,
                                unless the call names another squant_output_t */
  float* scales;             /* out: device, cout binary32 */
  int32_t cout, cin, kh, kw;
} squant_tensor_t;

/* Quantize one tensor (Algorithm 1 over all output channels).
 * d_w [cout*cin*kh*kw] in, d_codes [same count] out, d_scales [cout] out. */
int squant_quantize(const float* d_w, int32_t cout, int32_t cin, int32_t kh, int32_t kw,
                    int32_t bits, squant_mode_t mode, int8_t* d_codes, float* d_scales,
                    void* stream);

/* Device bytes squant_quantize_batched asks for as workspace: 0.  The kernels carry the
 * tensor descriptors in their kernel arguments (up to 256 per launch) and need no memory
 * beyond the inputs and outputs; the size calls and the workspace arguments stay in the
 * signatures so that callers written against them keep working. */
size_t squant_batched_workspace_bytes(int32_t n_tensors);

/* Quantize a set of tensors (the layers of a network are independent, Section 4.2)
 * with a few launches for the whole set instead of one per tensor.
 * h_tensors: HOST array of n_tensors descriptors holding DEVICE pointers; it may be
 * freed or reused as soon as the call returns.  d_workspace / workspace_bytes: may be
 * NULL / 0 (squant_batched_workspace_bytes is 0); a buffer that is passed is neither read
 * nor written; a size without a pointer is SQUANT_ERR_WORKSPACE.  n_tensors = 0 is a no-op. */
int squant_quantize_batched(const squant_tensor_t* h_tensors, int32_t n_tensors, int32_t bits,
                            squant_mode_t mode, void* d_workspace, size_t workspace_bytes,
                            void* stream);

/* Bytes of the output buffer of one tensor in the given format (0 on invalid arguments). */
size_t squant_output_bytes(int32_t cout, int32_t cin, int32_t kh, int32_t kw, squant_output_t output);

/* squant_quantize / squant_quantize_batched with the weight type and the output format
 * chosen by the caller (Algorithm 1; Section 2.2 for the dequantised form).  d_w holds
 * cout*cin*kh*kw elements of `wtype`, aligned to their size; d_out is a buffer of
 * squant_output_bytes() bytes, aligned to 4 bytes for F32 and to 2 for BF16 output; in the batched call the
 * `w` and `codes` members of each descriptor play these two roles and every tensor shares
 * wtype and output.  SQUANT_OUT_INT4 needs bits <= 4 (SQUANT_ERR_BITS otherwise).  With
 * SQUANT_W_F32 and SQUANT_OUT_INT8 the calls are the plain ones above. */
int squant_quantize_ex(const void* d_w, squant_wtype_t wtype, int32_t cout, int32_t cin,
                       int32_t kh, int32_t kw, int32_t bits, squant_mode_t mode,
                       squant_output_t output, void* d_out, float* d_scales, void* stream);
int squant_quantize_batched_ex(const squant_tensor_t* h_tensors, int32_t n_tensors,
                               squant_wtype_t wtype, int32_t bits, squant_mode_t mode,
                               squant_output_t output, void* d_workspace, size_t workspace_bytes,
                               void* stream);

/* Activation ranges without data (Section 4, experimental set-up: a wide, batch-norm based
 * range per activation tensor, clipped per tensor).  The output of a batch-norm layer is
 * taken as N(beta_c, gamma_c^2) per channel c, so channel c spans
 * [beta_c - n_sigma*|gamma_c|, beta_c + n_sigma*|gamma_c|] (each bound: one binary32 multiply,
 * one add / subtract); the tensor's range is [min_c, max_c] of these, with the lower end (and
 * the upper, should it be negative) raised to 0 when a ReLU follows.  The uniform quantizer
 * on that range with 2^bits levels: scale = (hi - lo) / (2^bits - 1) (1.0f for an empty range),
 * zero_point = round-half-even(-lo / scale) clamped to [0, 2^bits - 1]. */
typedef struct {
  const float* gamma;  /* in : device, `channels` binary32 batch-norm weights */
  const float* beta;   /* in : device, `channels` binary32 batch-norm biases */
  int32_t channels;
  int32_t relu;        /* non-zero: a ReLU follows the batch norm */
} squant_bn_t;

typedef struct {
  float lo, hi, scale;
  int32_t zero_point;
} squant_act_range_t;

/* Device bytes squant_activation_ranges asks for as workspace: 0 (the layer descriptors
 * travel in the kernel arguments, 256 per launch). */
size_t squant_activation_workspace_bytes(int32_t n_layers);

/* h_layers: HOST array of n_layers descriptors holding DEVICE pointers (reusable as soon as
 * the call returns); d_ranges: device, n_layers results; d_workspace as for
 * squant_quantize_batched (may be NULL / 0).
 * bits in [2, 16], n_sigma finite and >= 0 (SQUANT_ERR_BITS / SQUANT_ERR_SHAPE otherwise). */
int squant_activation_ranges(const squant_bn_t* h_layers, int32_t n_layers, float n_sigma,
                             int32_t bits, squant_act_range_t* d_ranges, void* d_workspace,
                             size_t workspace_bytes, void* stream);

/* One layer of a network: its weight tensor and, where a batch norm follows it, that
 * layer's parameters (bn.gamma == NULL: no activation range for this layer). */
typedef struct {
  squant_tensor_t weight;
  squant_bn_t bn;
} squant_layer_t;

/* Device bytes squant_quantize_network asks for as workspace: 0. */
size_t squant_network_workspace_bytes(int32_t n_layers);

/* The data-free pipeline of Section 4 for a whole network in one call: every weight tensor
 * through the SQuant solver (binary32 weights, int8 codes, as squant_quantize_batched) and
 * every batch-norm output through squant_activation_ranges, on the same stream.  d_ranges
 * holds n_layers entries; entry i is written only when layer i has batch-norm parameters. */
int squant_quantize_network(const squant_layer_t* h_layers, int32_t n_layers, int32_t weight_bits,
                            squant_mode_t mode, int32_t act_bits, float n_sigma,
                            squant_act_range_t* d_ranges, void* d_workspace,
                            size_t workspace_bytes, void* stream);

/* Largest cin*kh*kw one output channel may have: 2^30, the bound of the shape check (0 for an
 * invalid kernel size).  Channels that fit none of the kernels which keep a channel on chip
 * (3x3 beyond cin 4096, other kernel sizes beyond about 32 K elements, 1x1 / FC rows beyond
 * about 160 K elements or off 16-byte alignment beyond 64 K) go through a streaming kernel
 * that walks the weights several times: correct for any shape, a fraction of the speed. */
int64_t squant_max_channel_elems(int32_t kh, int32_t kw);

/* ---------------------------------------------------------------------------
 * Operators on quantised layers: products with the solver's codes, their gradients, and the
 * cross entropy over a vocabulary whose output embedding is codes.  No weights are dequantised to memory.
 *
 * Element type: the activations' type, binary32, binary16 or bfloat16 (squant_wtype_t), shared by all
 * activation buffers of a call (x, bias, residual, y, dy, dx, dbias).  Codes times activations are
 * multiplied exactly (binary32 activations to 22 bits) and added in binary32; the outputs of a forward
 * call are rounded once.  dx and dh are rounded twice: what is multiplied by the codes is held in 11 bits
 * (binary32: 22), which for binary16 is as much again as the output's own rounding.  Rows may be any
 * distance apart (ld*, in elements, at least the row's length); activation buffers need the alignment of
 * their element type, codes none.  Where codes or rows do not lie as the matrix units' kernels read them
 * (cin a multiple of 64, 16-byte aligned; few rows: anything goes) a call copies them to its workspace
 * first.
 *
 * d_workspace: the *_workspace_bytes call's amount (which depends on the shapes, on ldx or ldh and on
 * whether x or h and the codes are 16-byte aligned; 0 for many calls, NULL then), 256-byte aligned, not
 * shared with a call that may run at the same time; it holds nothing between calls.  rows = 0 is a no-op,
 * apart from d_dbias, which becomes 0.  A call of which a launch would need 2^32 threads (among others the
 * loss of 2^24 rows, and a layer of as many binary32 rows) is refused with SQUANT_ERR_SHAPE before its
 * first launch, and its amount of workspace is 0.  The calls launch kernels only and may be captured into
 * a HIP graph.  Infinities and NaN in the activations act as IEEE arithmetic has it (an infinity times a code of
 * 0 is NaN, and a row that holds one may be NaN where exact arithmetic has an infinity). */

/* A quantised layer: codes as squant_quantize_ex writes them for SQUANT_OUT_INT8 or SQUANT_OUT_INT4,
 * rows of cin codes (cin * kh * kw of a convolution's unfolded input). */
typedef struct {
  const void* codes;      /* device */
  const float* scales;    /* device, cout binary32 */
  int32_t cout, cin;
  squant_output_t format; /* SQUANT_OUT_INT8 or SQUANT_OUT_INT4 */
} squant_codes_t;

typedef enum {
  SQUANT_ACT_NONE = 0,
  SQUANT_ACT_RELU = 1,
  SQUANT_ACT_GELU = 2, /* z * Phi(z), Phi the normal distribution's */
  SQUANT_ACT_SILU = 3  /* z / (1 + exp(-z)) */
} squant_activation_t;

/* How the pre-activation z is kept for the backward pass.
 *   INT8  [rows][cout] int8 and [rows][ceil(cout / 64)] binary32 scales: 64 columns of a row share
 *         scale = max|z| / 127 (1 where all are 0), code = round-half-even(z * (127 / max|z|)).  A NaN
 *         or an infinity among them makes the scale one.
 *   FULL  [rows][cout] of the element type. */
typedef enum {
  SQUANT_KEEP_NONE = 0,
  SQUANT_KEEP_INT8 = 1,
  SQUANT_KEEP_FULL = 2
} squant_keep_t;

/* y[m][n] = act(z[m][n]) + residual[m][n],  z[m][n] = scales[n] * sum_k x[m][k] * codes[n][k] + bias[n].
 * d_bias [cout], d_residual [rows][cout] (ldr) and, with SQUANT_KEEP_NONE, d_kept may be NULL;
 * d_kept_scales only with SQUANT_KEEP_INT8.  d_y may be d_residual (ldy == ldr) and overlaps nothing else. */
size_t squant_linear_workspace_bytes(const void* d_x, int64_t ldx, squant_wtype_t type, int64_t rows,
                                     const squant_codes_t* h_w, squant_keep_t keep);
int squant_linear(const void* d_x, int64_t ldx, squant_wtype_t type, int64_t rows,
                  const squant_codes_t* h_w, const void* d_bias, squant_activation_t act,
                  const void* d_residual, int64_t ldr, void* d_y, int64_t ldy, squant_keep_t keep,
                  void* d_kept, float* d_kept_scales, void* d_workspace, size_t workspace_bytes,
                  void* stream);

/* Gradients of squant_linear, codes and scales held fixed (the residual's is dy itself):
 * dz = dy * act'(z), z as kept;  dx[m][k] = sum_n dz[m][n] * scales[n] * codes[n][k];
 * dbias[n] = sum_m dz[m][n].  d_dbias may be NULL.  With SQUANT_ACT_NONE keep is SQUANT_KEEP_NONE, with
 * the others it is not (SQUANT_ERR_MODE).  dz * scale is held in binary16 with an exponent for each row
 * (11 bits; binary32: 22). */
size_t squant_linear_backward_workspace_bytes(squant_wtype_t type, int64_t rows, const squant_codes_t* h_w);
int squant_linear_backward(const void* d_dy, int64_t lddy, squant_wtype_t type, int64_t rows,
                           const squant_codes_t* h_w, squant_activation_t act, squant_keep_t keep,
                           const void* d_kept, const float* d_kept_scales, void* d_dx, int64_t lddx,
                           void* d_dbias, void* d_workspace, size_t workspace_bytes, void* stream);

/* Softmax cross entropy of hidden states h [rows][cin] against a vocabulary of cout entries, without the
 * logits in memory:  l[t][v] = scales[v] * sum_d h[t][d] * codes[v][d],  lse[t] = log sum_v exp l[t][v],
 * loss[t] = lse[t] - l[t][label[t]];  0 where the label is ignore_index, NaN where it is neither that
 * nor in [0, cout).  loss and lse are binary32. */
size_t squant_cross_entropy_workspace_bytes(const void* d_h, int64_t ldh, squant_wtype_t type,
        int64_t rows, const squant_codes_t* h_w);
int squant_cross_entropy(const void* d_h, int64_t ldh, squant_wtype_t type, int64_t rows,
                         const squant_codes_t* h_w, const int64_t* d_labels, int64_t ignore_index,
                         float* d_loss, float* d_lse, void* d_workspace, size_t workspace_bytes,
                         void* stream);

/* dh[t][d] = dloss[t] * sum over v != y of p[t][v] * (scales[v] * codes[v][d] - scales[y] * codes[y][d])
 * with p = exp(l - lse) and y the label (lse of the call above; its own gradient is not taken), which is the
 * gradient in the form that keeps its precision where the label is likely; 0 where the label is
 * ignore_index, NaN where it is no entry.  p * scale is held in binary16 (11 bits; binary32: 22), or to 2^-38 of
 * the vocabulary's largest scale where that is more.  The vocabulary is walked in pieces whose
 * probabilities are in the workspace: about 256 MB, or 4096 entries of each row where that is more. */
size_t squant_cross_entropy_backward_workspace_bytes(const void* d_h, int64_t ldh, squant_wtype_t type,
        int64_t rows, const squant_codes_t* h_w);
int squant_cross_entropy_backward(const void* d_h, int64_t ldh, squant_wtype_t type, int64_t rows,
                                  const squant_codes_t* h_w, const int64_t* d_labels,
                                  int64_t ignore_index, const float* d_lse, const float* d_dloss,
                                  void* d_dh, int64_t lddh, void* d_workspace, size_t workspace_bytes,
                                  void* stream);

/* ---------------------------------------------------------------------------
 * Attention, and a cache of keys and values in 4 or 8 bits: what a language model of quantised layers has between
 * its projections.
 *
 * Element type (squant_wtype_t): that of queries, keys, values, outputs and gradients of a call.  Over prompts products
 * are taken of the elements as they are and added in binary32, softmax statistics are binary32; what is multiplied by the
 * values (and, in a backward pass, by queries, keys and output gradients) is rounded to the element type first (binary32:
 * not).  Gradients take weights as exp(score - log-sum-exp), which makes them off by 2^-21 |log-sum-exp| (relative), however
 * large scores are.  Every output is rounded once.
 *
 * Over a cache matrix products are of binary16 numbers, with shared powers of two:
 *   elements code * scale: all bits (4-bit codes 11, 8-bit ones 15), but 11 of 8-bit ones in bfloat16 calls;
 *   queries: all bits, binary32 22 (the last of these do not meet the last 4 of an 8-bit element);
 *   weights: 11 bits, binary32 22.
 * What is small against others keeps less: an element is off by up to 2^-24 of the largest scale times qmax, of the head's
 * keys or values, that the row sees; a query's by 2^-35 of its row's largest; a weight by 2^-39 of its row's largest.
 *
 * Rows are tokens.  Sequences lie one after the other: sequence b has the rows starts[b] to starts[b + 1] - 1, starts
 * holding sequences + 1 numbers that begin with 0 and do not fall; sequences may be empty.  Rows from
 * starts[sequences] on belong to no sequence (padding): what is computed for them is 0, nothing is written to a cache for
 * them, and what they hold does not matter.  A row that sees no key gets 0 (and a log-sum-exp of minus infinity); keys and
 * values that a row does not see do not reach its output, whatever they hold.  starts, lengths and tables are read on the
 * device; numbers there that break the rules give unspecified values, never an access out of the buffers.
 *
 * Query heads share key heads in groups: heads is a multiple of the key heads, query head h goes with key head
 * h / (heads / key heads).  No atomics: results are the same from run to run.  The calls launch kernels only and may be
 * captured into a HIP graph.  rows = 0 is a no-op unless said otherwise.  Workspaces as for the calls above.  Results overlap
 * neither each other nor what is read, but attention's output may be its queries' own buffer (the same steps). */

/* [rows][heads][head_dim] elements; a head's elements lie beside each other. */
typedef struct {
  void* data;      /* device, aligned to its element type */
  int64_t row;     /* elements between rows, from head_dim to 2^22, */
  int64_t head;    /* and between heads, from head_dim to 2^31; any number where there is one row or one head */
} squant_heads_t;

/* A paged cache of keys and values.  Codes [pages][heads][page_size][head_dim], int8 (SQUANT_OUT_INT8) or two 4-bit
 * codes a byte (SQUANT_OUT_INT4, as squant_output_t has them); each 32 consecutive elements of a head share a scale,
 * [pages][heads][page_size][head_dim / 32] bfloat16:
 *   scale = max|x| / qmax in binary32, rounded to bfloat16 (qmax = 7 or 127),
 *   code  = round-half-even(x / scale), at most qmax in magnitude; 0 where the scale is 0.
 * A NaN or an infinity among the 32 makes the scale NaN and the codes 0.  The value held is code * scale.
 * head_dim is 32, 64, 96, 128, 192 or 256; codes are aligned to 16 bytes; pages * heads * page_size < 2^31 and
 * heads * head_dim <= 2^17. */
typedef struct {
  void* key_codes;    /* all: device */
  void* key_scales;
  void* value_codes;
  void* value_scales;
  int32_t pages, page_size, heads, head_dim;
  squant_output_t format;
} squant_cache_t;

/* Where sequences lie in a cache, and which of their tokens a call is about.  Token t of sequence b is in slot
 * t % page_size of page table[b][t / page_size].  lengths[b] tokens of it count, the call's own among them: row r of
 * sequence b is token lengths[b] - (starts[b + 1] - r), the rows being its last ones.  starts NULL: one row for each
 * sequence.  A table's entry that is no page, or lengths beyond the table: nothing is written there, and NaN is read.  A row
 * that sees such a token, or one with a scale that is NaN or infinite, is NaN.  For attention a table holds at most 2^30
 * tokens. */
typedef struct {
  const int32_t* table;   /* device, [sequences][table_width] */
  const int32_t* lengths; /* device, [sequences] */
  const int32_t* starts;  /* device, [sequences + 1], or NULL */
  int32_t sequences, table_width;
} squant_paged_t;

/* Quantises keys and values of `rows` tokens, [rows][heads][head_dim], into their slots; other slots stay as they are.
 * A slot that two rows name (a page in two places of the table) holds a mixture of them afterwards. */
int squant_cache_write(const squant_heads_t* h_k, const squant_heads_t* h_v, squant_wtype_t type, int64_t rows,
                       const squant_cache_t* h_cache, const squant_paged_t* h_where, void* stream);

/* The values of these tokens' keys and values, code * scale rounded to the element type.  Rows of no sequence, and tokens
 * before the first, are written as 0. */
int squant_cache_read(const squant_cache_t* h_cache, const squant_paged_t* h_where, squant_wtype_t type, int64_t rows,
                      const squant_heads_t* h_k, const squant_heads_t* h_v, void* stream);

/* out[r][h] = sum_t p[t] value[t],  p = softmax over t of scale * q[r][h] . key[t],  t the tokens up to the row's own
 * (which are in the cache already).  scale is finite and not negative.  For one or a few rows a sequence: 16 or 32 rows
 * times grouped heads share a pass over the cache.  The workspace is about 128 MiB at most. */
size_t squant_cache_attention_workspace_bytes(int64_t rows, int32_t heads, const squant_cache_t* h_cache,
                                              const squant_paged_t* h_where);
int squant_cache_attention(const squant_heads_t* h_q, squant_wtype_t type, int64_t rows, int32_t heads,
                           const squant_cache_t* h_cache, const squant_paged_t* h_where, float scale,
                           const squant_heads_t* h_out, void* d_workspace, size_t workspace_bytes, void* stream);

/* Whole prompts: queries [q_rows][heads][head_dim] against keys and values [k_rows][kv_heads][head_dim].
 * causal: the last row of a sequence sees all of its keys, the row before it one less, and so on. */
typedef struct {
  const int32_t* q_starts; /* device, [sequences + 1], or NULL: one sequence of all rows */
  const int32_t* k_starts; /* the same for keys; both or neither */
  int32_t sequences;
  int64_t q_rows, k_rows;
  int32_t heads, kv_heads, head_dim; /* head_dim a multiple of 8 up to 256 */
  int32_t causal;
  float scale;             /* finite, not negative */
} squant_packed_t;

/* out[r][h] = sum_t p[t] v[t],  lse[h][r] = log sum_t exp(scale * q[r][h] . k[t])  (binary32 [heads][q_rows]; may be NULL). */
size_t squant_attention_workspace_bytes(const squant_packed_t* h_packed, squant_wtype_t type);
int squant_attention(const squant_heads_t* h_q, const squant_heads_t* h_k, const squant_heads_t* h_v, squant_wtype_t type,
                     const squant_packed_t* h_packed, const squant_heads_t* h_out, float* d_lse, void* d_workspace,
                     size_t workspace_bytes, void* stream);

/* Gradients of squant_attention for the output's gradient (lse's own is not taken): with p = exp(scale * q . k - lse),
 * dv = sum p dout,  ds = p (dout . v - dout . out),  dq = scale * sum ds k,  dk = scale * sum ds q, the latter two sums
 * over the query heads of a group as well.  Rows of no sequence get 0.  A NaN or an infinity in a position that a row
 * does not see may make gradients of up to 128 rows beside it NaN.  rows = 0: keys without queries get 0. */
size_t squant_attention_backward_workspace_bytes(const squant_packed_t* h_packed, squant_wtype_t type);
int squant_attention_backward(const squant_heads_t* h_dout, const squant_heads_t* h_q, const squant_heads_t* h_k,
                              const squant_heads_t* h_v, const squant_heads_t* h_out, const float* d_lse,
                              squant_wtype_t type, const squant_packed_t* h_packed, const squant_heads_t* h_dq,
                              const squant_heads_t* h_dk, const squant_heads_t* h_dv, void* d_workspace,
                              size_t workspace_bytes, void* stream);

const char* squant_status_string(int status);
int squant_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SQUANT_H_ */
