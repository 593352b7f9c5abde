/*
 * cdsgd_block.h -- what stands between the products of a transformer block in training: attention over packed sequences, the norms before
 * and after a block with its gate and residual scale, gated activations, each forward and backward, and activations held in 8 bits
 * (MXINT8) from the one pass to the other.
 *
 * The conventions are those of cdsgd.h and cdsgd_ops.h: DEVICE pointers owned by the caller unless a parameter says "host", a stream as
 * void*, a cdsgd_status returned, arguments checked on the host before anything is enqueued, nothing synchronised, nothing allocated.
 * Outputs must not overlap inputs or other outputs (CDSGD_ERR_ALIAS).  Results do not depend on the launch shape, and are the same bit for
 * bit from run to run.  Element types are the values of cdsgd_grad_dtype.  A matrix has `rows` rows of `cols` neighbouring elements,
 * ld >= cols elements apart, and needs no more than its own type's alignment; rows and cols are positive and below 2^31, ld at most 2^40
 * (CDSGD_ERR_SIZE).  The launch's device is the current one, on which the buffers are.
 */
#ifndef CDSGD_BLOCK_H
#define CDSGD_BLOCK_H

#include "cdsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Matrices in 8 bits (the MXINT8 of the OCP Microscaling Formats specification 1.0): 32 elements in a row share a power of two.  With
 * g = ceil(cols / 32):
 *   codes   int8[rows][32 g]   cdsgd_mxint8_code_bytes(rows, cols), 16-byte aligned; 0 behind the end of a row
 *   scales  uint8[rows][g]     cdsgd_mxint8_scale_bytes(rows, cols)
 * An element is code * 2^(s - 133) with its block's s; s = 255 is NaN throughout the block.
 * cdsgd_mxint8_quantize    s is the exponent field of the block's largest magnitude as an fp32 number, the code x * 2^(133 - s) rounded to
 *                          nearest, ties to even, and to 127 at most.  A NaN or an infinity in a block makes its s 255 and its codes 0.
 * cdsgd_mxint8_dequantize  the values, rounded once where the type has no such number (fp16 has none above 65504, and small ones with fewer bits).
 *                          A code of -128, which nothing here writes, is read as -128.
 */
size_t cdsgd_mxint8_code_bytes(size_t rows, size_t cols);
size_t cdsgd_mxint8_scale_bytes(size_t rows, size_t cols);
int cdsgd_mxint8_quantize(const void *x, int dtype, size_t rows, size_t cols, size_t ld, int8_t *codes, uint8_t *scales, void *hip_stream);
int cdsgd_mxint8_dequantize(const int8_t *codes, const uint8_t *scales, size_t rows, size_t cols, void *out, int dtype, size_t ld,
                            void *hip_stream);

/* A matrix that a call reads, as it is or in 8 bits (then codes and scales are set, and p is NULL); all NULL: none. */
typedef struct {
    const void *p;
    size_t ld;
    const int8_t *codes;
    const uint8_t *scales;
} cdsgd_held;

/*
 * y = act(a) * u, in fp32 and rounded once.
 *   CDSGD_ACT_SILU       act(a) = a / (1 + exp(-a))
 *   CDSGD_ACT_GELU_TANH  act(a) = a / 2 * (1 + tanh(sqrt(2 / pi) * (a + 0.044715 a^3)))
 * forward   a8_* and u8_*: where not NULL (all four or none) they receive a and u as cdsgd_mxint8_quantize would write them, for the backward pass
 * backward  da = dy * u * act'(a), du = dy * act(a), at a and u as they are or as 8 bits hold them (both the same way)
 * All matrices are rows by cols, of element type dtype.  An exponential below 2^-126 counts as 0.
 */
typedef enum { CDSGD_ACT_SILU = 0, CDSGD_ACT_GELU_TANH = 1 } cdsgd_act;
int cdsgd_gated_forward(int act, int dtype, size_t rows, size_t cols, const void *a, size_t ld_a, const void *u, size_t ld_u, void *y, size_t ld_y,
                        int8_t *a8_codes, uint8_t *a8_scales, int8_t *u8_codes, uint8_t *u8_scales, void *hip_stream);
int cdsgd_gated_backward(int act, int dtype, size_t rows, size_t cols, const void *dy, size_t ld_dy, const cdsgd_held *a, const cdsgd_held *u,
                         void *da, size_t ld_da, void *du, size_t ld_du, void *hip_stream);

/*
 * The end of one block and the beginning of the next, over rows of `cols` elements:
 *   n = 1 / sqrt(mean(b^2) + eps)                                (block_weight NULL: n = 1, no norm after the block)
 *   h_out = h + scale * gate * block_weight * b * n              (gate or block_weight NULL: 1)
 *   r = 1 / sqrt(mean(h_out^2) + eps)
 *   y = h_out * r * weight
 * and, from h_out, b, n and r as they were saved, with x = h_out r, c = b n, means over a row and sums over the rows:
 *   t = dh_out + r * (dy weight - x mean(dy weight x))           (dh_out NULL: 0)
 *   dh = t;  dweight = sum(dy x)
 *   e = scale gate block_weight t;  db = n * (e - c mean(e c))   (block_weight NULL: db = e)
 *   dblock_weight = scale gate sum(t c);  dgate = scale block_weight sum(t c)
 * h_out is formed in 64 bits and rounded to fp32, and from there to a 16-bit type; r, y and the gradients are formed in fp32 from what was not yet
 * rounded to 16 bits (the sums over rows in parts in fp32, joined in 64 bits) and rounded once.  eps keeps a row of zeros at 0.  Rows that are not
 * finite go as the formulas do: a NaN in h_out makes its row's y NaN; an infinity makes r 0, and y NaN at its place and 0 elsewhere; a NaN or an
 * infinity in b makes that row's y NaN where there is a block_weight.
 *   stream_dtype  of h, h_out, dh_out, dh: CDSGD_GRAD_F32, or dtype, which is that of b, y, dy, db
 *   rstd          fp32[2][rows]: r, and n (the second row is left as it is without a block_weight), from forward to backward
 *   b NULL        there is no block yet: h_out is h and must be NULL, b8, db, gate, block_weight and their gradients too; scale does nothing
 *   h8, b8        where not NULL they receive h_out and b as cdsgd_mxint8_quantize would write them; either, both or none
 *   dblock_weight, dgate  NULL if and only if the weight is.  The weights' gradients, fp32[cols], are stored, not added
 *   workspace     of the backward pass: cdsgd_block_norm_workspace(rows, cols) bytes, 16-byte aligned.  Calls that share one must be ordered
 * Weights and their gradients are fp32 and 4-byte aligned, as rstd is.  cols is at most 16384 (CDSGD_ERR_SIZE).  scale finite, eps finite and
 * >= 0 (CDSGD_ERR_PARAM).
 */
typedef struct {
    int dtype, stream_dtype;
    size_t rows, cols;
    const float *weight, *block_weight, *gate;
    double scale, eps;
} cdsgd_block_norm;

int cdsgd_block_norm_forward(const cdsgd_block_norm *norm, const void *h, size_t ld_h, const void *b, size_t ld_b, void *h_out, size_t ld_h_out,
                             void *y, size_t ld_y, float *rstd, int8_t *h8_codes, uint8_t *h8_scales, int8_t *b8_codes, uint8_t *b8_scales,
                             void *hip_stream);
size_t cdsgd_block_norm_workspace(size_t rows, size_t cols);
int cdsgd_block_norm_backward(const cdsgd_block_norm *norm, const void *dy, size_t ld_dy, const void *dh_out, size_t ld_dh_out,
                              const cdsgd_held *h_out, const cdsgd_held *b, const float *rstd, void *dh, size_t ld_dh, void *db, size_t ld_db,
                              float *dweight, float *dblock_weight, float *dgate, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Attention over a packed batch.  Sequence s has the queries of rows starts_q[s] ... starts_q[s + 1] - 1 and the keys and values of rows
 * starts_k[s] ... starts_k[s + 1] - 1.  Head h reads key head h / (heads / kv_heads).  For query i and key j of a sequence, counted in it,
 *   S = scale * q . k, hidden where causal and j > i + (keys - queries)
 *   lse = log sum exp S;  out = sum over j of exp(S - lse) v
 * A query that sees no key has out = 0 and lse = -infinity, and passes no gradient on.  The backward pass gives
 *   P = exp(S - lse);  dP = dout . v;  dS = P (dP - dout . out)
 *   dq = scale sum over j of dS k;  dk = scale sum over i, heads of dS q;  dv = sum over i, heads of P dout
 * Rows that belong to no sequence are neither read nor written.  A NaN or an infinity of a token reaches no other sequence, no other group of heads,
 * and, with `causal`, of its own sequence only what the formulas lead it to: a key's the queries that see it, a query's its own row and the keys
 * that it sees (and from a row that one key has made NaN all keys that the row sees).  What it does not reach is the same to the bit without it.
 * Products are summed in fp32; P and dS are rounded to the tensors' type as operands of the second products.  Of fp16 tensors they are multiplied by
 * powers of two first, which are divided out again: P by 2^7 over its row's largest in the forward pass (give or take 2^8) and 2^15 in the
 * backward pass, so that what is lost of it beside its rounding is below 2^-32 and 2^-40; dS by one of its row for dq, of its key for dk, up to 2^60,
 * so that nothing overflows on the way and what is lost is below 2^-32 of the largest |dS| that it is summed up with, or below 2^-85.
 * Where a batch has too few rows of queries to fill the card, the forward pass takes their keys in parts, as many as tokens, sequences and heads of the
 * whole batch say: out and lse of a sequence are then the same from run to run, but may be rounded otherwise in another batch (its gradients not).
 *   dtype         CDSGD_GRAD_BF16 or CDSGD_GRAD_F16
 *   dim           elements of a head: a multiple of 8, at most 128
 *   q, out, dout, dq  [tokens_q][heads][dim];  k, v, dk, dv  [tokens_k][kv_heads][dim]: the heads of a token in a row, tokens ld elements
 *                 apart, 16-byte aligned, ld a multiple of 8 and at most 2^20 (CDSGD_ERR_ALIGN, CDSGD_ERR_SIZE)
 *   lse           fp32[heads][tokens_q], natural logarithms; the forward pass takes NULL for none.  The backward pass is given the forward pass's;
 *                 where it is beyond 2800 or so, of which fp32 leaves too few bits, a row's sum is formed from its logits again
 *   starts_q, starts_k  int32[num_seqs + 1], not falling, from 0 or more to tokens_q (tokens_k) or less.  They are not looked at on the host:
 *                 what is out of range is cut to it, and starts that fall give rows of no meaning, but nothing outside the tensors is
 *                 touched.  starts_k NULL: starts_q.  Both NULL: one sequence, all rows (num_seqs 1).
 *   workspace     cdsgd_attention_workspace bytes for either pass, 16-byte aligned, NULL where that is 0.  Calls that share one must be ordered;
 *                 its content means nothing between calls.
 *   errors        CDSGD_ERR_PARAM: dtype, causal not 0 or 1, heads not a multiple of kv_heads, starts_k without starts_q, no starts and
 *                 num_seqs not 1, scale below 1e-30 or above 1e30.  CDSGD_ERR_SIZE: dim, a count of 0, tokens 2^31 and more, num_seqs 2^24 and more,
 *                 heads above 65535, more work than a launch holds, too small a workspace.
 */
typedef struct {
    int dtype, causal;
    size_t tokens_q, tokens_k, num_seqs;
    const int32_t *starts_q, *starts_k;
    int heads, kv_heads, dim;
    double scale; /* from 1e-30 to 1e30 */
} cdsgd_attention;

size_t cdsgd_attention_workspace(const cdsgd_attention *batch, int backward);
int cdsgd_attention_forward(const cdsgd_attention *batch, const void *q, size_t ld_q, const void *k, size_t ld_k, const void *v, size_t ld_v, void *out,
                            size_t ld_out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);
int cdsgd_attention_backward(const cdsgd_attention *batch, const void *dout, size_t ld_dout, const void *q, size_t ld_q, const void *k, size_t ld_k,
                             const void *v, size_t ld_v, const void *out, size_t ld_out, const float *lse, void *dq, size_t ld_dq, void *dk,
                             size_t ld_dk, void *dv, size_t ld_dv, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CDSGD_BLOCK_H */
