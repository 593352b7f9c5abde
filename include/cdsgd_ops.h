/*
 * cdsgd_ops.h -- what a training step needs next to the compressed gradient exchange of cdsgd.h: the
 * norm of a layer list's gradients, AdamW over the list with states in 32 or in 8 bits, and matrices in
 * microscaled 4-bit floating point (MXFP4) with the products of linear layers, forward and backward.
 *
 * The conventions are those of cdsgd.h: DEVICE pointers owned by the caller unless a parameter says
 * "host", a stream as void*, a cdsgd_status returned, arguments checked on the host before anything is
 * enqueued, nothing synchronised.  Outputs must not overlap inputs or other outputs (CDSGD_ERR_ALIAS).
 * Results do not depend on the launch shape, and are the same bit for bit from run to run.
 */
#ifndef CDSGD_OPS_H
#define CDSGD_OPS_H

#include "cdsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of tensors: the values of cdsgd_grad_dtype (CDSGD_GRAD_F32, CDSGD_GRAD_BF16, CDSGD_GRAD_F16). */

/*
 * Norm of a list of gradients, for clipping.  With s = grad_scale and the sum over every element of the list,
 *   out[0] = norm = sqrt(sum (s g)^2)
 *   out[1] = norm > max_norm ? max_norm / norm : 1
 * Squares, sums and both results are formed in 64 bits, where no finite 32-bit gradient overflows, and rounded once; the sum's
 * order is fixed by the list.  out[0] is not finite if the list holds a NaN or an infinity, and also if the norm itself is above the
 * largest fp32 number, though every gradient is finite; out[1] is right then, but a step that takes the two is skipped.
 *   grads, sizes  host arrays [num_tensors]: device pointers (16-byte aligned) and element counts (> 0)
 *   grad_dtype    a cdsgd_grad_dtype
 *   out           out fp32[2], 4-byte aligned, apart from the gradients (CDSGD_ERR_ALIAS)
 *   max_norm      > 0; INFINITY computes the norm alone (out[1] = 1)
 * The handle keeps a table and the partial sums in one device allocation and borrows the gradients: calls on
 * one handle must be ordered (same stream, or events).
 */
typedef struct cdsgd_grad_norm cdsgd_grad_norm;
int cdsgd_grad_norm_create(const void *const *grads, const size_t *sizes, int num_tensors, int grad_dtype,
                           cdsgd_grad_norm **out);
int cdsgd_grad_norm_compute(cdsgd_grad_norm *norm, double grad_scale, double max_norm, float *out, void *hip_stream);
int cdsgd_grad_norm_destroy(cdsgd_grad_norm *norm);

/*
 * One AdamW step (decoupled weight decay) over a layer list, one launch for all tensors.  Per element, in
 * fp32 and in this order, each operation rounded by itself:
 *   g = grad * (grad_scale * clip[1])
 *   m = m * beta1 + g * (1 - beta1)
 *   v = v * beta2 + (g * g) * (1 - beta2)
 *   weight = weight * (1 - lr * weight_decay)
 *          - (m / (sqrt(v) * (1 / sqrt(1 - beta2^step)) + eps)) * (lr / (1 - beta1^step))
 * (square root and reciprocal to one unit in the last place).  The factors are formed in 64 bits and rounded once;
 * where there is no clip, its factor is 1.  If clip[0] is not finite the pass writes nothing at all: a step whose
 * gradients overflowed is skipped, as under a loss scale.
 *
 * States in 8 bits.  A tensor's elements form blocks of CDSGD_STATE_BLOCK.  m and v are one byte an element, and
 * m_scale and v_scale one byte a block: the exponent field b of the block's largest magnitude as an fp32 number.
 * With T = 14 for m and T = 30 for v, the code of x is
 *   ((fp32 pattern of |x| * 2^(T - b)) + 16 * d) >> 20
 * (m: 7 bits, and the sign as bit 7; v: 8 bits, at least 1 where x > 0), and it stands for the number with pattern
 * code << 20, times 2^(b - T).  That is a float with 3 mantissa bits and 4 (m) or 5 (v) exponent bits, with
 * denormals, under a power of two.  b = 255 (a NaN or an infinity in the block) reads as NaN throughout the block.
 * All bytes 0 is a state of zeros.  d is the dither, 16 bits for each of the two states:
 *   c = counter of the element: its number in the list (mod 2^32), every tensor beginning at a multiple of
 *       CDSGD_STATE_BLOCK
 *   s = z' ^ (z' >> 32) mod 2^32 where z = seed + 0x9E3779B97F4A7C15, z' = (z ^ (z >> 32)) * 0xD6E8FEB86659FD93 mod 2^64
 *   x = c * 0x9E3779B9 + s;  x = (x ^ (x >> 15)) * 0xBB67AE85;  x = (x ^ (x >> 13)) * 0x6A09E667;  x = x ^ (x >> 16)
 *   d = low half of x for m, high half for v
 * so that a state is right on average: rounded to the nearest code, an average whose weight is 0.999 would never
 * move.  Give every step another seed.  States in 32 bits use neither scales nor seed.
 *
 *   weight        i/o fp32[n]
 *   weight16      out [n] in the gradients' type, a 16-bit copy of the new weights; NULL for none (it must be NULL
 *                 where the gradients are fp32: CDSGD_ERR_PARAM)
 *   grad          in  [n], grad_dtype
 *   m, v          i/o fp32[n] (state_bits 32) or uint8[n] (state_bits 8)
 *   m_scale, v_scale  i/o uint8[cdsgd_state_blocks(n)] (state_bits 8); NULL where state_bits is 32
 *   weight_decay  this tensor's (finite, >= 0)
 * weight, weight16, grad, m and v are 16-byte aligned; what a step writes overlaps no other buffer of the whole
 * list.  The plan copies a table to the device and borrows the buffers; passes of one plan must be ordered.
 *   step          number of this step, from 1 on;  lr, betas, eps, grad_scale: finite, lr >= 0, 0 <= beta < 1,
 *                 eps >= 1e-37 (CDSGD_ERR_PARAM)
 *   clip          in  fp32[2] as cdsgd_grad_norm_compute writes it, apart from what the step writes (CDSGD_ERR_ALIAS), or NULL
 */
#define CDSGD_STATE_BLOCK 256
typedef struct {
    float *weight;
    void *weight16;
    const void *grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    size_t n;
    float weight_decay;
} cdsgd_adamw_tensor;
typedef struct cdsgd_adamw_plan cdsgd_adamw_plan;

size_t cdsgd_state_blocks(size_t n);
int cdsgd_adamw_plan_create(const cdsgd_adamw_tensor *tensors, int num_tensors, int grad_dtype, int state_bits,
                            cdsgd_adamw_plan **out);
int cdsgd_adamw_plan_destroy(cdsgd_adamw_plan *plan);
int cdsgd_adamw_step(cdsgd_adamw_plan *plan, long step, double lr, double beta1, double beta2, double eps,
                     double grad_scale, uint64_t seed, const float *clip, void *hip_stream);
/* cdsgd_grad_norm_compute over the plan's own gradients. */
int cdsgd_adamw_grad_norm(cdsgd_adamw_plan *plan, double grad_scale, double max_norm, float *out, void *hip_stream);
/*
 * The values that 8-bit states stand for, in fp32 or bf16 (four significant bits: exact in either, but for numbers
 * below the type's smallest).  cdsgd_adamw_bind_readout takes host arrays [num_tensors] of device pointers, 16-byte
 * aligned, and their type (CDSGD_GRAD_F32 or CDSGD_GRAD_BF16), copies them into the plan's table with a synchronous
 * copy and borrows the buffers; it may be called again to rebind, while no pass of the plan may be running.
 * CDSGD_ERR_PARAM for a plan with 32-bit states; cdsgd_adamw_read_states without bound buffers is CDSGD_ERR_NULL.
 */
int cdsgd_adamw_bind_readout(cdsgd_adamw_plan *plan, void *const *m_out, void *const *v_out, int dtype);
int cdsgd_adamw_read_states(cdsgd_adamw_plan *plan, void *hip_stream);

/*
 * Matrices in microscaled 4-bit floating point (the MXFP4 of the OCP Microscaling Formats specification 1.0).
 * Values are 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign; 32 values in a row share a power of two.  A matrix of `rows` by
 * `cols` is held in two buffers, with g = ceil(cols / 128):
 *   codes   uint8[rows][64 g]   cdsgd_mxfp4_code_bytes(rows, cols).  Element c of a row is half c % 2 (0: the low one) of byte
 *                               c / 2: magnitude 0..7 in the order above, sign as bit 3.  16-byte aligned.
 *   scales  uint8[g][rows][4]   cdsgd_mxfp4_scale_bytes(rows, cols).  Byte j of (i, r) belongs to elements 128 i + 32 j ... + 31 of
 *                               row r and stands for 2^(byte - 127); 255 is NaN.  4-byte aligned.
 * Everything from `cols` to 128 g is 0.  (Whole rows of 128: a product's loads need no test along the axis that it sums
 * over, and the four scales that a matrix instruction takes for a row are one word.)
 *
 * cdsgd_mxfp4_quantize   of a matrix x: `codes` / `scales` receive it in blocks along its rows, codes_t / scales_t its
 *                        transpose in blocks along the transpose's rows, i.e. down x's columns (a matrix of `cols` by `rows`).
 *                        Either pair may be NULL, not both.  A block's scale is 2^(floor(log2 of the largest magnitude) - 2),
 *                        not below 2^-127; values are rounded to the nearest, ties to the even code, and above 6 they are 6.
 *                        A NaN or an infinity in a block makes its scale NaN.  x may have rows further apart than `cols`
 *                        elements (ld), and needs no more than its own type's alignment.
 * cdsgd_mxfp4_dequantize the values that a matrix stands for, rounded once if the type has not enough bits; out has rows
 *                        ld elements apart.
 * x and out have element type `dtype` (the values of cdsgd_grad_dtype); rows and cols are positive and below 2^31, ld at most 2^40
 * (CDSGD_ERR_SIZE).
 */
size_t cdsgd_mxfp4_code_bytes(size_t rows, size_t cols);
size_t cdsgd_mxfp4_scale_bytes(size_t rows, size_t cols);
int cdsgd_mxfp4_quantize(const void *x, int dtype, size_t rows, size_t cols, size_t ld, uint8_t *codes, uint8_t *scales,
                         uint8_t *codes_t, uint8_t *scales_t, void *hip_stream);
int cdsgd_mxfp4_dequantize(const uint8_t *codes, const uint8_t *scales, size_t rows, size_t cols, void *out, int dtype,
                           size_t ld, void *hip_stream);

/*
 * out[m, n] = sum over k of A[m, k] B[n, k], A (M by K) and B (N by K) as above, summed in fp32 and rounded once to
 * out's type.  A linear layer's forward pass is x w^T with x and w in blocks along their rows; with the transposes that
 * cdsgd_mxfp4_quantize writes, the gradients are dx = dy (w^T)^T, summed over the outputs, and dw = dy^T (x^T)^T, summed over
 * the tokens.  accumulate != 0 adds the product to what out holds (gradients of several micro-batches).
 *   out        [M][ld], element type `dtype`, aligned to its type
 *   workspace  cdsgd_mxfp4_matmul_workspace(M, N, K) bytes, 16-byte aligned, NULL where that is 0: room for the partial
 *              sums of a product with few outputs, whose long axis is split over many workgroups.  Calls that share one
 *              must be ordered; its content means nothing between calls.
 *   M, N       positive, at most 2^29;  K positive, at most 2^24
 *   errors     CDSGD_ERR_SIZE also if workspace_bytes is less than what is needed
 */
size_t cdsgd_mxfp4_matmul_workspace(size_t M, size_t N, size_t K);
int cdsgd_mxfp4_matmul(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes, const uint8_t *b_scales, size_t M,
                       size_t N, size_t K, void *out, int dtype, size_t ld, int accumulate, void *workspace,
                       size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CDSGD_OPS_H */
