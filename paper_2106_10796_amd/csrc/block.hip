// Norms around a block, gated activations and matrices in 8 bits (include/cdsgd_block.h): the C ABI's host side.  The kernels are in
// kernels_held8.hpp (8 bits, gated activations) and kernels_block_norm.hpp.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "cdsgd_block.h"

#include "host_common.hpp"
#include "tuning.hpp"
#include "device_common.hpp"
#include "host_matrix.hpp"

#include "kernels_block_norm.hpp"
#include "kernels_held8.hpp"

namespace {

inline int check_extents(size_t rows, size_t cols) { return good_extent(rows) && good_extent(cols) ? CDSGD_OK : CDSGD_ERR_SIZE; }
inline bool good_ld(size_t ld, size_t cols) { return ld >= cols && ld <= (size_t)1 << 40; }

// How a launch over a matrix is laid out: 2^lanes_log2 lanes to a row, `rows` rows to a lane.
struct Layout {
    unsigned lanes_log2, rows;
    unsigned long long groups;
};

// Rows to a lane: `many` on large matrices, 1 where that leaves compute units idle.  (8192 x 4096 in bf16, us: quantisation with 4 rows to a
// lane 24.0, 2 18.7; values 18.8, 16.5.)
inline Layout layout_of(size_t rows, size_t cols, unsigned each, unsigned many)
{
    Layout y = {each == 4 ? 3u : 2u, many, 0};
    while (y.lanes_log2 < 6u && ((size_t)each << y.lanes_log2) < cols) ++y.lanes_log2;
    const unsigned long long across = (cols + 64ull * each - 1) / (64ull * each), at_once = 4ull << (6u - y.lanes_log2);
    if (across * ((rows + at_once * many - 1) / (at_once * many)) < 1024) y.rows = 1;
    y.groups = across * ((rows + at_once * y.rows - 1) / (at_once * y.rows));
    return y;
}

// A held matrix that a backward pass reads: status, and whether it is in 8 bits.
inline int check_held(const cdsgd_held *x, size_t rows, size_t cols, int dtype, bool &eight, Span (&spans)[2])
{
    eight = x->codes != nullptr || x->scales != nullptr;
    spans[0] = spans[1] = Span{nullptr, 1, 0, 0};
    if (eight) {
        if (!x->codes || !x->scales) return CDSGD_ERR_NULL;
        if (x->p) return CDSGD_ERR_PARAM;
        if (!aligned(x->codes, 16)) return CDSGD_ERR_ALIGN;
        spans[0] = range_of(x->codes, cdsgd_mxint8_code_bytes(rows, cols));
        spans[1] = range_of(x->scales, cdsgd_mxint8_scale_bytes(rows, cols));
        return CDSGD_OK;
    }
    if (!x->p) return CDSGD_ERR_NULL;
    if (!good_ld(x->ld, cols)) return CDSGD_ERR_SIZE;
    if (!aligned(x->p, bytes_of(dtype))) return CDSGD_ERR_ALIGN;
    spans[0] = matrix_of(x->p, rows, cols, x->ld, dtype);
    return CDSGD_OK;
}

// The longest row: 16 waves of four fours to a lane.  Registers hold all of a row up to 8192 columns (of an fp32 matrix on an fp32 stream, backward, but
// for 3 to 9 of them); beyond, with 128 to a lane, 170 to 240 bytes of a lane's share are in scratch forward and 280 to 410 backward, and every row goes
// through them (2048 x 12288 in bf16 on an fp32 stream, us: 106, 236 of the 44 and 68 that its bytes take).
constexpr size_t kMostCols = 16384;

// Groups of the norm's backward pass, which leave their sums over rows: enough to fill the card, few enough that joining them
// costs little beside the pass (us, pass and join, 8192 x 4096: 1024 groups 113 + 8.7, 512 107 + 6.2; 1003 x 2049: 1003 16 + 9.5, 256 15 + 4.2).
inline unsigned norm_groups(size_t rows, size_t cols)
{
    const size_t most = ((size_t)1 << 21) / cols, want = most < 128 ? 128 : most > 2048 ? 2048 : most;
    const size_t few = rows / 4 < 256 ? (rows < 256 ? rows : 256) : rows / 4;
    return (unsigned)(few < want ? few : want);
}

// Calls f(waves to a row, fours of elements to a lane), both as integral constants, for rows of `cols` elements.  us, forward and backward:
// 8192 x 4096 in bf16 on an fp32 stream, 16 waves of one four 110, 117, 8 of two 94, 104, 4 of four 132, 135; 1003 x 2049 in fp16, saved in
// 8 bits, 16 of one 15.1, 11.8, 8 of two 13.0, 14.8, 4 of four 14.1, 18.9.
template <typename F>
void with_norm_shape(size_t cols, F f)
{
    const size_t units = (cols + 64 * kNormEach - 1) / (64 * kNormEach);
    typedef std::integral_constant<int, 1> i1;
    typedef std::integral_constant<int, 2> i2;
    typedef std::integral_constant<int, 4> i4;
    typedef std::integral_constant<int, 8> i8;
    typedef std::integral_constant<int, 16> i16;
    if (units <= 1) f(i1(), i1());
    else if (units <= 2) f(i2(), i1());
    else if (units <= 4) f(i4(), i1());
    else if (units <= 8) f(i8(), i1());
    else if (units <= 16) f(i8(), i2());
    else if (units <= 32) f(i8(), i4());
    else f(i16(), i4());
}

// Calls f(stream type, type) as integral constants.
template <typename F>
void with_norm_types(const cdsgd_block_norm &n, F f)
{
    with_dtype(n.dtype, [&](auto dt) {
        if constexpr (decltype(dt)::value != kGradF32) {
            if (n.stream_dtype != CDSGD_GRAD_F32) return f(dt, dt);
        }
        return f(std::integral_constant<int, kGradF32>(), dt);
    });
}

int check_norm(const cdsgd_block_norm *n)
{
    if (!n || !n->weight) return CDSGD_ERR_NULL;
    if (!good_dtype(n->dtype) || (n->stream_dtype != CDSGD_GRAD_F32 && n->stream_dtype != n->dtype)) return CDSGD_ERR_PARAM;
    if (!std::isfinite(n->scale) || !std::isfinite(n->eps) || n->eps < 0) return CDSGD_ERR_PARAM;
    const int rc = check_extents(n->rows, n->cols);
    if (rc != CDSGD_OK) return rc;
    if (n->cols > kMostCols) return CDSGD_ERR_SIZE;
    if (!aligned(n->weight, 4) || !aligned(n->block_weight, 4) || !aligned(n->gate, 4)) return CDSGD_ERR_ALIGN;
    return CDSGD_OK;
}

}  // namespace

extern "C" {

size_t cdsgd_mxint8_code_bytes(size_t rows, size_t cols) { return rows * held_groups(cols) * 32u; }
size_t cdsgd_mxint8_scale_bytes(size_t rows, size_t cols) { return rows * held_groups(cols); }

int cdsgd_mxint8_quantize(const void *x, int dtype, size_t rows, size_t cols, size_t ld, int8_t *codes, uint8_t *scales, void *hip_stream)
{
    if (!x || !codes || !scales) return CDSGD_ERR_NULL;
    if (!good_dtype(dtype)) return CDSGD_ERR_PARAM;
    int status = check_extents(rows, cols);
    if (status != CDSGD_OK) return status;
    if (!good_ld(ld, cols)) return CDSGD_ERR_SIZE;
    if (!aligned(x, bytes_of(dtype)) || !aligned(codes, 16)) return CDSGD_ERR_ALIGN;
    const Span out[] = {range_of(codes, cdsgd_mxint8_code_bytes(rows, cols)), range_of(scales, cdsgd_mxint8_scale_bytes(rows, cols))};
    const Span in[] = {matrix_of(x, rows, cols, ld, dtype)};
    if (any_overlap(out, 2, in, 1)) return CDSGD_ERR_ALIAS;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const Layout y = layout_of(rows, cols, kEach<DT>, 2);
        status = in_launches(y.groups, 256, [&](dim3 grid, unsigned first) {
            const auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)hip_stream, static_cast<const Elem<DT> *>(x), ld, (unsigned)rows,
                                   (unsigned)cols, codes, scales, y.lanes_log2, first);
            };
            if (y.rows == 2) launch(k_held8_quantize<DT, 2>);
            else launch(k_held8_quantize<DT, 1>);
        });
    });
    return status;
}

int cdsgd_mxint8_dequantize(const int8_t *codes, const uint8_t *scales, size_t rows, size_t cols, void *out, int dtype, size_t ld, void *hip_stream)
{
    if (!codes || !scales || !out) return CDSGD_ERR_NULL;
    if (!good_dtype(dtype)) return CDSGD_ERR_PARAM;
    int status = check_extents(rows, cols);
    if (status != CDSGD_OK) return status;
    if (!good_ld(ld, cols)) return CDSGD_ERR_SIZE;
    if (!aligned(out, bytes_of(dtype)) || !aligned(codes, 16)) return CDSGD_ERR_ALIGN;
    const Span in[] = {range_of(codes, cdsgd_mxint8_code_bytes(rows, cols)), range_of(scales, cdsgd_mxint8_scale_bytes(rows, cols))};
    const Span to[] = {matrix_of(out, rows, cols, ld, dtype)};
    if (any_overlap(to, 1, in, 2)) return CDSGD_ERR_ALIAS;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const Layout y = layout_of(rows, cols, kEach<DT>, 2);
        status = in_launches(y.groups, 256, [&](dim3 grid, unsigned first) {
            const auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)hip_stream, codes, scales, (unsigned)rows, (unsigned)cols,
                                   static_cast<Elem<DT> *>(out), ld, y.lanes_log2, first);
            };
            if (y.rows == 2) launch(k_held8_values<DT, 2>);
            else launch(k_held8_values<DT, 1>);
        });
    });
    return status;
}

int cdsgd_gated_forward(int act, int dtype, size_t rows, size_t cols, const void *a, size_t ld_a, const void *u, size_t ld_u, void *y, size_t ld_y,
                        int8_t *a8_codes, uint8_t *a8_scales, int8_t *u8_codes, uint8_t *u8_scales, void *hip_stream)
{
    const bool save = a8_codes || a8_scales || u8_codes || u8_scales;
    if (!a || !u || !y || (save && !(a8_codes && a8_scales && u8_codes && u8_scales))) return CDSGD_ERR_NULL;
    if (!good_dtype(dtype) || (act != CDSGD_ACT_SILU && act != CDSGD_ACT_GELU_TANH)) return CDSGD_ERR_PARAM;
    int status = check_extents(rows, cols);
    if (status != CDSGD_OK) return status;
    if (!good_ld(ld_a, cols) || !good_ld(ld_u, cols) || !good_ld(ld_y, cols)) return CDSGD_ERR_SIZE;
    const unsigned size = (unsigned)bytes_of(dtype);
    if (!aligned(a, size) || !aligned(u, size) || !aligned(y, size) || !aligned(a8_codes, 16) || !aligned(u8_codes, 16)) return CDSGD_ERR_ALIGN;
    const size_t codes = cdsgd_mxint8_code_bytes(rows, cols), scales = cdsgd_mxint8_scale_bytes(rows, cols);
    const Span out[] = {matrix_of(y, rows, cols, ld_y, dtype), range_of(a8_codes, codes), range_of(a8_scales, scales), range_of(u8_codes, codes),
                        range_of(u8_scales, scales)};
    const Span in[] = {matrix_of(a, rows, cols, ld_a, dtype), matrix_of(u, rows, cols, ld_u, dtype)};
    if (any_overlap(out, 5, in, 2)) return CDSGD_ERR_ALIAS;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const Layout l = layout_of(rows, cols, kEach<DT>, 2);
        status = in_launches(l.groups, 256, [&](dim3 grid, unsigned first) {
            const auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)hip_stream, static_cast<const Elem<DT> *>(a), ld_a,
                                   static_cast<const Elem<DT> *>(u), ld_u, static_cast<Elem<DT> *>(y), ld_y, (unsigned)rows, (unsigned)cols, a8_codes,
                                   a8_scales, u8_codes, u8_scales, l.lanes_log2, first);
            };
            const auto with_act = [&](auto kind) {
                constexpr int ACT = decltype(kind)::value;
                if (save && l.rows == 2) launch(k_gated_forward<DT, ACT, true, 2>);
                else if (save) launch(k_gated_forward<DT, ACT, true, 1>);
                else if (l.rows == 2) launch(k_gated_forward<DT, ACT, false, 2>);
                else launch(k_gated_forward<DT, ACT, false, 1>);
            };
            if (act == CDSGD_ACT_SILU) with_act(std::integral_constant<int, CDSGD_ACT_SILU>());
            else with_act(std::integral_constant<int, CDSGD_ACT_GELU_TANH>());
        });
    });
    return status;
}

int cdsgd_gated_backward(int act, int dtype, size_t rows, size_t cols, const void *dy, size_t ld_dy, const cdsgd_held *a, const cdsgd_held *u,
                         void *da, size_t ld_da, void *du, size_t ld_du, void *hip_stream)
{
    if (!dy || !a || !u || !da || !du) return CDSGD_ERR_NULL;
    if (!good_dtype(dtype) || (act != CDSGD_ACT_SILU && act != CDSGD_ACT_GELU_TANH)) return CDSGD_ERR_PARAM;
    int status = check_extents(rows, cols);
    if (status != CDSGD_OK) return status;
    if (!good_ld(ld_dy, cols) || !good_ld(ld_da, cols) || !good_ld(ld_du, cols)) return CDSGD_ERR_SIZE;
    const unsigned size = (unsigned)bytes_of(dtype);
    if (!aligned(dy, size) || !aligned(da, size) || !aligned(du, size)) return CDSGD_ERR_ALIGN;
    bool eight, eight_u;
    Span sa[2], su[2];
    if ((status = check_held(a, rows, cols, dtype, eight, sa)) != CDSGD_OK || (status = check_held(u, rows, cols, dtype, eight_u, su)) != CDSGD_OK)
        return status;
    if (eight != eight_u) return CDSGD_ERR_PARAM;
    const Span out[] = {matrix_of(da, rows, cols, ld_da, dtype), matrix_of(du, rows, cols, ld_du, dtype)};
    const Span in[] = {matrix_of(dy, rows, cols, ld_dy, dtype), sa[0], sa[1], su[0], su[1]};
    if (any_overlap(out, 2, in, 5)) return CDSGD_ERR_ALIAS;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const Layout l = layout_of(rows, cols, kEach<DT>, 2);
        status = in_launches(l.groups, 256, [&](dim3 grid, unsigned first) {
            const auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)hip_stream, static_cast<const Elem<DT> *>(dy), ld_dy,
                                   eight ? (const void *)a->codes : a->p, a->ld, a->scales, eight ? (const void *)u->codes : u->p, u->ld, u->scales,
                                   static_cast<Elem<DT> *>(da), ld_da, static_cast<Elem<DT> *>(du), ld_du, (unsigned)rows, (unsigned)cols,
                                   l.lanes_log2, first);
            };
            const auto with_act = [&](auto kind) {
                constexpr int ACT = decltype(kind)::value;
                if (eight && l.rows == 2) launch(k_gated_backward<DT, ACT, true, 2>);
                else if (eight) launch(k_gated_backward<DT, ACT, true, 1>);
                else if (l.rows == 2) launch(k_gated_backward<DT, ACT, false, 2>);
                else launch(k_gated_backward<DT, ACT, false, 1>);
            };
            if (act == CDSGD_ACT_SILU) with_act(std::integral_constant<int, CDSGD_ACT_SILU>());
            else with_act(std::integral_constant<int, CDSGD_ACT_GELU_TANH>());
        });
    });
    return status;
}

int cdsgd_block_norm_forward(const cdsgd_block_norm *norm, const void *h, size_t ld_h, const void *b, size_t ld_b, void *h_out, size_t ld_h_out,
                             void *y, size_t ld_y, float *rstd, int8_t *h8_codes, uint8_t *h8_scales, int8_t *b8_codes, uint8_t *b8_scales,
                             void *hip_stream)
{
    const int rc = check_norm(norm);
    if (rc != CDSGD_OK) return rc;
    const cdsgd_block_norm &n = *norm;
    if (!h || !y || !rstd || (b && !h_out) || (h8_codes != nullptr) != (h8_scales != nullptr) || (b8_codes != nullptr) != (b8_scales != nullptr))
        return CDSGD_ERR_NULL;
    if (!b && (h_out || b8_codes || n.block_weight || n.gate)) return CDSGD_ERR_PARAM;
    if (!good_ld(ld_h, n.cols) || !good_ld(ld_y, n.cols) || (b && (!good_ld(ld_b, n.cols) || !good_ld(ld_h_out, n.cols)))) return CDSGD_ERR_SIZE;
    const unsigned size = (unsigned)bytes_of(n.dtype), stream = (unsigned)bytes_of(n.stream_dtype);
    if (!aligned(h, stream) || !aligned(h_out, stream) || !aligned(b, size) || !aligned(y, size) || !aligned(rstd, 4) || !aligned(h8_codes, 16) ||
        !aligned(b8_codes, 16))
        return CDSGD_ERR_ALIGN;
    const size_t codes = cdsgd_mxint8_code_bytes(n.rows, n.cols), scales = cdsgd_mxint8_scale_bytes(n.rows, n.cols), w = n.cols * sizeof(float);
    const Span out[] = {matrix_of(h_out, n.rows, n.cols, ld_h_out, n.stream_dtype), matrix_of(y, n.rows, n.cols, ld_y, n.dtype),
                        range_of(rstd, 2 * n.rows * sizeof(float)), range_of(h8_codes, codes), range_of(h8_scales, scales),
                        range_of(b8_codes, codes), range_of(b8_scales, scales)};
    const Span in[] = {matrix_of(h, n.rows, n.cols, ld_h, n.stream_dtype), matrix_of(b, n.rows, n.cols, ld_b, n.dtype), range_of(n.weight, w),
                       range_of(n.block_weight, w), range_of(n.gate, w)};
    if (any_overlap(out, 7, in, 5)) return CDSGD_ERR_ALIAS;
    with_norm_types(n, [&](auto st, auto dt) {
        constexpr int ST = decltype(st)::value, DT = decltype(dt)::value;
        with_norm_shape(n.cols, [&](auto waves, auto v) {
            constexpr int W = decltype(waves)::value, V = decltype(v)::value;
            // (8192 rows of 4096, 8 waves each, us: 512 groups 88, 1024 90, 2048 94, 8192 115)
            const unsigned groups = n.rows < 4096 / W ? (unsigned)n.rows : 4096 / W;
            hipLaunchKernelGGL((k_block_norm_forward<ST, DT, W, V>), dim3(groups), dim3(64 * W), 0, (hipStream_t)hip_stream,
                               NormWeights{n.weight, n.block_weight, n.gate, n.scale, n.eps}, (unsigned)n.rows, (unsigned)n.cols,
                               Rows<const Elem<ST>>{static_cast<const Elem<ST> *>(h), ld_h}, Rows<const Elem<DT>>{static_cast<const Elem<DT> *>(b), ld_b},
                               Rows<Elem<ST>>{static_cast<Elem<ST> *>(h_out), ld_h_out}, Rows<Elem<DT>>{static_cast<Elem<DT> *>(y), ld_y}, rstd,
                               HeldOut{h8_codes, h8_scales}, HeldOut{b8_codes, b8_scales});
        });
    });
    return launch_status();
}

size_t cdsgd_block_norm_workspace(size_t rows, size_t cols)
{
    if (check_extents(rows, cols) != CDSGD_OK || cols > kMostCols) return 0;
    return (size_t)norm_groups(rows, cols) * 2u * ((cols + 3u) / 4u * 4u) * sizeof(float);
}

int cdsgd_block_norm_backward(const cdsgd_block_norm *norm, const void *dy, size_t ld_dy, const void *dh_out, size_t ld_dh_out,
                              const cdsgd_held *h_out, const cdsgd_held *b, const float *rstd, void *dh, size_t ld_dh, void *db, size_t ld_db,
                              float *dweight, float *dblock_weight, float *dgate, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_norm(norm);
    if (rc != CDSGD_OK) return rc;
    const cdsgd_block_norm &n = *norm;
    const bool block = b && (b->p || b->codes || b->scales);
    if (!dy || !h_out || !rstd || !dh || !dweight || !workspace || (block && !db) || (n.block_weight && block && !dblock_weight) ||
        (n.gate && block && !dgate))
        return CDSGD_ERR_NULL;
    if ((dblock_weight && !n.block_weight) || (dgate && !n.gate) || (!block && (db || n.block_weight || n.gate))) return CDSGD_ERR_PARAM;
    if (!good_ld(ld_dy, n.cols) || !good_ld(ld_dh, n.cols) || (dh_out && !good_ld(ld_dh_out, n.cols)) || (block && !good_ld(ld_db, n.cols)) ||
        workspace_bytes < cdsgd_block_norm_workspace(n.rows, n.cols))
        return CDSGD_ERR_SIZE;
    const unsigned size = (unsigned)bytes_of(n.dtype), stream = (unsigned)bytes_of(n.stream_dtype);
    if (!aligned(dy, size) || !aligned(db, size) || !aligned(dh_out, stream) || !aligned(dh, stream) || !aligned(rstd, 4) || !aligned(dweight, 4) ||
        !aligned(dblock_weight, 4) || !aligned(dgate, 4) || !aligned(workspace, 16))
        return CDSGD_ERR_ALIGN;
    bool eight_h, eight_b = false;
    Span sh[2], sb[2] = {{nullptr, 1, 0, 0}, {nullptr, 1, 0, 0}};
    if ((rc = check_held(h_out, n.rows, n.cols, n.stream_dtype, eight_h, sh)) != CDSGD_OK) return rc;
    if (block && (rc = check_held(b, n.rows, n.cols, n.dtype, eight_b, sb)) != CDSGD_OK) return rc;
    const size_t w = n.cols * sizeof(float);
    const Span out[] = {matrix_of(dh, n.rows, n.cols, ld_dh, n.stream_dtype), matrix_of(db, n.rows, n.cols, ld_db, n.dtype), range_of(dweight, w),
                        range_of(dblock_weight, w), range_of(dgate, w), range_of(workspace, cdsgd_block_norm_workspace(n.rows, n.cols))};
    const Span in[] = {matrix_of(dy, n.rows, n.cols, ld_dy, n.dtype), matrix_of(dh_out, n.rows, n.cols, ld_dh_out, n.stream_dtype), sh[0], sh[1],
                       sb[0], sb[1], range_of(rstd, 2 * n.rows * sizeof(float)), range_of(n.weight, w), range_of(n.block_weight, w),
                       range_of(n.gate, w)};
    if (any_overlap(out, 6, in, 10)) return CDSGD_ERR_ALIAS;
    const unsigned groups = norm_groups(n.rows, n.cols);
    const NormWeights by = {n.weight, n.block_weight, n.gate, n.scale, n.eps};
    float *const parts = static_cast<float *>(workspace);
    const HeldIn in_h = {eight_h ? (const void *)h_out->codes : h_out->p, h_out->ld, h_out->scales};
    const HeldIn in_b = block ? HeldIn{eight_b ? (const void *)b->codes : b->p, b->ld, b->scales} : HeldIn{nullptr, 0, nullptr};
    with_norm_types(n, [&](auto st, auto dt) {
        constexpr int ST = decltype(st)::value, DT = decltype(dt)::value;
        with_norm_shape(n.cols, [&](auto waves, auto v) {
            constexpr int W = decltype(waves)::value, V = decltype(v)::value;
            const auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3(groups), dim3(64 * W), 0, (hipStream_t)hip_stream, by, (unsigned)n.rows, (unsigned)n.cols,
                                   Rows<const Elem<DT>>{static_cast<const Elem<DT> *>(dy), ld_dy},
                                   Rows<const Elem<ST>>{static_cast<const Elem<ST> *>(dh_out), ld_dh_out}, in_h, in_b, rstd,
                                   Rows<Elem<ST>>{static_cast<Elem<ST> *>(dh), ld_dh}, Rows<Elem<DT>>{static_cast<Elem<DT> *>(db), ld_db}, parts);
            };
            if (eight_h && eight_b) launch(k_block_norm_backward<ST, DT, W, V, true, true>);
            else if (eight_h) launch(k_block_norm_backward<ST, DT, W, V, true, false>);
            else if (eight_b) launch(k_block_norm_backward<ST, DT, W, V, false, true>);
            else launch(k_block_norm_backward<ST, DT, W, V, false, false>);
        });
    });
    hipLaunchKernelGGL(k_block_norm_join, dim3((unsigned)((n.cols + 31) / 32), dblock_weight || dgate ? 2 : 1), dim3(1024), 0, (hipStream_t)hip_stream,
                       (const float *)parts, groups, (unsigned)n.cols, by, dweight, dblock_weight, dgate);
    return launch_status();
}

}  // extern "C"
