// Matrices in microscaled 4-bit floating point (include/cdsgd_ops.h): the C ABI's host side.  The kernels are in
// kernels_mxfp4.hpp.

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "cdsgd_ops.h"

#include "host_common.hpp"
#include "tuning.hpp"
#include "device_common.hpp"

#include "kernels_mxfp4.hpp"

namespace {

inline bool good_dtype(int t) { return t == CDSGD_GRAD_F32 || t == CDSGD_GRAD_BF16 || t == CDSGD_GRAD_F16; }
inline size_t bytes_of(int dtype) { return dtype == CDSGD_GRAD_F32 ? 4u : 2u; }
inline size_t groups_of(size_t cols) { return (cols + kGroup - 1) / kGroup; }
inline bool good_extent(size_t n) { return n > 0 && n <= 0x7FFFFFFFu; }

// Bytes from the first element of a matrix to the last, both included.
inline size_t extent_bytes(size_t rows, size_t cols, size_t ld, size_t elem) { return ((rows - 1) * ld + cols) * elem; }

// Calls f(std::integral_constant<int, element type>).
template <typename F>
void with_dtype(int dtype, F f)
{
    if (dtype == CDSGD_GRAD_BF16) f(std::integral_constant<int, kGradBF16>());
    else if (dtype == CDSGD_GRAD_F16) f(std::integral_constant<int, kGradF16>());
    else f(std::integral_constant<int, kGradF32>());
}

// Of a matrix in MXFP4 and its place in a launch: sizes that the kernels hold in 32 bits.
inline int check_matrix(size_t rows, size_t cols)
{
    if (!good_extent(rows) || !good_extent(cols)) return CDSGD_ERR_SIZE;
    return CDSGD_OK;
}

constexpr unsigned long long kMostGroups = 0xFFFFFFFFull / 256;  // workgroups of 256 lanes in a launch

}  // namespace

extern "C" {

size_t cdsgd_mxfp4_code_bytes(size_t rows, size_t cols) { return rows * groups_of(cols) * 64u; }
size_t cdsgd_mxfp4_scale_bytes(size_t rows, size_t cols) { return rows * groups_of(cols) * 4u; }

int cdsgd_mxfp4_quantize(const void *x, int dtype, size_t rows, size_t cols, size_t ld, uint8_t *codes, uint8_t *scales,
                         uint8_t *codes_t, uint8_t *scales_t, void *hip_stream)
{
    if (!x || (!codes && !codes_t) || (codes != nullptr) != (scales != nullptr) || (codes_t != nullptr) != (scales_t != nullptr))
        return CDSGD_ERR_NULL;
    if (!good_dtype(dtype)) return CDSGD_ERR_PARAM;
    const int rc = check_matrix(rows, cols);
    if (rc != CDSGD_OK) return rc;
    if (ld < cols || ld > (size_t)1 << 40) return CDSGD_ERR_SIZE;
    if (!aligned(x, bytes_of(dtype)) || !aligned(codes, 16) || !aligned(codes_t, 16) || !aligned(scales, 4) || !aligned(scales_t, 4))
        return CDSGD_ERR_ALIGN;
    const void *const buffer[] = {codes, scales, codes_t, scales_t, x};
    const size_t bytes[] = {cdsgd_mxfp4_code_bytes(rows, cols), cdsgd_mxfp4_scale_bytes(rows, cols), cdsgd_mxfp4_code_bytes(cols, rows),
                            cdsgd_mxfp4_scale_bytes(cols, rows), extent_bytes(rows, cols, ld, bytes_of(dtype))};
    for (int a = 0; a < 5; ++a)
        for (int b = a + 1; b < 5; ++b)
            if (overlap2(buffer[a], bytes[a], buffer[b], bytes[b])) return CDSGD_ERR_ALIAS;
    hipStream_t s = (hipStream_t)hip_stream;
    const unsigned r = (unsigned)rows, c = (unsigned)cols;
    constexpr unsigned kRows = 4;
    const unsigned long long groups = codes_t ? (unsigned long long)((rows + kTile - 1) / kTile) * ((cols + kTile - 1) / kTile)
                                              : (unsigned long long)((rows + 4 * kRows - 1) / (4 * kRows)) * ((cols + kRowCols - 1) / kRowCols);
    if (groups > kMostGroups) return CDSGD_ERR_SIZE;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const Elem<DT> *from = static_cast<const Elem<DT> *>(x);
        const dim3 grid((unsigned)groups), block(256);
        if (!codes_t) hipLaunchKernelGGL((k_quantize_rows<DT, kRows>), grid, block, 0, s, from, ld, r, c, codes, scales);
        else if (codes) hipLaunchKernelGGL((k_quantize_tiles<DT, true>), grid, block, 0, s, from, ld, r, c, codes, scales, codes_t, scales_t);
        else hipLaunchKernelGGL((k_quantize_tiles<DT, false>), grid, block, 0, s, from, ld, r, c, codes, scales, codes_t, scales_t);
    });
    return launch_status();
}

int cdsgd_mxfp4_dequantize(const uint8_t *codes, const uint8_t *scales, size_t rows, size_t cols, void *out, int dtype, size_t ld,
                           void *hip_stream)
{
    if (!codes || !scales || !out) return CDSGD_ERR_NULL;
    if (!good_dtype(dtype)) return CDSGD_ERR_PARAM;
    const int rc = check_matrix(rows, cols);
    if (rc != CDSGD_OK) return rc;
    if (ld < cols || ld > (size_t)1 << 40) return CDSGD_ERR_SIZE;
    if (!aligned(out, bytes_of(dtype)) || !aligned(codes, 16) || !aligned(scales, 4)) return CDSGD_ERR_ALIGN;
    const size_t ob = extent_bytes(rows, cols, ld, bytes_of(dtype));
    if (overlap2(out, ob, codes, cdsgd_mxfp4_code_bytes(rows, cols)) || overlap2(out, ob, scales, cdsgd_mxfp4_scale_bytes(rows, cols)))
        return CDSGD_ERR_ALIAS;
    constexpr unsigned kRows = 4;
    const unsigned long long groups = (unsigned long long)((rows + 4 * kRows - 1) / (4 * kRows)) * ((cols + kRowCols - 1) / kRowCols);
    if (groups > kMostGroups) return CDSGD_ERR_SIZE;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        hipLaunchKernelGGL((k_dequantize<DT, kRows>), dim3((unsigned)groups), dim3(256), 0, (hipStream_t)hip_stream, codes, scales,
                           (unsigned)rows, (unsigned)cols, static_cast<Elem<DT> *>(out), ld);
    });
    return launch_status();
}

size_t cdsgd_mxfp4_matmul_workspace(size_t, size_t, size_t) { return 0; }

int cdsgd_mxfp4_matmul(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes, const uint8_t *b_scales, size_t M,
                       size_t N, size_t K, void *out, int dtype, size_t ld, int accumulate, void *workspace, size_t workspace_bytes,
                       void *hip_stream)
{
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return CDSGD_ERR_NULL;
    if (!good_dtype(dtype)) return CDSGD_ERR_PARAM;
    if (!good_extent(M) || !good_extent(N) || !good_extent(K) || ld < N || ld > (size_t)1 << 40) return CDSGD_ERR_SIZE;
    const size_t want = cdsgd_mxfp4_matmul_workspace(M, N, K);
    if (want && !workspace) return CDSGD_ERR_NULL;
    if (workspace_bytes < want) return CDSGD_ERR_SIZE;
    if (!aligned(a_codes, 16) || !aligned(b_codes, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) ||
        !aligned(out, bytes_of(dtype)) || !aligned(workspace, 16))
        return CDSGD_ERR_ALIGN;
    const void *const in[] = {a_codes, a_scales, b_codes, b_scales};
    const size_t bytes[] = {cdsgd_mxfp4_code_bytes(M, K), cdsgd_mxfp4_scale_bytes(M, K), cdsgd_mxfp4_code_bytes(N, K),
                            cdsgd_mxfp4_scale_bytes(N, K)};
    const size_t ob = extent_bytes(M, N, ld, bytes_of(dtype));
    for (int i = 0; i < 4; ++i)
        if (overlap2(out, ob, in[i], bytes[i]) || (want && overlap2(workspace, want, in[i], bytes[i]))) return CDSGD_ERR_ALIAS;
    if (want && overlap2(out, ob, workspace, want)) return CDSGD_ERR_ALIAS;
    const unsigned long long tiles = (unsigned long long)((M + 31) / 32) * ((N + 31) / 32);
    if (tiles > 0xFFFFFFFFull / 64) return CDSGD_ERR_SIZE;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        hipLaunchKernelGGL((k_mxfp4_simple<DT>), dim3((unsigned)tiles), dim3(64), 0, (hipStream_t)hip_stream, a_codes, a_scales, b_codes,
                           b_scales, (unsigned)M, (unsigned)N, (unsigned)groups_of(K), static_cast<Elem<DT> *>(out), ld, accumulate);
    });
    return launch_status();
}

}  // extern "C"
