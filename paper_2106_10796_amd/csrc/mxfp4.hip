// Matrices in microscaled 4-bit floating point (include/cdsgd_ops.h): the C ABI's host side.  The kernels are in
// kernels_mxfp4.hpp (quantisation, values) and kernels_mxfp4_product.hpp.

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "cdsgd_ops.h"

#include "host_common.hpp"
#include "tuning.hpp"
#include "device_common.hpp"
#include "mxfp4_choice.hpp"

#include "kernels_mxfp4.hpp"
#include "kernels_mxfp4_product.hpp"

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

// Calls launch(groups, number of the first) for launches below 2^32 lanes; all but the last hold a multiple of 32 groups, what
// k_quantize_tiles numbers together.  (One but for matrices of 2^27 rows and more.)  The kernels number groups in 32 bits.
template <typename F>
int in_launches(unsigned long long groups, unsigned lanes, F launch)
{
    if (groups > 0xFFFFFFFFull) return CDSGD_ERR_SIZE;
    const unsigned long long most = 0xFFFFFFFFull / lanes / 32 * 32;
    for (unsigned long long first = 0; first < groups; first += most)
        launch(dim3((unsigned)(groups - first < most ? groups - first : most)), (unsigned)first);
    return launch_status();
}

// Calls f(kernel, groups, lanes) with the ring that `how` names, for results of type DT.
template <int DT, typename F>
void with_ring(const Product &how, size_t M, size_t N, F f)
{
    const auto ring = [&](auto kernel) { f(kernel, (unsigned)rings_of(how, M, N), 64u * how.ring_waves); };
    if (how.ring_rows == 1 && how.ring_waves == 8) ring(k_ring<DT, 1, 1, 2, 8>);
    else if (how.ring_rows == 1) ring(k_ring<DT, 1, 1, 2, 4>);
    else if (how.ring_rows == 2 && how.ring_waves == 8) ring(k_ring<DT, 2, 1, 2, 8>);
    else if (how.ring_rows == 2) ring(k_ring<DT, 2, 1, 2, 4>);
    else ring(k_ring<DT, 4, 1, 2, 4>);
}

// The same with the kernel for tiles.
template <int DT, typename F>
void with_tiles(Tile tile, F f)
{
    if (tile == k64By64) f(k_tiles<DT, 64, 64, 2, 2, 4>);
    else if (tile == k128By128) f(k_tiles<DT, 128, 128, 2, 2, 2>);
    else if (tile == k128By256) f(k_tiles<DT, 128, 256, 2, 4, 3>);
    else f(k_tiles<DT, 256, 256, 2, 4, 2>);
}

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
    // rows to a wave: 4 on large matrices, 1 where that leaves compute units idle (us, 1003 x 2049 in fp16: 2.8 with 4, 2.4 with 1;
    // 8192 x 4096 in bf16 12.8 and 14.1)
    const unsigned long long across = count_of(cols, kRowCols);
    const bool many = across * count_of(rows, 16) >= 256;
    const unsigned long long groups = codes_t ? tile_groups(rows, cols) : across * count_of(rows, many ? 16 : 4);
    int status = CDSGD_OK;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const Elem<DT> *from = static_cast<const Elem<DT> *>(x);
        const dim3 block(codes_t ? kTileLanes<DT> : 256u);
        status = in_launches(groups, block.x, [&](dim3 grid, unsigned first) {
            if (!codes_t && many) hipLaunchKernelGGL((k_quantize_rows<DT, 4>), grid, block, 0, s, from, ld, r, c, codes, scales, first);
            else if (!codes_t) hipLaunchKernelGGL((k_quantize_rows<DT, 1>), grid, block, 0, s, from, ld, r, c, codes, scales, first);
            else if (codes) hipLaunchKernelGGL((k_quantize_tiles<DT, true>), grid, block, 0, s, from, ld, r, c, codes, scales, codes_t, scales_t, first);
            else hipLaunchKernelGGL((k_quantize_tiles<DT, false>), grid, block, 0, s, from, ld, r, c, codes, scales, codes_t, scales_t, first);
        });
    });
    return status;
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
    const unsigned long long across = count_of(cols, dtype == CDSGD_GRAD_F32 ? kValueCols<kGradF32> : kValueCols<kGradBF16>);
    const bool many = across * count_of(rows, 16) >= 256;
    const unsigned long long groups = across * count_of(rows, many ? 16 : 4);
    int status = CDSGD_OK;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto launch = [&](auto kernel) {
            status = in_launches(groups, 256, [&](dim3 grid, unsigned first) {
                hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)hip_stream, codes, scales, (unsigned)rows, (unsigned)cols,
                                   static_cast<Elem<DT> *>(out), ld, first);
            });
        };
        if (many) launch(k_dequantize<DT, 4>);
        else launch(k_dequantize<DT, 1>);
    });
    return status;
}

size_t cdsgd_mxfp4_matmul_workspace(size_t M, size_t N, size_t K)
{
    if (!good_product(M, N, K)) return 0;
    const unsigned splits = product_of(M, N, K).splits;
    return splits > 1 ? (splits * M * N * sizeof(float) + 15u) / 16u * 16u : 0;
}

int cdsgd_mxfp4_matmul(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes, const uint8_t *b_scales, size_t M,
                       size_t N, size_t K, void *out, int dtype, size_t ld, int accumulate, void *workspace, size_t workspace_bytes,
                       void *hip_stream)
{
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return CDSGD_ERR_NULL;
    if (!good_dtype(dtype)) return CDSGD_ERR_PARAM;
    if (!good_product(M, N, K) || ld < N || ld > (size_t)1 << 40) return CDSGD_ERR_SIZE;
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
    const Product how = product_of(M, N, K);
    if (lanes_of(how, M, N) > 0xFFFFFFFFull) return CDSGD_ERR_SIZE;
    hipStream_t s = (hipStream_t)hip_stream;
    const unsigned m = (unsigned)M, n = (unsigned)N, groups = (unsigned)groups_of(K);
    // rows [m0, m1) and columns [n0, n1) of the result, in tiles
    const auto tiles = [&](auto dt, Tile tile, size_t m0, size_t n0, size_t m1, size_t n1, auto *to, size_t row, int add) {
        with_tiles<decltype(dt)::value>(tile, [&](auto kernel) {
            const unsigned tiles_m = (unsigned)tiles_of(tile, m1 - m0, 1), tiles_n = (unsigned)tiles_of(tile, 1, n1 - n0);
            hipLaunchKernelGGL(kernel, dim3(tiles_m * tiles_n * how.splits), dim3(lanes_of(tile)), 0, s, a_codes, a_scales, b_codes, b_scales,
                               m, n, groups, to, row, add, how.splits, (unsigned)m0, (unsigned)n0, tiles_m, tiles_n);
        });
    };
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        Elem<DT> *const to = static_cast<Elem<DT> *>(out);
        if (how.ring_rows) {
            with_ring<DT>(how, M, N, [&](auto kernel, unsigned count, unsigned lanes) {
                hipLaunchKernelGGL(kernel, dim3(count), dim3(lanes), 0, s, a_codes, a_scales, b_codes, b_scales, m, n, groups, to, ld,
                                   accumulate);
            });
        } else if (how.splits > 1) {
            float *const parts = static_cast<float *>(workspace);
            tiles(std::integral_constant<int, kGradF32>(), how.tile, 0, 0, M, N, parts, N, 0);
            hipLaunchKernelGGL((k_join<DT>), dim3((unsigned)joins_of(M, N)), dim3(256), 0, s, parts, m, n, how.splits, to, ld, accumulate);
        } else {
            tiles(dt, how.tile, 0, 0, how.rest_m ? how.rest_m : M, how.rest_n ? how.rest_n : N, to, ld, accumulate);
            if (how.rest_tile) tiles(dt, how.rest_tile, how.rest_m, how.rest_n, M, N, to, ld, accumulate);
        }
    });
    return launch_status();
}

}  // extern "C"
