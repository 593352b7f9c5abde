// Matrices in microscaled 4-bit floating point (include/cdsgd_ops.h): the C ABI's host side.  The kernels are in
// kernels_mxfp4.hpp (quantisation, values) and kernels_mxfp4_product.hpp.

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "cdsgd_ops.h"

#include "host_common.hpp"
#include "tuning.hpp"
#include "device_common.hpp"

#include "kernels_mxfp4.hpp"
#include "kernels_mxfp4_product.hpp"

namespace {

inline bool good_dtype(int t) { return t == CDSGD_GRAD_F32 || t == CDSGD_GRAD_BF16 || t == CDSGD_GRAD_F16; }
inline size_t bytes_of(int dtype) { return dtype == CDSGD_GRAD_F32 ? 4u : 2u; }
inline size_t groups_of(size_t cols) { return (cols + kGroup - 1) / kGroup; }
inline bool good_extent(size_t n) { return n > 0 && n <= 0x7FFFFFFFu; }

// Sizes of a product that the kernels hold in 32 bits: offsets inside a tile of 256 rows, and scale words of two groups.
inline bool good_product(size_t M, size_t N, size_t K)
{
    constexpr size_t kMostRows = (size_t)1 << 29, kMostSum = (size_t)1 << 24;
    return M > 0 && M <= kMostRows && N > 0 && N <= kMostRows && K > 0 && K <= kMostSum;
}

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

inline unsigned long long count_of(size_t n, size_t each) { return (n + each - 1) / each; }

constexpr unsigned long long kMostGroups = 0xFFFFFFFFull / 256;  // workgroups of 256 lanes in a launch

// How a product is computed.  Few rows of A, and a matrix B that is read once: rings of a wave's own (ring: fragments of 16 rows of
// A to a group, and its waves).  Otherwise tiles, whose sum is split over groups where it is long and the tiles are few, and whose last
// rows or columns may be left to a second launch with smaller ones.
enum Tile { kNoTile, k64By64, k128By128, k128By256, k256By256 };
struct Product {
    int ring_rows, ring_waves;  // 0: tiles
    Tile tile;
    unsigned splits;
    Tile rest_tile = kNoTile;  // else the rows from rest_m on or the columns from rest_n on are the second launch's
    size_t rest_m = 0, rest_n = 0;
};

inline unsigned long long tiles_of(Tile t, size_t M, size_t N)
{
    return count_of(M, t == k64By64 ? 64 : (t == k256By256 ? 256 : 128)) * count_of(N, t == k64By64 ? 64 : (t == k128By128 ? 128 : 256));
}

// Tiles run in rounds, 256 large ones at a time.  Where the last round would be nearly empty, its part of the result is taken off along
// one of the two extents: no more smaller tiles than run at a time, of the smallest 512 (us, bf16 results, in one launch and in two:
// 4352 x 4096 x 4096 56.4 and 44.1, 5120 x 4096 x 4096 56.7 and 52.7, 8190 x 4098 x 4096 103 and 90; not below eight stages:
// 4352 x 4096 x 1024 19.6 and 21.2).
inline Product without_a_last_round(Product p, size_t M, size_t N)
{
    const unsigned long long tiles_m = count_of(M, 256), tiles_n = count_of(N, 256), full = tiles_m * tiles_n / 256 * 256;
    const size_t rest_n = full / tiles_m * 256, rest_m = full / tiles_n * 256;
    if (full == 0 || full == tiles_m * tiles_n) return p;
    for (const Tile t : {k64By64, k128By256}) {
        const unsigned long long most = t == k64By64 ? 512 : 256;
        if (rest_n && rest_n < N && tiles_of(t, M, N - rest_n) <= most) {
            p.rest_tile = t, p.rest_n = rest_n;
            return p;
        }
        if (rest_m && rest_m < M && tiles_of(t, M - rest_m, N) <= most) {
            p.rest_tile = t, p.rest_m = rest_m;
            return p;
        }
    }
    return p;
}

// us, bf16 results, three sets of operands in turn; rWxF: rings of W waves, F fragments; t64, t128, t256: tiles of 64 by 64, 128 by 256,
// 256 by 256; /S: split S ways
//   16 x 8192 x 8192    r8x1 9.0, r4x1 10.6, t64 11.2            5 x 8192 x 300     r8x1 2.7, r4x1 2.5;  1 x 25088 x 512 6.1, 4.0
//   32 x 8192 x 8192    r8x2 12.0, r4x2 10.7, t64 11.3           32 x 4096 x 4096   r8x2 3.4, r4x2 3.6
//   128 x 1000 x 25088  r8x2 11.7, r4x4 15.0, t64 28.5           96 x 4096 x 4096   r8x2 9.8, r4x2 7.1, t64 6.9
//   64 x 4096 x 4096    r8x2 7.0, r4x4 4.8, t64 6.5              64 x 8192 x 8192   r4x4 14.5, t64 11.8
//   256 x 512 x 8192    r8x2 5.4, r4x4 6.9, t64 11.2             256 x 1000 x 4096  r8x2 6.7, r4x4 4.8, t64 7.2
//   200 x 500 x 2048    r8x2 3.0, t64 5.2                        400 x 1000 x 4096  r8x2 11.6, r4x4 9.1, t64 7.3
//   64 x 4096 x 25088   r4x4 16.5, t64 30.1, /2 19.4, /4 15.5    128 x 4096 x 25088 t64 30.9, /2 21.9, /4 21.2
//   65 x 4096 x 8192    t64 11.8, /2 10.6, /4 11.2               256 x 4096 x 8192  t64 12.5, /2 15.5
//   1024 x 1024 x 25088 t64 34.2, /2 28.2, t128/4 28.7           512 x 4096 x 25088 t64 44.5, t128 73.4, /2 46.2, /4 39.6
//   1024 x 4096 x 25088 t128 74.1, /2 68.0                       1024 x 4096 x 12544 t128 40.5, /2 41.0
//   512 x 4096 x 4096   t64 10.6, t256 24.3                      1024 x 4096 x 4096 t64 18.2, t128 16.1, t256 24.6
//   2048 x 4096 x 4096  t128 21.0, t256 25.3                     2176 x 4096 x 4096 t128 34.1, t256 26.7
// and 128 by 128, two groups to a compute unit, whose stores and products overlap by themselves, but which read more:
//   16384 x 8192 x 512  82.5, t128 92.3                          4096 x 25088 x 256 52, t128 60
//   16384 x 8192 x 1024 125, t256 105                            2048 x 4096 x 25088 114, t128 106
inline Product product_of(size_t M, size_t N, size_t K)
{
    const unsigned long long n16 = count_of(N, 16);
    if (M <= 16) return {1, n16 <= 512 ? 8 : 4, kNoTile, 1};
    if (n16 * count_of(M, 32) <= 256) return {2, 8, kNoTile, 1};
    if (M <= 32) return {2, 4, kNoTile, 1};
    if (n16 * count_of(M, 64) <= 256) return {4, 4, kNoTile, 1};
    const unsigned long long t64 = tiles_of(k64By64, M, N), t128 = tiles_of(k128By256, M, N), stages = count_of(K, 256);
    if (stages >= 32 && (t64 <= 128 || (t64 <= 256 && stages >= 64))) return {0, 0, k64By64, 2};
    if (stages >= 64 && t128 <= 128) return {0, 0, k128By256, t128 <= 64 ? 4u : 2u};
    if (t64 <= 512) return {0, 0, k64By64, 1};
    if (t128 <= 256) return {0, 0, k128By256, 1};
    if (stages < 4) return {0, 0, k128By128, 1};
    const Product p = {0, 0, k256By256, 1};
    return stages < 8 ? p : without_a_last_round(p, M, N);
}

// Calls f(kernel, groups, lanes) with the ring that `how` names, for results of type DT.
template <int DT, typename F>
void with_ring(const Product &how, size_t M, size_t N, F f)
{
    const auto ring = [&](auto kernel) { f(kernel, count_of(M, 16u * how.ring_rows) * count_of(N, 16), 64u * how.ring_waves); };
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
    if (tile == k64By64) f(k_tiles<DT, 64, 64, 2, 2, 4>, 256u);
    else if (tile == k128By128) f(k_tiles<DT, 128, 128, 2, 2, 2>, 256u);
    else if (tile == k128By256) f(k_tiles<DT, 128, 256, 2, 4, 3>, 512u);
    else f(k_tiles<DT, 256, 256, 2, 4, 2>, 512u);
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
    if (groups > kMostGroups / 2) return CDSGD_ERR_SIZE;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const Elem<DT> *from = static_cast<const Elem<DT> *>(x);
        const dim3 grid((unsigned)groups), block(codes_t ? kTileLanes<DT> : 256u);
        if (!codes_t && many) hipLaunchKernelGGL((k_quantize_rows<DT, 4>), grid, block, 0, s, from, ld, r, c, codes, scales);
        else if (!codes_t) hipLaunchKernelGGL((k_quantize_rows<DT, 1>), grid, block, 0, s, from, ld, r, c, codes, scales);
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
    const unsigned long long across = count_of(cols, dtype == CDSGD_GRAD_F32 ? kValueCols<kGradF32> : kValueCols<kGradBF16>);
    const bool many = across * count_of(rows, 16) >= 256;
    const unsigned long long groups = across * count_of(rows, many ? 16 : 4);
    if (groups > kMostGroups) return CDSGD_ERR_SIZE;
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)hip_stream, codes, scales, (unsigned)rows,
                               (unsigned)cols, static_cast<Elem<DT> *>(out), ld);
        };
        if (many) launch(k_dequantize<DT, 4>);
        else launch(k_dequantize<DT, 1>);
    });
    return launch_status();
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
    int status = CDSGD_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    const unsigned m = (unsigned)M, n = (unsigned)N, groups = (unsigned)groups_of(K);
    const auto fits = [&](unsigned long long count, unsigned lanes) {
        if (count > 0xFFFFFFFFull / lanes) status = CDSGD_ERR_SIZE;
        return status == CDSGD_OK;
    };
    // rows [m0, m1) and columns [n0, n1) of the result, in tiles
    const auto tiles = [&](auto dt, Tile tile, size_t m0, size_t n0, size_t m1, size_t n1, auto *to, size_t row, int add) {
        with_tiles<decltype(dt)::value>(tile, [&](auto kernel, unsigned lanes) {
            const unsigned long long tiles_m = tiles_of(tile, m1 - m0, 1), tiles_n = tiles_of(tile, 1, n1 - n0), count = tiles_m * tiles_n * how.splits;
            if (fits(count, lanes))
                hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(lanes), 0, s, a_codes, a_scales, b_codes, b_scales, m, n, groups, to,
                                   row, add, how.splits, (unsigned)m0, (unsigned)n0, (unsigned)tiles_m, (unsigned)tiles_n);
        });
    };
    with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        Elem<DT> *const to = static_cast<Elem<DT> *>(out);
        if (how.ring_rows) {
            with_ring<DT>(how, M, N, [&](auto kernel, unsigned long long count, unsigned lanes) {
                if (fits(count, lanes))
                    hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(lanes), 0, s, a_codes, a_scales, b_codes, b_scales, m, n, groups,
                                       to, ld, accumulate);
            });
        } else if (how.splits > 1) {
            float *const parts = static_cast<float *>(workspace);
            const unsigned long long join = count_of(count_of(N, 4) * M, 256);
            if (!fits(join, 256)) return;
            tiles(std::integral_constant<int, kGradF32>(), how.tile, 0, 0, M, N, parts, N, 0);
            if (status == CDSGD_OK)
                hipLaunchKernelGGL((k_join<DT>), dim3((unsigned)join), dim3(256), 0, s, parts, m, n, how.splits, to, ld, accumulate);
        } else {
            tiles(dt, how.tile, 0, 0, how.rest_m ? how.rest_m : M, how.rest_n ? how.rest_n : N, to, ld, accumulate);
            if (how.rest_tile && status == CDSGD_OK) tiles(dt, how.rest_tile, how.rest_m, how.rest_n, M, N, to, ld, accumulate);
        }
    });
    if (status != CDSGD_OK) return status;
    return launch_status();
}

}  // extern "C"
