// Which kernels compute a product of two matrices in MXFP4, by its sizes.  Plain C++: no header of the GPU's is needed.
#pragma once

#include <cstddef>
#include <initializer_list>

namespace {

// Sizes of a product that the kernels hold in 32 bits: offsets inside a tile of 256 rows, and scale words of two groups.
inline bool good_product(size_t M, size_t N, size_t K)
{
    constexpr size_t kMostRows = (size_t)1 << 29, kMostSum = (size_t)1 << 24;
    return M > 0 && M <= kMostRows && N > 0 && N <= kMostRows && K > 0 && K <= kMostSum;
}

inline unsigned long long count_of(size_t n, size_t each) { return (n + each - 1) / each; }

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

// us, bf16 results, three sets of operands in turn, without the wait states of the loads to LDS, which add up to 3 %; rWxF: rings of W waves, F fragments; t64, t128, t256: tiles of 64 by 64, 128 by 256,
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
// Rings of so many columns that a launch would pass its 2^32 lanes (n16 groups of 256) leave them to tiles of 64.
inline Product product_of(size_t M, size_t N, size_t K)
{
    const unsigned long long n16 = count_of(N, 16);
    if (M <= 32 && n16 >= 1ull << 24) return {0, 0, k64By64, 1};
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

inline unsigned lanes_of(Tile t) { return t == k64By64 || t == k128By128 ? 256 : 512; }
inline unsigned long long rings_of(const Product &p, size_t M, size_t N) { return count_of(M, 16u * p.ring_rows) * count_of(N, 16); }

// Groups of 256 lanes that add up a sum's parts, four neighbouring results to a lane.
inline unsigned long long joins_of(size_t M, size_t N) { return count_of(count_of(N, 4) * M, 256); }

// Lanes of the largest launch.
inline unsigned long long lanes_of(const Product &p, size_t M, size_t N)
{
    if (p.ring_rows) return rings_of(p, M, N) * 64 * p.ring_waves;
    const unsigned long long tiles = tiles_of(p.tile, p.rest_m ? p.rest_m : M, p.rest_n ? p.rest_n : N) * p.splits * lanes_of(p.tile);
    const unsigned long long rest = p.rest_tile ? tiles_of(p.rest_tile, M - p.rest_m, N - p.rest_n) * lanes_of(p.rest_tile) : 0;
    const unsigned long long join = p.splits > 1 ? joins_of(M, N) * 256 : 0;
    return tiles > rest ? (tiles > join ? tiles : join) : (rest > join ? rest : join);
}

}  // namespace
