// Matrices in microscaled 4-bit floating point: quantisation along rows and columns, values, the matrix instruction.
#pragma once

namespace {

typedef unsigned u4 __attribute__((ext_vector_type(4)));

constexpr unsigned kGroup = 128;  // elements of a row that one scale word covers

// Element types of matrices in ordinary floating point.
template <int DT>
using Elem = typename std::conditional<DT == kGradF32, float, typename std::conditional<DT == kGradBF16, __bf16, _Float16>::type>::type;

// Eight elements in a row, at any address that is a multiple of the type's size.
template <int DT>
struct Eight {
    Elem<DT> v[8];
};
template <int DT>
struct __attribute__((packed, aligned(sizeof(Elem<DT>)))) EightAt {
    Eight<DT> e;
};

// ---------------------------------------------------------------------------
// quantisation
// ---------------------------------------------------------------------------
// The scale byte for a block with that largest magnitude (as bits; denormal ones and zero have exponent field 0).
__device__ __forceinline__ unsigned scale_of(unsigned most)
{
    const unsigned field = most >> 23;
    return field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
}

// What the conversion instructions take: the exponent as a float's.  Byte 0 gives the pattern 0, which they read as 2^-127.
__device__ __forceinline__ float scale_operand(unsigned scale) { return __builtin_bit_cast(float, scale << 23); }

// Eight codes of a block in a word.
__device__ __forceinline__ unsigned encode8(const float (&x)[8], float scale)
{
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    return w;
}

__device__ __forceinline__ unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu; }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

__device__ __forceinline__ unsigned most_of(const float (&x)[8])
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = larger(m, magnitude(x[i]));
    return m;
}

// ... over the four lanes that hold a block.
__device__ __forceinline__ unsigned most_of_quad(unsigned m)
{
    m = larger(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));
    return larger(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
}

template <int DT>
__device__ __forceinline__ void widen8(const Eight<DT> &e, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)e.v[i];
}

// Eight elements of row `r` from column `c` on; what lies outside the matrix is 0.  The loads of an edge are as independent of
// one another as those of the interior: addresses are moved inside, and the values dropped.
template <int DT, bool EDGE>
__device__ __forceinline__ Eight<DT> load8(const Elem<DT> *x, size_t ld, unsigned rows, unsigned cols, unsigned r, unsigned c)
{
    if constexpr (!EDGE) {
        return reinterpret_cast<const EightAt<DT> *>(x + (size_t)r * ld + c)->e;
    } else {
        Eight<DT> e;
        const Elem<DT> *row = x + (size_t)(r < rows ? r : rows - 1u) * ld;
#pragma unroll
        for (unsigned i = 0; i < 8; ++i) e.v[i] = row[c + i < cols ? c + i : cols - 1u];
#pragma unroll
        for (unsigned i = 0; i < 8; ++i)
            if (!(r < rows && c + i < cols)) e.v[i] = (Elem<DT>)0.0f;
        return e;
    }
}

// Blocks along the rows alone.  A wave takes 512 columns of ROWS rows, eight elements a lane, four lanes a block.
constexpr unsigned kRowCols = 512;
template <int DT, int ROWS, bool EDGE>
__device__ __forceinline__ void quantize_rows(const Elem<DT> *x, size_t ld, unsigned rows, unsigned cols, unsigned r0, unsigned c,
                                              uint8_t *codes, uint8_t *scales)
{
    const unsigned groups = (cols + kGroup - 1) / kGroup;
    Eight<DT> e[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) e[i] = load8<DT, EDGE>(x, ld, rows, cols, r0 + i, c);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        float v[8];
        widen8<DT>(e[i], v);
        const unsigned s = scale_of(most_of_quad(most_of(v)));
        const unsigned w = encode8(v, scale_operand(s));
        const unsigned r = r0 + i;
        if (EDGE && (r >= rows || c >= groups * kGroup)) continue;
        reinterpret_cast<unsigned *>(codes + (size_t)r * (groups * 64u))[c / 8u] = w;
        if (threadIdx.x % 4u == 0u) scales[((size_t)(c / kGroup) * rows + r) * 4u + c / 32u % 4u] = (uint8_t)s;
    }
}

template <int DT, int ROWS>
__global__ __launch_bounds__(256) void k_quantize_rows(const Elem<DT> *__restrict__ x, size_t ld, unsigned rows, unsigned cols,
                                                       uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const unsigned col_blocks = (cols + kRowCols - 1) / kRowCols;
    const unsigned r0 = (blockIdx.x / col_blocks * 4u + threadIdx.x / 64u) * ROWS, c0 = blockIdx.x % col_blocks * kRowCols;
    if (r0 >= rows) return;
    const unsigned c = c0 + threadIdx.x % 64u * 8u;
    if (r0 + ROWS <= rows && c0 + kRowCols <= cols) quantize_rows<DT, ROWS, false>(x, ld, rows, cols, r0, c, codes, scales);
    else quantize_rows<DT, ROWS, true>(x, ld, rows, cols, r0, c, codes, scales);
}

// Blocks down the columns, and along the rows in the same pass if ROW.  A group takes a tile of 128 by 128: 64 bytes of every
// row of either result, and the scale words of 128 of them in a row.  The tile goes through LDS in the matrix's own type; a band
// of 32 rows is turned by a quarter of a row against the one above, so that the lanes that read one column in four bands
// meet different banks.
constexpr unsigned kTile = 128;
template <int DT>
__device__ __forceinline__ unsigned lds_at(unsigned r, unsigned c)  // in elements
{
    constexpr unsigned turn = kTile / 4;
    return r * kTile + ((c + r / 32u * turn) & (kTile - 1u));
}

template <int DT, bool ROW, bool EDGE>
__device__ __forceinline__ void load_tile(const Elem<DT> *x, size_t ld, unsigned rows, unsigned cols, unsigned r0, unsigned c0,
                                          uint8_t *codes, uint8_t *scales, Elem<DT> *tile)
{
    const unsigned groups = (cols + kGroup - 1) / kGroup, c = threadIdx.x % 16u * 8u;
    Eight<DT> e[8];
#pragma unroll
    for (unsigned i = 0; i < 8; ++i) e[i] = load8<DT, EDGE>(x, ld, rows, cols, r0 + i * 16u + threadIdx.x / 16u, c0 + c);
#pragma unroll
    for (unsigned i = 0; i < 8; ++i) {
        const unsigned r = i * 16u + threadIdx.x / 16u;
        *reinterpret_cast<Eight<DT> *>(__builtin_assume_aligned(tile + lds_at<DT>(r, c), 16)) = e[i];
        if constexpr (ROW) {
            float v[8];
            widen8<DT>(e[i], v);
            const unsigned s = scale_of(most_of_quad(most_of(v)));
            const unsigned w = encode8(v, scale_operand(s));
            if (EDGE && r0 + r >= rows) continue;
            reinterpret_cast<unsigned *>(codes + (size_t)(r0 + r) * (groups * 64u))[(c0 + c) / 8u] = w;
            if (threadIdx.x % 4u == 0u) scales[((size_t)(c0 / kGroup) * rows + r0 + r) * 4u + c / 32u] = (uint8_t)s;
        }
    }
}

template <int DT, bool ROW>
__global__ __launch_bounds__(256) void k_quantize_tiles(const Elem<DT> *__restrict__ x, size_t ld, unsigned rows, unsigned cols,
                                                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                        uint8_t *__restrict__ codes_t, uint8_t *__restrict__ scales_t)
{
    __shared__ __align__(16) Elem<DT> tile[kTile * kTile];
    const unsigned across = (cols + kTile - 1) / kTile;
    const unsigned r0 = blockIdx.x / across * kTile, c0 = blockIdx.x % across * kTile;
    if (r0 + kTile <= rows && c0 + kTile <= cols) load_tile<DT, ROW, false>(x, ld, rows, cols, r0, c0, codes, scales, tile);
    else load_tile<DT, ROW, true>(x, ld, rows, cols, r0, c0, codes, scales, tile);
    __syncthreads();
    // two neighbouring columns of one band to a lane; four lanes in a row hold the bands of a column
    const unsigned band = threadIdx.x % 4u, c = threadIdx.x / 4u * 2u;
    struct __attribute__((aligned(2 * sizeof(Elem<DT>)))) Two {
        Elem<DT> a, b;
    } e[32];
#pragma unroll
    for (unsigned i = 0; i < 32; ++i) e[i] = *reinterpret_cast<const Two *>(tile + lds_at<DT>(band * 32u + i, c));
    unsigned most[2] = {0, 0};
#pragma unroll
    for (unsigned i = 0; i < 32; ++i) {
        most[0] = larger(most[0], magnitude((float)e[i].a));
        most[1] = larger(most[1], magnitude((float)e[i].b));
    }
    const unsigned groups_t = (rows + kGroup - 1) / kGroup;
#pragma unroll
    for (unsigned k = 0; k < 2; ++k) {
        const unsigned s = scale_of(most[k]), col = c0 + c + k;
        u4 w;
#pragma unroll
        for (unsigned q = 0; q < 4; ++q) {
            float v[8];
#pragma unroll
            for (unsigned i = 0; i < 8; ++i) v[i] = (float)(k ? e[8 * q + i].b : e[8 * q + i].a);
            w[q] = encode8(v, scale_operand(s));
        }
        if (col < cols) {
            *reinterpret_cast<u4 *>(codes_t + (size_t)col * (groups_t * 64u) + r0 / 2u + band * 16u) = w;
            scales_t[((size_t)(r0 / kGroup) * cols + col) * 4u + band] = (uint8_t)s;
        }
    }
}

// ---------------------------------------------------------------------------
// values
// ---------------------------------------------------------------------------
template <int DT, int ROWS>
__global__ __launch_bounds__(256) void k_dequantize(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                    unsigned rows, unsigned cols, Elem<DT> *__restrict__ out, size_t ld)
{
    const unsigned col_blocks = (cols + kRowCols - 1) / kRowCols, groups = (cols + kGroup - 1) / kGroup;
    const unsigned r0 = (blockIdx.x / col_blocks * 4u + threadIdx.x / 64u) * ROWS;
    const unsigned c = blockIdx.x % col_blocks * kRowCols + threadIdx.x % 64u * 8u;
    if (r0 >= rows || c >= cols) return;
    unsigned w[ROWS], s[ROWS];
#pragma unroll
    for (unsigned i = 0; i < ROWS; ++i) {
        const unsigned r = r0 + i < rows ? r0 + i : rows - 1u;
        w[i] = reinterpret_cast<const unsigned *>(codes + (size_t)r * (groups * 64u))[c / 8u];
        s[i] = scales[((size_t)(c / kGroup) * rows + r) * 4u + c / 32u % 4u];
    }
#pragma unroll
    for (unsigned i = 0; i < ROWS; ++i) {
        if (r0 + i >= rows) break;
        typedef float f2 __attribute__((ext_vector_type(2)));
        const float scale = scale_operand(s[i]);
        const f2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 3)};
        EightAt<DT> e;
#pragma unroll
        for (unsigned k = 0; k < 8; ++k) e.e.v[k] = s[i] == 255u ? (Elem<DT>)__builtin_nanf("") : (Elem<DT>)v[k / 2][k % 2];
        Elem<DT> *to = out + (size_t)(r0 + i) * ld + c;
        if (c + 8u <= cols) {
            *reinterpret_cast<EightAt<DT> *>(to) = e;
        } else {
#pragma unroll
            for (unsigned k = 0; k < 8; ++k)
                if (c + k < cols) to[k] = e.e.v[k];
        }
    }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
// v_mfma_scale_f32_16x16x128: lane l holds elements 32 (l / 16) ... + 31 of row l % 16 of either operand in 16 bytes, their
// scale in a byte, and of the result rows 4 (l / 16) ... + 3 (A) of column l % 16 (B).
typedef int i8v __attribute__((ext_vector_type(8)));
typedef int i4v __attribute__((ext_vector_type(4)));

template <int SEL_A, int SEL_B>
__device__ __forceinline__ f4 mfma16(i4v a, i4v b, f4 c, int sa, int sb)
{
    const i8v wa = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, wb = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, SEL_A, sa, SEL_B, sb);
}

template <int DT>
__device__ __forceinline__ void put(Elem<DT> *p, float v, bool add)
{
    *p = (Elem<DT>)(add ? (float)*p + v : v);
}

}  // namespace
