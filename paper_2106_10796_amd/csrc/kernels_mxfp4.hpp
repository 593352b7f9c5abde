// Matrices in microscaled 4-bit floating point: quantisation along rows and columns, values, the matrix instruction.
#pragma once

namespace {

typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u4_by2 __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any address of a 16-bit (32-bit) element
typedef unsigned u4_by4 __attribute__((ext_vector_type(4), aligned(4)));

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

__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

// Elements as words: an fp32 one each, or two of 16 bits, which are compared and converted in pairs as they are: a third of the
// instructions that widening them takes (4096 x 4095 in bf16 in both forms: 14.4 us widened, 12.9 so; large ones the same).
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

// The larger magnitudes (of each half) of two words; `a` has no sign bits.
template <int DT>
__device__ __forceinline__ unsigned most_of(unsigned a, unsigned b)
{
    if constexpr (DT == kGradF32) return larger(a, b & 0x7FFFFFFFu);
    else return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b & 0x7FFF7FFFu)));
}

// A magnitude (of 16 bits: in the low half) as fp32 bits.
template <int DT>
__device__ __forceinline__ unsigned fp32_bits(unsigned a)
{
    if constexpr (DT == kGradF32) return a;
    else return __builtin_bit_cast(unsigned, widen16<DT>(a & 0xFFFFu));
}

// Two codes into byte `at` of w: of two fp32 words, or of the pair in word a.
template <int DT, int at>
__device__ __forceinline__ unsigned encode2(unsigned w, unsigned a, unsigned b, float scale)
{
    if constexpr (DT == kGradF32) {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __builtin_bit_cast(float, a), __builtin_bit_cast(float, b), scale, at);
    } else if constexpr (DT == kGradBF16) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(b2, a), scale, at);
    } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, a), scale, at);
    }
}

// Eight elements in a row.
template <int DT>
constexpr int kWords = DT == kGradF32 ? 8 : 4;
template <int DT>
struct Words {
    unsigned w[kWords<DT>];
};

template <int DT>
__device__ __forceinline__ unsigned encode8(const unsigned (&x)[kWords<DT>], float scale)
{
    constexpr int k = kWords<DT> / 4;
    unsigned w = 0;
    w = encode2<DT, 0>(w, x[0], x[k - 1], scale);
    w = encode2<DT, 1>(w, x[k], x[2 * k - 1], scale);
    w = encode2<DT, 2>(w, x[2 * k], x[3 * k - 1], scale);
    w = encode2<DT, 3>(w, x[3 * k], x[4 * k - 1], scale);
    return w;
}

template <int DT>
__device__ __forceinline__ unsigned most_of_eight(const unsigned (&x)[kWords<DT>])
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < kWords<DT>; ++i) m = most_of<DT>(m, x[i]);
    return fp32_bits<DT>(DT == kGradF32 ? m : larger(m & 0xFFFFu, m >> 16));
}

// ... over the four lanes that hold a block.
__device__ __forceinline__ unsigned most_of_quad(unsigned m)
{
    m = larger(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));
    return larger(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
}

// 16 bytes of a row, the first of which are elements `d` and on of those that were loaded: what is past them is 0.
template <int DT>
__device__ __forceinline__ u4 shifted(u4 w, unsigned d)
{
    const unsigned words = DT == kGradF32 ? d : d / 2u;
    u4 t = (words & 1u) ? u4{w.y, w.z, w.w, 0u} : w;
    t = (words & 2u) ? u4{t.z, t.w, 0u, 0u} : t;
    if (words > 3u) t = u4{0u, 0u, 0u, 0u};
    if constexpr (DT != kGradF32) {
        if (d & 1u) t = u4{t.x >> 16 | t.y << 16, t.y >> 16 | t.z << 16, t.z >> 16 | t.w << 16, t.w >> 16};
    }
    return t;
}

// Eight elements of row `r` from column `c` on; what lies outside the matrix is 0.  At an edge the load is moved inside the row and
// its elements back to their places, so that it is one load there, too.
template <int DT, bool EDGE>
__device__ __forceinline__ Eight<DT> load8(const Elem<DT> *x, size_t ld, unsigned rows, unsigned cols, unsigned r, unsigned c)
{
    if constexpr (!EDGE) {
        return reinterpret_cast<const EightAt<DT> *>(x + (size_t)r * ld + c)->e;
    } else {
        constexpr unsigned kEach = 16 / sizeof(Elem<DT>), kLoads = 8 / kEach;
        const Elem<DT> *row = x + (size_t)(r < rows ? r : rows - 1u) * ld;
        Eight<DT> e;
        if (cols >= kEach) {
            struct {
                u4 q[kLoads];
            } got;
#pragma unroll
            for (unsigned k = 0; k < kLoads; ++k) {
                struct __attribute__((packed, aligned(sizeof(Elem<DT>)))) At {
                    u4 v;
                };
                const unsigned from = c + k * kEach, at = from + kEach <= cols ? from : cols - kEach;
                got.q[k] = shifted<DT>(reinterpret_cast<const At *>(row + at)->v, from - at);
                if (r >= rows) got.q[k] = u4{0u, 0u, 0u, 0u};
            }
            e = __builtin_bit_cast(Eight<DT>, got);
        } else {
#pragma unroll
            for (unsigned i = 0; i < 8; ++i) e.v[i] = row[c + i < cols ? c + i : cols - 1u];
#pragma unroll
            for (unsigned i = 0; i < 8; ++i)
                if (!(r < rows && c + i < cols)) e.v[i] = (Elem<DT>)0.0f;
        }
        return e;
    }
}

// Blocks along the rows alone.  A wave takes 512 columns of ROWS rows, eight elements to a lane, four lanes to a block.  Bound by
// HBM: 5.5 TB/s over 2048 x 25088 in bf16, 5.6 over 4096 x 25088 in fp32 (4 rows; with loads that do not keep 22 and 92 us instead of
// 23 and 84, codes stored past the caches 21 and 81, but a product reads them next).
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
        const Words<DT> v = __builtin_bit_cast(Words<DT>, e[i]);
        const unsigned s = scale_of(most_of_quad(most_of_eight<DT>(v.w)));
        const unsigned w = encode8<DT>(v.w, scale_operand(s));
        const unsigned r = r0 + i;
        if (EDGE && (r >= rows || c >= groups * kGroup)) continue;
        reinterpret_cast<unsigned *>(codes + (size_t)r * (groups * 64u))[c / 8u] = w;
        if (threadIdx.x % 4u == 0u) scales[((size_t)(c / kGroup) * rows + r) * 4u + c / 32u % 4u] = (uint8_t)s;
    }
}

template <int DT, int ROWS>
__global__ __launch_bounds__(256) void k_quantize_rows(const Elem<DT> *__restrict__ x, size_t ld, unsigned rows, unsigned cols,
                                                       uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, unsigned first)
{
    const unsigned col_blocks = (cols + kRowCols - 1) / kRowCols, group = first + blockIdx.x;
    const unsigned r0 = (group / col_blocks * 4u + threadIdx.x / 64u) * ROWS, c0 = group % col_blocks * kRowCols;
    if (r0 >= rows) return;
    const unsigned c = c0 + threadIdx.x % 64u * 8u;
    if (r0 + ROWS <= rows && c0 + kRowCols <= cols) quantize_rows<DT, ROWS, false>(x, ld, rows, cols, r0, c, codes, scales);
    else quantize_rows<DT, ROWS, true>(x, ld, rows, cols, r0, c, codes, scales);
}

// Blocks down the columns, and along the rows in the same pass if ROW.  A group takes a tile of 128 by 128: 64 bytes of every
// row of either result, and the scale words of 128 of them in a row.  The tile goes through LDS in the matrix's own type; a band
// of 32 rows is turned by 64 bytes against the one above, so that the lanes that read one column in four bands meet different banks.
// Bound by HBM and by its stores of half lines: both forms of 4096 x 25088 in fp32 5.2 TB/s (100 us; 106 with neighbouring tiles on
// different XCDs), of 2048 x 25088 in bf16 4.5 (35 us; 37.5).
constexpr unsigned kTile = 128;
template <int DT>
__device__ __forceinline__ unsigned lds_at(unsigned r, unsigned c)  // in elements
{
    constexpr unsigned turn = 64 / sizeof(Elem<DT>);
    return r * kTile + ((c + r / 32u * turn) & (kTile - 1u));
}

inline unsigned long long tile_groups(size_t rows, size_t cols)
{
    const unsigned long long supers = (unsigned long long)((rows + 2 * kTile - 1) / (2 * kTile)) * ((cols + 2 * kTile - 1) / (2 * kTile));
    return (supers + 7u) / 8u * 32u;
}

// A lane's part of a column pass is 4 bytes of a row: one fp32 column, or two of 16 bits.
template <int DT>
constexpr unsigned kTileLanes = 512 / (4 / sizeof(Elem<DT>));

template <int DT, bool ROW, bool EDGE>
__device__ __forceinline__ void load_tile(const Elem<DT> *x, size_t ld, unsigned rows, unsigned cols, unsigned r0, unsigned c0,
                                          uint8_t *codes, uint8_t *scales, Elem<DT> *tile)
{
    constexpr unsigned kRows = kTileLanes<DT> / 16u;
    const unsigned groups = (cols + kGroup - 1) / kGroup, c = threadIdx.x % 16u * 8u;
    Eight<DT> e[kTile / kRows];
#pragma unroll
    for (unsigned i = 0; i < kTile / kRows; ++i) e[i] = load8<DT, EDGE>(x, ld, rows, cols, r0 + i * kRows + threadIdx.x / 16u, c0 + c);
#pragma unroll
    for (unsigned i = 0; i < kTile / kRows; ++i) {
        const unsigned r = i * kRows + threadIdx.x / 16u;
        *reinterpret_cast<Eight<DT> *>(__builtin_assume_aligned(tile + lds_at<DT>(r, c), 16)) = e[i];
        if constexpr (ROW) {
            const Words<DT> v = __builtin_bit_cast(Words<DT>, e[i]);
            const unsigned s = scale_of(most_of_quad(most_of_eight<DT>(v.w)));
            const unsigned w = encode8<DT>(v.w, scale_operand(s));
            if (EDGE && r0 + r >= rows) continue;
            reinterpret_cast<unsigned *>(codes + (size_t)(r0 + r) * (groups * 64u))[(c0 + c) / 8u] = w;
            if (threadIdx.x % 4u == 0u) scales[((size_t)(c0 / kGroup) * rows + r0 + r) * 4u + c / 32u] = (uint8_t)s;
        }
    }
}

template <int DT, bool ROW>
__global__ __launch_bounds__(kTileLanes<DT>) void k_quantize_tiles(const Elem<DT> *__restrict__ x, size_t ld, unsigned rows,
                                                                   unsigned cols, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                                   uint8_t *__restrict__ codes_t, uint8_t *__restrict__ scales_t,
                                                                   unsigned first)
{
    __shared__ __align__(16) Elem<DT> tile[kTile * kTile];
    // Four tiles, two by two, run on one XCD (group b on XCD b % 8) one after the other, so that the halves of a line of codes that
    // neighbouring tiles write meet in one L2.
    const unsigned supers_across = (cols + 2 * kTile - 1) / (2 * kTile), group = first + blockIdx.x, i = group / 8u, super = i / 4u * 8u + group % 8u;
    const unsigned r0 = (super / supers_across * 2u + i / 2u % 2u) * kTile, c0 = (super % supers_across * 2u + i % 2u) * kTile;
    if (r0 >= rows || c0 >= cols) return;
    if (r0 + kTile <= rows && c0 + kTile <= cols) load_tile<DT, ROW, false>(x, ld, rows, cols, r0, c0, codes, scales, tile);
    else load_tile<DT, ROW, true>(x, ld, rows, cols, r0, c0, codes, scales, tile);
    __syncthreads();
    // four lanes in a row hold the bands of a column (of two neighbouring ones)
    constexpr unsigned kCols = 4 / sizeof(Elem<DT>);
    const unsigned band = threadIdx.x % 4u, c = threadIdx.x / 4u * kCols;
    unsigned e[32];
#pragma unroll
    for (unsigned i = 0; i < 32; ++i) e[i] = *reinterpret_cast<const unsigned *>(__builtin_assume_aligned(tile + lds_at<DT>(band * 32u + i, c), 4));
    const unsigned groups_t = (rows + kGroup - 1) / kGroup;
    unsigned most = 0;
#pragma unroll
    for (unsigned i = 0; i < 32; ++i) most = most_of<DT>(most, e[i]);
#pragma unroll
    for (unsigned k = 0; k < kCols; ++k) {
        const unsigned s = scale_of(fp32_bits<DT>(k ? most >> 16 : most)), col = c0 + c + k;
        u4 w;
#pragma unroll
        for (unsigned q = 0; q < 4; ++q) {
            unsigned v[kWords<DT>];
#pragma unroll
            for (unsigned z = 0; z < kWords<DT>; ++z) {
                if constexpr (DT == kGradF32) v[z] = e[8 * q + z];
                else v[z] = __builtin_amdgcn_perm(e[8 * q + 2 * z + 1], e[8 * q + 2 * z], k ? 0x07060302u : 0x05040100u);  // this column's half of two rows
            }
            w[q] = encode8<DT>(v, scale_operand(s));
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
// 16 bytes of a row to a lane, so that a wave's store is to whole lines in a row, past the caches (fp32, 4096 x 25088: 88 us
// at the default policy, 66 so, 7.0 TB/s; eight elements to a lane 160.  In turn with the quantisation of such a matrix it takes 78).
template <int DT>
constexpr unsigned kValueCols = 64 * 16 / sizeof(Elem<DT>);
template <int DT, int ROWS>
__global__ __launch_bounds__(256) void k_dequantize(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                    unsigned rows, unsigned cols, Elem<DT> *__restrict__ out, size_t ld, unsigned first)
{
    constexpr unsigned E = 16 / sizeof(Elem<DT>);
    const unsigned col_blocks = (cols + kValueCols<DT> - 1) / kValueCols<DT>, groups = (cols + kGroup - 1) / kGroup, group = first + blockIdx.x;
    const unsigned r0 = (group / col_blocks * 4u + threadIdx.x / 64u) * ROWS;
    const unsigned c = group % col_blocks * kValueCols<DT> + threadIdx.x % 64u * E;
    if (r0 >= rows || c >= cols) return;
    unsigned w[ROWS], s[ROWS];
#pragma unroll
    for (unsigned i = 0; i < ROWS; ++i) {
        const unsigned r = r0 + i < rows ? r0 + i : rows - 1u;
        const uint8_t *row = codes + (size_t)r * (groups * 64u);
        w[i] = E == 8 ? reinterpret_cast<const unsigned *>(row)[c / 8u] : reinterpret_cast<const uint16_t *>(row)[c / 4u];
        s[i] = scales[((size_t)(c / kGroup) * rows + r) * 4u + c / 32u % 4u];
    }
#pragma unroll
    for (unsigned i = 0; i < ROWS; ++i) {
        if (r0 + i >= rows) break;
        typedef float f2 __attribute__((ext_vector_type(2)));
        const float scale = scale_operand(s[i]);
        f2 v[4];
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 1);
        if constexpr (E == 8) {
            v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 2);
            v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 3);
        }
        struct {
            Elem<DT> v[E];
        } e;
#pragma unroll
        for (unsigned k = 0; k < E; ++k) e.v[k] = s[i] == 255u ? (Elem<DT>)__builtin_nanf("") : (Elem<DT>)v[k / 2][k % 2];
        Elem<DT> *to = out + (size_t)(r0 + i) * ld + c;
        if (c + E <= cols) {
            typedef typename std::conditional<sizeof(Elem<DT>) == 4, u4_by4, u4_by2>::type u4_at;
            const u4 bits = __builtin_bit_cast(u4, e);
            __builtin_nontemporal_store(bits, reinterpret_cast<u4_at *>(to));
        } else {
#pragma unroll
            for (unsigned k = 0; k < E; ++k)
                if (c + k < cols) to[k] = e.v[k];
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
