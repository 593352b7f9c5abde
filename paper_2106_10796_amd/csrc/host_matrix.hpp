// Host side of entry points that take matrices.
#pragma once

#include <type_traits>

namespace {

inline bool good_dtype(int t) { return t == CDSGD_GRAD_F32 || t == CDSGD_GRAD_BF16 || t == CDSGD_GRAD_F16; }
inline size_t bytes_of(int dtype) { return dtype == CDSGD_GRAD_F32 ? 4u : 2u; }
inline bool good_extent(size_t n) { return n > 0 && n <= 0x7FFFFFFFu; }

// Bytes from the first element of a matrix to the last, both included.
inline size_t extent_bytes(size_t rows, size_t cols, size_t ld, size_t elem) { return ((rows - 1) * ld + cols) * elem; }

// A buffer as rows of `width` bytes, `ld` bytes apart; one row: a plain range of bytes.  (p NULL: nothing.)
struct Span {
    const void *p;
    size_t rows, width, ld;
};
inline Span range_of(const void *p, size_t bytes) { return {p, 1, bytes, bytes}; }
inline Span matrix_of(const void *p, size_t rows, size_t cols, size_t ld, int dtype) { return {p, rows, cols * bytes_of(dtype), ld * bytes_of(dtype)}; }

// Do two of them share a byte?  Slices of the columns of one matrix do not; ranges that overlap otherwise are taken to.
inline bool overlap(const Span &a, const Span &b)
{
    if (!overlap2(a.p, (a.rows - 1) * a.ld + a.width, b.p, (b.rows - 1) * b.ld + b.width)) return false;
    if (a.ld != b.ld) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const size_t after = y >= x ? (y - x) % a.ld : (a.ld - (x - y) % a.ld) % a.ld;  // from a row of a to the next row of b
    return !(after >= a.width && after + b.width <= a.ld);
}

// Does one of the outputs share a byte with another or with an input?
inline bool any_overlap(const Span *out, int outs, const Span *in, int ins)
{
    for (int i = 0; i < outs; ++i) {
        for (int k = i + 1; k < outs; ++k)
            if (overlap(out[i], out[k])) return true;
        for (int k = 0; k < ins; ++k)
            if (overlap(out[i], in[k])) return true;
    }
    return false;
}

// Calls f(std::integral_constant<int, element type>).
template <typename F>
void with_dtype(int dtype, F f)
{
    if (dtype == CDSGD_GRAD_BF16) f(std::integral_constant<int, kGradBF16>());
    else if (dtype == CDSGD_GRAD_F16) f(std::integral_constant<int, kGradF16>());
    else f(std::integral_constant<int, kGradF32>());
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

}  // namespace
