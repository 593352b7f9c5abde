// Matrices in 8 bits (MXINT8): quantisation, values, and the gated activation with its gradients, which saves and reads them.
//
// A wave takes 64 E neighbouring elements of a row, E to a lane, or E times a power of two of several rows where those are short; 32 / E
// lanes hold a block of the 8-bit form.
#pragma once

#include "device_matrix.hpp"

namespace {

// Elements to a lane: 16 bytes.
template <int DT>
constexpr int kEach = DT == kGradF32 ? 4 : 8;

// Blocks of a row.
template <typename T>
__host__ __device__ constexpr T held_groups(T cols)
{
    return (cols + 31u) / 32u;
}

__device__ __forceinline__ unsigned larger_of(unsigned a, unsigned b) { return a > b ? a : b; }

// The scale byte of the block that a lane's elements are of: the exponent field of its largest magnitude.
template <int E>
__device__ __forceinline__ unsigned block_scale(const float (&x)[E])
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) m = larger_of(m, __builtin_bit_cast(unsigned, x[i]) & 0x7FFFFFFFu);
    m = larger_of(m, moved<kDppXor1>(m));
    m = larger_of(m, moved<kDppXor2>(m));
    if constexpr (E == 4) m = larger_of(m, moved<kDppMirror8>(m));
    return m >> 23;
}

// E codes, four to a word.  x 2^(133 - s) is exact (two factors of 2 may not be: 2^133 is none of fp32), and adding 3 * 2^22 rounds it to a whole
// number, ties to even, which is then the sum's low byte in two's complement.
template <int E>
struct Codes {
    unsigned w[E / 4];
};
template <int E>
__device__ __forceinline__ Codes<E> encode(const float (&x)[E], unsigned s)
{
    Codes<E> c;
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
        unsigned b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float y = __builtin_amdgcn_ldexpf(x[4 * k + i], 133 - (int)s);
            b[i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_fmed3f(y, -127.0f, 127.0f) + 12582912.0f);
        }
        const unsigned low = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), high = __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
        c.w[k] = s == 255u ? 0u : low | high;
    }
    return c;
}

template <int E>
__device__ __forceinline__ void decode(const Codes<E> &c, unsigned s, float (&x)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int v = (int)(c.w[i / 4] << (24 - 8 * (i % 4))) >> 24;
        x[i] = s == 255u ? __builtin_nanf("") : __builtin_amdgcn_ldexpf((float)v, (int)s - 133);
    }
}

// E elements of a row to 8 bits: all of the padded row is written.  (Lanes behind it take part in the block's largest magnitude with zeros.)
template <int E>
__device__ __forceinline__ void save(int8_t *codes, uint8_t *scales, size_t r, unsigned cols, unsigned c, const float (&x)[E])
{
    const unsigned groups = held_groups(cols), s = block_scale<E>(x);
    const Codes<E> w = encode<E>(x, s);
    if (c >= groups * 32u) return;
    *reinterpret_cast<Codes<E> *>(__builtin_assume_aligned(codes + r * (groups * 32u) + c, E)) = w;
    if (c % 32u == 0u) scales[r * groups + c / 32u] = (uint8_t)s;
}

// What a lane reads of a matrix in 8 bits.
template <int E>
struct Saved {
    Codes<E> w;
    unsigned s;
};
template <int E>
__device__ __forceinline__ Saved<E> load_saved(const int8_t *codes, const uint8_t *scales, size_t r, unsigned cols, unsigned c)
{
    const unsigned groups = held_groups(cols);
    Saved<E> x = {};
    if (c < groups * 32u) {
        x.w = *reinterpret_cast<const Codes<E> *>(__builtin_assume_aligned(codes + r * (groups * 32u) + c, E));
        x.s = scales[r * groups + c / 32u];
    }
    return x;
}

template <int DT, int E>
__device__ __forceinline__ void widened(const Few<DT, E> &x, float (&v)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = (float)x.v[i];
}

// Where a lane works: `lanes` (a power of two, 32 / E to 64) lanes in a row hold a row's elements, waves take ROWS of such rows.
struct Place {
    size_t r;
    unsigned c;
};
template <int E, int ROWS>
__device__ __forceinline__ Place place_of(unsigned cols, unsigned lanes_log2, unsigned first)
{
    const unsigned lane = threadIdx.x % 64u, across = (cols + 64u * E - 1u) / (64u * E), group = first + blockIdx.x;
    const unsigned long long wave = (unsigned long long)(group / across) * 4u + threadIdx.x / 64u;
    return {(size_t)((wave * ROWS << (6u - lanes_log2)) + (lane >> lanes_log2)), group % across * (64u * E) + (lane & ((1u << lanes_log2) - 1u)) * E};
}

// Rows between a lane's one and its next.
__device__ __forceinline__ unsigned rows_apart(unsigned lanes_log2) { return 64u >> lanes_log2; }

template <int DT, int ROWS>
__global__ __launch_bounds__(256) void k_held8_quantize(const Elem<DT> *__restrict__ x, size_t ld, unsigned rows, unsigned cols,
                                                        int8_t *__restrict__ codes, uint8_t *__restrict__ scales, unsigned lanes_log2,
                                                        unsigned first)
{
    constexpr int E = kEach<DT>;
    const Place at = place_of<E, ROWS>(cols, lanes_log2, first);
    const unsigned apart = rows_apart(lanes_log2);
    Few<DT, E> e[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t r = at.r + i * apart;
        e[i] = load_few<DT, E>(x + (r < rows ? r : rows - 1u) * ld, cols, at.c);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        float v[E];
        widened<DT, E>(e[i], v);
        if (at.r + i * apart < rows) save<E>(codes, scales, at.r + i * apart, cols, at.c, v);
    }
}

template <int DT, int ROWS>
__global__ __launch_bounds__(256) void k_held8_values(const int8_t *__restrict__ codes, const uint8_t *__restrict__ scales, unsigned rows,
                                                      unsigned cols, Elem<DT> *__restrict__ out, size_t ld, unsigned lanes_log2, unsigned first)
{
    constexpr int E = kEach<DT>;
    const Place at = place_of<E, ROWS>(cols, lanes_log2, first);
    const unsigned apart = rows_apart(lanes_log2);
    Saved<E> e[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t r = at.r + i * apart;
        e[i] = load_saved<E>(codes, scales, r < rows ? r : rows - 1u, cols, at.c);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t r = at.r + i * apart;
        float v[E];
        decode<E>(e[i].w, e[i].s, v);
        if (r < rows) store_few<DT, E>(out + r * ld, cols, at.c, v);
    }
}

// ---------------------------------------------------------------------------
// gated activations
// ---------------------------------------------------------------------------
// Both activations are a sigmoid(z): z = a (SiLU), or 2 sqrt(2 / pi) (a + 0.044715 a^3), for (1 + tanh(w)) / 2 is sigmoid(2 w).  With
// e = exp(-|z|) at most 1, sigmoid and one minus it are 1 / (1 + e) and e / (1 + e), neither of which loses anything where it is small.
struct Act {
    float act, slope;
};
constexpr int kSilu = CDSGD_ACT_SILU;

template <int ACT>
__device__ __forceinline__ Act act_of(float a)
{
    float z = a, dz = 1.0f;
    if constexpr (ACT != kSilu) {
        constexpr float k = 1.5957691216057308f;
        const float b = __builtin_amdgcn_fmed3f(a, -64.0f, 64.0f), b2 = b * b;  // beyond 64 the sigmoid is 0 or 1, and a^2 would overflow in time
        z = k * __builtin_fmaf(0.044715f * b2, b, b);
        dz = k * __builtin_fmaf(3.0f * 0.044715f, b2, 1.0f);
    }
    // exp(-|z|) = 2^(-|z| log2 e): the product's rounding error comes back as a factor
    const float m = -__builtin_fabsf(z), t = m * 1.44269504f;
    const float rest = __builtin_fmaf(m, 1.44269504f, -t) + m * 1.92596300e-8f;
    float e = __builtin_amdgcn_exp2f(t);
    e = t < -200.0f ? 0.0f : __builtin_fmaf(e, rest * 0.69314718f, e);
    const float d = __builtin_amdgcn_rcpf(1.0f + e), ed = e * d;
    const float s = z < 0.0f ? ed : d, act = a * s;
    return {act, __builtin_fmaf(act * (z < 0.0f ? d : ed), dz, s)};
}

template <int DT, int ACT, bool SAVE, int ROWS>
__global__ __launch_bounds__(256) void k_gated_forward(const Elem<DT> *__restrict__ a, size_t ld_a, const Elem<DT> *__restrict__ u, size_t ld_u,
                                                       Elem<DT> *__restrict__ y, size_t ld_y, unsigned rows, unsigned cols,
                                                       int8_t *__restrict__ a8, uint8_t *__restrict__ a8_scales, int8_t *__restrict__ u8,
                                                       uint8_t *__restrict__ u8_scales, unsigned lanes_log2, unsigned first)
{
    constexpr int E = kEach<DT>;
    const Place at = place_of<E, ROWS>(cols, lanes_log2, first);
    const unsigned apart = rows_apart(lanes_log2);
    Few<DT, E> ea[ROWS], eu[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t r = at.r + i * apart < rows ? at.r + i * apart : rows - 1u;
        ea[i] = load_few<DT, E>(a + r * ld_a, cols, at.c);
        eu[i] = load_few<DT, E>(u + r * ld_u, cols, at.c);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t r = at.r + i * apart;
        if (r >= rows) continue;
        float va[E], vu[E], vy[E];
        widened<DT, E>(ea[i], va);
        widened<DT, E>(eu[i], vu);
#pragma unroll
        for (int k = 0; k < E; ++k) vy[k] = act_of<ACT>(va[k]).act * vu[k];
        store_few<DT, E>(y + r * ld_y, cols, at.c, vy);
        if constexpr (SAVE) {
            save<E>(a8, a8_scales, r, cols, at.c, va);
            save<E>(u8, u8_scales, r, cols, at.c, vu);
        }
    }
}

template <int DT, int ACT, bool HELD, int ROWS>
__global__ __launch_bounds__(256) void k_gated_backward(const Elem<DT> *__restrict__ dy, size_t ld_dy, const void *__restrict__ a, size_t ld_a,
                                                        const uint8_t *__restrict__ a8_scales, const void *__restrict__ u, size_t ld_u,
                                                        const uint8_t *__restrict__ u8_scales, Elem<DT> *__restrict__ da, size_t ld_da,
                                                        Elem<DT> *__restrict__ du, size_t ld_du, unsigned rows, unsigned cols,
                                                        unsigned lanes_log2, unsigned first)
{
    constexpr int E = kEach<DT>;
    typedef typename std::conditional<HELD, Saved<E>, Few<DT, E>>::type Held;
    const Place at = place_of<E, ROWS>(cols, lanes_log2, first);
    const unsigned apart = rows_apart(lanes_log2);
    Few<DT, E> ed[ROWS];
    Held ea[ROWS], eu[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t r = at.r + i * apart < rows ? at.r + i * apart : rows - 1u;
        ed[i] = load_few<DT, E>(dy + r * ld_dy, cols, at.c);
        if constexpr (HELD) {
            ea[i] = load_saved<E>(static_cast<const int8_t *>(a), a8_scales, r, cols, at.c);
            eu[i] = load_saved<E>(static_cast<const int8_t *>(u), u8_scales, r, cols, at.c);
        } else {
            ea[i] = load_few<DT, E>(static_cast<const Elem<DT> *>(a) + r * ld_a, cols, at.c);
            eu[i] = load_few<DT, E>(static_cast<const Elem<DT> *>(u) + r * ld_u, cols, at.c);
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t r = at.r + i * apart;
        if (r >= rows) continue;
        float va[E], vu[E], vd[E];
        widened<DT, E>(ed[i], vd);
        if constexpr (HELD) {
            decode<E>(ea[i].w, ea[i].s, va);
            decode<E>(eu[i].w, eu[i].s, vu);
        } else {
            widened<DT, E>(ea[i], va);
            widened<DT, E>(eu[i], vu);
        }
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const Act f = act_of<ACT>(va[k]);
            va[k] = vd[k] * vu[k] * f.slope;
            vu[k] = vd[k] * f.act;
        }
        store_few<DT, E>(da + r * ld_da, cols, at.c, va);
        store_few<DT, E>(du + r * ld_du, cols, at.c, vu);
    }
}

}  // namespace
