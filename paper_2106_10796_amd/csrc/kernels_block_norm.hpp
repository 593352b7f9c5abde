// The norms before and after a block, with its gate and residual scale (include/cdsgd_block.h), forward and backward.
//
// A group of WAVES waves takes a row, E elements V times to a lane, and keeps it in registers between the sums over it.
#pragma once

#include "device_matrix.hpp"
#include "kernels_held8.hpp"

namespace {

// Elements to a lane at a time: 16 bytes of the widest type, so that loads and stores of either type are to whole lines.
template <int ST>
constexpr int kNormEach = kEach<ST>;

struct NormWeights {
    const float *weight, *block_weight, *gate;
    double scale, eps;
};

template <typename T>
struct Rows {
    T *p;
    size_t ld;
};
struct HeldOut {
    int8_t *codes;
    uint8_t *scales;
};
struct HeldIn {
    const void *p;
    size_t ld;
    const uint8_t *scales;
};

template <int E>
__device__ __forceinline__ void load_weight(const float *w, unsigned cols, unsigned c, float (&v)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = 1.0f;
    if (w) widened<kGradF32, E>(load_few<kGradF32, E>(w, cols, c), v);
}

template <int ST, int DT, int WAVES, int V>
__global__ __launch_bounds__(64 * WAVES) void k_block_norm_forward(NormWeights by, unsigned rows, unsigned cols, Rows<const Elem<ST>> h,
                                                                   Rows<const Elem<DT>> b, Rows<Elem<ST>> h_out, Rows<Elem<DT>> y,
                                                                   float *__restrict__ rstd, HeldOut h8, HeldOut b8)
{
    constexpr int E = kNormEach<ST>;
    __shared__ double room[2 * WAVES];
    unsigned turn = 0;
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        Few<ST, E> eh[V];
        Few<DT, E> eb[V];
#pragma unroll
        for (int k = 0; k < V; ++k) eh[k] = load_few<ST, E>(h.p + r * h.ld, cols, (k * 64 * WAVES + threadIdx.x) * E);
        if (b.p) {
#pragma unroll
            for (int k = 0; k < V; ++k) eb[k] = load_few<DT, E>(b.p + r * b.ld, cols, (k * 64 * WAVES + threadIdx.x) * E);
        }
        double n = 1.0;
        if (by.block_weight) {
            double sum = 0;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) sum = __builtin_fma((double)eb[k].v[i], (double)eb[k].v[i], sum);
            n = 1.0 / __builtin_sqrt(group_sum<WAVES>(sum, room, turn++) / cols + by.eps);
        }
        float v[V][E];
        double sum = 0;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const unsigned c = (k * 64 * WAVES + threadIdx.x) * E;
            if (b.p) {
                float w[E], g[E];
                load_weight<E>(by.block_weight, cols, c, w);
                load_weight<E>(by.gate, cols, c, g);
#pragma unroll
                for (int i = 0; i < E; ++i)
                    v[k][i] = (float)__builtin_fma((double)g[i] * (double)w[i] * by.scale, (double)eb[k].v[i] * n, (double)eh[k].v[i]);
                if (c < cols) store_few<ST, E>(h_out.p + r * h_out.ld, cols, c, v[k]);
            } else {
                widened<ST, E>(eh[k], v[k]);
            }
#pragma unroll
            for (int i = 0; i < E; ++i) sum = __builtin_fma((double)v[k][i], (double)v[k][i], sum);
        }
        const float rr = (float)(1.0 / __builtin_sqrt(group_sum<WAVES>(sum, room, turn++) / cols + by.eps));
        if (threadIdx.x == 0) {
            rstd[r] = rr;
            if (by.block_weight) rstd[(size_t)rows + r] = (float)n;
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const unsigned c = (k * 64 * WAVES + threadIdx.x) * E;
            float w[E], out[E];
            load_weight<E>(by.weight, cols, c, w);
#pragma unroll
            for (int i = 0; i < E; ++i) out[i] = v[k][i] * rr * w[i];
            if (c < cols) store_few<DT, E>(y.p + r * y.ld, cols, c, out);
            if (h8.codes) {
#pragma unroll
                for (int i = 0; i < E; ++i) v[k][i] = (float)(Elem<ST>)v[k][i];
                save<E>(h8.codes, h8.scales, r, cols, c, v[k]);
            }
            if (b8.codes) {
                widened<DT, E>(eb[k], v[k]);
                save<E>(b8.codes, b8.scales, r, cols, c, v[k]);
            }
        }
    }
}

template <int DT, int E, bool HELD>
struct NormIn {
    typedef typename std::conditional<HELD, Saved<E>, Few<DT, E>>::type Type;
    static __device__ __forceinline__ Type load(const HeldIn &x, size_t r, unsigned cols, unsigned c)
    {
        if constexpr (HELD) return load_saved<E>(static_cast<const int8_t *>(x.p), x.scales, r, cols, c);
        else return load_few<DT, E>(static_cast<const Elem<DT> *>(x.p) + r * x.ld, cols, c);
    }
    static __device__ __forceinline__ void values(const Type &x, float (&v)[E])
    {
        if constexpr (HELD) decode<E>(x.w, x.s, v);
        else widened<DT, E>(x, v);
    }
};

// parts: [groups][2][cols], the sums over a group's rows of dy x and of t c.
template <int ST, int DT, int WAVES, int V, bool HELD_H, bool HELD_B>
__global__ __launch_bounds__(64 * WAVES) void k_block_norm_backward(NormWeights by, unsigned rows, unsigned cols, Rows<const Elem<DT>> dy,
                                                                    Rows<const Elem<ST>> dh_out, HeldIn h, HeldIn b,
                                                                    const float *__restrict__ rstd, Rows<Elem<ST>> dh, Rows<Elem<DT>> db,
                                                                    float *__restrict__ parts)
{
    constexpr int E = kNormEach<ST>;
    typedef NormIn<ST, E, HELD_H> H;
    typedef NormIn<DT, E, HELD_B> B;
    __shared__ float room[2 * WAVES];
    unsigned turn = 0;
    float sum_x[V][E] = {}, sum_c[V][E] = {};
    const float mean = 1.0f / (float)cols, scale = (float)by.scale;
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        Few<DT, E> ed[V];
        Few<ST, E> et[V] = {};
        typename H::Type eh[V];
        typename B::Type eb[V] = {};
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const unsigned c = (k * 64 * WAVES + threadIdx.x) * E;
            ed[k] = load_few<DT, E>(dy.p + r * dy.ld, cols, c);
            eh[k] = H::load(h, r, cols, c);
            if (dh_out.p) et[k] = load_few<ST, E>(dh_out.p + r * dh_out.ld, cols, c);
            if (b.p) eb[k] = B::load(b, r, cols, c);
        }
        const float rr = rstd[r], n = by.block_weight ? rstd[(size_t)rows + r] : 1.0f;
        float x[V][E], t[V][E], part = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const unsigned c = (k * 64 * WAVES + threadIdx.x) * E;
            float w[E];
            load_weight<E>(by.weight, cols, c, w);
            H::values(eh[k], x[k]);
            widened<DT, E>(ed[k], t[k]);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                x[k][i] *= rr;
                sum_x[k][i] = __builtin_fmaf(t[k][i], x[k][i], sum_x[k][i]);
                t[k][i] *= w[i];
                part = __builtin_fmaf(t[k][i], x[k][i], part);
            }
        }
        const float c1 = group_sum<WAVES>(part, room, turn++) * mean;
        part = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const unsigned c = (k * 64 * WAVES + threadIdx.x) * E;
#pragma unroll
            for (int i = 0; i < E; ++i) t[k][i] = __builtin_fmaf(rr, __builtin_fmaf(-c1, x[k][i], t[k][i]), (float)et[k].v[i]);
            if (c < cols) store_few<ST, E>(dh.p + r * dh.ld, cols, c, t[k]);
            if (b.p) {
                float w[E], g[E];
                load_weight<E>(by.block_weight, cols, c, w);
                load_weight<E>(by.gate, cols, c, g);
                B::values(eb[k], x[k]);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    x[k][i] *= n;
                    sum_c[k][i] = __builtin_fmaf(t[k][i], x[k][i], sum_c[k][i]);
                    t[k][i] *= scale * g[i] * w[i];
                    part = __builtin_fmaf(t[k][i], x[k][i], part);
                }
            }
        }
        if (!b.p) continue;
        const float c2 = by.block_weight ? group_sum<WAVES>(part, room, turn++) * mean : 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const unsigned c = (k * 64 * WAVES + threadIdx.x) * E;
#pragma unroll
            for (int i = 0; i < E; ++i) t[k][i] = n * __builtin_fmaf(-c2, x[k][i], t[k][i]);
            if (c < cols) store_few<DT, E>(db.p + r * db.ld, cols, c, t[k]);
        }
    }
    float *const mine = parts + (size_t)blockIdx.x * 2u * cols;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const unsigned c = (k * 64 * WAVES + threadIdx.x) * E;
        if (c < cols) {
            store_few<kGradF32, E>(mine, cols, c, sum_x[k]);
            store_few<kGradF32, E>(mine + cols, cols, c, sum_c[k]);
        }
    }
}

// The groups' sums, joined in 64 bits in an order of their own number alone: 16 lanes take every sixteenth of them for a column.
__global__ __launch_bounds__(256) void k_block_norm_join(const float *__restrict__ parts, unsigned groups, unsigned cols, NormWeights by,
                                                         float *__restrict__ dweight, float *__restrict__ dblock_weight,
                                                         float *__restrict__ dgate)
{
    __shared__ double room[16][17];
    const unsigned col = threadIdx.x % 16u, slice = threadIdx.x / 16u, c = blockIdx.x * 16u + col;
    const bool second = blockIdx.y != 0;
    double sum = 0;
    if (c < cols) {
        const float *p = parts + (second ? cols : 0u) + c;
        for (unsigned g = slice; g < groups; g += 16u) sum += (double)p[(size_t)g * 2u * cols];
    }
    room[slice][col] = sum;
    __syncthreads();
    if (slice != 0 || c >= cols) return;
#pragma unroll
    for (unsigned k = 1; k < 16; ++k) sum += room[k][col];
    if (!second) {
        dweight[c] = (float)sum;
    } else {
        sum *= by.scale;
        if (dblock_weight) dblock_weight[c] = (float)(sum * (by.gate ? (double)by.gate[c] : 1.0));
        if (dgate) dgate[c] = (float)(sum * (by.block_weight ? (double)by.block_weight[c] : 1.0));
    }
}

}  // namespace
