// The norms before and after a block, with its gate and residual scale (include/cdsgd_block.h), forward and backward.
//
// A group of WAVES waves takes a row, E elements V times to a lane, and keeps it in registers (of more than 8192 columns partly in scratch) between
// the sums over it.
#pragma once

#include "device_matrix.hpp"
#include "kernels_held8.hpp"

namespace {

// Elements to a lane at a time: 16 bytes of fp32, so that its loads and stores are to whole lines.
constexpr int kNormEach = 4;

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

// Weights of a lane's elements: in registers throughout where there are few of them, or read again (from L2) for every row.
constexpr int kKeptWeights = 8;

// The next row's elements are asked for ahead where there is room for them (forward and backward, us, 4096 x 8192 in bf16 on an fp32 stream, 8 waves
// of four fours: ahead 126, 147, not 103, 163;  2048 x 12288, 16 waves: 158, 368, not 106, 236).
template <int WAVES, int V>
constexpr bool kForwardAhead = V <= 2;
template <int WAVES, int V>
constexpr bool kBackwardAhead = V <= 2 || WAVES <= 8;

// A group goes from row to row, and asks for the next one's elements before it sums this one's.  Bound by HBM and by the two sums that a row
// waits for: 8192 x 4096 in bf16 on an fp32 stream 88 us, 4.6 TB/s (weights read again for every row, and nothing asked for ahead: 105).
template <int ST, int DT, int WAVES, int V>
__global__ __launch_bounds__(64 * WAVES) void k_block_norm_forward(NormWeights by, unsigned rows, unsigned cols, Rows<const Elem<ST>> h,
                                                                   Rows<const Elem<DT>> b, Rows<Elem<ST>> h_out, Rows<Elem<DT>> y,
                                                                   float *__restrict__ rstd, HeldOut h8, HeldOut b8)
{
    constexpr int E = kNormEach;
    constexpr bool kKept = V * E <= kKeptWeights;
    __shared__ double room[2 * WAVES];
    unsigned turn = 0;
    const auto place = [&](int k) __attribute__((always_inline)) { return (k * 64 * WAVES + threadIdx.x) * E; };
    // scale gate block_weight
    const auto load_into = [&](int k, double (&into)[E]) __attribute__((always_inline)) {
        float w[E], g[E];
        load_weight<E>(by.block_weight, cols, place(k), w);
        load_weight<E>(by.gate, cols, place(k), g);
#pragma unroll
        for (int i = 0; i < E; ++i) into[i] = (double)g[i] * (double)w[i] * by.scale;
    };
    double into[V][E];
    float weight[V][E];
    if constexpr (kKept) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            load_weight<E>(by.weight, cols, place(k), weight[k]);
            if (b.p) load_into(k, into[k]);
        }
    }
    Few<ST, E> next_h[V];
    Few<DT, E> next_b[V] = {};
    const auto ask = [&](size_t r) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            next_h[k] = load_few<ST, E>(h.p + r * h.ld, cols, place(k));
            if (b.p) next_b[k] = load_few<DT, E>(b.p + r * b.ld, cols, place(k));
        }
    };
    const double mean = 1.0 / cols;
    if constexpr (kForwardAhead<WAVES, V>) ask(blockIdx.x);
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        if constexpr (!kForwardAhead<WAVES, V>) ask(r);
        Few<DT, E> eb[V];
        float v[V][E];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            widened<ST, E>(next_h[k], v[k]);
            eb[k] = next_b[k];
        }
        if (kForwardAhead<WAVES, V> && r + gridDim.x < rows) ask(r + gridDim.x);
        double n = 1.0, sum = 0;
        if (by.block_weight) {
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) sum = __builtin_fma((double)eb[k].v[i], (double)eb[k].v[i], sum);
            n = 1.0 / __builtin_sqrt(group_sum<WAVES>(sum, room, turn++) * mean + by.eps);
            sum = 0;
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (b.p) {
                if constexpr (!kKept) load_into(k, into[k]);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const double x = __builtin_fma(into[k][i], (double)eb[k].v[i] * n, (double)v[k][i]);
                    v[k][i] = (float)x;  // (a 16-bit h_out is rounded from this, as torch takes 64 bits to 16: by way of fp32)
                    sum = __builtin_fma(x, x, sum);
                }
                if (place(k) < cols) store_few<ST, E>(h_out.p + r * h_out.ld, cols, place(k), v[k]);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) sum = __builtin_fma((double)v[k][i], (double)v[k][i], sum);
            }
        }
        const float rr = (float)(1.0 / __builtin_sqrt(group_sum<WAVES>(sum, room, turn++) * mean + by.eps));
        if (threadIdx.x == 0) {
            rstd[r] = rr;
            if (by.block_weight) rstd[(size_t)rows + r] = (float)n;
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float out[E];
            if constexpr (!kKept) load_weight<E>(by.weight, cols, place(k), weight[k]);
#pragma unroll
            for (int i = 0; i < E; ++i) out[i] = v[k][i] * rr * weight[k][i];
            if (place(k) < cols) store_few<DT, E>(y.p + r * y.ld, cols, place(k), out);
            if (h8.codes) {
#pragma unroll
                for (int i = 0; i < E; ++i) v[k][i] = (float)(Elem<ST>)v[k][i];
                save<E>(h8.codes, h8.scales, r, cols, place(k), v[k]);
            }
            if (b8.codes) {
                widened<DT, E>(eb[k], out);
                save<E>(b8.codes, b8.scales, r, cols, place(k), out);
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

// parts: [groups][2][cols, to a whole four], the sums over a group's rows of dy x and of t c.  8192 x 4096 as above: 104 us, 5.8 TB/s.
template <int ST, int DT, int WAVES, int V, bool HELD_H, bool HELD_B>
__global__ __launch_bounds__(64 * WAVES) void k_block_norm_backward(NormWeights by, unsigned rows, unsigned cols, Rows<const Elem<DT>> dy,
                                                                    Rows<const Elem<ST>> dh_out, HeldIn h, HeldIn b,
                                                                    const float *__restrict__ rstd, Rows<Elem<ST>> dh, Rows<Elem<DT>> db,
                                                                    float *__restrict__ parts)
{
    constexpr int E = kNormEach;
    constexpr bool kKept = V * E <= kKeptWeights;
    typedef NormIn<ST, E, HELD_H> H;
    typedef NormIn<DT, E, HELD_B> B;
    __shared__ float room[2 * WAVES];
    unsigned turn = 0;
    const auto place = [&](int k) __attribute__((always_inline)) { return (k * 64 * WAVES + threadIdx.x) * E; };
    const float mean = 1.0f / (float)cols, scale = (float)by.scale;
    // scale gate block_weight
    const auto load_into = [&](int k, float (&into)[E]) __attribute__((always_inline)) {
        float g[E];
        load_weight<E>(by.block_weight, cols, place(k), into);
        load_weight<E>(by.gate, cols, place(k), g);
#pragma unroll
        for (int i = 0; i < E; ++i) into[i] *= scale * g[i];
    };
    float into[V][E], weight[V][E], sum_x[V][E] = {}, sum_c[V][E] = {};
    if constexpr (kKept) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            load_weight<E>(by.weight, cols, place(k), weight[k]);
            if (b.p) load_into(k, into[k]);
        }
    }
    struct {
        Few<DT, E> d[V];
        Few<ST, E> t[V] = {};
        typename H::Type h[V];
        typename B::Type b[V] = {};
        float r, n = 1.0f;
    } next;
    const auto ask = [&](size_t r) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            next.d[k] = load_few<DT, E>(dy.p + r * dy.ld, cols, place(k));
            next.h[k] = H::load(h, r, cols, place(k));
            if (dh_out.p) next.t[k] = load_few<ST, E>(dh_out.p + r * dh_out.ld, cols, place(k));
            if (b.p) next.b[k] = B::load(b, r, cols, place(k));
        }
        next.r = rstd[r];
        if (by.block_weight) next.n = rstd[(size_t)rows + r];
    };
    if constexpr (kBackwardAhead<WAVES, V>) ask(blockIdx.x);
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        if constexpr (!kBackwardAhead<WAVES, V>) ask(r);
        const auto now = next;
        if (kBackwardAhead<WAVES, V> && r + gridDim.x < rows) ask(r + gridDim.x);
        float x[V][E], t[V][E], part = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if constexpr (!kKept) load_weight<E>(by.weight, cols, place(k), weight[k]);
            H::values(now.h[k], x[k]);
            widened<DT, E>(now.d[k], t[k]);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                x[k][i] *= now.r;
                sum_x[k][i] = __builtin_fmaf(t[k][i], x[k][i], sum_x[k][i]);
                t[k][i] *= weight[k][i];
                part = __builtin_fmaf(t[k][i], x[k][i], part);
            }
        }
        const float c1 = group_sum<WAVES>(part, room, turn++) * mean;
        part = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
#pragma unroll
            for (int i = 0; i < E; ++i) t[k][i] = __builtin_fmaf(now.r, __builtin_fmaf(-c1, x[k][i], t[k][i]), (float)now.t[k].v[i]);
            if (place(k) < cols) store_few<ST, E>(dh.p + r * dh.ld, cols, place(k), t[k]);
            if (b.p) {
                if constexpr (!kKept) load_into(k, into[k]);
                B::values(now.b[k], x[k]);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    x[k][i] *= now.n;
                    sum_c[k][i] = __builtin_fmaf(t[k][i], x[k][i], sum_c[k][i]);
                    t[k][i] *= into[k][i];
                    part = __builtin_fmaf(t[k][i], x[k][i], part);
                }
            }
        }
        if (!b.p) continue;
        const float c2 = by.block_weight ? group_sum<WAVES>(part, room, turn++) * mean : 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
#pragma unroll
            for (int i = 0; i < E; ++i) t[k][i] = now.n * __builtin_fmaf(-c2, x[k][i], t[k][i]);
            if (place(k) < cols) store_few<DT, E>(db.p + r * db.ld, cols, place(k), t[k]);
        }
    }
    const unsigned pitch = (cols + 3u) / 4u * 4u;  // (whole fours: their sums are 0 behind the end)
    float *const mine = parts + (size_t)blockIdx.x * 2u * pitch;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if (place(k) < pitch) {
            store_few<kGradF32, E, false>(mine, pitch, place(k), sum_x[k]);
            store_few<kGradF32, E, false>(mine + pitch, pitch, place(k), sum_c[k]);
        }
    }
}

// The groups' sums, joined in 64 bits in an order of their own number alone: 8 lanes take 32 columns, and 128 times as many every 128th of the
// parts each (2048 parts of 1024 columns 21 us with 32 of them).
__global__ __launch_bounds__(1024) void k_block_norm_join(const float *__restrict__ parts, unsigned groups, unsigned cols, NormWeights by,
                                                         float *__restrict__ dweight, float *__restrict__ dblock_weight,
                                                         float *__restrict__ dgate)
{
    constexpr unsigned kJoined = 128;
    __shared__ double room[kJoined][33];
    const unsigned slice = threadIdx.x / 8u, first = threadIdx.x % 8u * 4u, c0 = blockIdx.x * 32u, pitch = (cols + 3u) / 4u * 4u;
    const bool second = blockIdx.y != 0;
    double sum[4] = {};
    const f4 *p = reinterpret_cast<const f4 *>(parts + (second ? pitch : 0u) + (c0 + first < pitch ? c0 + first : 0u));
#pragma unroll 8
    for (unsigned g = slice; g < groups; g += kJoined) {
        const f4 x = p[(size_t)g * (pitch / 2u)];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += (double)x[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) room[slice][first + i] = sum[i];
    __syncthreads();
    const unsigned c = c0 + threadIdx.x;
    if (threadIdx.x >= 32u || c >= cols) return;
    double all = room[0][threadIdx.x];
#pragma unroll 16
    for (unsigned k = 1; k < kJoined; ++k) all += room[k][threadIdx.x];
    if (!second) {
        dweight[c] = (float)all;
    } else {
        all *= by.scale;
        if (dblock_weight) dblock_weight[c] = (float)(all * (by.gate ? (double)by.gate[c] : 1.0));
        if (dgate) dgate[c] = (float)(all * (by.block_weight ? (double)by.block_weight[c] : 1.0));
    }
}

}  // namespace
