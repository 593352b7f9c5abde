// What kernels on matrices share: element types, a few elements of a row at any address, and sums over the lanes of a wave.
#pragma once

namespace {

// Element types of matrices in ordinary floating point.
template <int DT>
using Elem = typename std::conditional<DT == kGradF32, float, typename std::conditional<DT == kGradBF16, __bf16, _Float16>::type>::type;

// E elements in a row.
template <int DT, int E>
struct Few {
    Elem<DT> v[E];
};
template <int DT, int E>
struct __attribute__((packed, aligned(sizeof(Elem<DT>)))) FewAt {
    Few<DT, E> e;
};

// Elements c ... c + E - 1 of a row, 0 where it has ended.
template <int DT, int E>
__device__ __forceinline__ Few<DT, E> load_few(const Elem<DT> *row, unsigned cols, unsigned c)
{
    if (c + E <= cols) return reinterpret_cast<const FewAt<DT, E> *>(row + c)->e;
    Few<DT, E> x = {};
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (c + i < cols) x.v[i] = row[c + i];
    return x;
}

// ... rounded once and stored.  PAST: past the caches, for rows that are read again a pass later at the earliest (8192 x 4096, us: the norms' backward
// pass 116 to the caches, 104 past them, 8-bit values 20.3 and 18.8, the gated activation's forward pass over 8192 x 16384 208 and 200, backward
// 196 and 203).
template <int DT, int E, bool PAST = true>
__device__ __forceinline__ void store_few(Elem<DT> *row, unsigned cols, unsigned c, const float (&v)[E])
{
    Few<DT, E> x;
#pragma unroll
    for (int i = 0; i < E; ++i) x.v[i] = (Elem<DT>)v[i];
    if (c + E <= cols) {
        typedef unsigned words __attribute__((ext_vector_type(E * sizeof(Elem<DT>) / 4), aligned(sizeof(Elem<DT>))));
        if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(words, x), reinterpret_cast<words *>(row + c));
        else *reinterpret_cast<words *>(row + c) = __builtin_bit_cast(words, x);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (c + i < cols) row[c + i] = x.v[i];
    }
}

// v of another lane of the wave, as a DPP control says; 0 where `rows` (a bit for each sixteen lanes) leaves the lane out.
template <int CONTROL, int ROWS = 0xF, typename T>
__device__ __forceinline__ T moved(T v)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, ROWS, 0xF, false));
    } else {
        typedef int i2 __attribute__((ext_vector_type(2)));
        const i2 w = __builtin_bit_cast(i2, v);
        return __builtin_bit_cast(T, i2{__builtin_amdgcn_update_dpp(0, w.x, CONTROL, ROWS, 0xF, false),
                                        __builtin_amdgcn_update_dpp(0, w.y, CONTROL, ROWS, 0xF, false)});
    }
}

constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppMirror8 = 0x141, kDppMirror16 = 0x140, kDppBcast15 = 0x142, kDppBcast31 = 0x143;

// The sum over the lanes of a wave, the same in all of them.
template <typename T>
__device__ __forceinline__ T wave_sum(T v)
{
    v += moved<kDppXor1>(v);
    v += moved<kDppXor2>(v);
    v += moved<kDppMirror8>(v);
    v += moved<kDppMirror16>(v);
    v += moved<kDppBcast15, 0xA>(v);
    v += moved<kDppBcast31, 0xC>(v);
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    } else {
        typedef int i2 __attribute__((ext_vector_type(2)));
        const i2 w = __builtin_bit_cast(i2, v);
        return __builtin_bit_cast(T, i2{__builtin_amdgcn_readlane(w.x, 63), __builtin_amdgcn_readlane(w.y, 63)});
    }
}

// ... over those of a group of WAVES waves.  room: [2][WAVES]; `turn` alternates from one call to the next, so that one barrier is enough.
template <int WAVES, typename T>
__device__ __forceinline__ T group_sum(T v, T *room, unsigned turn)
{
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        T *const at = room + (turn & 1u) * WAVES;
        if (threadIdx.x % 64u == 0u) at[threadIdx.x / 64u] = v;
        __syncthreads();
        v = at[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += at[w];
    }
    return v;
}

}  // namespace
