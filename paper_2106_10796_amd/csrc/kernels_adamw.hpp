// AdamW over a layer list, states in 32 or 8 bits; the values that 8-bit states stand for; norms of gradients.
#pragma once

namespace {

typedef unsigned u4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// tables
// ---------------------------------------------------------------------------
// A list is cut into chunks of kStepChunk elements; only a tensor's last one is ragged.  An entry holds every address of its
// chunk, so that a wave is one trip to memory away from its first loads.
constexpr unsigned kStepChunk = 4096;
struct StepChunk {
    float *weight;
    const void *grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    void *weight16;
    void *m_out, *v_out;  // cdsgd_adamw_bind_readout
    unsigned elems;       // elements of the chunk
    unsigned counter;     // number of its first element in the list
    float weight_decay;
    unsigned pad_;
};

struct StepFactors {
    double lr;
    float beta1, one_minus_beta1, beta2, one_minus_beta2, inv_sqrt_bias2, eps, lr_over_bias1, grad_scale;
    unsigned seed;
};

// ---------------------------------------------------------------------------
// loads and stores of E consecutive elements of a lane
// ---------------------------------------------------------------------------
// Every buffer is accessed through a descriptor that ends with the chunk.  RAGGED: elements narrower than a word are loaded
// and stored one by one, so that the range check clips each of them; what lies past the end is loaded as 0.
template <int E, int LOAD = 0, int STORE = 0>
struct Span {
    __amdgpu_buffer_rsrc_t rsrc;
    unsigned at;  // the lane's first element

    __device__ __forceinline__ Span(const void *base, unsigned elems, unsigned elem_bytes, unsigned first)
        : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)(elems * elem_bytes), kBufferFlags)), at(first)
    {
    }

    __device__ __forceinline__ void load32(float (&x)[E]) const
    {
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            const f4 t = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(at * 4u + 16u * q), 0, LOAD));
#pragma unroll
            for (int c = 0; c < 4; ++c) x[4 * q + c] = t[c];
        }
    }
    __device__ __forceinline__ void store32(const float (&x)[E]) const
    {
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            const f4 t = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, t), rsrc, (int)(at * 4u + 16u * q), 0, STORE);
        }
    }
    // two elements to a word
    template <bool RAGGED>
    __device__ __forceinline__ void load16(unsigned (&w)[E / 2]) const
    {
        if constexpr (RAGGED) {
            unsigned h[E];
#pragma unroll
            for (int i = 0; i < E; ++i)
                h[i] = (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(rsrc, (int)(at * 2u + 2u * i), 0, LOAD);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) w[i] = h[2 * i] | (h[2 * i + 1] << 16);
        } else if constexpr (E == 8) {
            const u4 t = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(at * 2u), 0, LOAD));
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = t[i];
        } else {
            const u2 t = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)(at * 2u), 0, LOAD));
            w[0] = t.x;
            w[1] = t.y;
        }
    }
    template <bool RAGGED>
    __device__ __forceinline__ void store16(const unsigned (&w)[2]) const
    {
        static_assert(E == 4, "a quad to a lane");
        if constexpr (RAGGED) {
#pragma unroll
            for (int i = 0; i < E; ++i)
                __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(w[i / 2] >> (16 * (i % 2))), rsrc, (int)(at * 2u + 2u * i), 0, STORE);
        } else {
            __builtin_amdgcn_raw_buffer_store_b64(u2{w[0], w[1]}, rsrc, (int)(at * 2u), 0, STORE);
        }
    }
    // four elements to a word
    template <bool RAGGED>
    __device__ __forceinline__ unsigned load8() const
    {
        static_assert(E == 4, "a quad to a lane");
        if constexpr (RAGGED) {
            unsigned b[E];
#pragma unroll
            for (int i = 0; i < E; ++i) b[i] = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(rsrc, (int)(at + i), 0, LOAD);
            return b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
        } else {
            return (unsigned)__builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)at, 0, LOAD);
        }
    }
    template <bool RAGGED>
    __device__ __forceinline__ void store8(unsigned w) const
    {
        static_assert(E == 4, "a quad to a lane");
        if constexpr (RAGGED) {
#pragma unroll
            for (int i = 0; i < E; ++i) __builtin_amdgcn_raw_buffer_store_b8((unsigned char)(w >> (8 * i)), rsrc, (int)(at + i), 0, STORE);
        } else {
            __builtin_amdgcn_raw_buffer_store_b32(w, rsrc, (int)at, 0, STORE);
        }
    }
};

// A gradient as it was loaded, and widened.
template <int GT, int E>
struct GradSpan {
    unsigned w[GT == kGradF32 ? E : E / 2];
    template <bool RAGGED, int LOAD, int STORE>
    __device__ __forceinline__ void load(const Span<E, LOAD, STORE> &s)
    {
        if constexpr (GT == kGradF32) {
            float x[E];
            s.load32(x);
#pragma unroll
            for (int i = 0; i < E; ++i) w[i] = __builtin_bit_cast(unsigned, x[i]);
        } else {
            s.template load16<RAGGED>(w);
        }
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (GT == kGradF32) return __builtin_bit_cast(float, w[i]);
        else if constexpr (GT == kGradBF16) return __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else return widen16<GT>(i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu);
    }
};

// Two fp32 values rounded to nearest even in 16 bits (NaN stays NaN).
template <int GT>
__device__ __forceinline__ unsigned narrow2(float a, float b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    if constexpr (GT == kGradBF16) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{a, b}), b2));
    } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{a, b}), h2));
    }
}

// ---------------------------------------------------------------------------
// the step
// ---------------------------------------------------------------------------
// The factor that decays a tensor's weights, in 64 bits and rounded once, as the other factors are on the host.
__device__ __forceinline__ float keep_of(const StepFactors &f, const StepChunk &c) { return (float)(1.0 - f.lr * (double)c.weight_decay); }

// One element: m, v and the weight.
__device__ __forceinline__ void adamw1(float g, float &m, float &v, float &w, const StepFactors &f, float keep)
{
    m = m * f.beta1 + g * f.one_minus_beta1;
    v = v * f.beta2 + (g * g) * f.one_minus_beta2;
    // (one unit in the last place each, of an update that is lr times the size of a weight; the instruction takes a denormal for 0)
    const bool small = v < 0x1p-96f;
    const float denom = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? 0x1p-32f : 1.0f) * f.inv_sqrt_bias2 + f.eps;
    w = w * keep - (m * __builtin_amdgcn_rcpf(denom)) * f.lr_over_bias1;
}

// States in 32 bits: 26 to 28 bytes an element and some forty operations, bound by HBM: 25.6 M elements, bf16 gradients and a copy, 111 us,
// 6.4 TB/s.  One wave per piece, one quad to a lane: every access of a wave is to whole lines in a row.
constexpr unsigned kStepLanes = 64;
template <int GT, bool COPY, bool RAGGED, int LOAD, int STORE>
__device__ __forceinline__ void adamw32_piece(const StepChunk &c, unsigned first, const StepFactors &f, float gs)
{
    constexpr int E = 4;
    const Span<E, LOAD, STORE> sw(c.weight, c.elems, 4, first), sm(c.m, c.elems, 4, first), sv(c.v, c.elems, 4, first);
    const Span<E, LOAD, STORE> sg(c.grad, c.elems, grad_bytes<GT>(), first);
    float w[E], m[E], v[E];
    GradSpan<GT, E> g;
    g.template load<RAGGED>(sg);
    sm.load32(m);
    sv.load32(v);
    sw.load32(w);
    const float keep = keep_of(f, c);
#pragma unroll
    for (int i = 0; i < E; ++i) adamw1(g[i] * gs, m[i], v[i], w[i], f, keep);
    sm.store32(m);
    sv.store32(v);
    sw.store32(w);
    if constexpr (COPY) {
        const unsigned h[2] = {narrow2<GT>(w[0], w[1]), narrow2<GT>(w[2], w[3])};
        Span<E, LOAD, STORE>(c.weight16, c.elems, 2, first).template store16<RAGGED>(h);
    }
}

// The factor on the gradients; false where the step is to be skipped.
__device__ __forceinline__ bool step_scale(const StepFactors &f, const float *clip, float &gs)
{
    gs = f.grad_scale;
    if (!clip) return true;
    gs *= clip[1];
    return (__builtin_bit_cast(unsigned, clip[0]) & 0x7F800000u) != 0x7F800000u;
}

template <int GT, bool COPY, int LOAD, int STORE>
__global__ __launch_bounds__(64) void k_adamw32(const StepChunk *__restrict__ chunks, unsigned per_chunk,
                                                const float *__restrict__ clip, StepFactors f)
{
    float gs;
    if (!step_scale(f, clip, gs)) return;
    const StepChunk c = chunks[blockIdx.x / per_chunk];
    const unsigned piece = blockIdx.x % per_chunk * (kStepLanes * 4u), first = piece + threadIdx.x * 4u;
    if (piece >= c.elems) return;
    if (piece + kStepLanes * 4u <= c.elems) adamw32_piece<GT, COPY, false, LOAD, STORE>(c, first, f, gs);
    else adamw32_piece<GT, COPY, true, LOAD, STORE>(c, first, f, gs);
}

// ---------------------------------------------------------------------------
// states in 8 bits
// ---------------------------------------------------------------------------
// fp32's own bit pattern, scaled so that its lowest binades are those of the code: the fp32 denormals stand where the
// code's denormals do, and encoding is an addition and a shift.  T: the exponent field of a block's largest magnitude.
constexpr int kTopM = 14, kTopV = 30;
static_assert(CDSGD_STATE_BLOCK == 4 * 64, "a wave holds a block, a quad to a lane");

// The code in byte `i` of a word, moved to where its bits are those of an fp32 number.
template <int i>
__device__ __forceinline__ float decode_m(unsigned word, int down)
{
    constexpr int k = 20 - 8 * i, z = 24 - 8 * i;
    const unsigned mag = (k >= 0 ? word << (k >= 0 ? k : 0) : word >> (k < 0 ? -k : 0)) & 0x07F00000u;
    return __builtin_amdgcn_ldexpf(__builtin_bit_cast(float, mag | (word << z & 0x80000000u)), down);
}

template <int i>
__device__ __forceinline__ float decode_v(unsigned word, int down)
{
    constexpr int k = 20 - 8 * i;
    return __builtin_amdgcn_ldexpf(__builtin_bit_cast(float, (k >= 0 ? word << (k >= 0 ? k : 0) : word >> (k < 0 ? -k : 0)) & 0x0FF00000u), down);
}

// Four values of a state under one scale; NaN if that is 255.
template <bool SIGNED>
__device__ __forceinline__ void decode4(unsigned w, unsigned scale, float (&x)[4])
{
    const int down = (int)scale - (SIGNED ? kTopM : kTopV);
    x[0] = SIGNED ? decode_m<0>(w, down) : decode_v<0>(w, down);
    x[1] = SIGNED ? decode_m<1>(w, down) : decode_v<1>(w, down);
    x[2] = SIGNED ? decode_m<2>(w, down) : decode_v<2>(w, down);
    x[3] = SIGNED ? decode_m<3>(w, down) : decode_v<3>(w, down);
    if (__any(scale == 255u)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = scale == 255u ? __builtin_nanf("") : x[i];
    }
}

// The code as the uppermost byte; `dither8`: the dither 8 bits up.  (The sign and the exponent bits that are 0 fall out of the
// word.)
__device__ __forceinline__ unsigned encode_m(float x, int up, unsigned dither8)
{
    const unsigned y = __builtin_bit_cast(unsigned, __builtin_amdgcn_ldexpf(x, up));
    return (((y << 4) + dither8) & 0x7FFFFFFFu) | (y & 0x80000000u);
}

__device__ __forceinline__ unsigned encode_v(float x, int up, unsigned dither8)
{
    const unsigned y = __builtin_bit_cast(unsigned, __builtin_amdgcn_ldexpf(x, up));
    const unsigned code = (y << 4) + dither8, least = x > 0.0f ? 1u << 24 : 0u;
    return code > least ? code : least;
}

// The uppermost bytes of four words.
__device__ __forceinline__ unsigned upper_bytes(unsigned a, unsigned b, unsigned c, unsigned d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x07030c0cu), __builtin_amdgcn_perm(b, a, 0x0c0c0703u), 0x07060100u);
}

// The largest of each half of x over the wave, in every lane.
__device__ __forceinline__ unsigned max_of_wave(unsigned x)
{
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    const auto most = [](unsigned p, unsigned q) {
        return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(us2, p), __builtin_bit_cast(us2, q)));
    };
    x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));   // quad_perm: neighbours
    x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));   // quad_perm: pairs
    x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));  // row_half_mirror: the other quad of eight lanes
    x = most(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true));  // row_mirror: the other half of sixteen
    const auto rows = __builtin_amdgcn_permlane16_swap(x, x, false, false);                 // the other row of 32 lanes
    x = most(rows[0], rows[1]);
    const auto halves = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return most(halves[0], halves[1]);
}

// 14 to 16 bytes an element and some seventy operations, bound by HBM: 138 M elements, bf16 with a copy, 362 us, 6.1 TB/s (the operations
// alone take two thirds of that).  A wave takes two blocks, a quad of each to a lane, so that every access of the wave is to whole
// lines in a row; a block's scale is a reduction over the wave that never leaves the registers.  (Eight elements in a row to a lane:
// a store of the weights leaves half of every line to the next one; 138 M elements 395 us, and 524 with stores written through.)
constexpr int kStep8Blocks = 2;
constexpr unsigned kStep8Elems = kStep8Blocks * CDSGD_STATE_BLOCK;
template <int GT, bool COPY, bool RAGGED, int LOAD, int STORE>
__device__ __forceinline__ void adamw8_piece(const StepChunk &c, unsigned piece, const StepFactors &f, float gs)
{
    constexpr int E = 4, B = kStep8Blocks;
    const unsigned lane4 = threadIdx.x * 4u, block = piece / CDSGD_STATE_BLOCK;
    // the blocks' scale bytes are the same in all lanes; one lane stores them (past the end: 0, and not)
    const unsigned blocks = (c.elems + CDSGD_STATE_BLOCK - 1) / CDSGD_STATE_BLOCK;
    const Span<E> sms(c.m_scale, blocks, 1, 0), svs(c.v_scale, blocks, 1, 0);
    unsigned bm[B], bv[B], mw[B], vw[B];
    float w[B][E];
    GradSpan<GT, E> g[B];
#pragma unroll
    for (int k = 0; k < B; ++k) {
        bm[k] = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(sms.rsrc, (int)(block + k), 0, 0);
        bv[k] = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(svs.rsrc, (int)(block + k), 0, 0);
    }
#pragma unroll
    for (int k = 0; k < B; ++k) {
        const unsigned first = piece + k * CDSGD_STATE_BLOCK + lane4;
        mw[k] = Span<E, LOAD, STORE>(c.m, c.elems, 1, first).template load8<RAGGED>();
        vw[k] = Span<E, LOAD, STORE>(c.v, c.elems, 1, first).template load8<RAGGED>();
        g[k].template load<RAGGED>(Span<E, LOAD, STORE>(c.grad, c.elems, grad_bytes<GT>(), first));
        Span<E, LOAD, STORE>(c.weight, c.elems, 4, first).load32(w[k]);
    }
    const float keep = keep_of(f, c);
    float m[B][E], v[B][E];
    unsigned most[B];
#pragma unroll
    for (int k = 0; k < B; ++k) {
        decode4<true>(mw[k], bm[k], m[k]);
        decode4<false>(vw[k], bv[k], v[k]);
        unsigned am = 0, av = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (RAGGED) {  // (what lies past the end takes no part in the scales)
                if (piece + k * CDSGD_STATE_BLOCK + lane4 + i >= c.elems) m[k][i] = v[k][i] = 0.0f;
            }
            adamw1(g[k][i] * gs, m[k][i], v[k][i], w[k][i], f, keep);
            const unsigned xm = __builtin_bit_cast(unsigned, m[k][i]) & 0x7FFFFFFFu, xv = __builtin_bit_cast(unsigned, v[k][i]) & 0x7FFFFFFFu;
            am = xm > am ? xm : am;
            av = xv > av ? xv : av;
        }
        most[k] = (am >> 23) | (av >> 23 << 16);
    }
#pragma unroll
    for (int k = 0; k < B; ++k) {
        most[k] = max_of_wave(most[k]);
        bm[k] = most[k] & 0xFFFFu;
        bv[k] = most[k] >> 16;
    }
#pragma unroll
    for (int k = 0; k < B; ++k) {
        const unsigned first = piece + k * CDSGD_STATE_BLOCK + lane4;
        const unsigned x0 = (c.counter + first) * 0x9E3779B9u + f.seed;
        unsigned cm[E], cv[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            unsigned x = x0 + (unsigned)i * 0x9E3779B9u;
            x = (x ^ (x >> 15)) * 0xBB67AE85u;
            x = (x ^ (x >> 13)) * 0x6A09E667u;
            x ^= x >> 16;
            cm[i] = encode_m(m[k][i], kTopM - (int)bm[k], (x & 0xFFFFu) << 8);
            cv[i] = encode_v(v[k][i], kTopV - (int)bv[k], x >> 16 << 8);
        }
        Span<E, LOAD, STORE>(c.m, c.elems, 1, first).template store8<RAGGED>(upper_bytes(cm[0], cm[1], cm[2], cm[3]));
        Span<E, LOAD, STORE>(c.v, c.elems, 1, first).template store8<RAGGED>(upper_bytes(cv[0], cv[1], cv[2], cv[3]));
        Span<E, LOAD, STORE>(c.weight, c.elems, 4, first).store32(w[k]);
        if constexpr (COPY) {
            const unsigned h[2] = {narrow2<GT>(w[k][0], w[k][1]), narrow2<GT>(w[k][2], w[k][3])};
            Span<E, LOAD, STORE>(c.weight16, c.elems, 2, first).template store16<RAGGED>(h);
        }
        if (threadIdx.x == 0u) {
            __builtin_amdgcn_raw_buffer_store_b8((unsigned char)bm[k], sms.rsrc, (int)(block + k), 0, 0);
            __builtin_amdgcn_raw_buffer_store_b8((unsigned char)bv[k], svs.rsrc, (int)(block + k), 0, 0);
        }
    }
}

template <int GT, bool COPY, int LOAD, int STORE>
__global__ __launch_bounds__(64) void k_adamw8(const StepChunk *__restrict__ chunks, unsigned per_chunk,
                                               const float *__restrict__ clip, StepFactors f)
{
    float gs;
    if (!step_scale(f, clip, gs)) return;
    const StepChunk c = chunks[blockIdx.x / per_chunk];
    const unsigned piece = blockIdx.x % per_chunk * kStep8Elems;
    if (piece >= c.elems) return;
    if (piece + kStep8Elems <= c.elems) adamw8_piece<GT, COPY, false, LOAD, STORE>(c, piece, f, gs);
    else adamw8_piece<GT, COPY, true, LOAD, STORE>(c, piece, f, gs);
}

// What 8-bit states stand for: OT is kGradF32 or kGradBF16.  Six bytes an element in bf16, bound by HBM: 138 M 134 us, 6.2 TB/s.
template <int OT, bool RAGGED, int LOAD, int STORE>
__device__ __forceinline__ void read_states_piece(const StepChunk &c, unsigned piece)
{
    constexpr int E = 4, B = kStep8Blocks;
    const unsigned blocks = (c.elems + CDSGD_STATE_BLOCK - 1) / CDSGD_STATE_BLOCK, block = piece / CDSGD_STATE_BLOCK;
    const Span<E> sms(c.m_scale, blocks, 1, 0), svs(c.v_scale, blocks, 1, 0);
    unsigned b[2][B], w[2][B];
#pragma unroll
    for (int k = 0; k < B; ++k) {
        const unsigned first = piece + k * CDSGD_STATE_BLOCK + threadIdx.x * 4u;
        b[0][k] = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(sms.rsrc, (int)(block + k), 0, 0);
        b[1][k] = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(svs.rsrc, (int)(block + k), 0, 0);
        w[0][k] = Span<E, LOAD, STORE>(c.m, c.elems, 1, first).template load8<RAGGED>();
        w[1][k] = Span<E, LOAD, STORE>(c.v, c.elems, 1, first).template load8<RAGGED>();
    }
#pragma unroll
    for (int k = 0; k < B; ++k) {
        const unsigned first = piece + k * CDSGD_STATE_BLOCK + threadIdx.x * 4u;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            float x[E];
            if (z == 0) decode4<true>(w[0][k], b[0][k], x);
            else decode4<false>(w[1][k], b[1][k], x);
            void *const out = z == 0 ? c.m_out : c.v_out;
            if constexpr (OT == kGradF32) {
                Span<E, LOAD, STORE>(out, c.elems, 4, first).store32(x);
            } else {
                const unsigned h[2] = {narrow2<OT>(x[0], x[1]), narrow2<OT>(x[2], x[3])};
                Span<E, LOAD, STORE>(out, c.elems, 2, first).template store16<RAGGED>(h);
            }
        }
    }
}

template <int OT, int LOAD, int STORE>
__global__ __launch_bounds__(64) void k_read_states(const StepChunk *__restrict__ chunks, unsigned per_chunk)
{
    const StepChunk c = chunks[blockIdx.x / per_chunk];
    const unsigned piece = blockIdx.x % per_chunk * kStep8Elems;
    if (piece >= c.elems) return;
    if (piece + kStep8Elems <= c.elems) read_states_piece<OT, false, LOAD, STORE>(c, piece);
    else read_states_piece<OT, true, LOAD, STORE>(c, piece);
}

// ---------------------------------------------------------------------------
// norm of a list
// ---------------------------------------------------------------------------
struct NormChunk {
    const void *grad;
    unsigned elems;
    unsigned pad_;
};
constexpr unsigned kNormLanes = 512, kNormLoads = 4, kNormBytes = kNormLanes * 16 * kNormLoads;  // bytes of a chunk: four loads to a lane
template <int GT>
constexpr unsigned kNormElems = kNormBytes / grad_bytes<GT>();

__device__ __forceinline__ double sum_of_group(double x, double *lds)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d, 64);
    if (threadIdx.x % 64u == 0u) lds[threadIdx.x / 64u] = x;
    __syncthreads();
    double s = 0.0;
    for (unsigned i = 0; i < kNormLanes / 64u; ++i) s += lds[i];
    return s;
}

// Sums of squares in 64 bits (a product of two fp32 numbers is exact there); bound by HBM, 6.9 TB/s over 138 M fp32 elements, 6.3
// in bf16, whose conversion to 64 bits takes as many instructions for half the bytes.  A group takes the chunks that have its number
// modulo the number of groups; the group that ends last adds up the groups' sums in their order, so that the result is the
// same whichever it is, and leaves the counter at 0 for the next call.
template <int GT>
__global__ __launch_bounds__(kNormLanes) void k_grad_norm(const NormChunk *__restrict__ chunks, unsigned num_chunks, double *partial,
                                                   unsigned *done, double scale, double max_norm, float *__restrict__ out)
{
    constexpr int E = GT == kGradF32 ? 4 : 8;
    __shared__ double lds[kNormLanes / 64u];
    __shared__ bool last;
    double s0 = 0.0, s1 = 0.0;
    for (unsigned k = blockIdx.x; k < num_chunks; k += gridDim.x) {
        const NormChunk c = chunks[k];
        GradSpan<GT, E> g[kNormLoads];
        if (c.elems == kNormElems<GT>) {
#pragma unroll
            for (unsigned q = 0; q < kNormLoads; ++q)
                g[q].template load<false>(Span<E, kStream>(c.grad, kNormElems<GT>, grad_bytes<GT>(), (q * kNormLanes + threadIdx.x) * E));
        } else {
#pragma unroll
            for (unsigned q = 0; q < kNormLoads; ++q) {
                g[q] = GradSpan<GT, E>();
                if (q * kNormLanes * E < c.elems)
                    g[q].template load<true>(Span<E, kStream>(c.grad, c.elems, grad_bytes<GT>(), (q * kNormLanes + threadIdx.x) * E));
            }
        }
#pragma unroll
        for (unsigned q = 0; q < kNormLoads; ++q)
#pragma unroll
            for (int i = 0; i < E; i += 2) {
                const double a = (double)g[q][i], b = (double)g[q][i + 1];
                s0 = __builtin_fma(a, a, s0);
                s1 = __builtin_fma(b, b, s1);
            }
    }
    const double mine = sum_of_group(s0 + s1, lds);
    if (threadIdx.x == 0u) {
        // Stores and loads of agent scope go past the compute dies' own caches to where all of them meet, and the counter is there,
        // too: it is enough that the sum has arrived before the counter moves.  (A release in its place writes an L2 back for every
        // group, 45 ns each: 138 M elements in 2048 groups 183 us.)
        __hip_atomic_store(&partial[blockIdx.x], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        last = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1u;
    }
    __syncthreads();
    if (!last) return;
    double t = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kNormLanes)
        t += __hip_atomic_load(&partial[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    t = sum_of_group(t, lds);
    if (threadIdx.x == 0u) {
        const double norm = sqrt(t) * scale;
        out[0] = (float)norm;
        out[1] = norm > max_norm ? (float)(max_norm / norm) : 1.0f;
        __hip_atomic_store(done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

}  // namespace
