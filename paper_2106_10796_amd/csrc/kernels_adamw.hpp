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
    float lr, beta1, one_minus_beta1, beta2, one_minus_beta2, inv_sqrt_bias2, eps, lr_over_bias1, grad_scale;
    unsigned seed;
};

// ---------------------------------------------------------------------------
// loads and stores of E consecutive elements of a lane
// ---------------------------------------------------------------------------
// Every buffer is accessed through a descriptor that ends with the chunk.  RAGGED: elements narrower than a word are loaded
// and stored one by one, so that the range check clips each of them; what lies past the end is loaded as 0.
template <int POLICY, int E>
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
            const f4 t = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(at * 4u + 16u * q), 0, POLICY));
#pragma unroll
            for (int c = 0; c < 4; ++c) x[4 * q + c] = t[c];
        }
    }
    __device__ __forceinline__ void store32(const float (&x)[E]) const
    {
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            const f4 t = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, t), rsrc, (int)(at * 4u + 16u * q), 0, POLICY);
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
                h[i] = (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(rsrc, (int)(at * 2u + 2u * i), 0, POLICY);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) w[i] = h[2 * i] | (h[2 * i + 1] << 16);
        } else if constexpr (E == 8) {
            const u4 t = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(at * 2u), 0, POLICY));
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = t[i];
        } else {
            const u2 t = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)(at * 2u), 0, POLICY));
            w[0] = t.x;
            w[1] = t.y;
        }
    }
    template <bool RAGGED>
    __device__ __forceinline__ void store16(const unsigned (&w)[E / 2]) const
    {
        if constexpr (RAGGED) {
#pragma unroll
            for (int i = 0; i < E; ++i)
                __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(w[i / 2] >> (16 * (i % 2))), rsrc, (int)(at * 2u + 2u * i), 0, POLICY);
        } else if constexpr (E == 8) {
            __builtin_amdgcn_raw_buffer_store_b128(u4{w[0], w[1], w[2], w[3]}, rsrc, (int)(at * 2u), 0, POLICY);
        } else {
            __builtin_amdgcn_raw_buffer_store_b64(u2{w[0], w[1]}, rsrc, (int)(at * 2u), 0, POLICY);
        }
    }
    // four elements to a word
    template <bool RAGGED>
    __device__ __forceinline__ void load8(unsigned (&w)[E / 4]) const
    {
        if constexpr (RAGGED) {
            unsigned b[E];
#pragma unroll
            for (int i = 0; i < E; ++i) b[i] = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(rsrc, (int)(at + i), 0, POLICY);
#pragma unroll
            for (int q = 0; q < E / 4; ++q) w[q] = b[4 * q] | (b[4 * q + 1] << 8) | (b[4 * q + 2] << 16) | (b[4 * q + 3] << 24);
        } else {
            const u2 t = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)at, 0, POLICY));
            w[0] = t.x;
            w[1] = t.y;
        }
    }
    template <bool RAGGED>
    __device__ __forceinline__ void store8(const unsigned (&w)[E / 4]) const
    {
        if constexpr (RAGGED) {
#pragma unroll
            for (int i = 0; i < E; ++i)
                __builtin_amdgcn_raw_buffer_store_b8((unsigned char)(w[i / 4] >> (8 * (i % 4))), rsrc, (int)(at + i), 0, POLICY);
        } else {
            __builtin_amdgcn_raw_buffer_store_b64(u2{w[0], w[1]}, rsrc, (int)at, 0, POLICY);
        }
    }
};

// A gradient as it was loaded, and widened.
template <int GT, int E>
struct GradSpan {
    unsigned w[GT == kGradF32 ? E : E / 2];
    template <bool RAGGED, int POLICY>
    __device__ __forceinline__ void load(const Span<POLICY, E> &s)
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
    if constexpr (GT == kGradBF16) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, b2{(__bf16)a, (__bf16)b});
    } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, h2{(_Float16)a, (_Float16)b});
    }
}

// ---------------------------------------------------------------------------
// the step
// ---------------------------------------------------------------------------
// One element: m, v and the weight.
__device__ __forceinline__ void adamw1(float g, float &m, float &v, float &w, const StepFactors &f, float keep)
{
    m = m * f.beta1 + g * f.one_minus_beta1;
    v = v * f.beta2 + (g * g) * f.one_minus_beta2;
    // (one unit in the last place each, of an update that is lr times the size of a weight)
    const float denom = __builtin_amdgcn_sqrtf(v) * f.inv_sqrt_bias2 + f.eps;
    w = w * keep - (m * __builtin_amdgcn_rcpf(denom)) * f.lr_over_bias1;
}

// States in 32 bits: 26 to 30 bytes an element and a dozen operations, bound by HBM.  One wave per piece, one quad a lane.
constexpr unsigned kStepLanes = 64;
template <int GT, bool COPY, bool RAGGED, int POLICY>
__device__ __forceinline__ void adamw32_piece(const StepChunk &c, unsigned first, const StepFactors &f, float gs)
{
    constexpr int E = 4;
    const Span<POLICY, E> sw(c.weight, c.elems, 4, first), sm(c.m, c.elems, 4, first), sv(c.v, c.elems, 4, first);
    const Span<POLICY, E> sg(c.grad, c.elems, grad_bytes<GT>(), first);
    float w[E], m[E], v[E];
    GradSpan<GT, E> g;
    g.template load<RAGGED>(sg);
    sm.load32(m);
    sv.load32(v);
    sw.load32(w);
    const float keep = 1.0f - f.lr * c.weight_decay;
#pragma unroll
    for (int i = 0; i < E; ++i) adamw1(g[i] * gs, m[i], v[i], w[i], f, keep);
    sm.store32(m);
    sv.store32(v);
    sw.store32(w);
    if constexpr (COPY) {
        const unsigned h[2] = {narrow2<GT>(w[0], w[1]), narrow2<GT>(w[2], w[3])};
        Span<POLICY, E>(c.weight16, c.elems, 2, first).template store16<RAGGED>(h);
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

template <int GT, bool COPY, int POLICY>
__global__ __launch_bounds__(64) void k_adamw32(const StepChunk *__restrict__ chunks, unsigned per_chunk,
                                                const float *__restrict__ clip, StepFactors f)
{
    float gs;
    if (!step_scale(f, clip, gs)) return;
    const StepChunk c = chunks[blockIdx.x / per_chunk];
    const unsigned piece = blockIdx.x % per_chunk * (kStepLanes * 4u), first = piece + threadIdx.x * 4u;
    if (piece >= c.elems) return;
    if (piece + kStepLanes * 4u <= c.elems) adamw32_piece<GT, COPY, false, POLICY>(c, first, f, gs);
    else adamw32_piece<GT, COPY, true, POLICY>(c, first, f, gs);
}

// ---------------------------------------------------------------------------
// states in 8 bits
// ---------------------------------------------------------------------------
// fp32's own bit pattern, scaled so that its lowest binades are those of the code: the fp32 denormals stand where the
// code's denormals do, and encoding is an addition and a shift.  T: the exponent field of a block's largest magnitude.
constexpr int kTopM = 14, kTopV = 30;
static_assert(CDSGD_STATE_BLOCK == 256, "32 lanes of 8 elements hold a block");

// 0, or the bits that make any pattern a NaN.
__device__ __forceinline__ unsigned poison_of(unsigned scale) { return scale == 255u ? 0x7FC00000u : 0u; }

__device__ __forceinline__ float decode_m(unsigned code, unsigned scale, unsigned poison)
{
    const unsigned x = ((code & 0x7Fu) << 20) | ((code & 0x80u) << 24) | poison;
    return __builtin_amdgcn_ldexpf(__builtin_bit_cast(float, x), (int)scale - kTopM);
}

__device__ __forceinline__ float decode_v(unsigned code, unsigned scale, unsigned poison)
{
    return __builtin_amdgcn_ldexpf(__builtin_bit_cast(float, (code << 20) | poison), (int)scale - kTopV);
}

__device__ __forceinline__ unsigned encode_m(float x, int up, unsigned dither16)
{
    const unsigned y = __builtin_bit_cast(unsigned, __builtin_amdgcn_ldexpf(x, up));
    return ((((y & 0x7FFFFFFFu) + dither16 * 16u) >> 20) & 0x7Fu) | ((y >> 24) & 0x80u);
}

__device__ __forceinline__ unsigned encode_v(float x, int up, unsigned dither16)
{
    const unsigned y = __builtin_bit_cast(unsigned, __builtin_amdgcn_ldexpf(x, up));
    const unsigned code = (((y & 0x7FFFFFFFu) + dither16 * 16u) >> 20) & 0xFFu;
    return code == 0u && x > 0.0f ? 1u : code;
}

// The largest value over the 32 lanes of this half of the wave.
__device__ __forceinline__ unsigned max_of_half_wave(unsigned x)
{
#define CDSGD_DPP_MAX(CTRL)                                                                              \
    do {                                                                                                 \
        const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);      \
        x = o > x ? o : x;                                                                               \
    } while (0)
    CDSGD_DPP_MAX(0xB1);   // quad_perm: neighbours
    CDSGD_DPP_MAX(0x4E);   // quad_perm: pairs
    CDSGD_DPP_MAX(0x141);  // row_half_mirror: the other quad of eight lanes
    CDSGD_DPP_MAX(0x140);  // row_mirror: the other half of sixteen
#undef CDSGD_DPP_MAX
    const auto both = __builtin_amdgcn_permlane16_swap(x, x, false, false);  // the other row of 32 lanes
    return both[0] > both[1] ? both[0] : both[1];
}

// 14 to 16 bytes an element and about 65 operations: bound by HBM, with the vector units two thirds busy.  A lane holds eight
// elements in a row and half a wave holds a block, whose scale is a reduction over lanes that never leaves the registers.
constexpr unsigned kStep8Elems = kStepLanes * 8u;
template <int GT, bool COPY, bool RAGGED, int POLICY>
__device__ __forceinline__ void adamw8_piece(const StepChunk &c, unsigned first, const StepFactors &f, float gs)
{
    constexpr int E = 8;
    const Span<POLICY, E> sw(c.weight, c.elems, 4, first), sm(c.m, c.elems, 1, first), sv(c.v, c.elems, 1, first);
    const Span<POLICY, E> sg(c.grad, c.elems, grad_bytes<GT>(), first);
    // scale bytes, one for 32 lanes (a whole chunk's at most; past the end: 0)
    const unsigned blocks = (c.elems + CDSGD_STATE_BLOCK - 1) / CDSGD_STATE_BLOCK, block = first / CDSGD_STATE_BLOCK;
    const Span<0, E> sms(c.m_scale, blocks, 1, block), svs(c.v_scale, blocks, 1, block);
    unsigned mw[2], vw[2];
    float w[E];
    GradSpan<GT, E> g;
    unsigned bm = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(sms.rsrc, (int)block, 0, 0);
    unsigned bv = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(svs.rsrc, (int)block, 0, 0);
    sm.template load8<RAGGED>(mw);
    sv.template load8<RAGGED>(vw);
    g.template load<RAGGED>(sg);
    sw.load32(w);
    const float keep = 1.0f - f.lr * c.weight_decay;
    const unsigned pm = poison_of(bm), pv = poison_of(bv);
    float m[E], v[E];
    unsigned most_m = 0, most_v = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const float gi = g[i] * gs;
        m[i] = decode_m((mw[i / 4] >> (8 * (i % 4))) & 0xFFu, bm, pm);
        v[i] = decode_v((vw[i / 4] >> (8 * (i % 4))) & 0xFFu, bv, pv);
        if constexpr (RAGGED) {  // (what lies past the end takes no part in the scales)
            if (first + i >= c.elems) m[i] = v[i] = 0.0f;
        }
        adamw1(gi, m[i], v[i], w[i], f, keep);
        const unsigned am = __builtin_bit_cast(unsigned, m[i]) & 0x7FFFFFFFu, av = __builtin_bit_cast(unsigned, v[i]) & 0x7FFFFFFFu;
        most_m = am > most_m ? am : most_m;
        most_v = av > most_v ? av : most_v;
    }
    bm = max_of_half_wave(most_m) >> 23;
    bv = max_of_half_wave(most_v) >> 23;
    const unsigned x0 = (c.counter + first) * 0x9E3779B9u + f.seed;
    mw[0] = mw[1] = vw[0] = vw[1] = 0u;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        unsigned x = x0 + (unsigned)i * 0x9E3779B9u;
        x = (x ^ (x >> 15)) * 0xBB67AE85u;
        x = (x ^ (x >> 13)) * 0x6A09E667u;
        x ^= x >> 16;
        mw[i / 4] |= encode_m(m[i], kTopM - (int)bm, x & 0xFFFFu) << (8 * (i % 4));
        vw[i / 4] |= encode_v(v[i], kTopV - (int)bv, x >> 16) << (8 * (i % 4));
    }
    sm.template store8<RAGGED>(mw);
    sv.template store8<RAGGED>(vw);
    sw.store32(w);
    if constexpr (COPY) {
        unsigned h[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) h[i] = narrow2<GT>(w[2 * i], w[2 * i + 1]);
        Span<POLICY, E>(c.weight16, c.elems, 2, first).template store16<RAGGED>(h);
    }
    if (threadIdx.x % 32u == 0u) {
        __builtin_amdgcn_raw_buffer_store_b8((unsigned char)bm, sms.rsrc, (int)block, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b8((unsigned char)bv, svs.rsrc, (int)block, 0, 0);
    }
}

template <int GT, bool COPY, int POLICY>
__global__ __launch_bounds__(64) void k_adamw8(const StepChunk *__restrict__ chunks, unsigned per_chunk,
                                               const float *__restrict__ clip, StepFactors f)
{
    float gs;
    if (!step_scale(f, clip, gs)) return;
    const StepChunk c = chunks[blockIdx.x / per_chunk];
    const unsigned piece = blockIdx.x % per_chunk * kStep8Elems, first = piece + threadIdx.x * 8u;
    if (piece >= c.elems) return;
    if (piece + kStep8Elems <= c.elems) adamw8_piece<GT, COPY, false, POLICY>(c, first, f, gs);
    else adamw8_piece<GT, COPY, true, POLICY>(c, first, f, gs);
}

// What 8-bit states stand for: OT is kGradF32 or kGradBF16.
template <int OT, bool RAGGED>
__device__ __forceinline__ void read_states_piece(const StepChunk &c, unsigned first)
{
    constexpr int E = 8;
    const unsigned blocks = (c.elems + CDSGD_STATE_BLOCK - 1) / CDSGD_STATE_BLOCK, block = first / CDSGD_STATE_BLOCK;
    const Span<0, E> sms(c.m_scale, blocks, 1, block), svs(c.v_scale, blocks, 1, block);
    const unsigned bm = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(sms.rsrc, (int)block, 0, 0);
    const unsigned bv = (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(svs.rsrc, (int)block, 0, 0);
    unsigned mw[2], vw[2];
    Span<kStream, E>(c.m, c.elems, 1, first).template load8<RAGGED>(mw);
    Span<kStream, E>(c.v, c.elems, 1, first).template load8<RAGGED>(vw);
    float m[E], v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        m[i] = decode_m((mw[i / 4] >> (8 * (i % 4))) & 0xFFu, bm, poison_of(bm));
        v[i] = decode_v((vw[i / 4] >> (8 * (i % 4))) & 0xFFu, bv, poison_of(bv));
    }
    if constexpr (OT == kGradF32) {
        Span<kStream, E>(c.m_out, c.elems, 4, first).store32(m);
        Span<kStream, E>(c.v_out, c.elems, 4, first).store32(v);
    } else {
        unsigned h[E / 2], k[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            h[i] = narrow2<OT>(m[2 * i], m[2 * i + 1]);
            k[i] = narrow2<OT>(v[2 * i], v[2 * i + 1]);
        }
        Span<kStream, E>(c.m_out, c.elems, 2, first).template store16<RAGGED>(h);
        Span<kStream, E>(c.v_out, c.elems, 2, first).template store16<RAGGED>(k);
    }
}

template <int OT>
__global__ __launch_bounds__(64) void k_read_states(const StepChunk *__restrict__ chunks, unsigned per_chunk)
{
    const StepChunk c = chunks[blockIdx.x / per_chunk];
    const unsigned piece = blockIdx.x % per_chunk * kStep8Elems, first = piece + threadIdx.x * 8u;
    if (piece >= c.elems) return;
    if (piece + kStep8Elems <= c.elems) read_states_piece<OT, false>(c, first);
    else read_states_piece<OT, true>(c, first);
}

// ---------------------------------------------------------------------------
// norm of a list
// ---------------------------------------------------------------------------
struct NormChunk {
    const void *grad;
    unsigned elems;
    unsigned pad_;
};
constexpr unsigned kNormLanes = 256, kNormChunk = 16384;

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

// Sums of squares in 64 bits (a product of two fp32 numbers is exact there).  A group takes the chunks that have its number
// modulo the number of groups; the group that ends last adds up the groups' sums in their order, so that the result is the
// same whichever it is, and leaves the counter at 0 for the next call.
template <int GT>
__global__ __launch_bounds__(256) void k_grad_norm(const NormChunk *__restrict__ chunks, unsigned num_chunks, double *partial,
                                                   unsigned *done, double scale, double max_norm, float *__restrict__ out)
{
    constexpr int E = GT == kGradF32 ? 4 : 8;
    __shared__ double lds[kNormLanes / 64u];
    __shared__ bool last;
    double s0 = 0.0, s1 = 0.0;
    for (unsigned k = blockIdx.x; k < num_chunks; k += gridDim.x) {
        const NormChunk c = chunks[k];
        if (c.elems == kNormChunk) {
#pragma unroll 4
            for (unsigned first = threadIdx.x * E; first < kNormChunk; first += kNormLanes * E) {
                GradSpan<GT, E> g;
                g.template load<false>(Span<kStream, E>(c.grad, kNormChunk, grad_bytes<GT>(), first));
#pragma unroll
                for (int i = 0; i < E; i += 2) {
                    const double a = (double)g[i], b = (double)g[i + 1];
                    s0 = __builtin_fma(a, a, s0);
                    s1 = __builtin_fma(b, b, s1);
                }
            }
        } else {
            for (unsigned first = threadIdx.x * E; first < c.elems; first += kNormLanes * E) {
                GradSpan<GT, E> g;
                g.template load<true>(Span<kStream, E>(c.grad, c.elems, grad_bytes<GT>(), first));
#pragma unroll
                for (int i = 0; i < E; ++i) s0 = __builtin_fma((double)g[i], (double)g[i], s0);
            }
        }
    }
    const double mine = sum_of_group(s0 + s1, lds);
    if (threadIdx.x == 0u) {
        __hip_atomic_store(&partial[blockIdx.x], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1u;
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
