// Attention over packed sequences (include/cdsgd_block.h), forward and backward.
//
// The heads that share a key head are rows of one matrix: row i of a sequence is query i / G under head i % G of the group's G, so that a
// tile of keys and values serves all of them, and a single query's heads share its instructions.  A wave takes 32 rows (or, for the gradients of
// keys and values, 32 keys) and keeps what belongs to them in registers; what it runs over goes through LDS, a tile at a time.
//
// Matrix instructions (32 x 32 x 16): lane l holds of the first operand row l % 32, of the second column l % 32, elements 8 (l / 32) ... + 7 of
// the axis that is summed over, and of the result rows 8 (r / 4) + 4 (l / 32) + r % 4, r = 0 ... 15, of column l % 32.  Products are taken so that a
// lane's results are already its elements of the next product's second operand: S^T = K Q^T has a query in every lane (the sum and the largest
// of its row need one exchange between two lanes), and the sum over keys in O^T = V^T P^T may run in any order, as long as both operands
// have the same one: slot e of lane l / 32 = h is key 4 h + e, or 4 + 4 h + e from e = 4 on, which is where S^T left it.  V^T comes from LDS by the
// reads that transpose: four lanes' 8 bytes of four rows each become four rows' elements of one column.
#pragma once

#include "device_matrix.hpp"
#include "kernels_mxfp4.hpp"
#include "kernels_mxfp4_product.hpp"  // loads to LDS

namespace {

typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.44269504088896f;
constexpr float kInfinity = __builtin_inff();
constexpr unsigned kRecords = 0x40000000u, kOutside = 0x7FFFFFF0u;  // of a buffer; a place behind every buffer's end, which loads 0

// Probabilities of fp16 tensors are operands of the second products times a power of two, 2^15 being the largest that 1 can be multiplied with
// there: numbers below 2^-14 lose bits in fp16, and a row of 2^14 keys has no others.  The forward pass leaves room for kSlack.
constexpr float kSlack = 8.0f;
constexpr float kFar = 1048576.0f;
template <int DT>
constexpr float kLift = DT == kGradF16 ? 7.0f : 0.0f;
template <int DT>
constexpr float kLiftBack = DT == kGradF16 ? 15.0f : 0.0f;
template <int DT>
constexpr float kLifted = DT == kGradF16 ? 32768.0f : 1.0f;

// The backward pass takes a row's logits less lse log2 e, in fp32.  Of 2^12 that leaves P a share of 2^-12 off, half a step of fp16; rows beyond it have their
// largest logit and their sum formed again, and take the largest off first.
constexpr float kFarBack = 4096.0f;

constexpr unsigned kTileRows = 128;  // rows of a group of the forward pass and of dq, and keys of a group of dk and dv
constexpr unsigned kMostSplits = 256;
constexpr unsigned kTileKeys = 64;   // what a group takes at a time of the other side

template <int DT>
__device__ __forceinline__ f16v mfma(s8v a, s8v b, f16v c)
{
    if constexpr (DT == kGradBF16) {
        typedef __bf16 b8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    } else {
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
}

// The lane's number, worked out where it is used, and what follows from it too: in and behind loops that have no registers left to keep that in.
__device__ __forceinline__ unsigned lane_now()
{
    unsigned lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(lane));
    return lane;
}

// The row of a result's element r.
__device__ __forceinline__ constexpr unsigned row_of(unsigned r, unsigned half) { return 8u * (r / 4u) + 4u * half + r % 4u; }

struct AttentionSizes {
    unsigned tokens_q, tokens_k, num_seqs, kv_heads, group, dim;
    const int *starts_q, *starts_k;
    int causal;
    float scale;
};

template <typename T>
struct Heads {
    T *p;
    unsigned ld;  // elements from one token to the next
};

// A sequence, cut to the tensors: its first rows and its lengths.
struct Sequence {
    unsigned q0, queries, k0, keys;
};

__device__ __forceinline__ unsigned cut(int at, unsigned from, unsigned to)
{
    const unsigned a = at < 0 ? 0u : (unsigned)at;
    return a < from ? from : a > to ? to : a;
}

__device__ __forceinline__ Sequence sequence_of(const AttentionSizes &z, unsigned s)
{
    Sequence x = {0u, z.tokens_q, 0u, z.tokens_k};
    if (z.starts_q) {
        const auto at = [](const int *p) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(*p); };
        const int *k = z.starts_k ? z.starts_k : z.starts_q;
        x.q0 = cut(at(z.starts_q + s), 0u, z.tokens_q);
        x.queries = cut(at(z.starts_q + s + 1u), x.q0, z.tokens_q) - x.q0;
        x.k0 = cut(at(k + s), 0u, z.tokens_k);
        x.keys = cut(at(k + s + 1u), x.k0, z.tokens_k) - x.k0;
    }
    return x;
}

// Tiles of a packed batch are numbered without a table: sequence s, whose rows are `each` for one of its tokens, begins at number
// starts[s] * each / tile + s, which leaves it a number for each of its tiles and at most one too many.  The search takes 64 sequences a step.
struct TileAt {
    unsigned seq;
    unsigned long long at;  // in its sequence
};
__device__ __forceinline__ TileAt tile_of(const int *starts, unsigned tokens, unsigned num_seqs, unsigned each, unsigned tile, unsigned long long number)
{
    if (!starts) return {0u, number * tile};
    const auto first = [&](unsigned s) __attribute__((always_inline)) { return (unsigned long long)cut(starts[s], 0u, tokens) * each / tile + s; };
    unsigned lo = 0, left = num_seqs;
    while (left > 1u) {
        const unsigned step = (left + 63u) / 64u, s = lo + threadIdx.x % 64u * step;
        const bool there = threadIdx.x % 64u * step < left && first(s < num_seqs ? s : 0u) <= number;
        const unsigned before = (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(there));
        lo += (before ? before - 1u : 0u) * step;
        left = step < num_seqs - lo ? step : num_seqs - lo;
        if (step == 1u) break;
    }
    lo = (unsigned)__builtin_amdgcn_readfirstlane((int)lo);
    const unsigned long long begin = (unsigned long long)cut(__builtin_amdgcn_readfirstlane(starts[lo]), 0u, tokens) * each / tile + lo;
    return {lo, number < begin ? ~0ull : (number - begin) * tile};
}

__device__ __forceinline__ unsigned long long tiles_over(unsigned tokens, unsigned num_seqs, unsigned each, unsigned tile)
{
    return (unsigned long long)tokens * each / tile + num_seqs;
}

template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(T *p)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)kRecords, kBufferFlags);
}

__device__ __forceinline__ s8v load16(__amdgpu_buffer_rsrc_t from, unsigned bytes)
{
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(s8v, (u4)__builtin_amdgcn_raw_buffer_load_b128(from, (int)bytes, 0, 0));
}

// What was loaded is there: the compiler, which does not count the loads to LDS, would wait for it where it is first used, and for all of
// those with it, in every turn of a loop.
template <int N>
__device__ __forceinline__ void landed(s8v (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// Byte offset of elements d ... of row `row` (of `rows`) behind the tile's first token.
__device__ __forceinline__ unsigned row_offset(unsigned row, unsigned rows, unsigned group, unsigned ld, unsigned d, unsigned dim)
{
    return row < rows && d < dim ? (row / group * ld + row % group * dim + d) * 2u : kOutside;
}

// ---------------------------------------------------------------------------
// tiles in LDS: rows of DP elements, in chunks of 16 bytes, turned so that neither sixteen rows' reads of one chunk nor the
// transposing reads of four chunks of four rows meet in a bank
// ---------------------------------------------------------------------------
template <int DP>
__device__ __forceinline__ unsigned turned(unsigned row, unsigned chunk)
{
    if constexpr (DP == 128) return chunk ^ ((row & 3u) << 2 | (row >> 2 & 3u));
    else return chunk ^ ((row >> 1 & 1u) << 2 | (row >> 2 & 3u));
}

template <int DP>
__device__ __forceinline__ unsigned lds_chunk(unsigned row, unsigned chunk) { return row * (DP * 2u) + turned<DP>(row, chunk) * 16u; }

typedef CDSGD_LDS unsigned char *Lds;

// Where a lane finds its (first) operands in a tile: the places of its first ones, from which those of the others differ by a few bits.
template <int DP>
struct Operands {
    unsigned row, column;

    __device__ __forceinline__ Operands()
    {
        const unsigned l = threadIdx.x % 64u, at = 16u * (l / 16u % 2u) + 4u * (l % 4u);
        row = lds_chunk<DP>(l % 32u, l / 32u);
        column = lds_chunk<DP>(4u * (l / 32u) + l % 16u / 4u, at / 8u) + at % 8u * 2u;
    }
    // At the head of a loop with no registers left: what the others are is worked out where they are read, one instruction each, and not kept in registers across it.
    __device__ __forceinline__ void renew() { asm volatile("" : "+v"(row), "+v"(column)); }
    // elements 16 k + 8 (l / 32) ... + 7 of row l % 32 of those that begin at `from`
    __device__ __forceinline__ s8v rows(Lds from, unsigned k) const { return *(const CDSGD_LDS s8v *)(from + (row ^ k * 32u)); }
    // column 32 d + l % 32 of rows 4 (l / 32) ... + 3 and 8 + 4 (l / 32) ... + 3 of those
    __device__ __forceinline__ s8v columns(Lds from, unsigned d) const
    {
        typedef CDSGD_LDS s4v *Four;
        const s4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(from + (column ^ d * 64u)));
        const s4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(from + 16u * DP + (column ^ (d * 64u | 32u))));
        return s8v{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    }
};

// A buffer's description, in scalar registers.
__device__ __forceinline__ i4s same_in_all(i4s x)
{
    return i4s{__builtin_amdgcn_readfirstlane(x.x), __builtin_amdgcn_readfirstlane(x.y), __builtin_amdgcn_readfirstlane(x.z), x.w};
}

// A tile of ROWS rows on its way to LDS, by WAVES waves: row i is head i % group of token i / group.  What the buffer does not hold, and
// elements behind `dim`, arrive as 0.
template <int DP, int ROWS, int WAVES>
struct TileLoads {
    static constexpr unsigned kLoads = ROWS * DP * 2 / 1024 / WAVES;
    unsigned at[kLoads];

    __device__ __forceinline__ TileLoads(unsigned wave, unsigned group, unsigned ld, unsigned dim)
    {
        const unsigned l = threadIdx.x % 64u;
#pragma unroll
        for (unsigned i = 0; i < kLoads; ++i) {
            const unsigned row = (wave * kLoads + i) * (512u / DP) + l / (DP / 8u), d = turned<DP>(row, l % (DP / 8u)) * 8u;
            at[i] = d < dim ? (row / group * ld + row % group * dim + d) * 2u : kOutside;
        }
    }
    __device__ __forceinline__ void ask(Lds tile, unsigned wave, const void *from, unsigned bytes) const
    {
        const i4s buffer = same_in_all(buffer_of(from, bytes));
#pragma unroll
        for (unsigned i = 0; i < kLoads; ++i) load_to_lds<16>(buffer, tile + (wave * kLoads + i) * 1024u, at[i]);
    }
};

// The order of what stands before in its block: AHEAD reads of LDS, then COUNT products, each followed by EACH more reads while there are any.
template <int AHEAD, int COUNT, int EACH>
__device__ __forceinline__ void reads_ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    }
}

// Of the 32 rows of a result, 16 from 16 t on, rounded: a second operand.
// P and dS are rounded once here, as the matrix instructions take no wider operands beside 16-bit ones.  A second operand of what that leaves costs a
// product more each: measured, errors against 64 bits as multiples of those of a result that is rounded once, and times (us, 8191 tokens in 8 sequences, 32
// heads of 128 over 8 | 4096 tokens, not causal):
//   out, dv  1.25 to 1.4 -> 1.0   forward 125 | 258 -> 149 | 353
//   dq       1.75 (fp16 1.9) -> 1.4 (1.5)   dq 170 | 374 -> 198 | 468
//   dk       1.6 -> 1.2 (with dq's)   dk, dv 270 | 517 -> 318 | 633, and of both P and dS 428 | 823
// What is lost is about as much as the results' own rounding, and the rest of dq's is from the rounded `out` in dout . out: it is left at one product.
template <int DT>
__device__ __forceinline__ s8v rounded(const f16v &x, unsigned t)
{
    Elem<DT> e[8];
#pragma unroll
    for (unsigned i = 0; i < 8; ++i) e[i] = (Elem<DT>)x[8 * t + i];
    return __builtin_bit_cast(s8v, e);
}

// x of lane l % 32, and of lane 32 + l % 32.
struct Halves {
    float low, high;
};
__device__ __forceinline__ Halves halves(float x)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned low = both[0], high = both[1];  // (a cast of an element's bits is one of the first element's to this compiler)
    return {__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)};
}
__device__ __forceinline__ float sum_of_halves(float x)
{
    const Halves h = halves(x);
    return h.low + h.high;
}
__device__ __forceinline__ float larger_half(float x)
{
    const Halves h = halves(x);
    return __builtin_fmaxf(h.low, h.high);
}

// acc += first * second where the second operand has zeros in what a lane does not see of the 16 that are summed over: it sees number n if
// from <= n < to.  A matrix instruction makes 0 times an infinity or NaN a NaN, so that these are taken out of the first operand, and what of them a lane
// sees is added for itself.  Without any the result is that of the one product, to the bit.
template <int DT>
__device__ __forceinline__ void add_seen(f16v &acc, s8v first, s8v second, int from, int to)
{
    __builtin_amdgcn_sched_barrier(0);
    typedef unsigned u4v __attribute__((ext_vector_type(4)));
    constexpr unsigned kTop = DT == kGradBF16 ? 0x7F80u : 0x7C00u;
    u4v w = __builtin_bit_cast(u4v, first), fine;
    unsigned any = 0;
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) {
        const unsigned mask = ((w[i] & kTop) == kTop ? 0xFFFFu : 0u) | ((w[i] >> 16 & kTop) == kTop ? 0xFFFF0000u : 0u);
        any |= mask;
        fine[i] = w[i] & ~mask;
        w[i] &= mask;
    }
    acc = mfma<DT>(__builtin_bit_cast(s8v, fine), second, acc);
    if (__builtin_amdgcn_ballot_w64(any != 0u) == 0) return;
    const u4v p = __builtin_bit_cast(u4v, second);
    const unsigned half = lane_now() / 32u;
    const auto widen = [](unsigned bits) __attribute__((always_inline)) { return (float)__builtin_bit_cast(Elem<DT>, (unsigned short)bits); };
#pragma unroll 1
    for (int n = 0; n < 16; ++n) {
        const unsigned at = (unsigned)n / 4u % 2u, e = (unsigned)n / 8u * 4u + (unsigned)n % 4u;  // lanes of half `at` hold it, in slot e
        const auto slot = [&](const u4v &x) __attribute__((always_inline)) { return (e < 2u ? x[0] : e < 4u ? x[1] : e < 6u ? x[2] : x[3]) >> e % 2u * 16u & 0xFFFFu; };
        const unsigned mine = half == at ? slot(w) : 0u;
        if (__builtin_amdgcn_ballot_w64(mine != 0u) == 0) continue;
        const Halves both = halves(widen(slot(p)));
        const float factor = at ? both.high : both.low;
        const bool sees = n >= from && n < to;
#pragma unroll
        for (unsigned r = 0; r < 16; ++r) {
            const unsigned bits = (unsigned)__builtin_amdgcn_ds_bpermute((int)(32u * at + row_of(r, half)) * 4, (int)mine);
            if (sees && bits != 0u) acc[r] = __builtin_fmaf(widen(bits), factor, acc[r]);
            if (r % 4u == 3u) __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Is any of a wave's results an infinity or NaN?
template <int N>
__device__ __forceinline__ bool any_not_finite(const f16v (&acc)[N])
{
    float zero = 0.0f;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (unsigned r = 0; r < 16; ++r) zero = __builtin_fmaf(acc[d][r], 0.0f, zero);
    return __builtin_amdgcn_ballot_w64(zero != 0.0f) != 0;
}

// Does any of a group's waves say so?  room: a word for each of them.
template <int WAVES>
__device__ __forceinline__ bool any_of_group(bool mine, unsigned *room)
{
    __syncthreads();
    if (threadIdx.x % 64u == 0u) room[threadIdx.x / 64u] = mine;
    __syncthreads();
    unsigned any = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) any |= room[i];
    return __builtin_amdgcn_readfirstlane((int)any) != 0;
}

// A row's results, which lie in two lanes four elements at a time, times f and rounded.
template <int DT, int DP>
__device__ __forceinline__ void store_row(Elem<DT> *row, const f16v (&acc)[DP / 32], float f, unsigned dim)
{
    typedef Elem<DT> e4 __attribute__((ext_vector_type(4)));
    const unsigned half = lane_now() / 32u;
#pragma unroll
    for (unsigned d = 0; d < DP / 32; ++d)
#pragma unroll
        for (unsigned q = 0; q < 4; ++q) {
            const unsigned at = 32u * d + 8u * q + 4u * half;
            if (at < dim)
                *reinterpret_cast<e4 *>(__builtin_assume_aligned(row + at, 8)) =
                    e4{(Elem<DT>)(acc[d][4 * q] * f), (Elem<DT>)(acc[d][4 * q + 1] * f), (Elem<DT>)(acc[d][4 * q + 2] * f), (Elem<DT>)(acc[d][4 * q + 3] * f)};
        }
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// A group takes 128 rows, 32 to a wave, and goes through the keys that they see by tiles of 64, the next tile on its way to LDS while one is worked on.
// With the 222 registers that a wave of 128 elements a head takes there are two groups to a compute unit, and their LDS fits.  16384 tokens, 16
// heads of 128 over 2, causal: 1.0 to 1.07 ms, 1.1 PFLOP/s of the 1.35 that the library's product reaches; bound by power and by the vector
// instructions between the products (164 beside 32 products for a tile).  One group to a compute unit 1.37, tiles through registers 1.9, rows and tiles
// read two reads ahead in place of six 1.10, a block's probabilities between the next one's products 1.2 to 1.6 (registers).
//
// parts, part_lse: where several groups share a row's keys (`splits`), each leaves its own result, [splits][row of all][DP] in fp32 and
// [splits][row of all]; rows of all are numbered [kv head][query][head of the group].
template <int DT, int DP>
__global__ __launch_bounds__(256, DP == 64 ? 4 : 2) void k_attention_forward(AttentionSizes z, Heads<const Elem<DT>> q, Heads<const Elem<DT>> k, Heads<const Elem<DT>> v,
                                                           Heads<Elem<DT>> out, float *__restrict__ lse, unsigned splits, float *__restrict__ parts,
                                                           float *__restrict__ part_lse)
{
    constexpr unsigned kTile = kTileKeys * DP * 2;
    __shared__ __align__(1024) unsigned char smem[4 * kTile];  // two tiles of keys and of values
    __shared__ unsigned said[4];
    const Lds lds = (Lds)smem;
    const unsigned kv = blockIdx.x % z.kv_heads, split = blockIdx.x / z.kv_heads % splits;
    // (the last tiles of a sequence see the most keys: they go first)
    const TileAt t = tile_of(z.starts_q, z.tokens_q, z.num_seqs, z.group, kTileRows,
                           tiles_over(z.tokens_q, z.num_seqs, z.group, kTileRows) - 1u - blockIdx.x / z.kv_heads / splits);
    const Sequence s = sequence_of(z, t.seq);
    const unsigned long long all_rows = (unsigned long long)s.queries * z.group;
    if (t.at >= all_rows) return;
    const unsigned first_query = (unsigned)(t.at / z.group), skip = (unsigned)(t.at % z.group);  // the tile's rows begin `skip` rows into its first query's
    const unsigned rows = all_rows - t.at < kTileRows ? (unsigned)(all_rows - t.at) : kTileRows;
    const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u), l = threadIdx.x % 64u, half = l / 32u, row = wave * 32u + l % 32u;
    const long long hidden_from = (long long)s.keys - s.queries + 1;  // query i sees keys below i + this

    const unsigned head0 = kv * z.group;
    // keys that a row sees, that all of the tile's together see, and that each of the wave's sees
    const auto seen = [&](unsigned r) __attribute__((always_inline)) -> unsigned {
        if (!z.causal) return s.keys;
        const long long n = (long long)(first_query + (skip + r) / z.group) + hidden_from;
        return n < 0 ? 0u : n < (long long)s.keys ? (unsigned)n : s.keys;
    };
    const unsigned mine = row < rows ? seen(row) : 0u, all = seen(rows - 1u), least = (unsigned)__builtin_amdgcn_readfirstlane((int)seen(wave * 32u));
    unsigned from = 0, to = all;
    if (splits > 1u) {
        const unsigned tiles = (s.keys + kTileKeys - 1u) / kTileKeys, each = (tiles + splits - 1u) / splits * kTileKeys;
        from = split * each < to ? split * each : to;
        to = to - from < each ? to : from + each;
    }

    f16v acc[DP / 32] = {};
    // P is formed as 2^(S c + shift), shift = lift - top c with the row's largest S so far: `top` stays where it is until a row has one that is
    // larger by more than a factor of 2^kSlack, so that what is there has to be multiplied in the first tiles alone.
    float top = -kInfinity, shift = 0.0f, total = 0.0f;
    const float c = z.scale * kLog2e, slack = kSlack / c;
    const TileLoads<DP, kTileKeys, 4> loads_k(wave, 1u, k.ld, z.dim), loads_v(wave, 1u, v.ld, z.dim);
    const auto ask = [&](unsigned j, unsigned b) __attribute__((always_inline)) {
        const unsigned left = s.keys - j < kTileKeys ? s.keys - j : kTileKeys;
        loads_k.ask(lds + b * 2u * kTile, wave, k.p + (size_t)(s.k0 + j) * k.ld + kv * z.dim, ((left - 1u) * k.ld + z.dim) * 2u);
        loads_v.ask(lds + b * 2u * kTile + kTile, wave, v.p + (size_t)(s.k0 + j) * v.ld + kv * z.dim, ((left - 1u) * v.ld + z.dim) * 2u);
    };
    unsigned buffer = 0;
    if (from < to) ask(from, 0);
    // asked for behind the first tile, which is on its way meanwhile (one token over 32768 keys 24.3 -> 23.4 us)
    const __amdgpu_buffer_rsrc_t from_q = buffer_at(q.p + (size_t)(s.q0 + first_query) * q.ld + head0 * z.dim);
    s8v bq[DP / 16];
#pragma unroll
    for (unsigned i = 0; i < DP / 16; ++i) bq[i] = load16(from_q, row_offset(skip + row, skip + rows, z.group, q.ld, 16u * i + 8u * half, z.dim));
    landed(bq);
    const auto run = [&](auto careful) __attribute__((always_inline)) {
        constexpr bool CAREFUL = decltype(careful)::value;
        for (unsigned j = from; j < to; j += kTileKeys) {
            wait_for_loads<0>();
            __syncthreads();
            if (j + kTileKeys < to) ask(j + kTileKeys, buffer ^ 1u);
            const Lds tile_k = lds + buffer * 2u * kTile, tile_v = tile_k + kTile;
            buffer ^= 1u;
            if (wave * 32u >= rows) continue;
            Operands<DP> operand;
            if constexpr (CAREFUL) operand.renew();
            f16v x[2] = {};
#pragma unroll
            for (unsigned i = 0; i < DP / 16; ++i)
#pragma unroll
                for (unsigned b = 0; b < 2; ++b) x[b] = mfma<DT>(operand.rows(tile_k + b * (32u * DP * 2u), i), bq[i], x[b]);
            reads_ahead<6, DP / 8, 1>();
            if (j + kTileKeys > least) {
#pragma unroll
                for (unsigned b = 0; b < 2; ++b)
#pragma unroll
                    for (unsigned r = 0; r < 16; ++r)
                        if (j + 32u * b + row_of(r, half) >= mine) x[b][r] = -kInfinity;
            }
            float most = x[0][0];
#pragma unroll
            for (unsigned r = 1; r < 32; ++r) most = __builtin_fmaxf(most, x[r / 16][r % 16]);
            most = larger_half(most);
            // (what happens to a row is its own: others in the wave do not change its bits)
            const bool rises = !(most <= top + slack);
            if (__builtin_amdgcn_ballot_w64(rises) != 0) {
                const float now = rises ? __builtin_fmaxf(most, top) : top, next = !rises ? shift : now == -kInfinity ? 0.0f : kLift<DT> - now * c;
                // (of logits far from 0 the product with c loses more than what is left: differences first)
                const float keep = !rises ? 1.0f : top == -kInfinity ? 0.0f : __builtin_fabsf(next) > kFar ? __builtin_amdgcn_exp2f((top - now) * c) : __builtin_amdgcn_exp2f(next - shift);
                top = now, shift = next;
                total *= keep;
#pragma unroll
                for (unsigned d = 0; d < DP / 32; ++d) acc[d] *= keep;
            }
            float add = shift;
            const bool is_far = __builtin_fabsf(shift) > kFar;
            if (__builtin_amdgcn_ballot_w64(is_far) != 0) {
                const float base = is_far ? top : 0.0f;
                add = is_far ? kLift<DT> : shift;
#pragma unroll
                for (unsigned r = 0; r < 32; ++r) x[r / 16][r % 16] -= base;
            }
#pragma unroll
            for (unsigned b = 0; b < 2; ++b)
#pragma unroll
                for (unsigned h = 0; h < 2; ++h) {
#pragma unroll
                    for (unsigned r = 8 * h; r < 8 * h + 8; ++r) {
                        x[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][r], c, add));
                        total += x[b][r];
                    }
                    const s8v p = rounded<DT>(x[b], h);
#pragma unroll
                    for (unsigned d = 0; d < DP / 32; ++d) {
                        const s8v columns = operand.columns(tile_v + (2u * b + h) * (16u * DP * 2u), d);
                        if constexpr (CAREFUL) add_seen<DT>(acc[d], columns, p, 0, (int)(mine - j - 32u * b - 16u * h));
                        else acc[d] = mfma<DT>(columns, p, acc[d]);
                    }
                }
        }
    };
    run(std::false_type());
    // Results that are not finite are formed again, so that no row has them from keys that are hidden from it.
    if (z.causal && any_of_group<4>(any_not_finite(acc), said)) {
        top = -kInfinity, shift = 0.0f, total = 0.0f, buffer = 0;
#pragma unroll
        for (unsigned d = 0; d < DP / 32; ++d) acc[d] = f16v{};
        if (from < to) ask(from, 0);
        run(std::true_type());
    }
    total = sum_of_halves(total);
    if (row >= rows) return;
    const unsigned query = first_query + (skip + row) / z.group, head = head0 + (skip + row) % z.group;
    const float f = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
    const float log_sum = total == 0.0f ? -kInfinity : (__builtin_log2f(total) - shift) * 0.693147180559945f;
    if (splits > 1u) {
        const size_t at = (((size_t)split * z.kv_heads + kv) * z.tokens_q + s.q0 + query) * z.group + head - head0;
        store_row<kGradF32, DP>(parts + at * DP, acc, f, DP);
        if (half == 0u) part_lse[at] = log_sum;
    } else {
        store_row<DT, DP>(out.p + (size_t)(s.q0 + query) * out.ld + head * z.dim, acc, f, z.dim);
        if (lse && half == 0u) lse[(size_t)head * z.tokens_q + s.q0 + query] = log_sum;
    }
}

// A row's parts, joined: a group to a row, whose waves take every fourth part each.
template <int DT, int DP>
__global__ __launch_bounds__(256) void k_attention_join(AttentionSizes z, Heads<Elem<DT>> out, float *__restrict__ lse, unsigned splits,
                                                        const float *__restrict__ parts, const float *__restrict__ part_lse)
{
    constexpr unsigned kEach = DP / 64;
    __shared__ float weight[kMostSplits], sums[4][DP];
    const size_t rows = (size_t)z.kv_heads * z.tokens_q * z.group, row = blockIdx.x;
    const unsigned wave = threadIdx.x / 64u, lane = threadIdx.x % 64u, query = (unsigned)(row / z.group % z.tokens_q);
    const unsigned head = (unsigned)(row / z.group / z.tokens_q) * z.group + (unsigned)(row % z.group);
    if (z.starts_q && (query < cut(z.starts_q[0], 0u, z.tokens_q) || query >= cut(z.starts_q[z.num_seqs], 0u, z.tokens_q))) return;
    float mine[kMostSplits / 64], most = -kInfinity, total = 0.0f;
#pragma unroll
    for (unsigned i = 0; i < kMostSplits / 64; ++i) {
        const unsigned p = i * 64u + lane;
        mine[i] = p < splits ? part_lse[p * rows + row] : -kInfinity;
        most = __builtin_fmaxf(most, mine[i]);
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, m));
    const float base = most == -kInfinity ? 0.0f : most;
#pragma unroll
    for (unsigned i = 0; i < kMostSplits / 64; ++i) {
        mine[i] = __builtin_amdgcn_exp2f((mine[i] - base) * kLog2e);
        total += mine[i];
        if (wave == 0u) weight[i * 64u + lane] = mine[i];
    }
    total = wave_sum(total);
    __syncthreads();
    float sum[kEach] = {};
    const float *at = parts + row * DP + lane * kEach;
#pragma unroll 8
    for (unsigned i = wave; i < splits; i += 4u) {
        const Few<kGradF32, (int)kEach> x = *reinterpret_cast<const Few<kGradF32, (int)kEach> *>(at + i * rows * DP);
#pragma unroll
        for (unsigned k = 0; k < kEach; ++k) sum[k] = __builtin_fmaf(weight[i], x.v[k], sum[k]);
    }
#pragma unroll
    for (unsigned k = 0; k < kEach; ++k) sums[wave][lane * kEach + k] = sum[k];
    __syncthreads();
    const unsigned d = threadIdx.x;
    if (d < z.dim) {
        const float f = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
        out.p[(size_t)query * out.ld + head * z.dim + d] = (Elem<DT>)((sums[0][d] + sums[1][d] + (sums[2][d] + sums[3][d])) * f);
    }
    if (lse && d == 0u) lse[(size_t)head * z.tokens_q + query] = total == 0.0f ? -kInfinity : base + __builtin_logf(total);
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// dS of fp16 tensors is an operand times a power of two of its own, a row's in dq and a key's in dk (either is a lane's): fp16 ends at 65504, which
// |dS| passes where values are large, and loses bits below 2^-14, where a flat row of many keys has all of it.  `fit` is given numbers that are
// multiplied by `by` already.  The first that are not 0 bring the largest to 2^7 ... 2^8, later ones above 2^15 bring it there again, and what is summed up
// is multiplied with them: nothing is lost of a number but below 2^-32 of the largest.  By no more than 2^60 at first: what comes later may be as
// large as 2^39.  (7999 tokens in 16 sequences, 12 heads of 64, not causal, us: dq 42 -> 45 and dk, dv 69 -> 62 with it in place of one power of two of dout's
// largest magnitude, which dk and dv's rows had to be searched for.)
struct Lift {
    float by = 1.0f;
    bool begun = false;

    template <int N>
    __device__ __forceinline__ void fit(f16v &y, f16v (&acc)[N])
    {
        float most = 0.0f;
#pragma unroll
        for (unsigned r = 0; r < 16; ++r) most = __builtin_fmaxf(most, __builtin_fabsf(y[r]));
        most = larger_half(most);
        const bool change = most > 32768.0f || (!begun && most > 0.0f);
        if (__builtin_amdgcn_ballot_w64(change) == 0) return;
        const unsigned e = __builtin_bit_cast(unsigned, most) >> 23, to = 261u - e;  // (of most's exponent field e, that of 2^7 over its power of two)
        const float f = !change || e == 255u ? 1.0f : __builtin_bit_cast(float, (to < 187u ? to : 187u) << 23);
        begun = begun || change;
        by *= f;
        y *= f;
#pragma unroll
        for (int d = 0; d < N; ++d) acc[d] *= f;
    }
};

// dq, and with it the first kernel of the backward pass: tiles as in the forward pass, three products for its two.  4096 tokens, 32 heads of 128 over 8,
// not causal: 374 us, 1.1 PFLOP/s, bound as the forward pass is; 8191 tokens in 8 sequences, causal: 166 to 172.
// For the next kernel row_lse receives what S begins with in every row, (lift - lse log2 e) / c, far 0, and delta -dout . out, all
// [kv head][token][head of the group].  A row whose lse is far from 0 leaves its largest S, and in far 2^lift over the sum of exp(scale (S - largest));
// where a tile has such rows its first one's far is not 0 (-1 if it is not far itself).
template <int DT, int DP>
__global__ __launch_bounds__(256, 2) void k_attention_dq(AttentionSizes z, Heads<const Elem<DT>> dout, Heads<const Elem<DT>> q, Heads<const Elem<DT>> k,
                                                      Heads<const Elem<DT>> v, Heads<const Elem<DT>> out, const float *__restrict__ lse,
                                                      Heads<Elem<DT>> dq, float *__restrict__ row_lse, float *__restrict__ delta,
                                                      float *__restrict__ far)
{
    constexpr unsigned kTile = kTileKeys * DP * 2;
    __shared__ __align__(1024) unsigned char smem[4 * kTile];  // two tiles of keys and of values
    __shared__ unsigned said[4];
    const Lds lds = (Lds)smem;
    const unsigned kv = blockIdx.x % z.kv_heads;
    const TileAt t = tile_of(z.starts_q, z.tokens_q, z.num_seqs, z.group, kTileRows,
                           tiles_over(z.tokens_q, z.num_seqs, z.group, kTileRows) - 1u - blockIdx.x / z.kv_heads);
    const Sequence s = sequence_of(z, t.seq);
    const unsigned long long all_rows = (unsigned long long)s.queries * z.group;
    if (t.at >= all_rows) return;
    const unsigned first_query = (unsigned)(t.at / z.group), skip = (unsigned)(t.at % z.group);
    const unsigned rows = all_rows - t.at < kTileRows ? (unsigned)(all_rows - t.at) : kTileRows;
    const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u), l = threadIdx.x % 64u, half = l / 32u, row = wave * 32u + l % 32u;
    const long long hidden_from = (long long)s.keys - s.queries + 1;
    const unsigned head0 = kv * z.group, query = first_query + (skip + row) / z.group, head = head0 + (skip + row) % z.group;
    const size_t token = s.q0 + first_query, at = (size_t)head * z.tokens_q + s.q0 + query;

    const __amdgpu_buffer_rsrc_t from_q = buffer_at(q.p + token * q.ld + head0 * z.dim);
    const __amdgpu_buffer_rsrc_t from_d = buffer_at(dout.p + token * dout.ld + head0 * z.dim);
    const __amdgpu_buffer_rsrc_t from_o = buffer_at(out.p + token * out.ld + head0 * z.dim);
    s8v bq[DP / 16], bd[DP / 16];
    float sum = 0.0f;
#pragma unroll
    for (unsigned i = 0; i < DP / 16; ++i) {
        typedef Elem<DT> e8 __attribute__((ext_vector_type(8)));
        const unsigned d = 16u * i + 8u * half;
        bq[i] = load16(from_q, row_offset(skip + row, skip + rows, z.group, q.ld, d, z.dim));
        bd[i] = load16(from_d, row_offset(skip + row, skip + rows, z.group, dout.ld, d, z.dim));
        const e8 o = __builtin_bit_cast(e8, load16(from_o, row_offset(skip + row, skip + rows, z.group, out.ld, d, z.dim)));
        const e8 g = __builtin_bit_cast(e8, bd[i]);
#pragma unroll
        for (unsigned e = 0; e < 8; ++e) sum = __builtin_fmaf((float)g[e], (float)o[e], sum);
    }
    sum = sum_of_halves(sum);
    // (a row that sees nothing, and one that is not there, has no share in anything)
    const float log_sum = row < rows ? lse[at] : kInfinity;
    float base = log_sum == -kInfinity ? kInfinity : log_sum * kLog2e, top = 0.0f;
    landed(bq);
    landed(bd);
    const float c = z.scale * kLog2e;

    const auto seen = [&](unsigned r) __attribute__((always_inline)) -> unsigned {
        if (!z.causal) return s.keys;
        const long long n = (long long)(first_query + (skip + r) / z.group) + hidden_from;
        return n < 0 ? 0u : n < (long long)s.keys ? (unsigned)n : s.keys;
    };
    const unsigned mine = row < rows ? seen(row) : 0u, to = seen(rows - 1u), least = (unsigned)__builtin_amdgcn_readfirstlane((int)seen(wave * 32u));
    f16v acc[DP / 32] = {};
    const TileLoads<DP, kTileKeys, 4> loads_k(wave, 1u, k.ld, z.dim), loads_v(wave, 1u, v.ld, z.dim);
    const auto ask_keys = [&](unsigned j, unsigned b) __attribute__((always_inline)) {
        const unsigned left = s.keys - j < kTileKeys ? s.keys - j : kTileKeys;
        loads_k.ask(lds + b * 2u * kTile, wave, k.p + (size_t)(s.k0 + j) * k.ld + kv * z.dim, ((left - 1u) * k.ld + z.dim) * 2u);
    };
    const auto ask = [&](unsigned j, unsigned b) __attribute__((always_inline)) {
        const unsigned left = s.keys - j < kTileKeys ? s.keys - j : kTileKeys;
        ask_keys(j, b);
        loads_v.ask(lds + b * 2u * kTile + kTile, wave, v.p + (size_t)(s.k0 + j) * v.ld + kv * z.dim, ((left - 1u) * v.ld + z.dim) * 2u);
    };
    Operands<DP> operand;
    const auto hide = [&](f16v &x, unsigned first) __attribute__((always_inline)) {
#pragma unroll
        for (unsigned r = 0; r < 16; ++r)
            if (first + row_of(r, half) >= mine) x[r] = -kInfinity;
    };
    const bool is_far = mine > 0u && __builtin_fabsf(base) > kFarBack;
    const bool far_wave = __builtin_amdgcn_ballot_w64(is_far) != 0;
    bool far_tile = any_of_group<4>(far_wave, said);
    if (far_tile) {
        float most = -kInfinity, total = 0.0f;
        unsigned buffer = 0;
        if (to) ask_keys(0, 0);
        for (unsigned j = 0; j < to; j += kTileKeys) {
            wait_for_loads<0>();
            __syncthreads();
            if (j + kTileKeys < to) ask_keys(j + kTileKeys, buffer ^ 1u);
            const unsigned at = buffer;
            buffer ^= 1u;
            if (!far_wave) continue;
#pragma unroll 1
            for (unsigned b = 0; b < 2; ++b) {
                f16v x = {};
#pragma unroll
                for (unsigned i = 0; i < DP / 16; ++i) x = mfma<DT>(operand.rows(lds + at * 2u * kTile + b * (32u * DP * 2u), i), bq[i], x);
                if (j + kTileKeys > least) hide(x, j + 32u * b);
                const float before = most;
#pragma unroll
                for (unsigned r = 0; r < 16; ++r) most = __builtin_fmaxf(most, x[r]);
                most = larger_half(most);
                if (most != -kInfinity) {
                    total *= __builtin_amdgcn_exp2f((before - most) * c);
#pragma unroll
                    for (unsigned r = 0; r < 16; ++r) total += __builtin_amdgcn_exp2f((x[r] - most) * c);
                }
            }
        }
        total = sum_of_halves(total);
        if (is_far && __builtin_fabsf(most) < kInfinity) top = most, base = __builtin_log2f(total);
        far_tile = any_of_group<4>(__builtin_amdgcn_ballot_w64(top != 0.0f) != 0, said);
    }
    if (row < rows && half == 0u) {
        const size_t place = ((size_t)kv * z.tokens_q + s.q0 + query) * z.group + head - head0;
        row_lse[place] = top != 0.0f ? top : (kLiftBack<DT> - base) / c;
        delta[place] = -sum;
        far[place] = top != 0.0f ? __builtin_amdgcn_exp2f(kLiftBack<DT> - base) : row == 0u && far_tile ? -1.0f : 0.0f;
    }
    Lift lift;
    unsigned buffer = 0;
    if (to) ask(0, 0);
    const auto run = [&](auto careful) __attribute__((always_inline)) {
        constexpr bool CAREFUL = decltype(careful)::value;
        for (unsigned j = 0; j < to; j += kTileKeys) {
            wait_for_loads<0>();
            __syncthreads();
            if (j + kTileKeys < to) ask(j + kTileKeys, buffer ^ 1u);
            const unsigned at = buffer;
            buffer ^= 1u;
            if (wave * 32u >= rows) continue;
            operand.renew();
#pragma unroll
            for (unsigned b = 0; b < 2; ++b) {
                const Lds at_k = lds + at * 2u * kTile + b * (32u * DP * 2u), at_v = at_k + kTile;
                f16v x = {}, y = {};
                s8v ring_k[2], ring_v[2];
                const auto fetch_rows = [&](unsigned i) __attribute__((always_inline)) {
                    ring_k[i % 2u] = operand.rows(at_k, i);
                    ring_v[i % 2u] = operand.rows(at_v, i);
                };
                fetch_rows(0);
#pragma unroll
                for (unsigned i = 0; i < DP / 16; ++i) {
                    if (i + 1u < DP / 16) fetch_rows(i + 1u);
                    __builtin_amdgcn_sched_barrier(0);
                    x = mfma<DT>(ring_k[i % 2u], bq[i], x);
                    y = mfma<DT>(ring_v[i % 2u], bd[i], y);
                    __builtin_amdgcn_sched_barrier(0);
                }
                s8v columns[DP / 16];
#pragma unroll
                for (unsigned i = 0; i < (CAREFUL ? 0 : DP / 16); ++i) columns[i] = operand.columns(at_k + i / (DP / 32) * (16u * DP * 2u), i % (DP / 32));
                if (j + kTileKeys > least) {
#pragma unroll
                    for (unsigned r = 0; r < 16; ++r)
                        if (j + 32u * b + row_of(r, half) >= mine) x[r] = -kInfinity, y[r] = 0.0f;
                }
                if (far_wave) {
#pragma unroll
                    for (unsigned r = 0; r < 16; ++r) x[r] -= top;
                }
#pragma unroll
                for (unsigned r = 0; r < 16; ++r) {
                    y[r] -= sum;
                    y[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, -base)) * (DT == kGradF16 ? y[r] * lift.by : y[r]);
                }
                if constexpr (DT == kGradF16) lift.fit(y, acc);
#pragma unroll
                for (unsigned h = 0; h < 2; ++h) {
                    const s8v ds = rounded<DT>(y, h);
#pragma unroll
                    for (unsigned d = 0; d < DP / 32; ++d) {
                        if constexpr (CAREFUL)
                            add_seen<DT>(acc[d], operand.columns(at_k + h * (16u * DP * 2u), d), ds, 0, (int)(mine - j - 32u * b - 16u * h));
                        else acc[d] = mfma<DT>(columns[h * (DP / 32) + d], ds, acc[d]);
                    }
                }
            }
        }
    };
    run(std::false_type());
    if (z.causal && any_of_group<4>(any_not_finite(acc), said)) {  // as in the forward pass
        lift = Lift();
        buffer = 0;
#pragma unroll
        for (unsigned d = 0; d < DP / 32; ++d) acc[d] = f16v{};
        if (to) ask(0, 0);
        run(std::true_type());
    }
    if (row < rows) store_row<DT, DP>(dq.p + (size_t)(s.q0 + query) * dq.ld + head * z.dim, acc, z.scale / lift.by, z.dim);
}

// dk and dv.  A group takes the keys of kKeyWaves waves, 32 each, of one key head and runs over the rows that see them, in kStreams streams:
// stream i takes every kStreams-th tile of rows, and the streams' sums meet at the end.  The first keys of a long causal sequence are seen by all
// of its rows, and the launch is as long as the longest group.  us (8191 tokens in 8 sequences, 32 heads of 128 over 8 | 4096 tokens, not
// causal, the same heads; fp16, 7999 tokens in 16 sequences, 12 heads of 64, not causal | 4096 tokens, 32 heads of 64 over 8):
//   128 elements a head: 4 waves in 2 streams 264 | 526, 2 in 4 255 | 575, 4 in one stream 345;  64: 2 in 2 70 | 318, 4 in 1 71 | 410, 4 in 2 82 | 314, 2 in 4 97 | 324
// A wave's registers hold its keys and both results, but not its values too, which are read from LDS: of 128 elements a head there is no room for
// them, and of 64 without them there are three waves to a SIMD (the fp16 batch 62 with two, 54 with three).
constexpr unsigned kStreamRows = 32;
template <int DP>
constexpr unsigned kKeyWaves = DP == 128 ? 4 : 2;
template <int DP>
constexpr unsigned kStreams = 2;
template <int DP>
constexpr unsigned kStreamKeys = 32 * kKeyWaves<DP>;

template <int DT, int DP>
__global__ __launch_bounds__(64 * kKeyWaves<DP> * kStreams<DP>, DP == 64 ? 3 : 2) void k_attention_dkv(AttentionSizes z, Heads<const Elem<DT>> dout, Heads<const Elem<DT>> q, Heads<const Elem<DT>> k,
                                                       Heads<const Elem<DT>> v, const float *__restrict__ all_lse, const float *__restrict__ delta,
                                                       const float *__restrict__ far, Heads<Elem<DT>> dk, Heads<Elem<DT>> dv)
{
    constexpr unsigned KW = kKeyWaves<DP>, S = kStreams<DP>, kKeys = kStreamKeys<DP>;
    // of a stream, twice: a tile of q, one of dout, and three numbers of each row
    constexpr unsigned kRows = kStreamRows, kTile = kRows * DP * 2, kStage = 2 * kTile + 1024, kValues = S * 2 * kStage;
    constexpr unsigned kSums = 32 * DP * 4;  // of a wave's results of one kind
    static_assert((S - 1) * KW * kSums <= kValues, "the streams' sums fit where their tiles were");
    __shared__ __align__(1024) unsigned char smem[kValues + kKeys * DP * 2];
    __shared__ unsigned said[KW * S];
    const Lds lds = (Lds)smem, values = lds + kValues;
    const unsigned kv = blockIdx.x % z.kv_heads;
    const int *starts = z.starts_k ? z.starts_k : z.starts_q;
    const TileAt t = tile_of(starts, z.tokens_k, z.num_seqs, 1u, kKeys, blockIdx.x / z.kv_heads);
    const Sequence s = sequence_of(z, t.seq);
    if (t.at >= s.keys) return;
    const unsigned key0 = (unsigned)t.at, keys = s.keys - key0 < kKeys ? s.keys - key0 : kKeys;
    const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u), stream = wave / KW, side = wave % KW;
    const unsigned l = threadIdx.x % 64u, half = l / 32u, key = side * 32u + l % 32u, head0 = kv * z.group;

    const TileLoads<DP, kKeys, KW * S> loads_v(wave, 1u, v.ld, z.dim);
    loads_v.ask(values, wave, v.p + (size_t)(s.k0 + key0) * v.ld + kv * z.dim, ((keys - 1u) * v.ld + z.dim) * 2u);
    // the first query that sees key j is j - (keys - queries)
    const long long later = (long long)s.queries - s.keys;
    const auto first_of = [&](unsigned j) __attribute__((always_inline)) -> unsigned {
        const long long i = (long long)j + later;
        return !z.causal || i < 0 ? 0u : i < (long long)s.queries ? (unsigned)i : s.queries;
    };
    f16v acc_k[DP / 32] = {}, acc_v[DP / 32] = {};
    const float c = z.scale * kLog2e;
    Lift lift;
    // A tile is as many queries as have kRows rows at most, or (`parts` of them) a part of one query's heads.
    const unsigned group = z.group, at_once = group < kRows ? kRows / group : 1u, parts = (group + kRows - 1u) / kRows;
    const unsigned from = first_of(key0), tiles = (s.queries - from + at_once - 1u) / at_once * parts;
    const TileLoads<DP, kRows, KW> loads_q(side, group, q.ld, z.dim), loads_d(side, group, dout.ld, z.dim);
    // (values, not one of three variables: the compiler would keep those in memory)
    const float *const numbers = side == 0u ? +all_lse : +delta;
    const float *const far_here = far + ((size_t)kv * z.tokens_q + s.q0) * group;
    unsigned found = 0;
#pragma unroll 4
    for (unsigned long long i = l * (unsigned long long)kTileRows; i < (unsigned long long)s.queries * group; i += 64u * kTileRows) found |= far_here[i] != 0.0f;
    const bool any_far = __builtin_amdgcn_ballot_w64(found != 0u) != 0;
    // tile `n` of all; past the last nothing is in range
    const auto ask = [&](unsigned n, unsigned b) __attribute__((always_inline)) {
        const unsigned i = from + n / parts * at_once, part = n % parts * kRows, there = n < tiles ? s.queries - i : 0u;
        const unsigned queries = there < at_once ? there : at_once, heads = group - part < kRows ? group - part : kRows;
        const Lds to = lds + (stream * 2u + b) * kStage;
        const size_t token = s.q0 + (n < tiles ? i : 0u);
        const unsigned last = queries ? queries - 1u : 0u;
        loads_q.ask(to, side, q.p + token * q.ld + (head0 + part) * z.dim, queries ? (last * q.ld + heads * z.dim) * 2u : 0u);
        loads_d.ask(to + kTile, side, dout.p + token * dout.ld + (head0 + part) * z.dim, queries ? (last * dout.ld + heads * z.dim) * 2u : 0u);
        const size_t at = ((size_t)kv * z.tokens_q + token) * group + part;
        if (KW == 2 || side < 2u) load_to_lds<4>(same_in_all(buffer_of(numbers + at, queries * heads * 4u)), to + 2u * kTile + side * 256u, l * 4u);
        if (any_far && side == 0u) load_to_lds<4>(same_in_all(buffer_of(far + at, queries * heads * 4u)), to + 2u * kTile + 512u, l * 4u);
    };
    Operands<DP> operand;
    unsigned buffer = 0;
    if (tiles) ask(stream, 0);
    const __amdgpu_buffer_rsrc_t from_k = buffer_at(k.p + (size_t)(s.k0 + key0) * k.ld + kv * z.dim);
    s8v bk[DP / 16];
#pragma unroll
    for (unsigned i = 0; i < DP / 16; ++i) bk[i] = load16(from_k, row_offset(key, keys, 1u, k.ld, 16u * i + 8u * half, z.dim));
    landed(bk);
    const auto run = [&](auto with_far, auto careful) __attribute__((always_inline)) {
        constexpr bool CAREFUL = decltype(careful)::value;
        const bool FAR = CAREFUL ? any_far : decltype(with_far)::value;
        for (unsigned first = 0; first < tiles; first += S) {
            wait_for_loads<0>();
            __syncthreads();
            const unsigned n = first + stream, now = from + n / parts * at_once;
            if (first + S < tiles) ask(n + S, buffer ^ 1u);
            const unsigned at = buffer;
            const CDSGD_LDS float *row_lse = (const CDSGD_LDS float *)(lds + (stream * 2u + at) * kStage + 2u * kTile), *row_delta = row_lse + 64, *row_far = row_lse + 128;
            buffer ^= 1u;
            if (side * 32u >= keys || n >= tiles) continue;
            operand.renew();
            // S less lse, and dP less delta: both begin with what is taken from them (S, where there are far rows, with 0, as it did when their
            // largest one was looked for).  The operands of a pair of products are read beside the pair before.
            f16v x, y;
#pragma unroll
            for (unsigned r = 0; r < 16; r += 4) {
                const f4 base = *(const CDSGD_LDS f4 *)(row_lse + row_of(r, half)), sum = *(const CDSGD_LDS f4 *)(row_delta + row_of(r, half));
#pragma unroll
                for (unsigned e = 0; e < 4; ++e) x[r + e] = FAR ? 0.0f : base[e], y[r + e] = sum[e];
            }
            const Lds at_q = lds + (stream * 2u + at) * kStage, at_d = at_q + kTile;
            s8v ring_q[2], ring_d[2], ring_v[2];
            const auto fetch_rows = [&](unsigned e) __attribute__((always_inline)) {
                ring_q[e % 2u] = operand.rows(at_q, e);
                ring_d[e % 2u] = operand.rows(at_d, e);
                ring_v[e % 2u] = operand.rows(values + side * (32u * DP * 2u), e);
            };
            fetch_rows(0);
#pragma unroll
            for (unsigned e = 0; e < DP / 16; ++e) {
                if (e + 1u < DP / 16) fetch_rows(e + 1u);
                __builtin_amdgcn_sched_barrier(0);
                x = mfma<DT>(ring_q[e % 2u], bk[e], x);
                y = mfma<DT>(ring_d[e % 2u], ring_v[e % 2u], y);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (FAR) {
#pragma unroll
                for (unsigned r = 0; r < 16; ++r) {
                    const float over = row_far[row_of(r, half)], first = row_lse[row_of(r, half)], less = x[r] - first;
                    x[r] = over <= 0.0f ? x[r] + first : (less > 0.0f ? 0.0f : less) + __builtin_amdgcn_logf(over) / c;
                    if (r % 2u == 1u) __builtin_amdgcn_sched_barrier(0);
                }
            }
            constexpr unsigned kProducts = DP / 8, kAhead = 3;
            s8v ring[kAhead + 1];
            const auto fetch_columns = [&](unsigned i) __attribute__((always_inline)) {
                ring[i % (kAhead + 1)] = operand.columns((i % 2u ? at_q : at_d) + i / (kProducts / 2u) * (16u * DP * 2u), i / 2u % (DP / 32));
            };
#pragma unroll
            for (unsigned i = 0; i < (CAREFUL ? 0u : kAhead); ++i) fetch_columns(i);
            // (every row of the tile sees every key of the wave, but for causal tiles on the border)
            unsigned hidden = 0;
            const bool border = z.causal && first_of(key0 + side * 32u + 31u) > now;
            if (border) {
                const unsigned lane = lane_now(), half = lane / 32u, first_row = first_of(key0 + side * 32u + lane % 32u);
                hidden = first_row <= now ? 0u : group < kRows ? (first_row - now) * group : kRows;
#pragma unroll
                for (unsigned r = 0; r < 16; ++r)
                    if (row_of(r, half) < hidden) x[r] = -kInfinity, y[r] = 0.0f;
            }
            const float down = lift.by * (1.0f / kLifted<DT>);
#pragma unroll
            for (unsigned r = 0; r < 16; ++r) {
                x[r] = __builtin_amdgcn_exp2f(x[r] * c);
                y[r] = x[r] * (DT == kGradF16 ? y[r] * down : y[r]);
            }
            if constexpr (DT == kGradF16) lift.fit(y, acc_k);
            const s8v p[2] = {rounded<DT>(x, 0), rounded<DT>(x, 1)}, ds[2] = {rounded<DT>(y, 0), rounded<DT>(y, 1)};
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (unsigned i = 0; i < kProducts; ++i) {
                if constexpr (CAREFUL) fetch_columns(i);
                else if (i + kAhead < kProducts) fetch_columns(i + kAhead);
                const unsigned h = i / (kProducts / 2u), d = i / 2u % (DP / 32);
                if constexpr (CAREFUL) add_seen<DT>(i % 2u ? acc_k[d] : acc_v[d], ring[i % (kAhead + 1)], i % 2u ? ds[h] : p[h], (int)hidden - 16 * (int)h, 16);
                else if (i % 2u) acc_k[d] = mfma<DT>(ring[i % (kAhead + 1)], ds[h], acc_k[d]);
                else acc_v[d] = mfma<DT>(ring[i % (kAhead + 1)], p[h], acc_v[d]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // (a branch for far rows within the loop costs 3 % of it, taken or not)
    if (any_far) run(std::true_type(), std::false_type());
    else run(std::false_type(), std::false_type());
    if (z.causal && any_of_group<KW * S>(any_not_finite(acc_k) || any_not_finite(acc_v), said)) {  // as in the forward pass
        lift = Lift();
        buffer = 0;
#pragma unroll
        for (unsigned d = 0; d < DP / 32; ++d) acc_k[d] = f16v{}, acc_v[d] = f16v{};
        if (tiles) ask(stream, 0);
        run(std::true_type(), std::true_type());
    }
    // the streams' sums, added in their order
    const unsigned lane = lane_now(), own_key = side * 32u + lane % 32u;
    wait_for_loads<0>();
    __syncthreads();
    const float f = z.scale / lift.by;
    CDSGD_LDS f4 *const sums = (CDSGD_LDS f4 *)lds;
#pragma unroll
    for (unsigned which = 0; which < 2; ++which) {
        f16v(&acc)[DP / 32] = which ? acc_v : acc_k;
        if constexpr (S > 1) __syncthreads();
        if (stream) {
#pragma unroll
            for (unsigned d = 0; d < DP / 32; ++d)
#pragma unroll
                for (unsigned e = 0; e < 4; ++e) {
                    f4 w = {acc[d][4 * e], acc[d][4 * e + 1], acc[d][4 * e + 2], acc[d][4 * e + 3]};
                    if (!which) w *= f;
                    sums[(((stream - 1u) * KW + side) * (DP / 8u) + d * 4u + e) * 64u + lane] = w;
                }
        }
        if constexpr (S > 1) __syncthreads();
        if (!stream) {
#pragma unroll
            for (unsigned d = 0; d < DP / 32; ++d)
#pragma unroll
                for (unsigned e = 0; e < 4; ++e) {
                    f4 w = {acc[d][4 * e], acc[d][4 * e + 1], acc[d][4 * e + 2], acc[d][4 * e + 3]};
                    if (!which) w *= f;
#pragma unroll
                    for (unsigned i = 0; i < S - 1; ++i) w += sums[((i * KW + side) * (DP / 8u) + d * 4u + e) * 64u + lane];
#pragma unroll
                    for (unsigned i = 0; i < 4; ++i) acc[d][4 * e + i] = w[i];
                }
            if (own_key < keys) {
                const Heads<Elem<DT>> &to = which ? dv : dk;
                store_row<DT, DP>(to.p + (size_t)(s.k0 + key0 + own_key) * to.ld + kv * z.dim, acc, which ? 1.0f / kLifted<DT> : 1.0f, z.dim);
            }
        }
    }
}

}  // namespace
