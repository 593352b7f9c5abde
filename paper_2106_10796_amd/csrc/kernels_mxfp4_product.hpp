// Products of two matrices in MXFP4: out = A B^T, both in blocks along the axis that is summed over.
//
// The kernels load codes and scale words from memory straight into LDS, a line of 128 bytes (256 elements) of a row at a time.
// Eight lanes in a row ask for one line, which is what the path from L2 is fast at: the operand layout of the matrix
// instructions puts neighbouring lanes in different rows, and loads in that order cost a compute unit 37 cycles each instead
// of 16 (64 x 1000 x 4096: 8.1 us with operands straight from memory, 3.8 so).  The line's eight chunks of 16 bytes lie in LDS
// turned by half the row's number (chunk c at c ^ (row / 2 % 8)), so that sixteen rows' reads of one chunk fill the banks.
#pragma once

namespace {

#define CDSGD_LDS __attribute__((address_space(3)))

typedef float f16v __attribute__((ext_vector_type(16)));
typedef int i4s __attribute__((ext_vector_type(4)));

// v_mfma_scale_f32_32x32x64: lane l holds elements 32 (l / 32) ... + 31 of row l % 32 of either operand and their scale, and of
// the result rows i % 4 + 8 (i / 4) + 4 (l / 32), i = 0 ... 15, of column l % 32.
template <int SEL>
__device__ __forceinline__ f16v mfma32(i4v a, i4v b, f16v c, int sa, int sb)
{
    const i8v wa = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, wb = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wa, wb, c, 4, 4, SEL, sa, SEL, sb);
}

// A buffer of `bytes` bytes from p on (uniform): what lies past them is not loaded.
__device__ __forceinline__ i4s buffer_of(const void *p, unsigned long long bytes)
{
    const unsigned long long at = (unsigned long long)p;
    return i4s{(int)(unsigned)at, (int)((unsigned)(at >> 32) & 0xFFFFu), (int)(bytes > 0xFFFFFFFFull ? 0xFFFFFFFFu : (unsigned)bytes),
               (int)kBufferFlags};
}

// Every lane's 16 (4) bytes from `offset` of the buffer on to to + 16 (4) lane.  (The instruction's scalar offset takes no part in
// the range check, so a place along the rows is a part of the buffer's address.)  The compiler does not know of these
// loads: wait_for_loads<N> waits until all but the wave's last N of them are in LDS.  (Its own form of the instruction makes it wait
// for all of them before the next read of any LDS.)  Nor does it look inside for the waits that gfx950 leaves to the program: one
// state between a scalar write of m0 and a load to LDS, and five between a vector instruction that writes a word of the buffer's
// description and the load; s_mov and s_nop are those five (up to 3 % against s_nop 0, 64 x 4096 x 4096 4.9 -> 5.05 us, large
// products the same).  m0 is reserved, so the compiler warns that it will not save it, but it takes the clobber for a write.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int BYTES>
__device__ __forceinline__ void load_to_lds(i4s buffer, CDSGD_LDS unsigned char *to, unsigned offset)
{
    const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)(unsigned long long)to);
    static_assert(BYTES == 16 || BYTES == 4, "sizes in use");
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(offset), "s"(buffer) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(at), "v"(offset), "s"(buffer) : "memory", "m0");
}
#pragma clang diagnostic pop

template <int N>
__device__ __forceinline__ void wait_for_loads()
{
    static_assert(N >= 0 && N < 64, "what the counter holds");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ unsigned last_of(unsigned r, unsigned n) { return r < n ? r : n - 1u; }

// Four neighbouring results of row m, from column n on, in fp32: rounded once, after what out holds has been added.
template <int DT>
__device__ __forceinline__ void put4(Elem<DT> *out, size_t ld, unsigned N, unsigned m, unsigned n, f4 v, bool add)
{
    typedef Elem<DT> e4 __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(sizeof(Elem<DT>)))) At {
        e4 v;
    };
    Elem<DT> *p = out + (size_t)m * ld + n;
    if (n + 4u <= N) {
        if (add) {
            const e4 old = reinterpret_cast<const At *>(p)->v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += (float)old[e];
        }
        reinterpret_cast<At *>(p)->v = e4{(Elem<DT>)v.x, (Elem<DT>)v.y, (Elem<DT>)v.z, (Elem<DT>)v.w};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < N) put<DT>(p + e, v[e], add);
    }
}

// What four neighbours of out hold; 0 where they are not within [M, N].
template <int DT>
__device__ __forceinline__ f4 get4(const Elem<DT> *out, size_t ld, unsigned M, unsigned N, unsigned m, unsigned n)
{
    typedef Elem<DT> e4 __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(sizeof(Elem<DT>)))) At {
        e4 v;
    };
    const Elem<DT> *p = out + (size_t)m * ld + n;
    f4 v = {};
    if (m < M && n + 4u <= N) {
        const e4 old = reinterpret_cast<const At *>(p)->v;
        v = f4{(float)old.x, (float)old.y, (float)old.z, (float)old.w};
    } else if (m < M) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < N) v[e] = (float)p[e];
    }
    return v;
}

// What the lanes of a wave wrote to LDS is there for its other lanes.  (LDS serves a wave in order: this is for the compiler.)
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------------
// few rows
// ---------------------------------------------------------------------------
// A group takes 16 FM rows of A and 16 FN of B; its W waves share the sum, line by line, and each has a ring of D slots in LDS of
// its own, so that no wave waits for another before the end.  Bound by reading B: 1 x 4096 x 25088 10.0 us, 5.5 TB/s of the whole call,
// 64 x 25088 x 4096 11.6 us, 5.0 TB/s; on small matrices by the launch (64 x 1000 x 4096: 3.8 us).
template <int FM, int FN>
constexpr unsigned kRingSlot = (FN + FM) * 2048u + ((FN + 1) / 2 + (FM + 1) / 2) * 256u;

template <int DT, int FM, int FN, int D, int W>
__global__ __launch_bounds__(64 * W) void k_ring(const uint8_t *__restrict__ a, const uint8_t *__restrict__ as,
                                                 const uint8_t *__restrict__ b, const uint8_t *__restrict__ bs, unsigned M, unsigned N,
                                                 unsigned groups, Elem<DT> *__restrict__ out, size_t ld, int add)
{
    constexpr unsigned kSlot = kRingSlot<FM, FN>, kSA = (FM + 1) / 2, kSB = (FN + 1) / 2, kLoads = 2 * FN + 2 * FM + kSB + kSA;
    constexpr unsigned kAtA = FN * 2048u, kAtSB = (FN + FM) * 2048u, kAtSA = kAtSB + kSB * 256u;
    static_assert(FN * FM * 1024u <= kSlot * D, "the parts of the sum fit where the rings were");
    __shared__ __align__(1024) unsigned char smem[kSlot * D * W];
    const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u), lane = threadIdx.x % 64u, l = lane % 16u, j = lane / 16u;
    CDSGD_LDS unsigned char *ring = (CDSGD_LDS unsigned char *)smem + wave * (kSlot * D);
    const unsigned tiles_m = (M + 16u * FM - 1u) / (16u * FM), n0 = blockIdx.x / tiles_m * (16u * FN), m0 = blockIdx.x % tiles_m * (16u * FM);
    const unsigned stride = groups * 64u;
    // codes: lane 8 r + c of load i has chunk c ^ (row / 2 % 8) of row 8 i + r
    unsigned va[2 * FM], vb[2 * FN], vsa[kSA], vsb[kSB];
#pragma unroll
    for (unsigned i = 0; i < 2 * FN; ++i) vb[i] = last_of(i * 8u + lane / 8u, N - n0) * stride + (lane % 8u ^ (i * 4u + lane / 16u) % 8u) * 16u;
#pragma unroll
    for (unsigned i = 0; i < 2 * FM; ++i) va[i] = last_of(i * 8u + lane / 8u, M - m0) * stride + (lane % 8u ^ (i * 4u + lane / 16u) % 8u) * 16u;
    // scale words: lane 32 f + 16 g + l of load i has row 16 (2 i + f) + l of group g (of one fragment: the same twice)
#pragma unroll
    for (unsigned i = 0; i < kSB; ++i) vsb[i] = (j % 2u * N + last_of((2u * i + (FN > 1 ? j / 2u : 0u)) * 16u + l, N - n0)) * 4u;
#pragma unroll
    for (unsigned i = 0; i < kSA; ++i) vsa[i] = (j % 2u * M + last_of((2u * i + (FM > 1 ? j / 2u : 0u)) * 16u + l, M - m0)) * 4u;
    const unsigned pairs = (groups + 1u) / 2u, count = wave < pairs ? (pairs - wave + W - 1u) / W : 0u;
    const auto ask = [&](unsigned i) __attribute__((always_inline)) {
        CDSGD_LDS unsigned char *slot = ring + i % D * kSlot;
        const unsigned p = wave + i * W;
        // (the last line of a row may be half a line, behind which the next row begins, or nothing)
        const i4s ra = buffer_of(a + (size_t)m0 * stride + p * 128u, (unsigned long long)(M - m0) * stride - p * 128u);
        const i4s rb = buffer_of(b + (size_t)n0 * stride + p * 128u, (unsigned long long)(N - n0) * stride - p * 128u);
#pragma unroll
        for (unsigned k = 0; k < 2 * FN; ++k) load_to_lds<16>(rb, slot + k * 1024u, vb[k]);
#pragma unroll
        for (unsigned k = 0; k < 2 * FM; ++k) load_to_lds<16>(ra, slot + kAtA + k * 1024u, va[k]);
        const i4s rsb = buffer_of(bs + ((size_t)(2u * p) * N + n0) * 4u, ((unsigned long long)(groups - 2u * p) * N - n0) * 4u);
        const i4s rsa = buffer_of(as + ((size_t)(2u * p) * M + m0) * 4u, ((unsigned long long)(groups - 2u * p) * M - m0) * 4u);
#pragma unroll
        for (unsigned k = 0; k < kSB; ++k) load_to_lds<4>(rsb, slot + kAtSB + k * 256u, vsb[k]);
#pragma unroll
        for (unsigned k = 0; k < kSA; ++k) load_to_lds<4>(rsa, slot + kAtSA + k * 256u, vsa[k]);
    };
    f4 c[FN][FM] = {};
#pragma unroll
    for (unsigned i = 0; i < D - 1; ++i)
        if (i < count) ask(i);
    for (unsigned i = 0; i < count; ++i) {
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): nothing of the slot that is asked for next is still being read
        if (i + D - 1 < count) {
            ask(i + D - 1);
            wait_for_loads<kLoads *(D - 1)>();
        } else {
            wait_for_loads<0>();
        }
        const CDSGD_LDS unsigned char *slot = ring + i % D * kSlot;
        const bool both = 2u * (wave + i * W) + 1u < groups;
#pragma unroll
        for (unsigned g = 0; g < 2; ++g) {
            if (g && !both) break;
            i4v xb[FN], xa[FM];
            int sb[FN], sa[FM];
            const unsigned at = l * 128u + ((4u * g + j) ^ (l / 2u)) * 16u;
#pragma unroll
            for (unsigned k = 0; k < FN; ++k) {
                xb[k] = *(const CDSGD_LDS i4v *)(slot + k * 2048u + at);
                sb[k] = *(slot + kAtSB + k / 2u * 256u + ((k % 2u * 2u + g) * 16u + l) * 4u + j);
            }
#pragma unroll
            for (unsigned k = 0; k < FM; ++k) {
                xa[k] = *(const CDSGD_LDS i4v *)(slot + kAtA + k * 2048u + at);
                sa[k] = *(slot + kAtSA + k / 2u * 256u + ((k % 2u * 2u + g) * 16u + l) * 4u + j);
            }
#pragma unroll
            for (unsigned i2 = 0; i2 < FN; ++i2)
#pragma unroll
                for (unsigned k = 0; k < FM; ++k) c[i2][k] = mfma16<0, 0>(xb[i2], xa[k], c[i2][k], sb[i2], sa[k]);
        }
    }
    // the waves' parts of the sum, added in their order
    __syncthreads();
    CDSGD_LDS f4 *part = (CDSGD_LDS f4 *)smem;
#pragma unroll
    for (unsigned i = 0; i < FN; ++i)
#pragma unroll
        for (unsigned k = 0; k < FM; ++k) part[((wave * FN + i) * FM + k) * 64u + lane] = c[i][k];
    __syncthreads();
    for (unsigned q = threadIdx.x; q < FN * FM * 64u; q += 64 * W) {
        f4 s = part[q];
#pragma unroll
        for (unsigned w = 1; w < W; ++w) s += part[w * FN * FM * 64u + q];
        const unsigned f = q / 64u, m = m0 + f % FM * 16u + q % 16u, n = n0 + f / FM * 16u + q % 64u / 16u * 4u;
        if (m >= M || n >= N) continue;
        put4<DT>(out, ld, N, m, n, s, add != 0);
    }
}

// The parts that the groups of a split sum left, added in their order.
template <int DT>
__global__ __launch_bounds__(256) void k_join(const float *__restrict__ partial, unsigned M, unsigned N, unsigned splits,
                                              Elem<DT> *__restrict__ out, size_t ld, int add)
{
    const unsigned across = (N + 3u) / 4u;
    const unsigned long long q = (unsigned long long)blockIdx.x * 256u + threadIdx.x;
    if (q >= (unsigned long long)across * M) return;
    const unsigned m = (unsigned)(q / across), n = (unsigned)(q % across) * 4u;
    f4 s = get4<kGradF32>(partial, N, M, N, m, n);
    for (unsigned k = 1; k < splits; ++k) s += get4<kGradF32>(partial + (size_t)k * M * N, N, M, N, m, n);
    put4<DT>(out, ld, N, m, n, s, add != 0);
}

// ---------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------
// A launch computes a part of the result: `tiles_m` by `tiles_n` tiles from row m_from and column n_from on.  `splits` groups may
// share a sum: out is then [splits][M][N], in fp32, for k_join.  A group of WM by WN waves takes BM rows of A and BN of B, a stage of
// one line of every row (four steps of 64 elements) at a time, D stages in LDS.
//
// The operands of a step are read from LDS while the products of the one before it run, and what is loaded for a later stage
// is asked for a few instructions at a time between the products: asked for at once, behind the barrier, the loads hold up every
// wave's products for as long as the line to L2 is busy (8192^3: 334 us, 303 so).
//
// Groups that begin together end together, round after round, and their stores wait for one another while no product runs.  Where
// there is more than one round, the groups of the first begin one after the other, over about the time that a round's stores take
// at the rate of HBM (kSpread, in sleeps of 256 cycles), which the others' products then fill.  us, without and with:
//   8192 x 4096 x 2048 fp32 65.2, 50.2, bf16 50.6, 44.9;  x 4096 fp32 95.0, 83.2, bf16 78.6, 75.8;  16384 x 8192 x 1024 bf16 115, 105;
//   128 by 128 8192 x 4096 x 1024 bf16 37.6, 34.1;  spread over a half and over twice as long: 8192 x 4096 x 2048 fp32 58, 56, bf16 47, 45
//
// 8192 x 4096 x 4096 in bf16, call after call, takes 71 us, 3.9 PFLOP/s; bound by the card's power, not by any path: it draws 1385 of its
// 1400 W at 1.82 GHz, and where all codes are the same 1190 W at 2.39 GHz for 57 us.  256 by 256 with 4 waves 82, 128 by 128 82; the next tile's loads ahead of the
// stores, in groups that go from tile to tile, 74.
template <int BM, int BN>
constexpr unsigned kTileStage = (BM + BN) * 136u;

template <int DT, int BM, int BN, int WM, int WN, int D>
__global__ __launch_bounds__(64 * WM * WN) void k_tiles(const uint8_t *__restrict__ a, const uint8_t *__restrict__ as,
                                                        const uint8_t *__restrict__ b, const uint8_t *__restrict__ bs, unsigned M,
                                                        unsigned N, unsigned all_groups, Elem<DT> *__restrict__ out, size_t ld, int add,
                                                        unsigned splits, unsigned m_from, unsigned n_from, unsigned tiles_m, unsigned tiles_n)
{
    constexpr unsigned W = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
    constexpr unsigned kA = BM * 128, kSA = (BM + BN) * 128, kSB = kSA + BM * 8, kStage = kTileStage<BM, BN>;
    constexpr unsigned kPitch = TN * sizeof(Elem<DT>) + 16u, kOut = 32u * kPitch * W;
    __shared__ __align__(1024) unsigned char smem[D * kStage > kOut ? D * kStage : kOut];
    CDSGD_LDS unsigned char *lds = (CDSGD_LDS unsigned char *)smem;
    const unsigned lane = threadIdx.x % 64u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);

    // The tiles that run on one XCD at a time lie next to one another: group b runs on XCD b % 8, which takes a run of
    // tiles, in bands of 8 rows of tiles.
    const unsigned total = tiles_m * tiles_n;
    const unsigned split = blockIdx.x / total, nth = blockIdx.x % total;
    const unsigned xcd = nth % 8u, id = xcd * (total / 8u) + (xcd < total % 8u ? xcd : total % 8u) + nth / 8u;
    constexpr unsigned kBand = 8;
    const unsigned band = id / (kBand * tiles_n), in = id % (kBand * tiles_n), left = tiles_m - band * kBand, high = left < kBand ? left : kBand;
    const unsigned m0 = m_from + (band * kBand + in % high) * BM, n0 = n_from + in / high * BN;

    // this group's part of the sum: lines `line` ... of every row
    const unsigned stride = all_groups * 64u, lines = (all_groups + 1u) / 2u, each = (lines + splits - 1u) / splits, line = split * each;
    const unsigned here = line < lines ? all_groups - 2u * line : 0u, groups = here < 2u * each ? here : 2u * each, stages = (groups + 1u) / 2u;
    out += (size_t)split * M * N;
    as += (size_t)(2u * line) * M * 4u;
    bs += (size_t)(2u * line) * N * 4u;
    const uint8_t *const at_a = a + (size_t)m0 * stride + line * 128u, *const at_b = b + (size_t)n0 * stride + line * 128u;
    const unsigned long long bytes_a = (unsigned long long)(M - m0) * stride - line * 128u,
                             bytes_b = (unsigned long long)(N - n0) * stride - line * 128u;
    constexpr unsigned JA = BM / 8 / W, JB = BN / 8 / W, kWords = 2 * (BM + BN) / 64, P = (kWords + W - 1) / W, kItems = JA + JB + P;
    static_assert(JA * 8 * W == BM && JB * 8 * W == BN, "every wave loads as much");
    unsigned va[JA], vb[JB];
#pragma unroll
    for (unsigned i = 0; i < JA; ++i) {
        const unsigned r = (wave * JA + i) * 8u + lane / 8u;
        va[i] = last_of(r, M - m0) * stride + (lane % 8u ^ r / 2u % 8u) * 16u;
    }
#pragma unroll
    for (unsigned i = 0; i < JB; ++i) {
        const unsigned r = (wave * JB + i) * 8u + lane / 8u;
        vb[i] = last_of(r, N - n0) * stride + (lane % 8u ^ r / 2u % 8u) * 16u;
    }
    // Load `item` of this wave's kItems for stage s.  Past the last stage nothing is in range, and nothing is loaded.
    const auto ask = [&](unsigned s, unsigned at, unsigned item) __attribute__((always_inline)) {
        CDSGD_LDS unsigned char *base = lds + at * kStage;
        if (item < JA + JB) {
            // (the last line of a row may be half a line, behind which the next row begins, or nothing)
            const bool is_a = item < JA;
            const i4s r = buffer_of((is_a ? at_a : at_b) + s * 128u, s < stages ? (is_a ? bytes_a : bytes_b) - s * 128u : 0ull);
            load_to_lds<16>(r, base + (is_a ? (wave * JA + item) * 1024u : kA + (wave * JB + item - JA) * 1024u),
                            is_a ? va[is_a ? item : 0u] : vb[is_a ? 0u : item - JA]);
        } else {
            // scale words of 64 rows: of A's first and second group, then of B's (the last ones twice where they do not go round)
            const unsigned p = last_of(wave + (item - JA - JB) * W, kWords);
            const bool is_b = p >= 2u * BM / 64u;
            const unsigned q = is_b ? p - 2u * BM / 64u : p, per = (is_b ? BN : BM) / 64u, g = q / per, part = q % per;
            const unsigned rows = is_b ? N : M, r0 = is_b ? n0 : m0;
            const bool real = 2u * s + g < groups;
            const i4s r = buffer_of((is_b ? bs : as) + ((size_t)(real ? 2u * s + g : 0u) * rows + r0) * 4u, real ? (unsigned long long)(rows - r0) * 4u : 0ull);
            load_to_lds<4>(r, base + (is_b ? kSB : kSA) + (g * (is_b ? BN : BM) + part * 64u) * 4u, lane * 4u + part * 256u);
        }
    };

    const unsigned wm = wave / WN * TM, wn = wave % WN * TN, hi = lane / 32u, l32 = lane % 32u;
    // The first operand of an instruction is B's, so that a lane's results are neighbours in a row of the output.
    f16v acc[FN][FM];
#pragma unroll
    for (unsigned i = 0; i < FN; ++i)
#pragma unroll
        for (unsigned j = 0; j < FM; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;
    struct Operands {
        i4v a[FM], b[FN];
    };
    struct Scales {
        int a[FM], b[FN];
    };
    const auto read = [&](unsigned at, unsigned h, Operands &x) __attribute__((always_inline)) {
        const CDSGD_LDS unsigned char *base = lds + at * kStage + l32 * 128u + ((2u * h + hi) ^ (l32 / 2u % 8u)) * 16u;
#pragma unroll
        for (unsigned j = 0; j < FM; ++j) x.a[j] = *(const CDSGD_LDS i4v *)(base + wm * 128u + j * 4096u);
#pragma unroll
        for (unsigned i = 0; i < FN; ++i) x.b[i] = *(const CDSGD_LDS i4v *)(base + kA + wn * 128u + i * 4096u);
    };
    const auto read_scales = [&](unsigned at, unsigned g, Scales &s) __attribute__((always_inline)) {
        const CDSGD_LDS unsigned char *base = lds + at * kStage + l32 * 4u;
#pragma unroll
        for (unsigned j = 0; j < FM; ++j) s.a[j] = *(const CDSGD_LDS int *)(base + kSA + (g * BM + wm + j * 32u) * 4u);
#pragma unroll
        for (unsigned i = 0; i < FN; ++i) s.b[i] = *(const CDSGD_LDS int *)(base + kSB + (g * BN + wn + i * 32u) * 4u);
    };
    // of a word's four bytes, the lanes of the upper half take the second and the fourth
    const auto turn = [&](Scales &s) __attribute__((always_inline)) {
#pragma unroll
        for (unsigned j = 0; j < FM; ++j) s.a[j] >>= hi * 8u;
#pragma unroll
        for (unsigned i = 0; i < FN; ++i) s.b[i] >>= hi * 8u;
    };
    const auto product = [&](unsigned i, unsigned j, const Operands &x, const Scales &s, bool odd) __attribute__((always_inline)) {
        acc[i][j] = odd ? mfma32<2>(x.b[i], x.a[j], acc[i][j], s.b[i], s.a[j]) : mfma32<0>(x.b[i], x.a[j], acc[i][j], s.b[i], s.a[j]);
    };

#pragma unroll
    for (unsigned t = 0; t < D - 1; ++t)
#pragma unroll
        for (unsigned i = 0; i < kItems; ++i) ask(t, t, i);
    if constexpr (BM == BN && BM > 64) {
        constexpr unsigned kAtOnce = BM == 256 ? 256 : 512, kSpread = BM == 256 ? 24 * sizeof(Elem<DT>) : 32;
        if (gridDim.x > kAtOnce && blockIdx.x < kAtOnce)
            for (unsigned i = blockIdx.x / 8u * kSpread / (kAtOnce / 8u); i > 0; --i) __builtin_amdgcn_s_sleep(4);
    }
    wait_for_loads<(D - 2) * kItems>();
    __syncthreads();
    unsigned at = 0, to = D - 1;
    const unsigned full = groups / 2u;
    if constexpr (FM * FN > 1) {
        constexpr unsigned kPart = (kItems + 2) / 3, kEvery = FM * FN / kPart;
        static_assert(kEvery >= 1, "every load finds a product to follow");
        Operands x[2];
        Scales s[2];
        // the products of a step, and among them a third of the loads for stage `later`
        const auto multiply = [&](unsigned h, unsigned part, unsigned later) __attribute__((always_inline)) {
            unsigned item = part * kPart;
#pragma unroll
            for (unsigned i = 0; i < FN; ++i)
#pragma unroll
                for (unsigned j = 0; j < FM; ++j) {
                    product(i, j, x[h % 2], s[h / 2], h % 2);
                    if ((i * FM + j) % kEvery == kEvery - 1u && item < (part + 1) * kPart && item < kItems) {
                        __builtin_amdgcn_sched_barrier(0);
                        ask(later, to, item);
                        __builtin_amdgcn_sched_barrier(0);
                        ++item;
                    }
                }
        };
#pragma unroll
        for (unsigned i = 0; i < kPart; ++i) ask(D - 1, to, i);
        read_scales(0, 0, s[0]);
        read(0, 0, x[0]);
        for (unsigned t = 0; t < full; ++t) {
#pragma unroll
            for (unsigned h = 0; h < 3; ++h) {
                if (h % 2 == 0) turn(s[h / 2]);
                if (h == 1) read_scales(at, 1, s[1]);
                read(at, h + 1, x[(h + 1) % 2]);
                __builtin_amdgcn_sched_barrier(0);
                multiply(h, h + 1, t + D - 1);  // (h = 2: none is left)
                __builtin_amdgcn_sched_barrier(0);
            }
            wait_for_loads<(D - 2) * kItems>();
            __syncthreads();
            to = at;
            at = at + 1 < D ? at + 1 : 0;
            read_scales(at, 0, s[0]);
            read(at, 0, x[0]);
            __builtin_amdgcn_sched_barrier(0);
            multiply(3, 0, t + D);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (groups % 2u) {
            turn(s[0]);
            read(at, 1, x[1]);
            multiply(0, 3, 0);
            multiply(1, 3, 0);
        }
    } else {
        // One product a step: shorter than a read of LDS takes.  All four steps of the next stage are read at once.
        Operands x[2][4];
        Scales s[2][2];
        const auto read_stage = [&](unsigned which) __attribute__((always_inline)) {
            read_scales(at, 0, s[which][0]);
            read_scales(at, 1, s[which][1]);
#pragma unroll
            for (unsigned h = 0; h < 4; ++h) read(at, h, x[which][h]);
        };
        const auto stage = [&](unsigned t, unsigned which) __attribute__((always_inline)) {
            wait_for_loads<(D - 3) * kItems>();
            __syncthreads();
            // (the buffer of the stage before last)
            at = at + 1 < D ? at + 1 : 0;
            read_stage(which ^ 1u);
            __builtin_amdgcn_sched_barrier(0);
            turn(s[which][0]);
            turn(s[which][1]);
#pragma unroll
            for (unsigned h = 0; h < 4; ++h) {
                product(0, 0, x[which][h], s[which][h / 2], h % 2);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (unsigned i = h * ((kItems + 3) / 4); i < (h + 1) * ((kItems + 3) / 4) && i < kItems; ++i) ask(t + D - 1, to, i);
                __builtin_amdgcn_sched_barrier(0);
            }
            to = to + 1 < D ? to + 1 : 0;
        };
        read_stage(0);
        unsigned t = 0;
        for (; t + 2 <= full; t += 2) {
            stage(t, 0);
            stage(t + 1, 1);
        }
        if (t < full) {
            stage(t, 0);
#pragma unroll
            for (unsigned h = 0; h < 2; ++h) x[0][h] = x[1][h];
            s[0][0] = s[1][0];
        }
        if (groups % 2u) {
            turn(s[0][0]);
#pragma unroll
            for (unsigned h = 0; h < 2; ++h) product(0, 0, x[0][h], s[0][0], h);
        }
    }
    wait_for_loads<0>();
    __syncthreads();

    // In the result's type through LDS, 32 rows of a wave at a time, so that rows are stored in pieces of 16 bytes to a lane: past
    // the caches, which hold the operands (4096 x 25088 x 2048 in fp32: 204 us at the default policy, 185 so, 144 with what else is
    // here).  What is added to is read as the products lie, so that the sum is rounded once, from fp32; the loads of 32 rows are all
    // under way before the first is used (8192 x 4096 x 4096 added to one bf16 result call after call: 87 us, to three in turn 96;
    // one load and one store after the other, 106).
    typedef Elem<DT> e4 __attribute__((ext_vector_type(4)));
    constexpr unsigned E = 16 / sizeof(Elem<DT>), kPerRow = TN / E, kAtOnce = 64 / kPerRow;
    CDSGD_LDS unsigned char *mine = lds + wave * (32u * kPitch);
#pragma unroll
    for (unsigned j = 0; j < FM; ++j) {
        if (add) {
            f4 old[FN][4];
#pragma unroll
            for (unsigned i = 0; i < FN; ++i)
#pragma unroll
                for (unsigned q = 0; q < 4; ++q) old[i][q] = get4<DT>(out, ld, M, N, m0 + wm + j * 32u + l32, n0 + wn + i * 32u + q * 8u + hi * 4u);
#pragma unroll
            for (unsigned i = 0; i < FN; ++i)
#pragma unroll
                for (unsigned q = 0; q < 4; ++q)
#pragma unroll
                    for (unsigned e = 0; e < 4; ++e) acc[i][j][4 * q + e] += old[i][q][e];
        }
#pragma unroll
        for (unsigned i = 0; i < FN; ++i)
#pragma unroll
            for (unsigned q = 0; q < 4; ++q)
                *(CDSGD_LDS e4 *)(mine + l32 * kPitch + (i * 32u + q * 8u + hi * 4u) * sizeof(Elem<DT>)) =
                    e4{(Elem<DT>)acc[i][j][4 * q], (Elem<DT>)acc[i][j][4 * q + 1], (Elem<DT>)acc[i][j][4 * q + 2], (Elem<DT>)acc[i][j][4 * q + 3]};
        wave_sync();
#pragma unroll
        for (unsigned r = 0; r < 32; r += kAtOnce) {
            const unsigned row = r + lane / kPerRow, col = lane % kPerRow * E;
            const u4 v = *(const CDSGD_LDS u4 *)(mine + row * kPitch + col * sizeof(Elem<DT>));
            const unsigned m = m0 + wm + j * 32u + row, n = n0 + wn + col;
            Elem<DT> *p = out + (size_t)m * ld + n;
            if (m < M && n + E <= N) {
                __builtin_nontemporal_store(v, reinterpret_cast<typename std::conditional<sizeof(Elem<DT>) == 4, u4_by4, u4_by2>::type *>(p));
            } else if (m < M) {
                struct Vec {
                    Elem<DT> v[E];
                };
                const Vec e = __builtin_bit_cast(Vec, v);
#pragma unroll
                for (unsigned k = 0; k < E; ++k)
                    if (n + k < N) p[k] = e.v[k];
            }
        }
        wave_sync();
    }
}

}  // namespace
