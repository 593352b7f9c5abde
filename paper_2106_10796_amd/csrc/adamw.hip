// Norms of gradients and AdamW over a layer list (include/cdsgd_ops.h): the C ABI's host side.  The kernels are in
// kernels_adamw.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>
#include <utility>
#include <vector>

#include "cdsgd_ops.h"

#include "host_common.hpp"
#include "tuning.hpp"
#include "device_common.hpp"
#include "kernels_adamw.hpp"

namespace {

constexpr int kState32 = 32, kState8 = 8;

inline bool good_dtype(int t) { return t == CDSGD_GRAD_F32 || t == CDSGD_GRAD_BF16 || t == CDSGD_GRAD_F16; }
inline size_t bytes_of(int dtype) { return dtype == CDSGD_GRAD_F32 ? 4u : 2u; }

// A launch of one wave per piece stays below 2^32 threads, and a table below 1 GiB.
constexpr unsigned long long kMaxStepChunks = (1ull << 22) - 1, kMaxNormChunks = 1ull << 24;

inline unsigned norm_elems(int dtype) { return kNormBytes / (unsigned)bytes_of(dtype); }

inline unsigned long long pieces(size_t n, unsigned each) { return (n + each - 1ull) / each; }

// Groups of k_grad_norm.  A group's turn at the counter takes 12 ns, so there are as few as keep the memory busy (us, fp32, 64 / 128
// / 256 / 512 / 1024 groups: 4 M elements 7.7 / 6.3 / 7.0 / 9.5 / 9.5, 8 M 13.2 / 9.1 / 9.2 / 11.9 / 17.2, 26 M 35.6 / 21.3 / 17.8 /
// 20.2 / 23.7, 138 M 183 / 109 / 80 / 83 / 89).
inline unsigned norm_groups(unsigned chunks) { return chunks <= 128 ? chunks : (chunks <= 512 ? 128 : 256); }

// How the caches are used, and LDS that a wave asks for to bound the waves resident (160 KiB / bytes), by the length of the list.
//   up to kShortList     loads keep what they find, stores are written through and stay in the memory-side cache
//   up to kLongList      loads keep, stores are written through and do not stay
//   above                loads do not keep either (states in 32 bits; in 8 bits as before)
// us, bf16 gradients with a copy, three sets of buffers in turn / ten, which no cache holds:
//   32 bits   non-temporal   2 M 10.1 / 10.6   4 M 19.2 / 19.6   8 M 36.0 / 36.4   26 M 109   138 M 594
//             first form     2 M  7.2 / 11.4   4 M 13.6 / 21.4   8 M 39.3 / 39.9   26 M 120   138 M 640
//             second         2 M 10.0 / 10.4   4 M 18.6 / 18.8   8 M 35.0 / 35.1   26 M 105   138 M 615
//             third          2 M     -         4 M 18.1          8 M 36.1          26 M 110   138 M 586
//   8 bits    non-temporal   2 M  7.6 /  8.1   4 M 13.6 / 14.4   8 M 24.2 / 24.5   26 M 69    138 M 364
//             first form     2 M  6.3 /  7.0   4 M 10.4 / 16.1   8 M 18.0 / 27.0   26 M 74    138 M 376
//             second         2 M  7.7 /  8.6   4 M 13.9 / 14.3   8 M 23.2 / 23.3   26 M 63    138 M 360
// Waves resident, second form: 32 bits 26 M, all 112, 20 waves 108, 16 107, 13 105, 10 107;  8 bits 26 M, all 65.0, 22 63.4, 20 64.7,
// 16 66.5;  138 M 393, 375, 360, 365.
constexpr unsigned long long kShortList = 2500000, kMidList = 16ull << 20, kLongList = 64ull << 20;

struct Block {  // device memory of a handle
    void *p = nullptr;
    ~Block()
    {
        if (p) (void)hipFree(p);
    }
    int fill(const void *image, size_t bytes)
    {
        if (hipMalloc(&p, bytes) != hipSuccess) {
            (void)hipGetLastError();
            p = nullptr;
            return CDSGD_ERR_DEVICE;
        }
        if (hipMemcpy(p, image, bytes, hipMemcpyHostToDevice) != hipSuccess) {
            (void)hipGetLastError();
            return CDSGD_ERR_DEVICE;
        }
        return CDSGD_OK;
    }
};

// The buffers of a list, for its check: nothing that is written shares a byte with another buffer.
struct Buffers {
    struct Range {
        uintptr_t from, to;
        bool written;
    };
    std::vector<Range> all;

    void add(const void *p, size_t bytes, bool written)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) all.push_back({at, at + bytes, written});
    }
    bool alias()
    {
        std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return a.from < b.from; });
        uintptr_t end = 0, end_written = 0;  // of what lies before
        for (const Range &r : all) {
            if (r.from < (r.written ? end : end_written)) return true;
            end = std::max(end, r.to);
            if (r.written) end_written = std::max(end_written, r.to);
        }
        return false;
    }
};

// Bytes that a handle's passes read, or write, against an argument of a call.
struct Extents {
    std::vector<std::pair<uintptr_t, uintptr_t>> all;

    void add(const void *p, size_t bytes)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) all.push_back({at, at + bytes});
    }
    void close()  // sorts, and joins what overlaps
    {
        std::sort(all.begin(), all.end());
        size_t n = 0;
        for (const auto &r : all) {
            if (n && r.first <= all[n - 1].second) all[n - 1].second = std::max(all[n - 1].second, r.second);
            else all[n++] = r;
        }
        all.resize(n);
    }
    bool touch(const void *p, size_t bytes) const
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        const auto after = std::lower_bound(all.begin(), all.end(), std::make_pair(at + bytes, (uintptr_t)0));  // begins behind p's bytes
        return p && after != all.begin() && (after - 1)->second > at;
    }
};

inline bool good_rate(double x) { return std::isfinite(x) && std::isfinite((float)x); }

}  // namespace

struct cdsgd_grad_norm {
    Block block;
    Extents read;
    NormChunk *chunks = nullptr;
    double *partial = nullptr;
    unsigned *done = nullptr;
    unsigned num_chunks = 0, groups = 0;
    int grad_dtype = 0;
};

struct cdsgd_adamw_plan {
    std::vector<StepChunk> host_chunks;
    std::vector<size_t> sizes;
    Block block;
    Extents written;  // by a step
    cdsgd_grad_norm norm;
    unsigned long long elements = 0;
    int grad_dtype = 0, state_bits = kState32, readout_dtype = -1;
    bool copies = false;

    const StepChunk *chunks() const { return static_cast<const StepChunk *>(block.p); }
};

namespace {

int norm_create(cdsgd_grad_norm &h, const void *const *grads, const size_t *sizes, int num_tensors, int grad_dtype)
{
    unsigned long long total = 0;
    for (int i = 0; i < num_tensors; ++i) {
        if (!grads[i]) return CDSGD_ERR_NULL;
        if (sizes[i] == 0 || sizes[i] > (size_t)1 << 40) return CDSGD_ERR_SIZE;
        if (!aligned(grads[i], 16)) return CDSGD_ERR_ALIGN;
        total += pieces(sizes[i], norm_elems(grad_dtype));
        if (total > kMaxNormChunks) return CDSGD_ERR_SIZE;
        h.read.add(grads[i], sizes[i] * bytes_of(grad_dtype));
    }
    h.read.close();
    h.grad_dtype = grad_dtype;
    h.num_chunks = (unsigned)total;
    h.groups = norm_groups(h.num_chunks);
    // counter, partial sums, chunks
    const size_t off_p = 256, off_c = off_p + ((sizeof(double) * h.groups + 255) & ~(size_t)255);
    std::vector<unsigned char> image(off_c + sizeof(NormChunk) * (size_t)total, 0);
    NormChunk *c = reinterpret_cast<NormChunk *>(image.data() + off_c);
    for (int i = 0; i < num_tensors; ++i)
        for (size_t at = 0; at < sizes[i]; at += norm_elems(grad_dtype), ++c) {
            c->grad = static_cast<const char *>(grads[i]) + at * bytes_of(grad_dtype);
            c->elems = (unsigned)(sizes[i] - at < norm_elems(grad_dtype) ? sizes[i] - at : norm_elems(grad_dtype));
        }
    const int rc = h.block.fill(image.data(), image.size());
    if (rc != CDSGD_OK) return rc;
    unsigned char *base = static_cast<unsigned char *>(h.block.p);
    h.done = reinterpret_cast<unsigned *>(base);
    h.partial = reinterpret_cast<double *>(base + off_p);
    h.chunks = reinterpret_cast<NormChunk *>(base + off_c);
    return CDSGD_OK;
}

int norm_compute(const cdsgd_grad_norm &h, double grad_scale, double max_norm, float *out, void *hip_stream)
{
    if (!out) return CDSGD_ERR_NULL;
    if (!std::isfinite(grad_scale) || !(max_norm > 0.0)) return CDSGD_ERR_PARAM;
    if (!aligned(out, 4)) return CDSGD_ERR_ALIGN;
    if (h.read.touch(out, 2 * sizeof(float))) return CDSGD_ERR_ALIAS;
    hipStream_t s = (hipStream_t)hip_stream;
    const double scale = std::fabs(grad_scale);
#define CDSGD_LAUNCH_NORM(GT)                                                                                   \
    hipLaunchKernelGGL((k_grad_norm<GT>), dim3(h.groups), dim3(kNormLanes), 0, s, h.chunks, h.num_chunks,      \
                       h.partial, h.done, scale, max_norm, out)
    if (h.grad_dtype == CDSGD_GRAD_BF16) CDSGD_LAUNCH_NORM(kGradBF16);
    else if (h.grad_dtype == CDSGD_GRAD_F16) CDSGD_LAUNCH_NORM(kGradF16);
    else CDSGD_LAUNCH_NORM(kGradF32);
#undef CDSGD_LAUNCH_NORM
    return launch_status();
}

int check_adamw_list(const cdsgd_adamw_tensor *tensors, int num_tensors, int grad_dtype, int state_bits, bool *copies)
{
    if (!tensors) return CDSGD_ERR_NULL;
    if (num_tensors < 1) return CDSGD_ERR_SIZE;
    if (!good_dtype(grad_dtype) || (state_bits != kState32 && state_bits != kState8)) return CDSGD_ERR_PARAM;
    unsigned long long total = 0;
    Buffers buffers;
    *copies = tensors[0].weight16 != nullptr;
    for (int i = 0; i < num_tensors; ++i) {
        const cdsgd_adamw_tensor &t = tensors[i];
        if (!t.weight || !t.grad || !t.m || !t.v) return CDSGD_ERR_NULL;
        if (state_bits == kState8 && (!t.m_scale || !t.v_scale)) return CDSGD_ERR_NULL;
        if (state_bits == kState32 && (t.m_scale || t.v_scale)) return CDSGD_ERR_PARAM;
        if (t.n == 0 || t.n > (size_t)1 << 40) return CDSGD_ERR_SIZE;
        total += pieces(t.n, kStepChunk);
        if (total > kMaxStepChunks) return CDSGD_ERR_SIZE;
        if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.0f) return CDSGD_ERR_PARAM;
        // copies for all tensors or for none, and none that would be no narrower than the weights
        if ((t.weight16 != nullptr) != *copies || (t.weight16 && grad_dtype == CDSGD_GRAD_F32)) return CDSGD_ERR_PARAM;
        if (!aligned(t.weight, 16) || !aligned(t.weight16, 16) || !aligned(t.grad, 16) || !aligned(t.m, 16) || !aligned(t.v, 16))
            return CDSGD_ERR_ALIGN;
        for (void *p : {t.m, t.v}) buffers.add(p, state_bits / 8 * t.n, true);
        for (void *p : {t.m_scale, t.v_scale}) buffers.add(p, cdsgd_state_blocks(t.n), true);
        buffers.add(t.weight, t.n * 4, true);
        buffers.add(t.weight16, t.n * 2, true);
        buffers.add(t.grad, t.n * bytes_of(grad_dtype), false);
    }
    if (buffers.alias()) return CDSGD_ERR_ALIAS;
    return CDSGD_OK;
}

template <typename T>
T *moved(T *p, size_t bytes)
{
    return p ? reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(p) + bytes) : nullptr;
}

}  // namespace

extern "C" {

size_t cdsgd_state_blocks(size_t n) { return (n + CDSGD_STATE_BLOCK - 1) / CDSGD_STATE_BLOCK; }

int cdsgd_grad_norm_create(const void *const *grads, const size_t *sizes, int num_tensors, int grad_dtype, cdsgd_grad_norm **out)
try {
    if (!out) return CDSGD_ERR_NULL;
    *out = nullptr;
    if (!grads || !sizes) return CDSGD_ERR_NULL;
    if (num_tensors < 1) return CDSGD_ERR_SIZE;
    if (!good_dtype(grad_dtype)) return CDSGD_ERR_PARAM;
    std::unique_ptr<cdsgd_grad_norm> h(new cdsgd_grad_norm);
    const int rc = norm_create(*h, grads, sizes, num_tensors, grad_dtype);
    if (rc != CDSGD_OK) return rc;
    *out = h.release();
    return CDSGD_OK;
} catch (...) {
    return CDSGD_ERR_DEVICE;
}

int cdsgd_grad_norm_compute(cdsgd_grad_norm *norm, double grad_scale, double max_norm, float *out, void *hip_stream)
{
    return norm ? norm_compute(*norm, grad_scale, max_norm, out, hip_stream) : CDSGD_ERR_NULL;
}

int cdsgd_grad_norm_destroy(cdsgd_grad_norm *norm)
{
    delete norm;
    return CDSGD_OK;
}

int cdsgd_adamw_plan_create(const cdsgd_adamw_tensor *tensors, int num_tensors, int grad_dtype, int state_bits, cdsgd_adamw_plan **out)
try {
    if (!out) return CDSGD_ERR_NULL;
    *out = nullptr;
    bool copies = false;
    int rc = check_adamw_list(tensors, num_tensors, grad_dtype, state_bits, &copies);
    if (rc != CDSGD_OK) return rc;
    std::unique_ptr<cdsgd_adamw_plan> plan(new cdsgd_adamw_plan);
    plan->grad_dtype = grad_dtype;
    plan->state_bits = state_bits;
    plan->copies = copies;
    const size_t gb = bytes_of(grad_dtype), sb = (size_t)state_bits / 8;
    std::vector<const void *> grads;
    unsigned counter = 0;
    for (int i = 0; i < num_tensors; ++i) {
        const cdsgd_adamw_tensor &t = tensors[i];
        grads.push_back(t.grad);
        plan->sizes.push_back(t.n);
        plan->elements += t.n;
        plan->written.add(t.weight, t.n * 4);
        plan->written.add(t.weight16, t.n * 2);
        for (void *p : {t.m, t.v}) plan->written.add(p, t.n * sb);
        for (void *p : {t.m_scale, t.v_scale}) plan->written.add(p, cdsgd_state_blocks(t.n));
        for (size_t at = 0; at < t.n; at += kStepChunk) {
            StepChunk c{};
            c.weight = t.weight + at;
            c.grad = moved(t.grad, at * gb);
            c.m = moved(t.m, at * sb);
            c.v = moved(t.v, at * sb);
            c.m_scale = moved(t.m_scale, at / CDSGD_STATE_BLOCK);
            c.v_scale = moved(t.v_scale, at / CDSGD_STATE_BLOCK);
            c.weight16 = moved(t.weight16, at * 2);
            c.elems = (unsigned)(t.n - at < kStepChunk ? t.n - at : kStepChunk);
            c.counter = counter + (unsigned)at;
            c.weight_decay = t.weight_decay;
            plan->host_chunks.push_back(c);
        }
        counter += (unsigned)(cdsgd_state_blocks(t.n) * CDSGD_STATE_BLOCK);
    }
    plan->written.close();
    rc = plan->block.fill(plan->host_chunks.data(), sizeof(StepChunk) * plan->host_chunks.size());
    if (rc == CDSGD_OK) rc = norm_create(plan->norm, grads.data(), plan->sizes.data(), num_tensors, grad_dtype);
    if (rc != CDSGD_OK) return rc;
    *out = plan.release();
    return CDSGD_OK;
} catch (...) {
    return CDSGD_ERR_DEVICE;
}

int cdsgd_adamw_plan_destroy(cdsgd_adamw_plan *plan)
{
    delete plan;
    return CDSGD_OK;
}

int cdsgd_adamw_step(cdsgd_adamw_plan *plan, long step, double lr, double beta1, double beta2, double eps, double grad_scale,
                     uint64_t seed, const float *clip, void *hip_stream)
{
    if (!plan) return CDSGD_ERR_NULL;
    if (step < 1 || !good_rate(lr) || lr < 0.0 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
        !good_rate(eps) || eps < 1e-37 || !good_rate(grad_scale))
        return CDSGD_ERR_PARAM;
    if (!aligned(clip, 4)) return CDSGD_ERR_ALIGN;
    if (plan->written.touch(clip, 2 * sizeof(float))) return CDSGD_ERR_ALIAS;
    StepFactors f;
    f.lr = lr;
    f.beta1 = (float)beta1;
    f.one_minus_beta1 = (float)(1.0 - beta1);
    f.beta2 = (float)beta2;
    f.one_minus_beta2 = (float)(1.0 - beta2);
    f.inv_sqrt_bias2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    f.eps = (float)eps;
    f.lr_over_bias1 = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    f.grad_scale = (float)grad_scale;
    uint64_t z = seed + 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 32)) * 0xD6E8FEB86659FD93ull;
    f.seed = (unsigned)(z ^ (z >> 32));
    hipStream_t s = (hipStream_t)hip_stream;
    const unsigned per = kStepChunk / (plan->state_bits == kState32 ? kStepLanes * 4u : kStep8Elems);
    const dim3 grid((unsigned)plan->host_chunks.size() * per), block(kStepLanes);
    const unsigned long long n = plan->elements;
#define CDSGD_LAUNCH_ADAMW(KERNEL, GT, COPY, LOAD, STORE, LDS) \
    hipLaunchKernelGGL((KERNEL<GT, COPY, LOAD, STORE>), grid, block, LDS, s, plan->chunks(), per, clip, f)
#define CDSGD_LAUNCH_ADAMW_T(KERNEL, LOAD, STORE, LDS)                                                                              \
    do {                                                                                                                            \
        if (plan->grad_dtype == CDSGD_GRAD_BF16 && plan->copies) CDSGD_LAUNCH_ADAMW(KERNEL, kGradBF16, true, LOAD, STORE, LDS);     \
        else if (plan->grad_dtype == CDSGD_GRAD_BF16) CDSGD_LAUNCH_ADAMW(KERNEL, kGradBF16, false, LOAD, STORE, LDS);               \
        else if (plan->grad_dtype == CDSGD_GRAD_F16 && plan->copies) CDSGD_LAUNCH_ADAMW(KERNEL, kGradF16, true, LOAD, STORE, LDS);  \
        else if (plan->grad_dtype == CDSGD_GRAD_F16) CDSGD_LAUNCH_ADAMW(KERNEL, kGradF16, false, LOAD, STORE, LDS);                 \
        else CDSGD_LAUNCH_ADAMW(KERNEL, kGradF32, false, LOAD, STORE, LDS);                                                         \
    } while (0)
    if (plan->state_bits == kState32) {
        if (n <= kShortList) CDSGD_LAUNCH_ADAMW_T(k_adamw32, 0, kThrough, 0);
        else if (n <= kLongList) CDSGD_LAUNCH_ADAMW_T(k_adamw32, 0, kThroughStream, n <= kMidList ? 10240 : 12288);
        else CDSGD_LAUNCH_ADAMW_T(k_adamw32, kStream, kThroughStream, 12288);
    } else {
        if (n <= kShortList) CDSGD_LAUNCH_ADAMW_T(k_adamw8, 0, kThrough, 0);
        else CDSGD_LAUNCH_ADAMW_T(k_adamw8, 0, kThroughStream, n <= kLongList ? 7168 : 8192);
    }
#undef CDSGD_LAUNCH_ADAMW_T
#undef CDSGD_LAUNCH_ADAMW
    return launch_status();
}

int cdsgd_adamw_grad_norm(cdsgd_adamw_plan *plan, double grad_scale, double max_norm, float *out, void *hip_stream)
{
    return plan ? norm_compute(plan->norm, grad_scale, max_norm, out, hip_stream) : CDSGD_ERR_NULL;
}

int cdsgd_adamw_bind_readout(cdsgd_adamw_plan *plan, void *const *m_out, void *const *v_out, int dtype)
try {
    if (!plan || !m_out || !v_out) return CDSGD_ERR_NULL;
    if (plan->state_bits != kState8 || (dtype != CDSGD_GRAD_F32 && dtype != CDSGD_GRAD_BF16)) return CDSGD_ERR_PARAM;
    const size_t ob = bytes_of(dtype);
    Buffers buffers;
    size_t c = 0;
    for (size_t i = 0; i < plan->sizes.size(); ++i) {
        const size_t n = plan->sizes[i];
        if (!m_out[i] || !v_out[i]) return CDSGD_ERR_NULL;
        if (!aligned(m_out[i], 16) || !aligned(v_out[i], 16)) return CDSGD_ERR_ALIGN;
        for (void *p : {m_out[i], v_out[i]}) buffers.add(p, n * ob, true);
        const StepChunk &t = plan->host_chunks[c];
        for (const void *p : {t.m, t.v}) buffers.add(p, n, false);
        for (const void *p : {t.m_scale, t.v_scale}) buffers.add(p, cdsgd_state_blocks(n), false);
        buffers.add(t.weight, n * 4, false);
        buffers.add(t.weight16, n * 2, false);
        buffers.add(t.grad, n * bytes_of(plan->grad_dtype), false);
        c += pieces(n, kStepChunk);
    }
    if (buffers.alias()) return CDSGD_ERR_ALIAS;
    c = 0;
    for (size_t i = 0; i < plan->sizes.size(); ++i)
        for (size_t at = 0; at < plan->sizes[i]; at += kStepChunk, ++c) {
            plan->host_chunks[c].m_out = moved(m_out[i], at * ob);
            plan->host_chunks[c].v_out = moved(v_out[i], at * ob);
        }
    plan->readout_dtype = -1;
    if (hipMemcpy(plan->block.p, plan->host_chunks.data(), sizeof(StepChunk) * plan->host_chunks.size(), hipMemcpyHostToDevice) !=
        hipSuccess) {
        (void)hipGetLastError();
        return CDSGD_ERR_DEVICE;
    }
    plan->readout_dtype = dtype;
    return CDSGD_OK;
} catch (...) {
    return CDSGD_ERR_DEVICE;
}

int cdsgd_adamw_read_states(cdsgd_adamw_plan *plan, void *hip_stream)
{
    if (!plan) return CDSGD_ERR_NULL;
    if (plan->state_bits != kState8) return CDSGD_ERR_PARAM;
    if (plan->readout_dtype < 0) return CDSGD_ERR_NULL;
    hipStream_t s = (hipStream_t)hip_stream;
    const unsigned per = kStepChunk / kStep8Elems;
    const dim3 grid((unsigned)plan->host_chunks.size() * per), block(kStepLanes);
    // us, bf16, three sets in turn: codes kept / not, 2 M 3.0 / 3.4, 8 M 7.6 / 10.4, 26 M 19.7 / 26.9, 138 M 142 / 134
    const bool keeps = plan->elements <= kLongList;
#define CDSGD_LAUNCH_READOUT(OT, LOAD) hipLaunchKernelGGL((k_read_states<OT, LOAD, kStream>), grid, block, 0, s, plan->chunks(), per)
    if (plan->readout_dtype == CDSGD_GRAD_F32 && keeps) CDSGD_LAUNCH_READOUT(kGradF32, 0);
    else if (plan->readout_dtype == CDSGD_GRAD_F32) CDSGD_LAUNCH_READOUT(kGradF32, kStream);
    else if (keeps) CDSGD_LAUNCH_READOUT(kGradBF16, 0);
    else CDSGD_LAUNCH_READOUT(kGradBF16, kStream);
#undef CDSGD_LAUNCH_READOUT
    return launch_status();
}

}  // extern "C"
