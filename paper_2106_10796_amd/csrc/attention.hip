// Attention over packed sequences (include/cdsgd_block.h): the C ABI's host side.  The kernels are in kernels_attention.hpp.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cdsgd_block.h"

#include "host_common.hpp"
#include "tuning.hpp"
#include "device_common.hpp"
#include "host_matrix.hpp"
#include "mxfp4_choice.hpp"

#include "kernels_attention.hpp"

namespace {

// Groups in a row of tiles: a launch's, for one split.
inline unsigned long long groups_over(size_t tokens, size_t num_seqs, size_t each, size_t tile, size_t kv_heads)
{
    return ((unsigned long long)tokens * each / tile + num_seqs) * kv_heads;
}

// Over how many groups the keys of a row are split: where the rows alone do not fill the card, as many as fill it, none of them with fewer keys
// (of a sequence of ordinary length) than four tiles.  One token of 32 heads over 8, 32768 keys, us, pass and join: 256 groups 23.4 + 5.7,
// 512 24.7 + 8.5, 1024 25.8 + 14.1.
inline unsigned splits_of(const cdsgd_attention &b)
{
    const unsigned long long groups = groups_over(b.tokens_q, b.num_seqs, (size_t)(b.heads / b.kv_heads), kTileRows, (size_t)b.kv_heads);
    if (groups >= 256) return 1;
    const unsigned long long want = (255 + groups) / groups, most = b.tokens_k / b.num_seqs / (4 * kTileKeys);
    static_assert(kMostSplits >= 256, "of 256 groups all may share one row's keys");
    return (unsigned)(want < most ? want : most < 1 ? 1 : most);
}

inline int padded_dim(int dim) { return dim <= 64 ? 64 : 128; }

int check_batch(const cdsgd_attention *a)
{
    if (!a) return CDSGD_ERR_NULL;
    if ((a->dtype != CDSGD_GRAD_BF16 && a->dtype != CDSGD_GRAD_F16) || (a->causal != 0 && a->causal != 1) || (a->starts_k && !a->starts_q) ||
        (!a->starts_q && a->num_seqs != 1) || !(a->scale >= 1e-30 && a->scale <= 1e30))
        return CDSGD_ERR_PARAM;
    if (!good_extent(a->tokens_q) || !good_extent(a->tokens_k) || a->num_seqs < 1 || a->num_seqs >= (size_t)1 << 24 || a->heads < 1 ||
        a->heads > 65535 || a->kv_heads < 1 || a->dim < 8 || a->dim > 128 || a->dim % 8)
        return CDSGD_ERR_SIZE;
    if (a->heads % a->kv_heads) return CDSGD_ERR_PARAM;
    if (!aligned(a->starts_q, 4) || !aligned(a->starts_k, 4)) return CDSGD_ERR_ALIGN;
    const size_t group = (size_t)(a->heads / a->kv_heads);
    if ((groups_over(a->tokens_q, a->num_seqs, group, kTileRows, (size_t)a->kv_heads) * splits_of(*a)) >> 23 ||
        groups_over(a->tokens_k, a->num_seqs, 1, kStreamKeys<64>, (size_t)a->kv_heads) >> 23)
        return CDSGD_ERR_SIZE;
    return CDSGD_OK;
}

// A tensor of a batch: [tokens][heads][dim] with tokens ld elements apart.
struct Tensor {
    const void *p;
    size_t ld;
    bool keys, written;
};

int check_tensors(const cdsgd_attention &a, const Tensor *t, int count, Span *in, int &ins, Span *out, int &outs)
{
    for (int i = 0; i < count; ++i) {
        if (!t[i].p) return CDSGD_ERR_NULL;
        const size_t row = (size_t)(t[i].keys ? a.kv_heads : a.heads) * a.dim;
        if (t[i].ld < row || t[i].ld > (size_t)1 << 20) return CDSGD_ERR_SIZE;
        if (t[i].ld % 8 || !aligned(t[i].p, 16)) return CDSGD_ERR_ALIGN;
        const Span s = matrix_of(t[i].p, t[i].keys ? a.tokens_k : a.tokens_q, row, t[i].ld, a.dtype);
        if (t[i].written) out[outs++] = s;
        else in[ins++] = s;
    }
    return CDSGD_OK;
}

AttentionSizes sizes_of(const cdsgd_attention &a)
{
    return {(unsigned)a.tokens_q, (unsigned)a.tokens_k, (unsigned)a.num_seqs, (unsigned)a.kv_heads, (unsigned)(a.heads / a.kv_heads), (unsigned)a.dim,
            a.starts_q, a.starts_k, a.causal, (float)a.scale};
}

template <int DT>
Heads<const Elem<DT>> read_of(const void *p, size_t ld) { return {static_cast<const Elem<DT> *>(p), (unsigned)ld}; }
template <int DT>
Heads<Elem<DT>> write_of(void *p, size_t ld) { return {static_cast<Elem<DT> *>(p), (unsigned)ld}; }

// Calls f(type, padded dim), as integral constants.
template <typename F>
void with_kernel(const cdsgd_attention &a, F f)
{
    const auto with_dim = [&](auto dt) {
        if (padded_dim(a.dim) == 64) f(dt, std::integral_constant<int, 64>());
        else f(dt, std::integral_constant<int, 128>());
    };
    if (a.dtype == CDSGD_GRAD_BF16) with_dim(std::integral_constant<int, kGradBF16>());
    else with_dim(std::integral_constant<int, kGradF16>());
}

}  // namespace

extern "C" {

size_t cdsgd_attention_workspace(const cdsgd_attention *batch, int backward)
{
    if (check_batch(batch) != CDSGD_OK) return 0;
    const size_t rows = batch->tokens_q * (size_t)batch->heads;
    if (backward) return (rows * 3 * sizeof(float) + 15u) & ~(size_t)15u;
    const unsigned splits = splits_of(*batch);
    return splits > 1 ? (splits * rows * (size_t)(padded_dim(batch->dim) + 1) * sizeof(float) + 15u) & ~(size_t)15u : 0;
}

int cdsgd_attention_forward(const cdsgd_attention *batch, const void *q, size_t ld_q, const void *k, size_t ld_k, const void *v, size_t ld_v, void *out,
                            size_t ld_out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_batch(batch);
    if (rc != CDSGD_OK) return rc;
    const cdsgd_attention &a = *batch;
    const Tensor tensors[] = {{q, ld_q, false, false}, {k, ld_k, true, false}, {v, ld_v, true, false}, {out, ld_out, false, true}};
    Span in[5], outs[3];
    int num_in = 0, num_out = 0;
    if ((rc = check_tensors(a, tensors, 4, in, num_in, outs, num_out)) != CDSGD_OK) return rc;
    const size_t want = cdsgd_attention_workspace(batch, 0), rows = a.tokens_q * (size_t)a.heads;
    if (want && !workspace) return CDSGD_ERR_NULL;
    if (workspace_bytes < want) return CDSGD_ERR_SIZE;
    if (!aligned(lse, 4) || !aligned(workspace, 16)) return CDSGD_ERR_ALIGN;
    outs[num_out++] = range_of(lse, rows * sizeof(float));
    outs[num_out++] = range_of(want ? workspace : nullptr, want);
    if (a.starts_q) in[num_in++] = range_of(a.starts_q, (a.num_seqs + 1) * sizeof(int32_t));
    if (a.starts_k) in[num_in++] = range_of(a.starts_k, (a.num_seqs + 1) * sizeof(int32_t));
    if (any_overlap(outs, num_out, in, num_in)) return CDSGD_ERR_ALIAS;
    const AttentionSizes z = sizes_of(a);
    const unsigned splits = splits_of(a);
    const unsigned groups = (unsigned)groups_over(a.tokens_q, a.num_seqs, z.group, kTileRows, z.kv_heads) * splits;
    hipStream_t stream = (hipStream_t)hip_stream;
    with_kernel(a, [&](auto dt, auto dim) {
        constexpr int DT = decltype(dt)::value, DP = decltype(dim)::value;
        float *const parts = splits > 1 ? static_cast<float *>(workspace) : nullptr, *const part_lse = parts ? parts + splits * rows * DP : nullptr;
        hipLaunchKernelGGL((k_attention_forward<DT, DP>), dim3(groups), dim3(256), 0, stream, z, read_of<DT>(q, ld_q), read_of<DT>(k, ld_k),
                           read_of<DT>(v, ld_v), write_of<DT>(out, ld_out), lse, splits, parts, part_lse);
        if (parts)
            hipLaunchKernelGGL((k_attention_join<DT, DP>), dim3((unsigned)rows), dim3(256), 0, stream, z, write_of<DT>(out, ld_out), lse,
                               splits, (const float *)parts, (const float *)part_lse);
    });
    return launch_status();
}

int cdsgd_attention_backward(const cdsgd_attention *batch, const void *dout, size_t ld_dout, const void *q, size_t ld_q, const void *k, size_t ld_k,
                             const void *v, size_t ld_v, const void *out, size_t ld_out, const float *lse, void *dq, size_t ld_dq, void *dk,
                             size_t ld_dk, void *dv, size_t ld_dv, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_batch(batch);
    if (rc != CDSGD_OK) return rc;
    const cdsgd_attention &a = *batch;
    if (!lse || !workspace) return CDSGD_ERR_NULL;
    const Tensor tensors[] = {{dout, ld_dout, false, false}, {q, ld_q, false, false}, {k, ld_k, true, false}, {v, ld_v, true, false},
                              {out, ld_out, false, false},   {dq, ld_dq, false, true}, {dk, ld_dk, true, true}, {dv, ld_dv, true, true}};
    Span in[8], outs[4];
    int num_in = 0, num_out = 0;
    if ((rc = check_tensors(a, tensors, 8, in, num_in, outs, num_out)) != CDSGD_OK) return rc;
    const size_t want = cdsgd_attention_workspace(batch, 1), rows = a.tokens_q * (size_t)a.heads;
    if (workspace_bytes < want) return CDSGD_ERR_SIZE;
    if (!aligned(lse, 4) || !aligned(workspace, 16)) return CDSGD_ERR_ALIGN;
    in[num_in++] = range_of(lse, rows * sizeof(float));
    outs[num_out++] = range_of(workspace, want);
    if (a.starts_q) in[num_in++] = range_of(a.starts_q, (a.num_seqs + 1) * sizeof(int32_t));
    if (a.starts_k) in[num_in++] = range_of(a.starts_k, (a.num_seqs + 1) * sizeof(int32_t));
    if (any_overlap(outs, num_out, in, num_in)) return CDSGD_ERR_ALIAS;
    const AttentionSizes z = sizes_of(a);
    hipStream_t stream = (hipStream_t)hip_stream;
    with_kernel(a, [&](auto dt, auto dim) {
        constexpr int DT = decltype(dt)::value, DP = decltype(dim)::value;
        float *const row_lse = static_cast<float *>(workspace), *const delta = row_lse + rows, *const far = delta + rows;
        hipLaunchKernelGGL((k_attention_dq<DT, DP>), dim3((unsigned)groups_over(a.tokens_q, a.num_seqs, z.group, kTileRows, z.kv_heads)), dim3(256), 0, stream, z,
                           read_of<DT>(dout, ld_dout), read_of<DT>(q, ld_q), read_of<DT>(k, ld_k), read_of<DT>(v, ld_v), read_of<DT>(out, ld_out), lse,
                           write_of<DT>(dq, ld_dq), row_lse, delta, far);
        hipLaunchKernelGGL((k_attention_dkv<DT, DP>), dim3((unsigned)groups_over(a.tokens_k, a.num_seqs, 1, kStreamKeys<DP>, z.kv_heads)), dim3(64 * kKeyWaves<DP> * kStreams<DP>), 0, stream, z,
                           read_of<DT>(dout, ld_dout), read_of<DT>(q, ld_q), read_of<DT>(k, ld_k), read_of<DT>(v, ld_v), (const float *)row_lse,
                           (const float *)delta, (const float *)far, write_of<DT>(dk, ld_dk), write_of<DT>(dv, ld_dv));
    });
    return launch_status();
}

}  // extern "C"
