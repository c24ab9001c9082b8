// C entry points of the softmax-attention layers: argument checks and the shape that the kernels of kda_attn_fwd.hip and
// kda_attn_bwd.hip see.
#include "kda_attn_tile.h"

namespace kda {

kda_status attn_fwd_dispatch(const attn::Shape &, int dim, bool out_bf16, const void *q, const void *k, const void *v, void *o, float *lse,
                             hipStream_t);
size_t attn_bwd_workspace(const attn::Shape &, int dim);
kda_status attn_bwd_dispatch(const attn::Shape &, int dim, const void *q, const void *k, const void *v, const void *o, const float *lse,
                             const void *d_o, void *dq, void *dk, void *dv, void *workspace, hipStream_t);

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A stride of 0 stands for contiguous tokens.  (A tile's rows are addressed by 32-bit byte offsets: 64 strides stay below 2^32.)
kda_status stride_of(int64_t given, int64_t row, const char *name, int64_t &out)
{
    out = given ? given : row;
    if (out < row || out % 8 || out > (1 << 24))
        return fail(KDA_ERR_INVALID_ARG, "%s_stride must be 0 or a multiple of 8 in [%lld, 2^24], got %lld", name, (long long)row, (long long)given);
    return KDA_OK;
}

kda_status check(const kda_attn_dims *d, const int32_t *cu, attn::Shape &s)
{
    if (!d) return fail(KDA_ERR_INVALID_ARG, "dims is NULL");
    if (d->batch < 0 || d->seqlen < 0 || d->num_seqs < 0 || d->heads_q < 0 || d->heads_kv < 0)
        return fail(KDA_ERR_INVALID_ARG, "negative size (batch %d, seqlen %lld, num_seqs %d, heads %d and %d)", d->batch, (long long)d->seqlen,
                    d->num_seqs, d->heads_q, d->heads_kv);
    if (d->in_dtype != KDA_F32 && d->in_dtype != KDA_BF16) return fail(KDA_ERR_INVALID_ARG, "in_dtype %d is not a kda_dtype", (int)d->in_dtype);
    if (d->out_dtype != KDA_F32 && d->out_dtype != KDA_BF16) return fail(KDA_ERR_INVALID_ARG, "out_dtype %d is not a kda_dtype", (int)d->out_dtype);
    if (d->in_dtype != KDA_BF16) return fail(KDA_ERR_UNSUPPORTED, "softmax attention is built for KDA_BF16 inputs");
    if (d->dim != 64 && d->dim != 128) return fail(KDA_ERR_UNSUPPORTED, "dim must be 64 or 128, got %d", d->dim);
    if (d->heads_q > 65535) return fail(KDA_ERR_UNSUPPORTED, "heads_q > 65535");
    if (d->heads_q && (d->heads_kv == 0 || d->heads_q % d->heads_kv))
        return fail(KDA_ERR_INVALID_ARG, "heads_q (%d) must be a multiple of heads_kv (%d)", d->heads_q, d->heads_kv);
    if (d->window < 0) return fail(KDA_ERR_INVALID_ARG, "window < 0");
    if (d->sinks < 0) return fail(KDA_ERR_INVALID_ARG, "sinks < 0");
    if (d->sinks > attn::kTile) return fail(KDA_ERR_UNSUPPORTED, "at most %d sinks, got %d", attn::kTile, d->sinks);
    if (!(d->scale >= 1e-30f && d->scale <= 1e30f)) return fail(KDA_ERR_INVALID_ARG, "scale must be positive, in [1e-30, 1e30]");
    if (cu) {
        if (d->batch != 1) return fail(KDA_ERR_INVALID_ARG, "packed batches need batch == 1");
        if (d->seqlen > 0x7fffffffLL) return fail(KDA_ERR_INVALID_ARG, "packed token count exceeds the int32 range of cu_seqlens");
        if (reinterpret_cast<uintptr_t>(cu) & 3u) return fail(KDA_ERR_INVALID_ARG, "cu_seqlens is misaligned");
    } else if (d->num_seqs != d->batch) {
        return fail(KDA_ERR_INVALID_ARG, "fixed-length batches need num_seqs == batch");
    }
    s = {};
    s.tokens = d->seqlen;
    s.num_seqs = d->num_seqs;
    s.heads_q = d->heads_q;
    s.heads_kv = d->heads_kv;
    s.group = d->heads_q ? d->heads_q / d->heads_kv : 0;
    s.sinks = d->sinks;
    s.scale = d->scale;
    s.cu = cu;
    // a window that no two tokens are apart by is none
    s.window = d->window >= d->seqlen ? 0 : (int32_t)d->window;
    if (s.window == 0) s.sinks = 0;
    if (d->seqlen > 1 << 30) return fail(KDA_ERR_UNSUPPORTED, "more than 2^30 tokens of a row");
    const int64_t tiles = (d->seqlen + attn::kCols - 1) / attn::kCols;
    const int64_t slots = cu ? d->seqlen / attn::kCols + d->num_seqs : tiles * d->batch;
    // (a launch has fewer than 2^32 threads; the dK / dV walk has the sinks' workgroups as well, no more than the others)
    if (slots > 0x7fffff || slots * 2 * (d->heads_q > 0 ? d->heads_q : 1) * attn::kThreads > 0xffffffffLL)
        return fail(KDA_ERR_UNSUPPORTED, "more than 2^23 tiles of %d tokens and heads", attn::kCols);
    s.slots = (int32_t)slots;
    s.tiles = cu ? 0 : (int32_t)tiles;
    kda_status st = stride_of(d->q_stride, (int64_t)d->heads_q * d->dim, "q", s.q_stride);
    if (st == KDA_OK) st = stride_of(d->k_stride, (int64_t)d->heads_kv * d->dim, "k", s.k_stride);
    if (st == KDA_OK) st = stride_of(d->v_stride, (int64_t)d->heads_kv * d->dim, "v", s.v_stride);
    return st;
}
bool nothing(const attn::Shape &s) { return s.slots == 0 || s.heads_q == 0 || s.tokens == 0 || s.num_seqs == 0; }

}  // namespace
}  // namespace kda

using namespace kda;

extern "C" kda_status kda_window_attn_fwd(const kda_attn_dims *dims, const void *q, const void *k, const void *v, const int32_t *cu_seqlens,
                                          void *o, float *lse, void *hip_stream)
{
    attn::Shape s;
    if (const kda_status st = check(dims, cu_seqlens, s); st != KDA_OK) return st;
    if (nothing(s)) return KDA_OK;
    if (!q || !k || !v || !o) return fail(KDA_ERR_INVALID_ARG, "kda_window_attn_fwd: q, k, v or o is NULL");
    for (const void *p : {q, k, v, (const void *)o, (const void *)lse})
        if (!aligned16(p)) return fail(KDA_ERR_INVALID_ARG, "kda_window_attn_fwd: tensors must be 16-byte aligned");
    return attn_fwd_dispatch(s, dims->dim, dims->out_dtype == KDA_BF16, q, k, v, o, lse, static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t kda_window_attn_bwd_workspace_size(const kda_attn_dims *dims)
{
    // (one row may come with cu_seqlens or without: sized for either)
    if (!dims) return 0;
    attn::Shape s;
    const int32_t some = 0;
    size_t most = 0;
    for (const int32_t *cu : {(const int32_t *)nullptr, &some})
        if (check(dims, cu, s) == KDA_OK && !nothing(s)) {
            const size_t n = attn_bwd_workspace(s, dims->dim);
            most = n > most ? n : most;
        }
    return most;
}

extern "C" kda_status kda_window_attn_bwd(const kda_attn_dims *dims, const void *q, const void *k, const void *v, const int32_t *cu_seqlens,
                                          const void *o, const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *workspace,
                                          size_t workspace_bytes, void *hip_stream)
{
    attn::Shape s;
    if (const kda_status st = check(dims, cu_seqlens, s); st != KDA_OK) return st;
    if (dims->out_dtype != KDA_BF16) return fail(KDA_ERR_UNSUPPORTED, "kda_window_attn_bwd takes o and d_o in bf16 (out_dtype KDA_BF16)");
    if (nothing(s)) return KDA_OK;
    if (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv) return fail(KDA_ERR_INVALID_ARG, "kda_window_attn_bwd: a tensor is NULL");
    for (const void *p : {q, k, v, o, (const void *)lse, d_o, (const void *)dq, (const void *)dk, (const void *)dv})
        if (!aligned16(p)) return fail(KDA_ERR_INVALID_ARG, "kda_window_attn_bwd: tensors must be 16-byte aligned");
    const size_t need = kda_window_attn_bwd_workspace_size(dims);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < need)
        return fail(KDA_ERR_WORKSPACE, "kda_window_attn_bwd: workspace must be 256-byte aligned and hold %zu bytes, got %zu", need, workspace_bytes);
    return attn_bwd_dispatch(s, dims->dim, q, k, v, o, lse, d_o, dq, dk, dv, workspace, static_cast<hipStream_t>(hip_stream));
}
