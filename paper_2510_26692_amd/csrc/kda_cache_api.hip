// C entry points of the paged 8-bit cache: argument checks and what the kernels of kda_cache_append.hip and kda_cache_attn.hip see.
#include "kda_cache.h"

namespace kda {

kda_status cache_append_dispatch(const cache::Cache &, const cache::Append &, int dim, hipStream_t);
kda_status cache_attn_dispatch(const cache::Cache &, const cache::Attend &, int dim, hipStream_t);
int32_t cache_attn_splits(const cache::Cache &, int64_t pairs, int64_t most_keys, int64_t window, int32_t sinks, int32_t tokens);

namespace {

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

kda_status stride_of(int64_t given, int64_t row, const char *name, int64_t &out)
{
    out = given ? given : row;
    if (out < row || out % 8 || out > (1 << 24))
        return fail(KDA_ERR_INVALID_ARG, "%s_stride must be 0 or a multiple of 8 in [%lld, 2^24], got %lld", name, (long long)row, (long long)given);
    return KDA_OK;
}

// Sizes alone where `buffers` is false.
kda_status check(const kda_cache *d, bool buffers, cache::Cache &c)
{
    if (!d) return fail(KDA_ERR_INVALID_ARG, "cache is NULL");
    if (d->num_seqs < 0 || d->heads_q < 0 || d->heads_kv < 0 || d->num_pages < 0 || d->max_pages < 0)
        return fail(KDA_ERR_INVALID_ARG, "negative size (num_seqs %d, heads %d and %d, num_pages %lld, max_pages %d)", d->num_seqs, d->heads_q,
                    d->heads_kv, (long long)d->num_pages, d->max_pages);
    if (d->dim != 64 && d->dim != 128) return fail(KDA_ERR_UNSUPPORTED, "dim must be 64 or 128, got %d", d->dim);
    if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128)
        return fail(KDA_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128, got %d", d->page_size);
    if (d->heads_q > 65535) return fail(KDA_ERR_UNSUPPORTED, "heads_q > 65535");
    if (d->heads_q && (d->heads_kv == 0 || d->heads_q % d->heads_kv))
        return fail(KDA_ERR_INVALID_ARG, "heads_q (%d) must be a multiple of heads_kv (%d)", d->heads_q, d->heads_kv);
    if ((int64_t)d->max_pages * d->page_size > 1 << 30) return fail(KDA_ERR_UNSUPPORTED, "more than 2^30 tokens a sequence (max_pages %d)", d->max_pages);
    if (d->num_pages > 0x7fffffffLL) return fail(KDA_ERR_INVALID_ARG, "num_pages exceeds the int32 range of block_table");
    c = {};
    c.num_pages = d->num_pages;
    c.num_seqs = d->num_seqs;
    c.heads_q = d->heads_q;
    c.heads_kv = d->heads_kv;
    c.group = d->heads_q ? d->heads_q / d->heads_kv : 0;
    c.page_size = d->page_size;
    c.page_log2 = d->page_size == 16 ? 4 : d->page_size == 32 ? 5 : d->page_size == 64 ? 6 : 7;
    c.max_pages = d->max_pages;
    if (!buffers || d->num_seqs == 0 || d->heads_q == 0) return KDA_OK;
    const bool pages = d->num_pages > 0;
    if (!d->kv_lens || (d->max_pages && !d->block_table) || (pages && (!d->k || !d->v || !d->k_scale || !d->v_scale)))
        return fail(KDA_ERR_INVALID_ARG, "a buffer of the cache is NULL");
    if (!aligned(d->k, 16) || !aligned(d->v, 16) || !aligned(d->k_scale, 4) || !aligned(d->v_scale, 4) || !aligned(d->block_table, 4) || !aligned(d->kv_lens, 4))
        return fail(KDA_ERR_INVALID_ARG, "a buffer of the cache is misaligned");
    c.k = static_cast<uint8_t *>(d->k);
    c.v = static_cast<uint8_t *>(d->v);
    c.k_scale = d->k_scale;
    c.v_scale = d->v_scale;
    c.table = d->block_table;
    c.lens = d->kv_lens;
    // (no pages or no columns: every entry is none, and the table is not read)
    if (!pages) c.max_pages = 0;
    return KDA_OK;
}

kda_status check(const kda_cache *d, bool buffers, const kda_cache_query *q, cache::Cache &c, cache::Attend &a)
{
    if (const kda_status st = check(d, buffers, c); st != KDA_OK) return st;
    if (!q) return fail(KDA_ERR_INVALID_ARG, "query is NULL");
    if (q->tokens < 0 || q->window < 0 || q->sinks < 0 || q->max_kv_len < 0)
        return fail(KDA_ERR_INVALID_ARG, "negative size (tokens %d, window %lld, sinks %d, max_kv_len %lld)", q->tokens, (long long)q->window, q->sinks,
                    (long long)q->max_kv_len);
    if (q->tokens > 8) return fail(KDA_ERR_UNSUPPORTED, "at most 8 new tokens a sequence, got %d", q->tokens);
    if (q->sinks > 64) return fail(KDA_ERR_UNSUPPORTED, "at most 64 sinks, got %d", q->sinks);
    if (!(q->scale >= 1e-30f && q->scale <= 1e30f)) return fail(KDA_ERR_INVALID_ARG, "scale must be positive, in [1e-30, 1e30]");
    if (q->out_dtype != KDA_F32 && q->out_dtype != KDA_BF16) return fail(KDA_ERR_INVALID_ARG, "out_dtype %d is not a kda_dtype", (int)q->out_dtype);
    a = {};
    // a window that no two tokens are apart by is none
    a.window = q->window > 0x7fffffffLL ? 0 : (int32_t)q->window;
    a.sinks = a.window ? q->sinks : 0;
    a.scale = q->scale;
    a.tokens = q->tokens;
    a.out_bf16 = q->out_dtype == KDA_BF16;
    if (const kda_status st = stride_of(q->q_stride, (int64_t)d->heads_q * d->dim, "q", a.q_stride); st != KDA_OK) return st;
    a.rows = q->tokens * c.group;
    a.row_tiles = (a.rows + 31) / 32;
    const int64_t pairs = (int64_t)c.num_seqs * c.heads_kv, held = (int64_t)d->max_pages * d->page_size;
    const int64_t most = q->max_kv_len && q->max_kv_len < held ? q->max_kv_len : held;
    a.splits = pairs && a.rows ? cache_attn_splits(c, pairs * a.row_tiles, most, a.window, a.sinks, a.tokens) : 1;
    // (a launch has fewer than 2^32 threads: 256 a workgroup, and 64 a row of the join)
    if (pairs * a.row_tiles * a.splits > 0xffffff || pairs * a.rows > 0x3ffffff) return fail(KDA_ERR_UNSUPPORTED, "more than 2^24 workgroups");
    return KDA_OK;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t stats_offset(const cache::Cache &c, const cache::Attend &a, int dim)
{
    return up256((size_t)c.num_seqs * c.heads_kv * a.splits * a.rows * dim * 4);
}

}  // namespace
}  // namespace kda

using namespace kda;

extern "C" kda_status kda_cache_append(const kda_cache *cache, int64_t seqlen, const void *k, const void *v, int64_t k_stride, int64_t v_stride,
                                       const int32_t *cu_seqlens, const kda_rope *rope, void *k_out, const void *q, int64_t q_stride, void *q_out,
                                       uint32_t flags, void *hip_stream)
{
    cache::Cache c;
    if (const kda_status st = check(cache, true, c); st != KDA_OK) return st;
    if (seqlen < 0) return fail(KDA_ERR_INVALID_ARG, "seqlen < 0");
    cache::Append a = {};
    const int64_t row = (int64_t)cache->heads_kv * cache->dim;
    if (rope) {
        if (rope->num_freqs < 0 || 2 * (int64_t)rope->num_freqs > cache->dim || rope->num_freqs % 8)
            return fail(KDA_ERR_INVALID_ARG, "num_freqs must be a multiple of 8 up to dim / 2, got %d", rope->num_freqs);
        if (rope->num_freqs && (!rope->inv_freq || !aligned(rope->inv_freq, 4))) return fail(KDA_ERR_INVALID_ARG, "inv_freq is NULL or misaligned");
        a.inv_freq = rope->inv_freq;
        a.n_freq = rope->num_freqs;
        a.interleaved = rope->interleaved != 0;
    }
    if (kda_status st = stride_of(k_stride, row, "k", a.k_stride); st != KDA_OK) return st;
    if (kda_status st = stride_of(v_stride, row, "v", a.v_stride); st != KDA_OK) return st;
    if (kda_status st = stride_of(q_stride, (int64_t)cache->heads_q * cache->dim, "q", a.q_stride); st != KDA_OK) return st;
    if ((q == nullptr) != (q_out == nullptr)) return fail(KDA_ERR_INVALID_ARG, "q and q_out come together");
    if (flags & ~(uint32_t)(KDA_APPEND_ZERO_Q | KDA_APPEND_ZERO_K)) return fail(KDA_ERR_INVALID_ARG, "flags %u", (unsigned)flags);
    if (seqlen == 0 || c.heads_q == 0 || (c.num_seqs == 0 && !cu_seqlens)) return KDA_OK;
    if (!k || !v) return fail(KDA_ERR_INVALID_ARG, "k or v is NULL");
    for (const void *p : {k, v, q, (const void *)k_out, (const void *)q_out})
        if (!aligned(p, 16)) return fail(KDA_ERR_INVALID_ARG, "kda_cache_append: tensors must be 16-byte aligned");
    if (cu_seqlens && (seqlen > 0x7fffffffLL || !aligned(cu_seqlens, 4))) return fail(KDA_ERR_INVALID_ARG, "cu_seqlens is misaligned or seqlen exceeds its int32 range");
    if (seqlen > 1 << 30) return fail(KDA_ERR_UNSUPPORTED, "more than 2^30 new tokens");
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.q = static_cast<const uint16_t *>(q);
    a.k_out = static_cast<uint16_t *>(k_out);
    a.q_out = static_cast<uint16_t *>(q_out);
    a.cu = cu_seqlens;
    a.zero_q = q_out && (flags & KDA_APPEND_ZERO_Q);
    a.zero_k = k_out && (flags & KDA_APPEND_ZERO_K);
    a.per_seq = cu_seqlens ? 0 : seqlen;
    a.tokens = cu_seqlens ? seqlen : seqlen * c.num_seqs;
    // pages that seqlen tokens can touch, wherever they begin
    const int64_t per_seq = cu_seqlens ? 0 : (seqlen + c.page_size - 2) / c.page_size + 1;
    const int64_t slots = c.num_seqs == 0 ? 0 : cu_seqlens ? seqlen / c.page_size + 2 * (int64_t)c.num_seqs : per_seq * c.num_seqs;
    // (a launch has fewer than 2^32 threads: up to 512 a page and head, and dim / 8 a row of q)
    if (slots > 0x1fffff || slots * c.heads_kv * 2 > 0x3fffff || a.tokens * c.heads_q > 0x7ffffff || a.tokens * c.heads_kv > 0x7ffffff)
        return fail(KDA_ERR_UNSUPPORTED, "more than 2^22 pages and heads, or 2^27 rows of k or q");
    a.slots = (int32_t)slots;
    a.slots_per_seq = (int32_t)per_seq;
    return cache_append_dispatch(c, a, cache->dim, static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t kda_cache_attn_workspace_size(const kda_cache *cache, const kda_cache_query *query)
{
    cache::Cache c;
    cache::Attend a;
    if (check(cache, false, query, c, a) != KDA_OK || a.splits <= 1) return 0;
    return stats_offset(c, a, cache->dim) + up256((size_t)c.num_seqs * c.heads_kv * a.splits * a.rows * 2 * 4);
}

extern "C" kda_status kda_cache_attn(const kda_cache *cache, const kda_cache_query *query, const void *q, void *o, void *workspace,
                                     size_t workspace_bytes, void *hip_stream)
{
    cache::Cache c;
    cache::Attend a;
    if (const kda_status st = check(cache, true, query, c, a); st != KDA_OK) return st;
    if (c.num_seqs == 0 || a.rows == 0) return KDA_OK;
    if (!q || !o || !aligned(q, 16) || !aligned(o, 16)) return fail(KDA_ERR_INVALID_ARG, "q or o is NULL or not 16-byte aligned");
    if (a.splits > 1) {
        const size_t need = kda_cache_attn_workspace_size(cache, query);
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
            return fail(KDA_ERR_WORKSPACE, "kda_cache_attn: workspace must be 256-byte aligned and hold %zu bytes, got %zu", need, workspace_bytes);
        a.part = static_cast<float *>(workspace);
        a.stats = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + stats_offset(c, a, cache->dim));
    }
    a.q = static_cast<const uint16_t *>(q);
    a.o = o;
    return cache_attn_dispatch(c, a, cache->dim, static_cast<hipStream_t>(hip_stream));
}
