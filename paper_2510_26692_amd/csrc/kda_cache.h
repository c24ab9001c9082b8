// The paged 8-bit cache as its kernels see it (kda_cache_append.hip, kda_cache_attn.hip).
#pragma once

#include "kda_common.h"

namespace kda {
namespace cache {

// Pages of page_size tokens, [num_pages][heads][page_size][dim] e4m3 codes for keys and as many for values, a scale [num_pages][heads] fp32
// each.  Sequence n's token t stands in page table[n][t / page_size]; an entry outside [0, num_pages) is no page.
struct Cache {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    const int32_t *table, *lens;
    int64_t num_pages;
    int32_t num_seqs, heads_q, heads_kv, group, page_size, page_log2, max_pages;
};
// A call of kda_cache_append.
struct Append {
    const uint16_t *k, *v, *q;
    uint16_t *k_out, *q_out;
    const float *inv_freq;
    const int32_t *cu;
    int64_t tokens;                  // rows of k, v and q in all
    int64_t per_seq;                 // tokens of a sequence (fixed)
    int64_t k_stride, v_stride, q_stride;
    int32_t n_freq;                  // half the rotated channels
    int32_t interleaved;
    int32_t slots;                   // pages that the call may touch: a workgroup has one of them for some heads
    int32_t slots_per_seq;           // 0: packed
    int32_t page_blocks;             // workgroups of pages; those behind them turn queries
    int32_t whole;                   // a slot is a sequence: its workgroups have all pages that its new tokens touch
    int32_t page_heads;              // heads of a page that a workgroup has
    int32_t q_heads;                 // query heads a thread turns
    int32_t zero_q, zero_k;          // rows that no sequence writes become zeros
};
// A call of kda_cache_attn.
struct Attend {
    const uint16_t *q;
    void *o;
    float *part, *stats;             // [N][Hk][splits][rows][D] and [..][2]: numerators' sums, maximum (in powers of two) and sum of the softmax
    int64_t q_stride;
    float scale;
    int32_t tokens, window, sinks, rows, row_tiles, splits, out_bf16;
};

// Number of the page that holds logical page p of sequence n, or -1.
__device__ __forceinline__ int32_t page_at(const Cache &c, int n, int64_t p)
{
    if (p < 0 || p >= c.max_pages) return -1;
    const int32_t id = c.table[(int64_t)n * c.max_pages + p];
    return id >= 0 && id < c.num_pages ? id : -1;
}

}  // namespace cache
}  // namespace kda
