// What the attention kernels over the paged cache share (kda_cache_attn.hip, kda_cache_tree.hip): the join of a row's parts, which used_parts of
// the call's type counts.
#pragma once

#include "kda_cache.h"

namespace kda {
namespace cache {

constexpr float kInf = __builtin_huge_valf();
constexpr int kWaves = 4;
constexpr int kJoinAlone = 32;       // parts of a row that one wave joins
constexpr float kLift = 64.f;        // what logits, in powers of two, count more to the maximum where a scale of their values has these bits
constexpr uint32_t kLargeScale = 0x5f800000u;                // or more: 2^64

// The splits' parts of a row, D / 64 channels a lane.  kPer waves have a row between them: one wave reads 8 parts at a time, and what a long
// sequence of few heads is split into would keep it waiting (the call for one of 131 072 tokens and 2 key heads, 256 parts: 37.7 us with one
// wave a row, 22.2 with four; 8 192 tokens and 8 heads, 32 parts, 11.2 and 11.1).
template <int D, int kPer, typename A>
__global__ __launch_bounds__(256) void kda_cache_join_kernel(const Cache c, const A a)
{
    constexpr int W = D / 64, kAhead = kPer > 1 ? 16 : 8;
    __shared__ float joined[kPer > 1 ? kPer : 1][D + 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t item = kPer > 1 ? blockIdx.x : (int64_t)blockIdx.x * kWaves + wave;         // (sequence, key head, row)
    if (item >= (int64_t)c.num_seqs * c.heads_kv * a.rows) return;                             // (whole workgroups, where they share a row)
    const int64_t pair = item / a.rows;
    const int row = (int)(item - pair * a.rows), n = (int)(pair / c.heads_kv), kv = (int)(pair - (int64_t)n * c.heads_kv);
    const int32_t used = used_parts(c, a, n), mine = (used + kPer - 1) / kPer, begin = kPer > 1 ? wave * mine : 0, end = min(begin + mine, used);
    // a lane has one split's maximum and sum, 64 splits at a time
    float m = -kInf, l = 0.f, y[W] = {};
    for (int s0 = begin; s0 < end; s0 += 64) {
        const int64_t part = (pair * a.splits + s0 + lane) * a.rows + row;
        float ms = -kInf, ls = 0.f;
        if (s0 + lane < end) {
            ms = a.stats[part * 2];
            ls = a.stats[part * 2 + 1];
        }
        float top = ms;
#pragma unroll
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float mn = fmaxf(m, top), old = m == -kInf ? 0.f : fast_exp2(m - mn), f = ms == -kInf ? 0.f : fast_exp2(ms - mn);
        m = mn;
        ls *= f;
#pragma unroll
        for (int o = 32; o; o >>= 1) ls += __shfl_xor(ls, o);
        l = l * old + ls;
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] *= old;
        const int count = end - s0 < 64 ? end - s0 : 64;
        const float *from = a.part + ((pair * a.splits + s0) * a.rows + row) * D + W * lane;
        const int64_t step = (int64_t)a.rows * D;
        for (int s = 0; s < count; s += kAhead) {
            float x[kAhead][W];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int i = 0; i < W; ++i) x[u][i] = from[(s + u < count ? s + u : count - 1) * step + i];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float g = s + u < count ? __shfl(f, s + u) : 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) y[i] += s + u < count ? x[u][i] * g : 0.f;
            }
        }
    }
    if constexpr (kPer > 1) {
#pragma unroll
        for (int i = 0; i < W; ++i) joined[wave][W * lane + i] = y[i];
        if (lane == 0) {
            joined[wave][D] = m;
            joined[wave][D + 1] = l;
        }
        __syncthreads();
        if (wave) return;
        float top = -kInf;
#pragma unroll
        for (int w = 0; w < kPer; ++w) top = fmaxf(top, joined[w][D]);
        l = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] = 0.f;
#pragma unroll
        for (int w = 0; w < kPer; ++w) {
            const float f = joined[w][D] == -kInf ? 0.f : fast_exp2(joined[w][D] - top);
            l += joined[w][D + 1] * f;
#pragma unroll
            for (int i = 0; i < W; ++i) y[i] += joined[w][W * lane + i] * f;
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int t = row / c.group, head = kv * c.group + row - t * c.group;
    const int64_t out = (((int64_t)n * a.tokens + t) * c.heads_q + head) * D + W * lane;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (a.out_bf16) static_cast<uint16_t *>(a.o)[out + i] = (uint16_t)pack_bf16x2(y[i] * inv, 0.f);
        else static_cast<float *>(a.o)[out + i] = y[i] * inv;
    }
}

template <int D, typename A> hipError_t launch_join(const Cache &c, const A &a, int64_t items, hipStream_t st)
{
    if (a.splits > kJoinAlone) hipLaunchKernelGGL((kda_cache_join_kernel<D, kWaves, A>), dim3((uint32_t)items), dim3(64 * kWaves), 0, st, c, a);
    else hipLaunchKernelGGL((kda_cache_join_kernel<D, 1, A>), dim3((uint32_t)((items + kWaves - 1) / kWaves)), dim3(64 * kWaves), 0, st, c, a);
    return hipGetLastError();
}

}  // namespace cache
}  // namespace kda
