// Moving what stands in the paged cache: whole pages (kda_cache_copy_pages), and the accepted tokens of a draft tree up to the end of what a
// sequence holds (kda_cache_keep), in every layer of a stack at once.
#include "kda_cache.h"

namespace kda {
namespace cache {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---- kda_cache_copy_pages.  An item is up to kPiece bytes of one page's codes in one layer; bound by reading and writing them. ----
constexpr int kPiece = 16384;
__global__ __launch_bounds__(256) void kda_cache_copy_kernel(const Cache c, const Copies a)
{
    for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
        int64_t i = item;
        const int piece = (int)(i % a.pieces);
        i /= a.pieces;
        const bool values = i & 1;
        i >>= 1;
        const int layer = (int)(i % a.layers);
        const int64_t pair = i / a.layers;
        const int64_t from = a.pairs[2 * pair], to = a.pairs[2 * pair + 1];
        if (from < 0 || from >= c.num_pages || to < 0 || to >= c.num_pages || from == to) continue;
        uint8_t *codes = (values ? c.v : c.k) + (int64_t)layer * c.num_pages * a.page_bytes;
        const uint8_t *src = codes + from * a.page_bytes;
        uint8_t *dst = codes + to * a.page_bytes;
        const int64_t begin = (int64_t)piece * kPiece + 16 * threadIdx.x;
        u32x4 w[kPiece / 4096];
#pragma unroll
        for (int j = 0; j < kPiece / 4096; ++j)
            if (begin + 4096 * j < a.page_bytes) w[j] = *reinterpret_cast<const u32x4 *>(src + begin + 4096 * j);
#pragma unroll
        for (int j = 0; j < kPiece / 4096; ++j)
            if (begin + 4096 * j < a.page_bytes) *reinterpret_cast<u32x4 *>(dst + begin + 4096 * j) = w[j];
        if (piece == 0) {
            float *scale = (values ? c.v_scale : c.k_scale) + (int64_t)layer * c.num_pages * c.heads_kv;
            for (int h = threadIdx.x; h < c.heads_kv; h += 256) scale[to * c.heads_kv + h] = scale[from * c.heads_kv + h];
        }
    }
}

// ---- kda_cache_keep.  A workgroup has the keys or the values of one sequence and head in one layer: everything is read, in
// registers, ahead of the first write.  The largest is 64 tokens, 8 KiB, and so what bounds it is latency: page numbers, scales, codes. ----
constexpr int kKept = 64, kPages = 6;                        // tokens; pages that they can go to (16 tokens a page: 5)

// codes times ratio, rounded to nearest even
__device__ __forceinline__ u32x4 rescale(const u32x4 &w, float ratio)
{
    if (ratio == 1.f) return w;                              // (codes that are no number keep their bits)
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(w[i], 0) * ratio, __builtin_amdgcn_cvt_f32_fp8(w[i], 1) * ratio, 0, false);
        o[i] = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(w[i], 2) * ratio, __builtin_amdgcn_cvt_f32_fp8(w[i], 3) * ratio, r, true);
    }
    return o;
}

template <int D>
__global__ __launch_bounds__(256) void kda_cache_keep_kernel(const Cache c, const Keep a)
{
    constexpr int kChunks = D / 16;                          // 16-byte pieces of a token
    __shared__ int32_t from_page[kKept], from_at[kKept], to_page[kPages], count_;
    __shared__ float from_scale[kKept];
    __shared__ uint32_t top[kPages];                         // scales' bits: positive numbers, in their order
    uint32_t id = blockIdx.x;
    const int head = id % c.heads_kv;
    id /= c.heads_kv;
    const bool values = id & 1;
    id >>= 1;
    const int layer = id % a.layers, n = id / a.layers;
    const int32_t len = c.lens[n];
    if (len < 0) return;
    const int64_t heads_pages = (int64_t)layer * c.num_pages * c.heads_kv;
    uint8_t *codes = (values ? c.v : c.k) + heads_pages * c.page_size * D;
    float *scales = (values ? c.v_scale : c.k_scale) + heads_pages;
    const int tid = threadIdx.x;
    const int32_t page0 = len >> c.page_log2, older = len & (c.page_size - 1);
    if (tid < 64) {
        const int32_t x = tid < a.most ? a.kept[(int64_t)n * a.most + tid] : -1;
        const int32_t before = __shfl_up(x, 1);
        const bool good = x >= 0 && (tid == 0 || x > before);
        const uint64_t bad = ~__ballot(good);
        const int32_t count = bad ? __builtin_ctzll(bad) : 64;
        if (tid == 0) count_ = count;
        if (tid < count) {
            const int64_t at = (int64_t)len + x;
            const int32_t p = page_at(c, n, at >> c.page_log2);
            from_page[tid] = p;
            from_at[tid] = (int32_t)(at & (c.page_size - 1));
            from_scale[tid] = p < 0 ? 0.f : scales[(int64_t)p * c.heads_kv + head];
        }
        if (tid < kPages) to_page[tid] = page_at(c, n, (int64_t)page0 + tid);
    }
    __syncthreads();
    const int32_t count = count_;
    if (count == 0) return;
    if (tid < kPages) {
        const int32_t p = to_page[tid];
        top[tid] = tid == 0 && older && p >= 0 ? __float_as_uint(scales[(int64_t)p * c.heads_kv + head]) : 0u;
    }
    const float scale0 = to_page[0] >= 0 ? scales[(int64_t)to_page[0] * c.heads_kv + head] : 0.f;
    auto place = [&](int i, int &page, int &at) {
        const int32_t to = older + i;
        page = to >> c.page_log2;
        at = to & (c.page_size - 1);
    };
    auto address = [&](int32_t page, int32_t at) { return codes + (((int64_t)page * c.heads_kv + head) * c.page_size + at) * D; };
    // the tokens' codes
    constexpr int kMine = (kKept * kChunks + 255) / 256;
    u32x4 w[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const int i = (tid + 256 * j) / kChunks;
        if (i < count && from_page[i] >= 0) w[j] = *reinterpret_cast<const u32x4 *>(address(from_page[i], from_at[i]) + 16 * (tid % kChunks));
    }
    __syncthreads();
    if (tid < count && from_page[tid] >= 0) {
        int page, at;
        place(tid, page, at);
        atomicMax(top + page, __float_as_uint(from_scale[tid]));
    }
    // (every code and scale has been read: the loads' values are waited for here)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const int i = (tid + 256 * j) / kChunks;
        if (i >= count || from_page[i] < 0) continue;
        int page, at;
        place(i, page, at);
        const int32_t p = to_page[page];
        if (p < 0) continue;
        const float scale = from_scale[i], now = __uint_as_float(top[page]);
        if (p == from_page[i] && at == from_at[i] && scale == now) continue;
        *reinterpret_cast<u32x4 *>(address(p, at) + 16 * (tid % kChunks)) = rescale(w[j], scale / now);
    }
    if (older && to_page[0] >= 0 && __uint_as_float(top[0]) != scale0) {
        uint8_t *page = address(to_page[0], 0);
        const float ratio = scale0 / __uint_as_float(top[0]);
        for (int i = tid; i < older * kChunks; i += 256) {
            u32x4 *at = reinterpret_cast<u32x4 *>(page + 16 * i);
            *at = rescale(*at, ratio);
        }
    }
    if (tid < kPages && to_page[tid] >= 0 && top[tid]) scales[(int64_t)to_page[tid] * c.heads_kv + head] = __uint_as_float(top[tid]);
}

}  // namespace cache
}  // namespace kda

using namespace kda;
using namespace kda::cache;

namespace kda {

kda_status cache_copy_dispatch(const Cache &c, Copies a, hipStream_t st)
{
    a.pieces = (int32_t)((a.page_bytes + kPiece - 1) / kPiece);
    a.items *= a.pieces;
    const uint32_t grid = (uint32_t)(a.items < 0xffffff ? a.items : 0xffffff);
    hipLaunchKernelGGL(kda_cache_copy_kernel, dim3(grid), dim3(256), 0, st, c, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_cache_copy_pages: %s", hipGetErrorString(e));
}

kda_status cache_keep_dispatch(const Cache &c, const Keep &a, int dim, hipStream_t st)
{
    const uint32_t grid = (uint32_t)c.num_seqs * a.layers * 2 * c.heads_kv;
    if (dim == 128) hipLaunchKernelGGL((kda_cache_keep_kernel<128>), dim3(grid), dim3(256), 0, st, c, a);
    else hipLaunchKernelGGL((kda_cache_keep_kernel<64>), dim3(grid), dim3(256), 0, st, c, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_cache_keep: %s", hipGetErrorString(e));
}

}  // namespace kda
