// Moving what stands in the paged cache: whole pages (kda_cache_copy_pages), and the accepted tokens of a draft tree up to the end of what a
// sequence holds (kda_cache_keep), in every layer of a stack at once.
#include "kda_cache.h"

namespace kda {
namespace cache {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---- kda_cache_copy_pages.  An item is up to kPiece bytes of one page's codes in one layer; bound by reading and writing them: 1.04 GB
// in 217 us, 4.8 TB/s, a plain copy's rate. ----
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

// ---- kda_cache_keep.  A workgroup has the keys or the values of one sequence in one layer, as many heads at a time as its registers hold:
// everything of a head is read ahead of the first write.  A path of six tokens is 6 KiB for eight heads, and so what bounds it is latency: lengths and
// path, page numbers, then scales and codes.  64 sequences x 16 layers x 8 heads 24 us with a workgroup for each head, which looked all of that up
// again, 11 so. ----
constexpr int kKept = 64, kPages = 6;                        // tokens; pages that they can go to (16 tokens a page: 5)
constexpr int kPieces = 4;                                   // of 16 codes, in a thread's registers

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
    constexpr int kMost = 256 * kPieces / kChunks;           // tokens x heads at a time
    __shared__ int32_t from_page[kKept], from_at[kKept], to_page[kPages], count_;
    __shared__ float from_scale[kMost], own_scale[kMost];
    __shared__ uint32_t top[kPages][kMost];                  // scales' bits: positive numbers, in their order
    uint32_t id = blockIdx.x;
    const bool values = id & 1;
    id >>= 1;
    const int layer = id % a.layers, n = id / a.layers;
    const int tid = threadIdx.x;
    const int32_t len = c.lens[n];
    if (tid < 64) {
        const int32_t x = tid < a.most ? a.kept[(int64_t)n * a.most + tid] : -1;
        const int32_t before = __shfl_up(x, 1);
        const uint64_t bad = ~__ballot(x >= 0 && (tid == 0 || x > before));
        const int32_t count = len < 0 ? 0 : bad ? __builtin_ctzll(bad) : 64;
        if (tid == 0) count_ = count;
        if (tid < count) {
            const int64_t at = (int64_t)len + x;
            from_page[tid] = page_at(c, n, at >> c.page_log2);
            from_at[tid] = (int32_t)(at & (c.page_size - 1));
        }
        if (tid < kPages) to_page[tid] = len < 0 ? -1 : page_at(c, n, (int64_t)(len >> c.page_log2) + tid);
    }
    __syncthreads();
    const int32_t count = count_, older = len & (c.page_size - 1);
    if (count == 0) return;
    const int64_t heads_pages = (int64_t)layer * c.num_pages * c.heads_kv;
    uint8_t *codes = (values ? c.v : c.k) + heads_pages * c.page_size * D;
    float *scales = (values ? c.v_scale : c.k_scale) + heads_pages;
    auto address = [&](int32_t page, int head, int32_t at) { return codes + (((int64_t)page * c.heads_kv + head) * c.page_size + at) * D; };
    const int at_once = min(c.heads_kv, kMost / count), chunk = tid % kChunks;
    for (int h0 = 0; h0 < c.heads_kv; h0 += at_once) {
        const int heads = min(at_once, c.heads_kv - h0), items = heads * count;        // an item: a head of a token
        u32x4 w[kPieces];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int item = (tid + 256 * j) / kChunks, head = item / count, i = item - head * count;
            if (item < items && from_page[i] >= 0) w[j] = *reinterpret_cast<const u32x4 *>(address(from_page[i], h0 + head, from_at[i]) + 16 * chunk);
        }
        for (int item = tid; item < items; item += 256) {
            const int head = item / count, i = item - head * count;
            from_scale[item] = from_page[i] >= 0 ? scales[(int64_t)from_page[i] * c.heads_kv + h0 + head] : 0.f;
        }
        for (int h = tid; h < heads; h += 256) {
            const float own = to_page[0] >= 0 ? scales[(int64_t)to_page[0] * c.heads_kv + h0 + h] : 0.f;
            own_scale[h] = own;
            top[0][h] = older ? __float_as_uint(own) : 0u;
#pragma unroll
            for (int p = 1; p < kPages; ++p) top[p][h] = 0u;
        }
        __syncthreads();
        for (int item = tid; item < items; item += 256) {
            const int head = item / count, i = item - head * count;
            if (from_page[i] >= 0) atomicMax(&top[(older + i) >> c.page_log2][head], __float_as_uint(from_scale[item]));
        }
        // (every code has been read: the loads' values are waited for here)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int item = (tid + 256 * j) / kChunks, head = item / count, i = item - head * count;
            if (item >= items || from_page[i] < 0) continue;
            const int page = (older + i) >> c.page_log2, at = (older + i) & (c.page_size - 1);
            const int32_t p = to_page[page];
            if (p < 0) continue;
            const float scale = from_scale[item], now = __uint_as_float(top[page][head]);
            if (p == from_page[i] && at == from_at[i] && scale == now) continue;
            *reinterpret_cast<u32x4 *>(address(p, h0 + head, at) + 16 * chunk) = rescale(w[j], scale / now);
        }
        // older tokens of the first page, where its scale has grown: a head a wave, four pieces of a lane on their way at once
        for (int h = tid >> 6; h < heads && to_page[0] >= 0 && older; h += 4) {
            const float now = __uint_as_float(top[0][h]);
            if (now == own_scale[h]) continue;
            u32x4 *page = reinterpret_cast<u32x4 *>(address(to_page[0], h0 + h, 0));
            const float ratio = own_scale[h] / now;
            for (int i0 = tid & 63; i0 < older * kChunks; i0 += 4 * 64) {
                u32x4 y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = page[min(i0 + 64 * j, older * kChunks - 1)];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i0 + 64 * j < older * kChunks) page[i0 + 64 * j] = rescale(y[j], ratio);
            }
        }
        for (int i = tid; i < heads * kPages; i += 256) {
            const int p = i / heads, h = i - p * heads;
            if (to_page[p] >= 0 && top[p][h]) scales[(int64_t)to_page[p] * c.heads_kv + h0 + h] = __uint_as_float(top[p][h]);
        }
        __syncthreads();
    }
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
    const uint32_t grid = (uint32_t)c.num_seqs * a.layers * 2;
    if (dim == 128) hipLaunchKernelGGL((kda_cache_keep_kernel<128>), dim3(grid), dim3(256), 0, st, c, a);
    else hipLaunchKernelGGL((kda_cache_keep_kernel<64>), dim3(grid), dim3(256), 0, st, c, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_cache_keep: %s", hipGetErrorString(e));
}

}  // namespace kda
