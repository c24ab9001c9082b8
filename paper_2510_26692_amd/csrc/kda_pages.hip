// Pages that several sequences share: forking and freeing rows of a block table, the pages that a step will write, and moving the pages in use
// to the front of the pool.  Tables and reference counts alone; the pages themselves are copied by kda_cache_copy_pages.
//
// A page is free where its count is zero, so there is no list to keep: free pages are taken the lowest-numbered first, in the order of
// rows and columns, and every answer is the same whatever the order in which workgroups run.  Counts change by integer atomics whose
// results nobody reads.
//
// What bounds these calls is latency: a table of 128 sequences and 17 columns and the counts of a thousand pages are some kilobytes.  Forked in 4 us, reserved
// in 7; 4 000 pages compacted in 7 and 5.
#include "kda_common.h"

namespace kda {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
constexpr int kMaxRows = 8192;

__device__ __forceinline__ bool is_page(int32_t e, int64_t pages) { return e >= 0 && e < pages; }

// ---- kda_pages_fork: a workgroup has all rows of some columns, read whole ahead of the first write ----
constexpr int kForkEntries = 8192;                           // of a workgroup, in LDS
__global__ __launch_bounds__(256) void kda_pages_fork_kernel(int32_t *table, int32_t rows, int32_t columns, int32_t width, int32_t *refs, int64_t pages,
                                                             const int32_t *source)
{
    extern __shared__ int32_t old[];
    const int32_t c0 = blockIdx.x * width, w = min(width, columns - c0), count = rows * w;
    for (int i = threadIdx.x; i < count; i += 256) old[i] = table[(int64_t)(i / w) * columns + c0 + i % w];
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += 256) {
        const int32_t n = i / w, s = source[n];
        if (s == n || s >= rows) continue;
        const int32_t was = old[i], is = s < 0 ? -1 : old[s * w + i % w];
        if (was == is) continue;
        table[(int64_t)n * columns + c0 + i % w] = is;
        if (is_page(was, pages)) atomicSub(refs + was, 1);
        if (is_page(is, pages)) atomicAdd(refs + is, 1);
    }
}

// ---- what one workgroup of 1024 threads shares ----
constexpr int kThreads = 1024;
// Sum of v over the threads before this one, and over all of them.
__device__ __forceinline__ int32_t sum_before(int32_t v, int32_t &all, int32_t (&lds)[kThreads / 64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                                         // (of the call before)
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    int32_t before = x - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        before += w < wave ? lds[w] : 0;
        all += lds[w];
    }
    return before;
}
// Counts of sixteen pages from `at` on, -1 behind the pool's last.
struct Sixteen {
    i32x4 v[4];
    __device__ __forceinline__ void load(const int32_t *refs, int64_t at, int64_t pages)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (at + 4 * i + 4 <= pages) v[i] = *reinterpret_cast<const i32x4 *>(refs + at + 4 * i);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = at + 4 * i + e < pages ? refs[at + 4 * i + e] : -1;
        }
    }
    __device__ __forceinline__ int32_t count(bool used) const
    {
        int32_t n = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) n += used ? v[i / 4][i % 4] > 0 : v[i / 4][i % 4] == 0;
        return n;
    }
};

// ---- kda_pages_reserve ----
struct Reserve {
    int32_t *table, *refs, *copies, *missing;
    const int32_t *lens, *after;
    i32x4 *wanted;                   // workspace: row, column, the entry that is replaced
    int32_t *free;                   // workspace: free pages, lowest first
    int64_t pages;
    int32_t rows, columns, page_log2, most;      // most: entries of the workspace's lists
};
__global__ __launch_bounds__(kThreads) void kda_pages_reserve_kernel(const Reserve a)
{
    extern __shared__ int32_t starts[];                      // [rows + 1]: entries that the rows ahead will write
    __shared__ int32_t sums[kThreads / 64];
    const int tid = threadIdx.x;
    int32_t all, total = 0;
    auto columns_of = [&](int32_t n, int32_t &first) -> int32_t {
        const int32_t l = a.lens[n], m = a.after[n];
        first = 0;
        if (l < 0 || m <= l) return 0;
        first = l >> a.page_log2;
        const int32_t end = min(((m - 1) >> a.page_log2) + 1, a.columns);
        return max(end - first, 0);
    };
    for (int32_t n0 = 0; n0 < a.rows; n0 += kThreads) {
        const int32_t n = n0 + tid;
        int32_t first, mine = 0;
        if (n < a.rows) {
            mine = columns_of(n, first);
            a.copies[2 * n] = a.copies[2 * n + 1] = -1;
        }
        const int32_t before = sum_before(mine, all, sums);
        if (n < a.rows) starts[n] = total + before;
        total += all;
    }
    if (tid == 0) starts[a.rows] = total;
    __syncthreads();
    // those that are no page, or another's too, in order
    int32_t want = 0;
    for (int32_t i0 = 0; i0 < total; i0 += kThreads) {
        const int32_t i = i0 + tid;
        i32x4 w = {0, 0, -1, 0};
        bool need = false;
        if (i < total) {
            int32_t lo = 0, hi = a.rows - 1;                 // the last row that starts at i or before
            while (lo < hi) {
                const int32_t mid = (lo + hi + 1) >> 1;
                if (starts[mid] <= i) lo = mid; else hi = mid - 1;
            }
            const int32_t column = (a.lens[lo] >> a.page_log2) + i - starts[lo], e = a.table[(int64_t)lo * a.columns + column];
            const bool page = is_page(e, a.pages);
            need = !page || a.refs[e] > 1;
            w = i32x4{lo, column, page ? e : -1, 0};
        }
        const int32_t rank = want + sum_before(need, all, sums);
        if (need && rank < a.most) a.wanted[rank] = w;
        want += all;
    }
    // as many free pages
    int32_t found = 0;
    for (int64_t p0 = 0; p0 < a.pages && found < want; p0 += kThreads * 16) {
        Sixteen s;
        s.load(a.refs, p0 + 16 * tid, a.pages);
        int32_t rank = found + sum_before(s.count(false), all, sums);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (s.v[i / 4][i % 4] == 0) {
                if (rank < want && rank < a.most) a.free[rank] = (int32_t)(p0 + 16 * tid + i);
                ++rank;
            }
        found += all;
    }
    if (tid == 0) *a.missing = want > found ? want - found : 0;
    if (want > found) return;
    __syncthreads();                                         // (the lists are written, and every count has been read)
    for (int32_t r = tid; r < want; r += kThreads) {
        const i32x4 w = a.wanted[r];
        const int32_t page = a.free[r], n = w[0], l = a.lens[n];
        a.table[(int64_t)n * a.columns + w[1]] = page;
        a.refs[page] = 1;
        if (w[2] >= 0) {
            atomicSub(a.refs + w[2], 1);
            if (w[1] == l >> a.page_log2 && (l & ((1 << a.page_log2) - 1))) {
                a.copies[2 * n] = w[2];
                a.copies[2 * n + 1] = page;
            }
        }
    }
}

// ---- kda_pages_compact ----
struct Compact {
    int32_t *table, *refs, *moves, *rank;        // rank, workspace: of a page in use at U and above among them
    int32_t *count;                              // workspace: moves
    int64_t pages, entries;
};
__global__ __launch_bounds__(kThreads) void kda_pages_moves_kernel(const Compact a)
{
    __shared__ int32_t sums[kThreads / 64], below;           // below: pages in use below U
    const int tid = threadIdx.x;
    int32_t all, used = 0;
    for (int64_t p0 = 0; p0 < a.pages; p0 += kThreads * 16) {
        Sixteen s;
        s.load(a.refs, p0 + 16 * tid, a.pages);
        sum_before(s.count(true), all, sums);
        used += all;
    }
    int32_t before = 0;
    if (tid == 0 && used == a.pages) below = used;           // (nothing stands at U)
    for (int64_t p0 = 0; p0 < a.pages; p0 += kThreads * 16) {
        Sixteen s;
        const int64_t at = p0 + 16 * tid;
        s.load(a.refs, at, a.pages);
        int32_t n = before + sum_before(s.count(true), all, sums);
        if (at <= used && used < at + 16 && used < a.pages) {
            int32_t x = n;
#pragma unroll
            for (int i = 0; i < 16; ++i) x += at + i < used && s.v[i / 4][i % 4] > 0;
            below = x;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t p = at + i;
            const int32_t r = s.v[i / 4][i % 4];
            if (p < used && r <= 0) a.moves[2 * (p - n) + 1] = (int32_t)p;          // (every page that is not in use: ranks have no gaps)
            if (p >= used && p < a.pages) {
                a.rank[p] = r > 0 ? n - below : -1;
                if (r > 0) a.moves[2 * (n - below)] = (int32_t)p;
            }
            n += r > 0;
        }
        before += all;
    }
    __syncthreads();
    const int32_t count = used - below;
    if (tid == 0) *a.count = count;
    for (int64_t i = count + tid; i < a.pages / 2; i += kThreads) a.moves[2 * i] = a.moves[2 * i + 1] = -1;
}
__global__ __launch_bounds__(256) void kda_pages_place_kernel(const Compact a)
{
    const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int32_t count = *a.count;
    if (count == 0) return;
    // (moves are ascending in both columns: the first from is the lowest page that moves)
    const int32_t lowest = a.moves[0];
    for (int64_t i = first; i < a.entries; i += step) {
        const int32_t e = a.table[i];
        if (e < lowest || e >= a.pages) continue;
        const int32_t r = a.rank[e];
        if (r >= 0) a.table[i] = a.moves[2 * r + 1];
    }
    for (int64_t i = first; i < count; i += step) {
        a.refs[a.moves[2 * i + 1]] = a.refs[a.moves[2 * i]];
        a.refs[a.moves[2 * i]] = 0;
    }
}

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
kda_status check(const int32_t *table, int32_t rows, int32_t columns, const int32_t *refs, int64_t pages)
{
    if (rows < 0 || columns < 0 || pages < 0)
        return fail(KDA_ERR_INVALID_ARG, "negative size (num_seqs %d, max_pages %d, num_pages %lld)", rows, columns, (long long)pages);
    if (pages > 0x7fffffffLL) return fail(KDA_ERR_INVALID_ARG, "num_pages exceeds the int32 range of block_table");
    if ((rows && columns && !table) || (pages && !refs)) return fail(KDA_ERR_INVALID_ARG, "block_table or page_refs is NULL");
    if (!aligned(table, 4) || !aligned(refs, 16)) return fail(KDA_ERR_INVALID_ARG, "block_table is misaligned, or page_refs not 16-byte aligned");
    return KDA_OK;
}
kda_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "%s: %s", what, hipGetErrorString(e));
}
// entries that one call can want: no more than the table or the pool has
int64_t reserve_most(int32_t rows, int32_t columns, int64_t pages)
{
    const int64_t n = (int64_t)rows * columns;
    return n < pages ? n : pages;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace
}  // namespace kda

using namespace kda;

extern "C" kda_status kda_pages_fork(int32_t *block_table, int32_t num_seqs, int32_t max_pages, int32_t *page_refs, int64_t num_pages,
                                     const int32_t *source, void *hip_stream)
{
    if (const kda_status st = check(block_table, num_seqs, max_pages, page_refs, num_pages); st != KDA_OK) return st;
    if (num_seqs > kMaxRows) return fail(KDA_ERR_UNSUPPORTED, "at most %d sequences, got %d", kMaxRows, num_seqs);
    if (num_seqs == 0 || max_pages == 0) return KDA_OK;
    if (!source || !aligned(source, 4)) return fail(KDA_ERR_INVALID_ARG, "source is NULL or misaligned");
    // columns of a workgroup: up to half a cache line's, as far as its rows fit the LDS and 64 workgroups are left (128 sequences x 17 columns: 7.6 us
    // with 16 columns, 4.1 with one)
    int64_t width = ((int64_t)max_pages + 63) / 64;
    width = width > kForkEntries / num_seqs ? kForkEntries / num_seqs : width;
    width = width > 16 ? 16 : width;
    const int64_t blocks = (max_pages + width - 1) / width;
    // (a launch has fewer than 2^32 threads)
    if (blocks > 0xffffff) return fail(KDA_ERR_UNSUPPORTED, "more than 2^24 workgroups (max_pages %d)", max_pages);
    hipLaunchKernelGGL(kda_pages_fork_kernel, dim3((uint32_t)blocks), dim3(256), (size_t)num_seqs * width * 4, static_cast<hipStream_t>(hip_stream),
                       block_table, num_seqs, max_pages, (int32_t)width, page_refs, num_pages, source);
    return launched("kda_pages_fork");
}

extern "C" size_t kda_pages_reserve_workspace_size(int32_t num_seqs, int32_t max_pages, int64_t num_pages)
{
    if (num_seqs < 0 || max_pages < 0 || num_pages < 0) return 0;
    const size_t most = reserve_most(num_seqs, max_pages, num_pages);
    return up256(most * sizeof(i32x4)) + up256(most * 4);
}

extern "C" kda_status kda_pages_reserve(int32_t *block_table, int32_t num_seqs, int32_t max_pages, int32_t page_size, int32_t *page_refs,
                                        int64_t num_pages, const int32_t *kv_lens, const int32_t *new_lens, int32_t *copies, int32_t *missing,
                                        void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (const kda_status st = check(block_table, num_seqs, max_pages, page_refs, num_pages); st != KDA_OK) return st;
    if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128)
        return fail(KDA_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128, got %d", page_size);
    if (num_seqs > kMaxRows) return fail(KDA_ERR_UNSUPPORTED, "at most %d sequences, got %d", kMaxRows, num_seqs);
    // (entries are counted in 32 bits, a workgroup's threads at a time)
    if ((int64_t)num_seqs * max_pages >= 0x7fffffffLL - kThreads + 1) return fail(KDA_ERR_UNSUPPORTED, "a table of 2^31 - 1024 entries or more");
    if (!missing || (num_seqs && (!kv_lens || !new_lens || !copies))) return fail(KDA_ERR_INVALID_ARG, "kv_lens, new_lens, copies or missing is NULL");
    for (const void *p : {(const void *)kv_lens, (const void *)new_lens, (const void *)copies, (const void *)missing})
        if (!aligned(p, 4)) return fail(KDA_ERR_INVALID_ARG, "kv_lens, new_lens, copies or missing is misaligned");
    const size_t need = kda_pages_reserve_workspace_size(num_seqs, max_pages, num_pages);
    if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return fail(KDA_ERR_WORKSPACE, "kda_pages_reserve: workspace must be 256-byte aligned and hold %zu bytes, got %zu", need, workspace_bytes);
    Reserve a = {};
    a.table = block_table;
    a.refs = page_refs;
    a.copies = copies;
    a.missing = missing;
    a.lens = kv_lens;
    a.after = new_lens;
    a.pages = num_pages;
    a.rows = num_seqs;
    a.columns = max_pages;
    a.page_log2 = page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7;
    a.most = (int32_t)reserve_most(num_seqs, max_pages, num_pages);
    a.wanted = static_cast<i32x4 *>(workspace);
    a.free = reinterpret_cast<int32_t *>(static_cast<uint8_t *>(workspace) + up256((size_t)a.most * sizeof(i32x4)));
    hipLaunchKernelGGL(kda_pages_reserve_kernel, dim3(1), dim3(kThreads), ((size_t)num_seqs + 1) * 4, static_cast<hipStream_t>(hip_stream), a);
    return launched("kda_pages_reserve");
}

extern "C" kda_status kda_pages_compact(int32_t *block_table, int32_t num_seqs, int32_t max_pages, int32_t *page_refs, int64_t num_pages, int32_t *moves,
                                        void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (const kda_status st = check(block_table, num_seqs, max_pages, page_refs, num_pages); st != KDA_OK) return st;
    if (num_pages == 0) return KDA_OK;
    if ((num_pages > 1 && !moves) || !aligned(moves, 4)) return fail(KDA_ERR_INVALID_ARG, "moves is NULL or misaligned");
    const size_t need = (size_t)num_pages * 4 + 256;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
        return fail(KDA_ERR_WORKSPACE, "kda_pages_compact: workspace must be 256-byte aligned and hold %zu bytes, got %zu", need, workspace_bytes);
    Compact a = {};
    a.table = block_table;
    a.refs = page_refs;
    a.moves = moves;
    a.count = static_cast<int32_t *>(workspace);
    a.rank = a.count + 64;
    a.pages = num_pages;
    a.entries = (int64_t)num_seqs * max_pages;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(kda_pages_moves_kernel, dim3(1), dim3(kThreads), 0, st, a);
    if (const kda_status s = launched("kda_pages_compact"); s != KDA_OK) return s;
    const int64_t work = a.entries > num_pages / 2 ? a.entries : num_pages / 2, blocks = (work + 255) / 256;
    if (blocks == 0) return KDA_OK;
    hipLaunchKernelGGL(kda_pages_place_kernel, dim3((uint32_t)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, st, a);
    return launched("kda_pages_compact");
}
