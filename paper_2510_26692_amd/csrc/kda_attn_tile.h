// Tiles shared by the softmax-attention kernels (kda_attn_fwd.hip, kda_attn_bwd.hip).
//
// A wave owns 32 columns (queries, or in the dK / dV kernel keys) whose operands stay in registers, and walks tiles of 32 or 64
// rows (keys, or queries) that the workgroup's four waves bring into LDS.  Every product is a 32x32x16 bf16 MFMA with the walked rows as
// the A operand:
//
//     X [row, column]    = sum_d  R[row, d] C[column, d]       A: rows of the LDS tile,            B: the wave's columns
//     Y^T [d, column]   += sum_row R[row, d] P[row, column]    A: the LDS tile read transposed,    B: X's accumulators, packed to bf16
//
// A lane of the accumulator (x = lane % 32, h = lane / 32) holds column x and the rows 8 (j / 4) + 4 h + j % 4, j = 0..15: eight of
// them in a row, packed, are a B operand of the second product for the contraction indices {16 s + 4 h + 0..3, 16 s + 8 + 4 h + 0..3},
// so that a softmax's numerators go from the one product to the next with no data movement.
#pragma once

#include "kda_common.h"

namespace kda {
namespace attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;            // rows of a walked tile
constexpr int kCols = 128;           // columns of a workgroup, 32 a wave
constexpr int kThreads = 256;
constexpr float kInf = __builtin_huge_valf();

// What a call's kernels know of its tensors: element counts, strides in elements.
struct Shape {
    int64_t tokens;                  // of a row of the batch, or packed
    int32_t num_seqs, heads_q, heads_kv, group;
    int32_t slots;                   // tiles of kCols tokens in the grid, for every head
    int32_t tiles;                   // of a sequence of a fixed batch; 0: packed
    int32_t window;                  // 0: none; below 2^30
    int32_t sinks;
    float scale;
    int64_t q_stride, k_stride, v_stride;
    const int32_t *cu;
};

// Sequence and first token of tile `slot`: tile t of sequence n of a packed batch has slot base(n) + t, base(n) = cu[n] / kCols + n,
// which leaves every sequence at least as many slots as it has tiles.  (cu is clamped to the tensor: entries that decrease or
// pass its end give empty or short sequences, never a row outside.)
struct Place {
    int64_t row0;                    // first token of the sequence in the tensors
    int32_t len;                     // its tokens
    int32_t first;                   // first token of the tile, relative to row0; len or beyond: nothing to do
    int32_t batch;                   // row of the batch (0: packed)
    int32_t seq;                     // which sequence
};
__device__ __forceinline__ int64_t cu_at(const Shape &s, int n)
{
    const int64_t v = s.cu[n];
    return v < 0 ? 0 : v < s.tokens ? v : s.tokens;
}
// by_rows orders the tiles of a fixed batch row after row, where neighbours' windows overlap (forward at 8 x 2048 tokens, 32 heads over 8,
// window 1024: 250 us, 256 in the other order); else tile after tile, so that no row's longest walks are begun late (forward at 4 x 4096 x 16
// heads causal 290 us, 300 in the other order; the whole backward pass 978 and 995, with a window 905 and 950).
__device__ __forceinline__ Place place_of(const Shape &s, int slot, bool by_rows)
{
    if (s.tiles) {
        const int b = by_rows ? slot / s.tiles : slot % s.num_seqs, t = by_rows ? slot - b * s.tiles : slot / s.num_seqs;
        return {(int64_t)b * s.tokens, (int32_t)s.tokens, t * kCols, b, b};
    }
    int lo = 0, hi = s.num_seqs - 1;                         // the last sequence whose base is not beyond the slot
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu_at(s, mid) / kCols + mid <= slot) lo = mid; else hi = mid - 1;
    }
    const int64_t a = cu_at(s, lo), e = cu_at(s, lo + 1);
    return {a, (int32_t)(e - a), (int32_t)(slot - (a / kCols + lo)) * kCols, 0, lo};
}

// What a column of a tile of 64 rows sees, as bits: row 32 b + r of the tile is bit r of w[b].  seen_rows: rows first .. last.
struct Seen { uint32_t w[2]; };
__device__ __forceinline__ int32_t clamp_tile(int32_t v) { return v < -1 ? -1 : v > kTile ? kTile : v; }
__device__ __forceinline__ Seen seen_rows(int32_t first, int32_t last)
{
    const uint64_t below = last < 0 ? 0ull : last >= 63 ? ~0ull : (2ull << last) - 1, m = below & (first <= 0 ? ~0ull : first > 63 ? 0ull : ~0ull << first);
    return {{(uint32_t)m, (uint32_t)(m >> 32)}};
}
// The keys k0 .. k0 + 63 that a query sees: not later, and in the window or among the sinks.
__device__ __forceinline__ Seen seen_keys(int32_t query, int32_t k0, int32_t window, int32_t sinks)
{
    const int32_t last = clamp_tile(query - k0), sink = clamp_tile(sinks - k0 - 1);
    Seen a = seen_rows(window ? clamp_tile(query - k0 - window + 1) : 0, last);
    const Seen b = seen_rows(0, last < sink ? last : sink);
    a.w[0] |= b.w[0];
    a.w[1] |= b.w[1];
    return a;
}
// All ones where accumulator register j of a lane in half h (the word shifted by 4 h) is seen.
__device__ __forceinline__ uint32_t seen_bit(uint32_t shifted, int j)
{
    return (uint32_t)((int32_t)(shifted << (31 - (8 * (j >> 2) + (j & 3)))) >> 31);
}
__device__ __forceinline__ float where_seen(uint32_t bit, float x, float other)
{
    return __uint_as_float((__float_as_uint(x) & bit) | (__float_as_uint(other) & ~bit));
}

// ---- LDS tiles of [kTile rows][D] bf16.  The 16-byte chunks of a row stand permuted so that both ways of reading a tile meet every
// bank once: 16 lanes on the same chunk of 16 rows (A operand of the first product), and 4 rows x 64 contiguous bytes (transposed). ----
template <int D> __device__ __forceinline__ constexpr int swizzle(int row)
{
    return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
}
template <int D> constexpr int kTileBytes = kTile * D * 2;

// Descriptor of the rows of one tile: reads behind `rows` rows give zeros.
__device__ __forceinline__ u32x4 rows_descriptor(const void *p, int32_t rows, uint32_t stride_bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    const uint32_t n = rows < 0 ? 0 : rows > kTile ? kTile : rows;
    u32x4 r = {(uint32_t)at, (uint32_t)(at >> 32), n * stride_bytes, 0x00020000u};
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
}
// One LDS-direct load of 4 bytes a lane, as dma16.
__device__ __forceinline__ void dma4(uint32_t m0, uint32_t voff, const u32x4 &rsrc)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "s_nop 3\n\t"
                 "buffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(m0), "v"(voff), "s"(rsrc) : "memory", "m0");
}
// One LDS-direct load of 16 bytes a lane: LDS byte m0 + 16 L <- byte voff(L) behind the descriptor's base.  The descriptor may come
// back from a spill by v_readlane, which a memory instruction written as text has to keep its distance from.
__device__ __forceinline__ void dma16(uint32_t m0, uint32_t voff, const u32x4 &rsrc)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "s_nop 3\n\t"
                 "buffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(m0), "v"(voff), "s"(rsrc) : "memory", "m0");
}
// A wave's quarter of a tile of kRows rows, 1 KiB an instruction.
template <int D, int kRows = kTile> struct TileLoader {
    static constexpr int kPer = 1024 / (2 * D);             // rows an instruction
    static constexpr int kLoads = kRows / 4 / kPer;
    uint32_t voff[kLoads];
    __device__ __forceinline__ void init(int wave, int lane, uint32_t stride_bytes)
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int r = kRows / 4 * wave + kPer * j + lane / (64 / kPer);
            voff[j] = r * stride_bytes + 16 * ((lane % (64 / kPer)) ^ swizzle<D>(r));
        }
    }
    __device__ __forceinline__ void issue(uint32_t lds, int wave, const u32x4 &rsrc) const
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) dma16(__builtin_amdgcn_readfirstlane(lds + wave * kRows / 4 * 2 * D + j * 1024), voff[j], rsrc);
    }
};
// every wave's part of the tile has landed, and every wave has left the tile before
__device__ __forceinline__ void tile_barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The kernels have no LDS but what their launch gives them, and that begins at byte 0.  Taken from an array's address the number is known
// to the linker only, and every read of a tile costs an addition of it.
constexpr uint32_t kLds = 0;
// Reads of a tile at LDS byte `tile`: A operands of the two products.  Where `tile` is a constant a read is its instruction alone, with
// one of the 16 permuted addresses.
typedef __attribute__((address_space(3))) const u32x4 *lds_u4;
typedef __attribute__((address_space(3))) s16x4 *lds_s4;
template <int D> struct TileReader {
    uint32_t row_at, tr_at[2];       // byte of the lane's row and first chunk; the chunk's number is changed by an exclusive or of bits above
    __device__ __forceinline__ void init(int lane)
    {
        const int x = lane & 31, h = lane >> 5, i = lane & 15, g = (lane >> 4) & 1;
        row_at = x * 2 * D + (swizzle<D>(x) ^ h) * 16;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int row = 8 * u + 4 * h + (i >> 2);
            tr_at[u] = row * 2 * D + ((2 * g + ((i >> 1) & 1)) ^ swizzle<D>(row)) * 16 + 8 * (i & 1);
        }
    }
    // The permuted addresses cost an operation each; kept across a walk they take 16 registers, which the backward kernels do not have (the
    // compiler then spills others): what this touches has to be formed again.  The whole backward pass at 4 x 4 096 tokens, 16 heads over 4, 128
    // wide: 1 047 us with the addresses of the dQ kernel kept, 1 015 with them formed again.
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(row_at), "+v"(tr_at[0]), "+v"(tr_at[1])); }
    // row 32 block + x, channels 16 s + 8 h ..
    __device__ __forceinline__ bf16x8 rows(uint32_t tile, int block, int s) const
    {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<lds_u4>((row_at ^ (32 * s)) + (tile + block * 32 * 2 * D)));
    }
    // channel 32 db + x, rows 16 ks + {4 h + 0..3, 8 + 4 h + 0..3}
    __device__ __forceinline__ bf16x8 transposed(uint32_t tile, int db, int ks) const
    {
        s16x4 r[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            r[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s4>((tr_at[u] ^ (64 * db)) + (tile + ks * 16 * 2 * D)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

__device__ __forceinline__ f32x16 mfma(const bf16x8 &a, const bf16x8 &b, const f32x16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Waits for operands loaded ahead of a walk.  Left to their first use, inside it, the wait would stand in every step, and as loads come
// back in order it would wait for the next tile's as well.
template <int N> __device__ __forceinline__ void arrived(bf16x8 (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        u32x4 w = __builtin_bit_cast(u32x4, f[i]);
        asm volatile("" : "+v"(w));
        f[i] = __builtin_bit_cast(bf16x8, w);
    }
}
__device__ __forceinline__ f32x16 zeros16()
{
    f32x16 z;
#pragma unroll
    for (int j = 0; j < 16; ++j) z[j] = 0.f;
    return z;
}
// the other half wave's value beside this one's: reductions over the rows of a column
__device__ __forceinline__ float other_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ __forceinline__ bf16x8 pack8(const float *p)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(p[2 * i], p[2 * i + 1]);
    return __builtin_bit_cast(bf16x8, w);
}

// The order in which a stretch without branches is issued: `lead` LDS reads first, then `per` of them behind each MFMA while there are
// any of the `reads`, then the rest of the `mfmas`.  Left to itself the compiler has one or two reads in flight and every MFMA, 32 cycles
// long, waits some 100 for its operand.
template <int lead, int per, int reads, int mfmas> __device__ __forceinline__ void reads_ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, lead, 0);
    constexpr int steps = (reads - lead) / per;
#pragma unroll
    for (int i = 0; i < steps; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, per, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, mfmas - steps, 0);
}

// ---- values that are not finite in masked places.  A product takes P = 0 times such a value for NaN.  Where that happened (the
// accumulators say so in the end), the walk is repeated with this on tiles that some column sees only in part: the value is taken
// out of the product, and every column that does see it becomes NaN.  (Forward, a sum of finite values may have left fp32 as well.) ----
__device__ __forceinline__ bf16x8 without_nonfinite(const bf16x8 &v, bf16x8 &marks, bool &any)
{
    u32x4 w = __builtin_bit_cast(u32x4, v), m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = (w[i] & 0x7f80u) == 0x7f80u, hi = (w[i] & 0x7f800000u) == 0x7f800000u;
        m[i] = (lo ? 0x3f80u : 0u) | (hi ? 0x3f800000u : 0u);
        w[i] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
        any |= lo | hi;
    }
    marks = __builtin_bit_cast(bf16x8, m);
    return __builtin_bit_cast(bf16x8, w);
}
// Y += A P for NK K-steps of one channel block, A read transposed; seen: a word for each 32 rows, shifted by 4 h.
template <int D, int NK>
__device__ __forceinline__ void careful_product(f32x16 &y, const TileReader<D> &rd, uint32_t tile, int db, int ks0, const bf16x8 *p, const uint32_t *seen)
{
    f32x16 count = zeros16();
#pragma unroll
    for (int k = 0; k < NK; ++k) {
        bool any = false;
        bf16x8 marks;
        const bf16x8 a = without_nonfinite(rd.transposed(tile, db, ks0 + k), marks, any);
        y = mfma(a, p[k], y);
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = (seen_bit(seen[k / 2], 8 * (k % 2) + 2 * i) & 0x3f80u) | (seen_bit(seen[k / 2], 8 * (k % 2) + 2 * i + 1) & 0x3f800000u);
        count = mfma(marks, __builtin_bit_cast(bf16x8, v), count);
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) y[j] = count[j] > 0.f ? __builtin_nanf("") : y[j];
}

// Whether a sum of the lane is not finite: 0 times an infinity or NaN is NaN.
template <int N> __device__ __forceinline__ bool not_finite(const f32x16 (&a)[N])
{
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) sum[j & 3] = fmaf(a[i][j], 0.f, sum[j & 3]);
    return !((sum[0] + sum[1]) + (sum[2] + sum[3]) == 0.f);
}
// Whether that is so anywhere in the workgroup: its walk is then repeated with care, and what it has stored stored again.  LDS is free when this
// is called, and when it returns.
__device__ __forceinline__ bool repeat(bool bad, uint32_t lds)
{
    typedef __attribute__((address_space(3))) uint32_t *lds_u1;
    typedef __attribute__((address_space(3))) u32x4 *lds_w4;
    const uint32_t any = __any(bad);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) *reinterpret_cast<lds_u1>(lds + (threadIdx.x >> 4)) = any;
    __syncthreads();
    const u32x4 w = *reinterpret_cast<lds_w4>(lds);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(w[0] | w[1] | w[2] | w[3]) != 0;
}

// Workgroup -> (slot, query head or key head): heads fastest, a group's key head fastest of all, so that the tiles that read the same
// keys run on the same die (workgroups go to the dies in turn) and meet in its L2; the longest walks first.
__device__ __forceinline__ void split_block(uint32_t id, uint32_t heads_kv, uint32_t per_kv, uint32_t &slot, uint32_t &kv, uint32_t &sub)
{
    kv = id % heads_kv;
    sub = (id / heads_kv) % per_kv;
    slot = id / (heads_kv * per_kv);
}

}  // namespace attn
}  // namespace kda
