// Attention of a draft tree's tokens over the paged cache of e4m3 codes.
//
// Rows are (drafted token, query head of the group), 64 or 128 of a key head to a workgroup.  Its four waves bring 64 keys and values
// at a time into LDS, widened to bf16 (exact) on the way, and walk them as the prefill does:
//
//     X^T [key, row] = K Q^T,   P^T = 2^(c X^T - m),   O^T [channel, row] += V^T P^T          (32x32x16 bf16 products, statistics in fp32)
//
// A page's scales are taken by its codes on their way to bf16, which is exact for the powers of two that the append makes; any others are on the logits and
// numerators of its keys, in fp32, with 64 more to the maximum for values with a scale of 2^64 or more (kda_cache_attn.hip).  With 128 rows a wave has 32 of them and all keys of a tile, with 64 half of the keys, and two
// waves' parts meet at the end.  The next tile's codes are on their way into registers while one is worked on, and their pages' numbers a tile
// ahead of that.
//
// What bounds it is no part of it alone: the matrix cores are 39 % busy, vector instructions 41 %, LDS 40 %.  Four sequences of up to 131 072 tokens, 8 key heads,
// trees of 64 tokens and 32 heads, take 535 to 566 us (780 to 820 TFLOP/s of visible pairs; a library product of 8192^3 1 379), 64 of up to 8 192 with 20 to 32 tokens 270
// to 279.  The forward kernel (kda_attn_fwd.hip) has the same products and exponentials at 1 055 TFLOP/s; what this one has beside them is the codes, widened by
// vector instructions and written to LDS, for every 128 rows again.  (Products and exponentials of two blocks of keys issued in turn by one wave take the same time.)
//
// The softmax's terms P are rounded to bf16 ahead of their product with V where the result is bf16: half a step, 2^-8, is what the result's own rounding may be off
// by.  Where it is fp32 they go as two bf16, P = p + rest, of which 2^-16 is left out, and V is multiplied twice.  Off the formulas in 64 bits, in the mean square, and time, for 64
// sequences of up to 8 192 with 20 to 32 tokens: bf16 results 2.3 10^-3 in 272 us (with two 1.7 10^-3 in 369: not taken), fp32 results 4.8 10^-6 in 354 (with one
// 1.6 10^-3 in 277).
//
// A row's token sees what is held (by the window and sinks of its position, len + depth) and its line, a bit for each drafted token; both
// become one word of bits a tile, made only for tiles that some row sees in part.
#include <atomic>
#include <type_traits>

#include "kda_attn_tile.h"
#include "kda_cache.h"
#include "kda_cache_join.h"
#include "kda_tree.h"

namespace kda {
namespace cache {

using attn::bf16x8;
using attn::f32x16;
using attn::TileReader;
using attn::u32x2;
using attn::u32x4;
constexpr int kKeys = 64;            // of a tile
constexpr int kLead = 4;             // operands read ahead of the products that take them

// The visible keys of a sequence's tree as tiles: those of the sinks where the window begins behind them, then the window's and the tree's.
struct Tiles {
    int32_t held, len, low, sink_tiles, count;
};
__device__ __forceinline__ Tiles tiles_of(const Cache &c, const TreeAttend &a, int n)
{
    const int32_t most = c.max_pages << c.page_log2, l = c.lens[n];
    Tiles t = {min(l, 1 << 30), 0, 0, 0, 0};                 // (no table has more)
    if (l < 0) return t;
    t.len = t.held < most - a.tokens ? t.held + a.tokens : most;
    // a token of depth 0 is at position l, and its window begins at l - window + 1
    t.low = a.window && t.held >= a.window ? (t.held - a.window + 1) / kKeys : 0;
    const int32_t high = (t.len + kKeys - 1) / kKeys;
    t.low = min(t.low, high);
    t.sink_tiles = min(t.low, (a.sinks + kKeys - 1) / kKeys);
    t.count = high - t.low + t.sink_tiles;
    return t;
}
__device__ __forceinline__ int32_t part_tiles(const Tiles &t, int splits) { return (t.count + splits - 1) / splits; }
__device__ __forceinline__ int32_t used_parts(const Cache &c, const TreeAttend &a, int n)
{
    const Tiles t = tiles_of(c, a, n);
    const int32_t per = part_tiles(t, a.splits);
    return per ? (t.count + per - 1) / per : 0;
}

// sixteen codes, times a power of two, as two pieces of eight bf16 (exact)
__device__ __forceinline__ void widen16(const u32x4 &w, float scale, u32x4 (&o)[2])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[i / 2][2 * (i % 2)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
        o[i / 2][2 * (i % 2) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
    }
}
// A scale that the codes can take on their way to bf16: a power of two, 2^-60 to 2^60.  (Of those that the append makes, 2^-100 and up, others are those of pages whose
// values are all zeros, below about 2^-52 or above 2^68: their tiles multiply logits and numerators.)
__device__ __forceinline__ bool is_plain(float scale)
{
    const uint32_t b = __float_as_uint(scale);
    return (b & 0x807fffffu) == 0 && b - (67u << 23) <= 120u << 23;
}

// x = p + rest in bf16: p what bf16's bits have of x, rest what is left, rounded (to 2^-16 of x)
__device__ __forceinline__ void two_of(const float *x, bf16x8 &p, bf16x8 &rest)
{
    u32x4 w;
    float r[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = __float_as_uint(x[2 * i]), hi = __float_as_uint(x[2 * i + 1]);
        w[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
        r[2 * i] = x[2 * i] - __uint_as_float(lo & 0xffff0000u);
        r[2 * i + 1] = x[2 * i + 1] - __uint_as_float(hi & 0xffff0000u);
    }
    p = __builtin_bit_cast(bf16x8, w);
    rest = attn::pack8(r);
}
__device__ __forceinline__ bf16x8 held(const bf16x8 &v)
{
    u32x4 w = __builtin_bit_cast(u32x4, v);
    asm volatile("" : "+v"(w));
    return __builtin_bit_cast(bf16x8, w);
}

// LDS: K and V of one tile, then of another; then what the waves share
template <int D> struct Lds {
    static constexpr int kT = kKeys * D * 2;
    static constexpr int kScales = 4 * kT;                   // [2][8] fp32: of the tile's four 16-key blocks, keys and values, what the codes have not taken
    static constexpr int kHave = kScales + 64;               // [2][4] words: the block has a page (1), its codes have taken its scales (2)
    static constexpr int kLine = kHave + 32;                 // [64] of 64 bits
    static constexpr int kBytes = kLine + 512;
};

// The sequence that workgroup `place` of the sequences takes.  Two workgroups or three share a compute unit, and those that a launch begins with are handed out
// round by round: in the first round the longest sequences, in falling order, in the second the next in rising order, and so on, the sums even
// out (64 trees of 32 tokens over 4 096 to 8 192 tokens, 8 heads: 266 us, as they come 285).
constexpr int kOrdered = 256;        // sequences that are ranked
__device__ __forceinline__ int sequence_of(const Cache &c, const TreeAttend &a, int place)
{
    if (!a.per_round) return place;
    extern __shared__ __align__(16) uint8_t lds[];
    int32_t *lens = reinterpret_cast<int32_t *>(lds);
    const int tid = threadIdx.x;
    if (tid < c.num_seqs) lens[tid] = c.lens[tid];
    __syncthreads();
    const int round = place / a.per_round, at = place % a.per_round, in_round = min(a.per_round, c.num_seqs - round * a.per_round);
    const int wanted = round * a.per_round + (round & 1 ? in_round - 1 - at : at);
    if (tid < c.num_seqs) {
        const int32_t mine = lens[tid];
        int rank = 0;
        for (int j = 0; j < c.num_seqs; ++j) rank += lens[j] > mine || (lens[j] == mine && j < tid);
        if (rank == wanted) lens[kOrdered] = tid;
    }
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(lens[kOrdered]);
    __syncthreads();
    return n;
}

// A tile of rows over a split's keys.  Returns true where the walk has to be repeated with care: a value that is not finite stood where some row does
// not see it.
template <int D, int WR, bool kFine, bool kCareful> __device__ __forceinline__ bool tree_tile(const Cache &c, const TreeAttend &a)
{
    constexpr int WK = 4 / WR, KB = 2 / WK;                  // waves along the keys; 32-key blocks of a wave
    constexpr int kT = Lds<D>::kT, kChunks = D / 16, kPieces = kKeys * kChunks / 256;     // 16-code pieces of a key; of a thread, keys or values
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), x = lane & 31, h = lane >> 5;
    const int wr = wave % WR, wk = WK == 1 ? 0 : wave / WR;
    uint32_t id = blockIdx.x;
    const int kv = id % c.heads_kv;
    id /= c.heads_kv;
    const int tile = id % a.row_tiles;
    id /= a.row_tiles;
    const int split = id % a.splits, n = sequence_of(c, a, id / a.splits);
    const Tiles t = tiles_of(c, a, n);
    const int32_t per = part_tiles(t, a.splits), begin = min(split * per, t.count), end = min(begin + per, t.count);
    if (a.splits > 1 && begin >= end) return false;          // (the join knows)

    // ---- the trees' lines, and what the window leaves of them ----
    uint64_t *lines = reinterpret_cast<uint64_t *>(lds + Lds<D>::kLine);
    if (wave == 0) lines[lane] = tree_line(lane < a.tokens ? a.parents[(int64_t)n * a.tokens + lane] : -2, a.tokens);
    __syncthreads();
    const int row0 = (tile * WR + wr) * 32, row = row0 + x;
    const bool working = row0 < a.rows;
    const int rr = min(row, a.rows - 1), tok = rr / c.group, head = kv * c.group + rr - tok * c.group;
    uint64_t line = lines[tok];
    const bool there = line != 0;
    const int32_t depth = __popcll(line) - 1, pos = t.held + depth;
    if (a.window && a.window < kTreeTokens)
        for (int j = 0; j < a.tokens; ++j) {
            const int32_t dj = __popcll(lines[j]) - 1;
            if (depth - dj >= a.window && t.held + dj >= a.sinks) line &= ~(1ull << j);
        }

    // ---- the loader: a wave has 16 keys of a tile, in one page, a thread 16 codes of kPieces of them ----
    const int key_of = 16 * wave + lane / kChunks, chunk = lane % kChunks;
    auto first_key = [&](int32_t u) { return (u < t.sink_tiles ? u : t.low + u - t.sink_tiles) * kKeys; };
    // some row may see some of the wave's keys (others' entries in the table may be another sequence's by now)
    auto sought = [&](int32_t key) -> bool {
        return (key < t.len) & !((a.window != 0) & (t.held - key - 15 >= a.window) & (key >= a.sinks));
    };
    // (Entries are read a tile ahead of their use, and judged then.  Where there is a tile the table has a column, and the pool a page: no load needs a
    // branch.)
    const int32_t *row_of_table = c.table + (int64_t)n * c.max_pages;
    int32_t entry = -1;
    auto look_up = [&](int32_t u) {
        const int32_t key = first_key(u) + 16 * wave;
        entry = row_of_table[sought(key) ? key >> c.page_log2 : 0];
    };
    u32x4 kc[kPieces], vc[kPieces];
    float k_scale = 0.f, v_scale = 0.f;
    int32_t count = 0;                                       // of the wave's keys, how many stand in a page
    const uint32_t in_page = (uint32_t)(lane / kChunks) * D + 16 * chunk;
    auto fetch = [&](int32_t u) {
        const int32_t key = first_key(u) + 16 * wave, e = __builtin_amdgcn_readfirstlane(entry);
        const bool in = sought(key) & (e >= 0) & (e < c.num_pages);
        count = in ? t.len - key : 0;
        const int64_t page = ((int64_t)(in ? e : 0) * c.heads_kv + kv);
        const int64_t at = (page * c.page_size + (key & (c.page_size - 1))) * D;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            kc[j] = *reinterpret_cast<const u32x4 *>(c.k + at + (in_page + j * 1024));
            vc[j] = *reinterpret_cast<const u32x4 *>(c.v + at + (in_page + j * 1024));
        }
        k_scale = c.k_scale[page];
        v_scale = c.v_scale[page];
    };
    auto leave = [&](uint32_t tile_at, int buf) {
        // what stands behind the last token, or in no page of the sequence, may be anything: the product takes zeros
        if (count < 16) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) vc[j][e] = lane / kChunks + j * (64 / kChunks) < count ? vc[j][e] : 0u;
        }
        const float ks = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(k_scale)));
        const float vs = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v_scale)));
        const bool pk = is_plain(ks), pv = is_plain(vs);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int r = key_of + j * (64 / kChunks);
            u32x4 o[2];
            widen16(kc[j], pk ? ks : 1.f, o);
            uint8_t *to = lds + tile_at + r * 2 * D;
#pragma unroll
            for (int e = 0; e < 2; ++e) *reinterpret_cast<u32x4 *>(to + 16 * ((2 * chunk + e) ^ attn::swizzle<D>(r))) = o[e];
            widen16(vc[j], pv ? vs : 1.f, o);
#pragma unroll
            for (int e = 0; e < 2; ++e) *reinterpret_cast<u32x4 *>(to + kT + 16 * ((2 * chunk + e) ^ attn::swizzle<D>(r))) = o[e];
        }
        if (lane == 0) {
            // what is left of the scales
            float *left = reinterpret_cast<float *>(lds + Lds<D>::kScales) + 8 * buf + wave;
            left[0] = pk || count <= 0 ? 1.f : ks;
            left[4] = pv || count <= 0 ? 1.f : vs;
            reinterpret_cast<uint32_t *>(lds + Lds<D>::kHave)[4 * buf + wave] = (count > 0 ? 1u : 0u) | (pk && pv || count <= 0 ? 2u : 0u);
        }
    };

    // ---- the rows ----
    TileReader<D> rd;
    rd.init(lane);
    bf16x8 qf[D / 16];
    {
        const uint16_t *from = a.q + ((int64_t)n * a.tokens + tok) * a.q_stride + (int64_t)head * D + 8 * h;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) qf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(from + 16 * i));
    }
    const float cs = a.scale * kLog2e;
    f32x16 acc[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = attn::zeros16();
    float m = -kInf, mref = 0.f, l = 0.f;

    auto work = [&](int32_t u, auto parity) {
        constexpr int buf = decltype(parity)::value;
        constexpr uint32_t kt = 2 * buf * kT, vt = kt + kT;
        const int32_t k0 = first_key(u);
        f32x16 st[KB];
        // (a wave at its products goes ahead of one at its exponentials: 2 %)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int b = 0; b < KB; ++b) st[b] = attn::zeros16();
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int b = 0; b < KB; ++b) st[b] = attn::mfma(rd.rows(kt, KB * wk + b, i), qf[i], st[b]);
        attn::reads_ahead<kLead, 1, KB * D / 16, KB * D / 16>();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        const u32x4 hv = *reinterpret_cast<const u32x4 *>(lds + Lds<D>::kHave + 16 * buf);
        const uint32_t every = __builtin_amdgcn_readfirstlane(hv[0] & hv[1] & hv[2] & hv[3]);
        // scales that the codes have not taken (of this wave's 16-key blocks)
        typedef float f32xb __attribute__((ext_vector_type(2 * KB)));
        f32xb vs;
        bool large = false;
        if (!(every & 2)) {
            const f32xb ks = *reinterpret_cast<const f32xb *>(lds + Lds<D>::kScales + 32 * buf + 8 * KB * wk);
            vs = *reinterpret_cast<const f32xb *>(lds + Lds<D>::kScales + 32 * buf + 16 + 8 * KB * wk);
#pragma unroll
            for (int b = 0; b < 2 * KB; ++b) large |= (__float_as_uint(vs[b]) & 0x7fffffffu) >= kLargeScale;
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) st[b][j] *= ks[2 * b + j / 8];
        }
        // some row does not see some key
        const bool edge = __builtin_amdgcn_readfirstlane(!(every & 1) || k0 + kKeys - 1 >= t.held || (a.window && t.held + a.tokens - 1 - k0 >= a.window));
        uint32_t seen[KB];
        if (edge) {
            const int32_t node = t.held - k0;                // the row of the first drafted token
            const attn::Seen ctx = attn::seen_rows(a.window ? attn::clamp_tile(pos - a.window + 1 - k0) : 0, attn::clamp_tile(node - 1));
            const attn::Seen sinks = attn::seen_rows(0, attn::clamp_tile(min(a.sinks, t.held) - 1 - k0));
            uint64_t w = ((uint64_t)(ctx.w[1] | sinks.w[1]) << 32) | (ctx.w[0] | sinks.w[0]);
            w |= node >= 64 || node <= -64 ? 0ull : node >= 0 ? line << node : line >> -node;
#pragma unroll
            for (int b = 0; b < 4; ++b) w &= hv[b] & 1 ? ~0ull : ~(0xffffull << (16 * b));
            w = there ? w : 0ull;
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                seen[b] = (uint32_t)(w >> (32 * (KB * wk + b))) >> (4 * h);
#pragma unroll
                for (int j = 0; j < 16; ++j) st[b][j] = attn::where_seen(attn::seen_bit(seen[b], j), st[b][j], -kInf);
            }
        }
        float top = st[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, st[b][j]);
        top = fmaxf(top, attn::other_half(top)) * cs + (large ? kLift : 0.f);
        if (__any(top > m + 8.f)) {
            const float mn = fmaxf(m, top), f = mn == -kInf ? 1.f : fast_exp2(m - mn);
            m = mn;
            mref = mn == -kInf ? 0.f : mn;
            l *= f;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[db][j] *= f;
        }
        bf16x8 p[2 * KB];
        [[maybe_unused]] bf16x8 rest[2 * KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            float e[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                e[j] = fast_exp2(fmaf(st[b][j], cs, -mref));
                l += e[j];
            }
            // (packed on either side of the branch, and held there: values that meet behind it would be moved)
            if constexpr (kFine) {
                if (!(every & 2))
#pragma unroll
                    for (int j = 0; j < 16; ++j) e[j] *= vs[2 * b + j / 8];
#pragma unroll
                for (int i = 0; i < 2; ++i) two_of(e + 8 * i, p[2 * b + i], rest[2 * b + i]);
            } else if (every & 2) {
                p[2 * b] = held(attn::pack8(e));
                p[2 * b + 1] = held(attn::pack8(e + 8));
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) e[j] *= vs[2 * b + j / 8];
                p[2 * b] = attn::pack8(e);
                p[2 * b + 1] = attn::pack8(e + 8);
            }
        }
        if (kCareful && edge) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                attn::careful_product<D, 2 * KB>(acc[db], rd, vt, db, 2 * KB * wk, p, seen);
                if constexpr (kFine) attn::careful_product<D, 2 * KB>(acc[db], rd, vt, db, 2 * KB * wk, rest, seen);
            }
        } else {
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int s = 0; s < 2 * KB; ++s)
#pragma unroll
                for (int db = 0; db < D / 32; ++db) {
                    const bf16x8 v = rd.transposed(vt, db, 2 * KB * wk + s);
                    acc[db] = attn::mfma(v, p[s], acc[db]);
                    if constexpr (kFine) acc[db] = attn::mfma(v, rest[s], acc[db]);
                }
            if constexpr (kFine) attn::reads_ahead<2 * kLead, 1, 2 * KB * D / 16, 2 * KB * D / 16>();
            else attn::reads_ahead<2 * kLead, 2, 2 * KB * D / 16, KB * D / 16>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
        }
    };

    if (begin < end) {
        look_up(begin);
        fetch(begin);
        look_up(min(begin + 1, end - 1));
        auto step = [&](int32_t u, auto parity) {
            constexpr int buf = decltype(parity)::value;
            leave(2 * buf * kT, buf);
            // (behind the last tile it is read again: a branch here would have the compiler move, and so wait for, what was read)
            fetch(min(u + 1, end - 1));
            look_up(min(u + 2, end - 1));
            __syncthreads();
            if (working) work(u, parity);
        };
        int32_t u = begin;
        for (; u + 1 < end; u += 2) {
            step(u, std::integral_constant<int, 0>{});
            step(u + 1, std::integral_constant<int, 1>{});
        }
        if (u < end) step(u, std::integral_constant<int, 0>{});
    }
    l += attn::other_half(l);

    // ---- two waves' parts of the same rows ----
    const bool again = !kCareful && attn::repeat(attn::not_finite(acc), 0);
    if constexpr (WK == 2) {
        __syncthreads();
        f32x4 *at = reinterpret_cast<f32x4 *>(lds) + wr * (D / 32 * 4) * 64 + lane;
        float *stats = reinterpret_cast<float *>(lds + WR * (D / 32 * 4) * 64 * 16) + (wr * 64 + lane) * 2;
        if (wk == 1) {
#pragma unroll
            for (int i = 0; i < D / 32 * 4; ++i) at[64 * i] = f32x4{acc[i / 4][4 * (i % 4)], acc[i / 4][4 * (i % 4) + 1], acc[i / 4][4 * (i % 4) + 2], acc[i / 4][4 * (i % 4) + 3]};
            stats[0] = m;
            stats[1] = l;
        }
        __syncthreads();
        if (wk == 1) return again;
        const float mo = stats[0], lo = stats[1], mn = fmaxf(m, mo);
        // (a part that saw nothing adds nothing; one that is NaN stays so)
        const float f0 = m == -kInf ? 0.f : fast_exp2(m - mn), f1 = mo == -kInf ? 0.f : fast_exp2(mo - mn);
        l = l * f0 + lo * f1;
#pragma unroll
        for (int i = 0; i < D / 32 * 4; ++i) {
            const f32x4 y = at[64 * i];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i / 4][4 * (i % 4) + e] = acc[i / 4][4 * (i % 4) + e] * f0 + y[e] * f1;
        }
        m = mn;
    }
    if (row >= a.rows) return again;
    if (!there || t.held < 0) {                              // (whatever tiles that every row sees whole have left)
        m = -kInf;
        l = 0.f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] = attn::zeros16();
    }
    if (a.splits > 1) {
        const int64_t part = (((int64_t)n * c.heads_kv + kv) * a.splits + split) * a.rows + row;
        float *to = a.part + part * D + 4 * h;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int b = 0; b < 4; ++b) *reinterpret_cast<f32x4 *>(to + 32 * db + 8 * b) = f32x4{acc[db][4 * b], acc[db][4 * b + 1], acc[db][4 * b + 2], acc[db][4 * b + 3]};
        if (h == 0) {
            a.stats[part * 2] = m;
            a.stats[part * 2 + 1] = l;
        }
        return again;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t out = (((int64_t)n * a.tokens + tok) * c.heads_q + head) * D + 4 * h;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 y = f32x4{acc[db][4 * b], acc[db][4 * b + 1], acc[db][4 * b + 2], acc[db][4 * b + 3]} * inv;
            const int64_t w = out + 32 * db + 8 * b;
            if (a.out_bf16) *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.o) + w) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
            else *reinterpret_cast<f32x4 *>(static_cast<float *>(a.o) + w) = y;
        }
    return again;
}
template <int D, int WR, bool kFine> __device__ __noinline__ void tree_tile_again(const Cache c, const TreeAttend a) { tree_tile<D, WR, kFine, true>(c, a); }
template <int D, int WR, bool kFine> __device__ __forceinline__ void tree_rows(const Cache &c, const TreeAttend &a)
{
    if (!tree_tile<D, WR, kFine, false>(c, a)) return;
    __syncthreads();                                         // (LDS is read to the end)
    tree_tile_again<D, WR, kFine>(c, a);
}
// (of heads of 64, three on a compute unit, as cache_tree_splits counts on)
template <int D, int WR>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void kda_cache_tree_kernel(const Cache c, const TreeAttend a) { tree_rows<D, WR, false>(c, a); }
// for results in fp32
template <int D, int WR>
__global__ __launch_bounds__(256, 2) void kda_cache_tree_fine_kernel(const Cache c, const TreeAttend a) { tree_rows<D, WR, true>(c, a); }

}  // namespace cache
}  // namespace kda

using namespace kda;
using namespace kda::cache;

namespace kda {

int32_t cache_tree_tile_rows(int32_t rows) { return rows <= 64 ? 64 : 128; }

// Workgroups of a tile of rows: as many as two on every compute unit hold, or one where that leaves each fewer than five tiles of keys, and each with two at
// least; none is split where one a compute unit has at most 16.  us with two / one on every compute unit (16 tokens x 32 heads over 8): four sequences of 2 000
// tokens 22.4 / 19.6, one of 16 000 22.5 / 21.6, 16 of 8 000 62 / 88; eight of 4 000 with trees of 32 36.3 / 38.7; 32 of 1 000 split in two / whole 34.3 / 27.8.
// A few more than they hold would leave a second round to a few of them: with the count rounded up / down, trees of 32 tokens, five sequences of 2 000 29.5 / 25.8,
// seven of 16 000 90 / 79, 20 of 4 000 82 / 70, 48 of 2 000 111 / 65.
// Of heads of 64 with bf16 results, as many as three on every compute unit hold where each has 16 tiles at least.  us with two / three: four of up to 100 000 with trees of
// 64 tokens 233 / 214, 16 of 8 000 with 64 rows 47 / 43, but eight of 4 000 with 32 28.5 / 33, and, in more than one round, 64 of 8 000 178 / 220.
// Where that would leave parts of more than 256 tiles, parts of about 64 and up to 2 048 workgroups: of a batch one sequence may be long and the others not, which
// only the device knows.  us for 64 sequences of 32 000 / one of them in 64, the others of 500 to 2 000: in 512 workgroups 994 / 784, in 2 048 1 060 / 276; 36 of
// 50 000, one in eight so long, 1 224 / 305; eight of 65 000 to 131 072 with trees of 64 1 058 / 1 005.
int32_t cache_tree_splits(int dim, bool fine, int64_t tiles, int64_t most_keys, int64_t window, int32_t sinks, int32_t tokens)
{
    int64_t keys = most_keys;
    if (window && window + tokens + sinks + 2 * kKeys < keys) keys = window + tokens + sinks + 2 * kKeys;
    const int64_t steps = (keys + kKeys - 1) / kKeys, most = (steps + 1) / 2, all = tiles > 0 ? tiles : 1;
    int64_t n = all < 512 ? 512 / all : 1;
    if (dim == 64 && !fine && 768 / all > n && steps >= 16 * (768 / all)) n = 768 / all;
    if (steps < 5 * n) n = all < 256 ? 256 / all : 1;
    if (all >= 256 && steps <= 16) n = 1;
    if (steps > 256 * n && 2048 / all > n) n = steps / 64 < 2048 / all ? steps / 64 : 2048 / all;
    n = n < most ? n : most;
    return (int32_t)(n < 1 ? 1 : n);
}

namespace {
template <int D, int WR, bool kFine> hipError_t launch(const Cache &c, const TreeAttend &a, hipStream_t st)
{
    constexpr auto kernel = kFine ? &kda_cache_tree_fine_kernel<D, WR> : &kda_cache_tree_kernel<D, WR>;
    const uint32_t grid = (uint32_t)c.num_seqs * c.heads_kv * a.row_tiles * a.splits;
    static std::atomic<bool> raised[64];                                  // per device: a workgroup's LDS passes the runtime's default
    if (Lds<D>::kBytes > 65536) {
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        if (dev < 0 || dev >= 64 || !raised[dev]) {
            e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Lds<D>::kBytes);
            if (e != hipSuccess) return e;
            if (dev >= 0 && dev < 64) raised[dev] = true;
        }
    }
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), Lds<D>::kBytes, st, c, a);
    return hipGetLastError();
}
template <int D> hipError_t launch(const Cache &c, TreeAttend a, hipStream_t st)
{
    // (with a workgroup for each sequence, head and tile of rows, and more than one round of them)
    const int32_t beside = c.heads_kv * a.row_tiles;
    a.per_round = a.splits == 1 && c.num_seqs <= kOrdered && beside <= 256 && c.num_seqs * beside > 256 ? 256 / beside : 0;
    const bool small = cache_tree_tile_rows(a.rows) == 64;
    hipError_t e = a.out_bf16 ? (small ? launch<D, 2, false>(c, a, st) : launch<D, 4, false>(c, a, st)) : small ? launch<D, 2, true>(c, a, st) : launch<D, 4, true>(c, a, st);
    if (e == hipSuccess && a.splits > 1) e = launch_join<D>(c, a, (int64_t)c.num_seqs * c.heads_kv * a.rows, st);
    return e;
}
}  // namespace

kda_status cache_tree_dispatch(const Cache &c, const TreeAttend &a, int dim, hipStream_t st)
{
    const hipError_t e = dim == 128 ? launch<128>(c, a, st) : launch<64>(c, a, st);
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_cache_tree_attn: %s", hipGetErrorString(e));
}

}  // namespace kda
