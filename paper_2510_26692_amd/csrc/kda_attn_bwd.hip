// Softmax attention, backward pass.  With P_ij = exp(x_ij - lse_i), x_ij = scale q_i . k_j, and the row sums d_i = do_i . o_i:
//
//     dV_j = sum_i P_ij do_i,     dS_ij = P_ij (do_i . v_j - d_i),     dQ_i = scale sum_j dS_ij k_j,     dK_j = scale sum_i dS_ij q_i
//
// Two walks: over the keys of 128 queries (dQ; it leaves d behind) and over the queries of 128 keys (dK, dV).  Each forms P and dS for
// itself: 7 products where one walk would need 5, but no sum is shared between workgroups, so that there are no atomics and the order
// of every sum is fixed.  A key head's gradients sum over its group's query heads inside a workgroup; where that leaves too few
// workgroups, over parts of the group, whose fp32 sums a last kernel adds.  The sinks' keys are seen by every later query: what lies beyond
// their window is walked by workgroups of its own, in parts.
//
// What bounds it is the matrix cores: 16 384 tokens x 16 heads of 128 causal in 3 550 us, 775 TFLOP/s for the 5 products that a gradient
// needs and 1 084 for the 7 done; 4 x 4 096 x 16 heads over 4 in 985 us (698 and 977), 29 of them for the sums of the parts.  A window of
// 1024 costs a fifth more a visible pair (65 536 x 16 heads over 2, 2 130 us): every walk has two partly seen ends.
#include <algorithm>
#include <type_traits>

#include "kda_attn_tile.h"

namespace kda {
namespace attn {

// What the backward pass has beyond the shape.
struct Back {
    const uint16_t *q, *k, *v, *o, *d_o;
    const float *lse;
    float *stats;                    // [2][B,Hq,T]: lse log2 e (+inf for a row that sees nothing), and d
    uint16_t *dq, *dk, *dv;
    float *part_k, *part_v;          // [splits][tokens][Hk][D] fp32, or with `heads_only` [num_seqs][64][Hk][D]
    float *sink_k, *sink_v;          // [sink_slots][2][splits][Hk][64][D] fp32
    int32_t splits;                  // parts that a group's heads are cut into
    int32_t sink_slots, sink_tiles;  // parts of the sinks' walks: how many, and tiles of 64 queries each
    int32_t sink_parts;              // of a sequence of a fixed batch; 0: packed
    bool direct;                     // nothing to be summed: gradients are written as they are
    bool heads_only;                 // nothing but the sinks' walks' parts, of each sequence's first 64 keys
};
// elements of one part of dK or dV
__device__ __forceinline__ int64_t part_size(const Shape &s, int d) { return (s.cu ? s.tokens : s.tokens * s.num_seqs) * s.heads_kv * d; }
__device__ __forceinline__ int64_t stats_size(const Shape &s) { return (s.cu ? s.tokens : s.tokens * s.num_seqs) * s.heads_q; }
// tiles of 64 queries that the first key tile's own walk covers
__device__ __forceinline__ int first_walk_tiles(const Shape &s, int len)
{
    const int all = (len + kTile - 1) / kTile, own = s.window ? (kCols + s.window - 2) / kTile + 1 : all;
    return own < all ? own : all;
}

// dQ of 128 queries.  Returns true where the walk has to be repeated with care.
template <int D, bool kCareful> __device__ __forceinline__ bool dq_tile(const Shape &s, const Back &g, const uint32_t lds)
{
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, x = lane & 31, h = lane >> 5;
    uint32_t slot, kv, sub;
    split_block(blockIdx.x, s.heads_kv, s.group, slot, kv, sub);
    const int head = kv * s.group + sub;
    const Place at = place_of(s, s.slots - 1 - slot, s.window != 0);
    if (at.first >= at.len || at.first < 0) return false;

    const int wq0 = at.first + 32 * wave;
    const int query = wq0 + x, last = min(at.first + kCols - 1, at.len - 1);
    const int wlast = wq0 > last ? -1 : min(wq0 + 31, last);
    const int64_t token = at.row0 + (query < at.len ? query : at.len - 1), stat = ((int64_t)at.batch * (s.heads_q - 1) + head) * s.tokens + token;

    bf16x8 qf[D / 16], df[D / 16];
    float delta = 0.f;
    {
        const uint16_t *qrow = g.q + token * s.q_stride + (int64_t)head * D + 8 * h;
        const int64_t row = (token * s.heads_q + head) * D + 8 * h;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            qf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qrow + 16 * i));
            const u32x4 dw = *reinterpret_cast<const u32x4 *>(g.d_o + row + 16 * i), ow = *reinterpret_cast<const u32x4 *>(g.o + row + 16 * i);
            df[i] = __builtin_bit_cast(bf16x8, dw);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float a, b, u, w;
                unpack_bf16x2(dw[e], a, b);
                unpack_bf16x2(ow[e], u, w);
                delta = fmaf(a, u, fmaf(b, w, delta));
            }
        }
    }
    delta += other_half(delta);
    const float lse = g.lse[stat], lse2 = lse == -kInf ? kInf : lse * kLog2e;

    arrived(qf);
    arrived(df);
    TileReader<D> rd;
    rd.init(lane);
    TileLoader<D> lk, lv;
    const uint32_t ks_bytes = s.k_stride * 2, vs_bytes = s.v_stride * 2;
    lk.init(wave, lane, ks_bytes);
    lv.init(wave, lane, vs_bytes);
    const uint16_t *kh = g.k + at.row0 * s.k_stride + (int64_t)kv * D, *vh = g.v + at.row0 * s.v_stride + (int64_t)kv * D;
    constexpr uint32_t kT = kTileBytes<D>;
    const int low = s.window && at.first >= s.window ? (at.first - s.window + 1) / kTile : 0, high = last / kTile;
    const int sink_first = s.sinks > 0 && low > 0, steps = high - low + 1 + sink_first;
    const float c = s.scale * kLog2e;
    auto first_key = [&](int it) { return (sink_first ? (it == 0 ? 0 : low + it - 1) : low + it) * kTile; };
    auto issue = [&](int it, uint32_t buf) {
        const int k0 = first_key(it);
        lk.issue(lds + 2 * buf * kT, wave, rows_descriptor(kh + k0 * s.k_stride, at.len - k0, ks_bytes));
        lv.issue(lds + (2 * buf + 1) * kT, wave, rows_descriptor(vh + k0 * s.v_stride, at.len - k0, vs_bytes));
    };

    // The sum of a row's dS is zero but for what o's rounding took from d: added to d, it gives the dK / dV walk the d of the unrounded o
    // (errors of dK 2.5e-3 to 2.8e-3 without, 2.4e-3 with).
    float rest = 0.f;
    f32x16 acc[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = zeros16();
    issue(0, 0);
    auto step = [&](int it, auto parity, auto sums_only) {
        constexpr int P = decltype(parity)::value;
        constexpr bool kSumsOnly = decltype(sums_only)::value;
        tile_barrier();
        if (it + 1 < steps) issue(it + 1, P ^ 1);
        const int k0 = first_key(it);
        const uint32_t kt = lds + 2 * P * kT, vt = kt + kT;
        if (k0 > wlast || (s.window && k0 + kTile - 1 <= wq0 - s.window && k0 >= s.sinks)) return;
        const bool edge = k0 + kTile - 1 > wq0 || (s.window && wq0 + 31 - k0 >= s.window);
        Seen seen;
        if (edge) {
            seen = seen_keys(query, k0, s.window, s.sinks);
            seen.w[0] >>= 4 * h;
            seen.w[1] >>= 4 * h;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            rd.forget();
            f32x16 st = zeros16(), dp = zeros16();
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                st = mfma(rd.rows(kt, b, i), qf[i], st);
                dp = mfma(rd.rows(vt, b, i), df[i], dp);
            }
            reads_ahead<8, 1, D / 8, D / 8>();
            float e[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) e[j] = fast_exp2(fmaf(st[j], c, -lse2)) * (dp[j] - delta);
            if (edge) {
#pragma unroll
                for (int j = 0; j < 16; ++j) e[j] = where_seen(seen_bit(seen.w[b], j), e[j], 0.f);
            }
            float four[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) four[j] = (e[j] + e[4 + j]) + (e[8 + j] + e[12 + j]);
            rest += (four[0] + four[1]) + (four[2] + four[3]);
            if constexpr (kSumsOnly) continue;
            const bf16x8 ds[2] = {pack8(e), pack8(e + 8)};
            if (kCareful && edge) {
#pragma unroll
                for (int db = 0; db < D / 32; ++db) careful_product<D, 2>(acc[db], rd, kt, db, 2 * b, ds, seen.w + b);
            } else {
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                    for (int db = 0; db < D / 32; ++db) acc[db] = mfma(rd.transposed(kt, db, 2 * b + ks), ds[ks], acc[db]);
                reads_ahead<8, 2, D / 8, D / 16>();
            }
        }
    };
    using First = std::integral_constant<int, 0>;
    using Second = std::integral_constant<int, 1>;
    // In a row that sees few keys d is as large as do . v, and o's rounding in it as large as that of dS.  Where all rows see few, in a
    // short walk or with a small window, d is summed from P and do . v first.  dQ at 2 x 200 tokens: 2.7e-3 off without, 2.4e-3 with, for 0.4 us;
    // with a window of 16 2.5e-3 and 2.35e-3, 16 384 tokens x 16 heads 202 and 217 us; of 64 2.4e-3 and 2.35e-3, 252 and 280 us.
    if (steps <= 2 || (s.window && s.window <= kCols)) {
        delta = 0.f;
        for (int it = 0; it < steps; it += 2) {
            step(it, First{}, std::true_type{});
            if (it + 1 < steps) step(it + 1, Second{}, std::true_type{});
        }
        delta = rest + other_half(rest);
        rest = 0.f;
        if (steps > 2) {                                     // (else both tiles are there still)
            tile_barrier();
            issue(0, 0);
        }
    }
    for (int it = 0; it < steps; it += 2) {
        step(it, First{}, std::false_type{});
        if (it + 1 < steps) step(it + 1, Second{}, std::false_type{});
    }
    rest += other_half(rest);
    // (formed again: held through the walk these would take registers from it)
    int again = tid;
    asm volatile("" : "+v"(again));
    const int mine = wq0 + (again & 31);
    const bool bad = !kCareful && not_finite(acc);
    if (mine < at.len) {
        const int64_t place = at.row0 + mine;
        g.stats[((int64_t)at.batch * (s.heads_q - 1) + head) * s.tokens + place + (again & 32 ? stats_size(s) : 0)] = again & 32 ? delta + rest : lse2;
        uint16_t *out = g.dq + (place * s.heads_q + head) * D + (again & 32) / 8;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const u32x2 y = {pack_bf16x2(acc[db][4 * b] * s.scale, acc[db][4 * b + 1] * s.scale),
                                 pack_bf16x2(acc[db][4 * b + 2] * s.scale, acc[db][4 * b + 3] * s.scale)};
                *reinterpret_cast<u32x2 *>(out + 32 * db + 8 * b) = y;
            }
    }
    return !kCareful && repeat(bad, lds);
}
// The walk with care is a call at d 128, where in line it takes registers from the loop that always runs (spilled in line: dQ 13, dK / dV 94; none
// as calls); at d 64 there are enough (dQ 2, dK / dV none), and the call's stack costs more.  us in line / called, d 64: 8 x 4096 x 32 heads 2 119 /
// 2 128, 2 x 200 x 4 heads 20.7 / 20.9; d 128: 4 x 4096 x 16 heads over 4 996 / 985.
template <int D> __device__ __noinline__ void dq_tile_again(const Shape s, const Back g, const uint32_t lds) { dq_tile<D, true>(s, g, lds); }
template <int D> __global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void kda_attn_dq_kernel(const Shape s, const Back g)
{
    constexpr uint32_t lds = kLds;
    if (!dq_tile<D, false>(s, g, lds)) return;
    if constexpr (D == 128) dq_tile_again<D>(s, g, lds);
    else dq_tile<D, true>(s, g, lds);
}

// dK and dV of 128 keys, or (the first workgroups) the sinks' part of a sequence's first 64, each half of the waves on every other tile of
// queries.
//
// At d 128 a wave's sums take 128 registers, K 32 and a block's X and dP 32 more: two waves a SIMD have no room for V, which is read from LDS
// as the tiles are, and the tiles are of 32 queries, so that V, Q and dO of two workgroups fit a compute unit.
template <int D> struct DkvLayout {
    static constexpr bool kVInLds = D == 128;
    static constexpr int kRows = D == 128 ? 32 : 64;         // queries of a tile
    static constexpr uint32_t kT = kRows * D * 2, kBuf = 2 * kT + 2 * 64 * 4;          // Q, dO, lse and d
    static constexpr uint32_t kV = 2 * kBuf;
    static constexpr uint32_t kBytes = kV + (kVInLds ? 2 * kTileBytes<D> : 0);
};
template <int D, bool kCareful> __device__ __forceinline__ bool dkv_tile(const Shape &s, const Back &g, const uint32_t lds)
{
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, x = lane & 31, h = lane >> 5;
    uint32_t slot, kv, sub;
    const uint32_t sink_blocks = (uint32_t)g.sink_slots * s.heads_kv * g.splits;
    const bool sink = blockIdx.x < sink_blocks;
    split_block(sink ? blockIdx.x : blockIdx.x - sink_blocks, s.heads_kv, g.splits, slot, kv, sub);
    const int heads = s.group / g.splits, head0 = kv * s.group + sub * heads;
    using L = DkvLayout<D>;
    constexpr int kRows = L::kRows;
    constexpr uint32_t kT = L::kT, kBuf = L::kBuf;
    Place at;
    int tile0, tiles;                                        // of queries
    if (sink) {
        int32_t part;
        if (g.sink_parts) {
            at = {(int64_t)(slot / g.sink_parts) * s.tokens, (int32_t)s.tokens, 0, (int32_t)(slot / g.sink_parts), (int32_t)(slot / g.sink_parts)};
            part = slot % g.sink_parts;
        } else {
            const int64_t per = (int64_t)kTile * g.sink_tiles;               // (slots as in place_of)
            int lo = 0, hi = s.num_seqs - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (cu_at(s, mid) / per + mid <= (int64_t)slot) lo = mid; else hi = mid - 1;
            }
            const int64_t a = cu_at(s, lo), e = cu_at(s, lo + 1), p = (int64_t)slot - (a / per + lo);
            if (p < 0) return false;
            at = {a, (int32_t)(e - a), 0, 0, lo};
            part = (int32_t)p;
        }
        if (at.len <= 0) return false;
        const int all = (at.len + kTile - 1) / kTile, from = first_walk_tiles(s, at.len) + part * g.sink_tiles, n = min(all - from, g.sink_tiles);
        if (n <= 0) return false;
        tile0 = from * kTile / kRows;
        tiles = n * kTile / kRows;
    } else {
        at = place_of(s, slot, false);
        if (at.first >= at.len || at.first < 0) return false;
        const int last = s.window ? min(at.first + kCols + s.window - 2, at.len - 1) : at.len - 1;
        tile0 = at.first / kRows;
        tiles = last / kRows - tile0 + 1;
        if (at.first == 0 && s.sinks) tiles = first_walk_tiles(s, at.len) * (kTile / kRows);          // (the sinks' walks begin behind them)
    }
    const int kw0 = at.first + 32 * (sink ? wave & 1 : wave), key = kw0 + x;
    const int64_t token = at.row0 + (key < at.len ? key : at.len - 1);

    bf16x8 kf[D / 16], vf[L::kVInLds ? 1 : D / 16];
    {
        const uint16_t *krow = g.k + token * s.k_stride + (int64_t)kv * D + 8 * h, *vrow = g.v + token * s.v_stride + (int64_t)kv * D + 8 * h;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            kf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(krow + 16 * i));
            if constexpr (!L::kVInLds) vf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(vrow + 16 * i));
        }
    }
    if constexpr (L::kVInLds) {
        TileLoader<D> lv;
        lv.init(wave, lane, s.v_stride * 2);
        const uint16_t *vh = g.v + (at.row0 + at.first) * s.v_stride + (int64_t)kv * D;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            lv.issue(lds + L::kV + i * kTileBytes<D>, wave, rows_descriptor(vh + i * kTile * s.v_stride, at.len - at.first - i * kTile, s.v_stride * 2));
    }
    const uint32_t vt = lds + L::kV + ((kw0 - at.first) / kTile) * kTileBytes<D>;         // the wave's 32 rows of V: block vb of this tile
    const int vb = ((kw0 - at.first) / 32) & 1;
    arrived(kf);
    if constexpr (!L::kVInLds) arrived(vf);
    TileReader<D> rd;
    rd.init(lane);
    TileLoader<D, kRows> lq, ld;
    const int64_t do_stride = (int64_t)s.heads_q * D;
    lq.init(wave, lane, s.q_stride * 2);
    ld.init(wave, lane, do_stride * 2);
    const float c = s.scale * kLog2e;
    const int steps = tiles * heads;

    int issue_head = 0, issue_tile = 0;                                  // the step to be issued next: (head, tile), tiles fastest
    auto issue = [&](uint32_t parity) {
        const int head = head0 + issue_head;
        const int q0 = (tile0 + issue_tile) * kRows, rows = at.len - q0;
        const uint32_t buf = lds + parity * kBuf;
        lq.issue(buf, wave, rows_descriptor(g.q + (at.row0 + q0) * s.q_stride + (int64_t)head * D, rows, s.q_stride * 2));
        ld.issue(buf + kT, wave, rows_descriptor(g.d_o + (at.row0 + q0) * do_stride + (int64_t)head * D, rows, do_stride * 2));
        if (wave < 2) {                                      // lse, then d: 64 values each
            const float *p = g.stats + (wave ? stats_size(s) : 0) + ((int64_t)at.batch * (s.heads_q - 1) + head) * s.tokens + at.row0 + q0;
            dma4(__builtin_amdgcn_readfirstlane(buf + 2 * kT + wave * 64 * 4), lane * 4, rows_descriptor(p, rows, 4));
        }
        if (++issue_tile == tiles) { issue_tile = 0; ++issue_head; }
    };

    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dk[db] = dv[db] = zeros16();
    issue(0);
    int tile = 0;
    for (int it = 0; it < steps; ++it) {
        tile_barrier();
        if (it + 1 < steps) issue((it + 1) & 1);
        const int q0 = (tile0 + tile) * kRows;
        if (++tile == tiles) tile = 0;
        const uint32_t qt = lds + (uint32_t)(it & 1) * kBuf, dt = qt + kT, stats = qt + 2 * kT;
        if (sink && (int)(it & 1) != wave >> 1) continue;
        if (kw0 >= at.len || q0 + kRows - 1 < kw0 || (s.window && q0 - (kw0 + 31) >= s.window && kw0 >= s.sinks)) continue;
        const bool edge = q0 < kw0 + 31 || (s.window && q0 + kRows - 1 - kw0 >= s.window);
        // the key is seen by its own query and later ones, to the window's end
        Seen seen;
        if (edge) {
            const int32_t last = s.window && key >= s.sinks ? key + s.window - 1 - q0 : kTile;
            seen = seen_rows(key - q0, last);
            seen.w[0] >>= 4 * h;
            seen.w[1] >>= 4 * h;
        }
#pragma unroll
        for (int b = 0; b < kRows / 32; ++b) {
            if constexpr (D == 128) rd.forget();
            f32x16 st = zeros16(), dp = zeros16();
#pragma unroll
            for (int i = 0; i < D / 16; ++i) st = mfma(rd.rows(qt, b, i), kf[i], st);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                if constexpr (L::kVInLds) dp = mfma(rd.rows(dt, b, i), rd.rows(vt, vb, i), dp);
                else dp = mfma(rd.rows(dt, b, i), vf[i], dp);
            }
            bf16x8 pb[2], ds[2];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                typedef __attribute__((address_space(3))) const f32x4 *lds_f4;
                float p[8], e[8];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t row = stats + (32 * b + 16 * ks + 8 * u + 4 * h) * 4;
                    const f32x4 ls = *reinterpret_cast<lds_f4>(row);
#pragma unroll
                    for (int j = 0; j < 4; ++j) p[4 * u + j] = fast_exp2(fmaf(st[8 * ks + 4 * u + j], c, -ls[j]));
                    const f32x4 de = *reinterpret_cast<lds_f4>(row + 64 * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[4 * u + j] = p[4 * u + j] * (dp[8 * ks + 4 * u + j] - de[j]);
                }
                if (edge) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t bit = seen_bit(seen.w[b], 8 * ks + j);
                        p[j] = where_seen(bit, p[j], 0.f);
                        e[j] = where_seen(bit, e[j], 0.f);
                    }
                }
                pb[ks] = pack8(p);
                ds[ks] = pack8(e);
            }
            if (kCareful && edge) {
#pragma unroll
                for (int db = 0; db < D / 32; ++db) {
                    careful_product<D, 2>(dv[db], rd, dt, db, 2 * b, pb, seen.w + b);
                    careful_product<D, 2>(dk[db], rd, qt, db, 2 * b, ds, seen.w + b);
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                    for (int db = 0; db < D / 32; ++db) {
                        dv[db] = mfma(rd.transposed(dt, db, 2 * b + ks), pb[ks], dv[db]);
                        dk[db] = mfma(rd.transposed(qt, db, 2 * b + ks), ds[ks], dk[db]);
                    }
                reads_ahead<8, 2, D / 4, D / 8>();
            }
        }
    }
    int again = tid;                                         // (as in dq_tile)
    asm volatile("" : "+v"(again));
    const bool bad = !kCareful && (not_finite(dk) || not_finite(dv));
    const int mine = kw0 + (again & 31), half = again & 32;
    if (sink || mine < at.len) {
        const int seq = !sink && g.heads_only && kw0 < kTile ? place_of(s, slot, false).seq : 0;         // (found again, as above)
        const int64_t row = ((at.row0 + mine) * s.heads_kv + kv) * D;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int ch = 32 * db + 8 * b + half / 8;
                f32x4 yk, yv;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    yk[j] = dk[db][4 * b + j] * s.scale;
                    yv[j] = dv[db][4 * b + j];
                }
                if (sink) {
                    const int64_t w = ((((int64_t)slot * 2 + (wave >> 1)) * g.splits + sub) * s.heads_kv + kv) * kTile * D + (int64_t)mine * D + ch;
                    *reinterpret_cast<f32x4 *>(g.sink_k + w) = yk;
                    *reinterpret_cast<f32x4 *>(g.sink_v + w) = yv;
                } else if (g.direct || (g.heads_only && kw0 >= kTile)) {
                    const u32x2 wk = {pack_bf16x2(yk[0], yk[1]), pack_bf16x2(yk[2], yk[3])}, wv = {pack_bf16x2(yv[0], yv[1]), pack_bf16x2(yv[2], yv[3])};
                    *reinterpret_cast<u32x2 *>(g.dk + row + ch) = wk;
                    *reinterpret_cast<u32x2 *>(g.dv + row + ch) = wv;
                } else {
                    const int64_t w = (g.heads_only ? (((int64_t)seq * kTile + mine) * s.heads_kv + kv) * D : (int64_t)sub * part_size(s, D) + row) + ch;
                    *reinterpret_cast<f32x4 *>(g.part_k + w) = yk;
                    *reinterpret_cast<f32x4 *>(g.part_v + w) = yv;
                }
            }
    }
    return !kCareful && repeat(bad, lds);
}
template <int D> __device__ __noinline__ void dkv_tile_again(const Shape s, const Back g, const uint32_t lds) { dkv_tile<D, true>(s, g, lds); }
template <int D> __global__ __launch_bounds__(kThreads, 2) void kda_attn_dkv_kernel(const Shape s, const Back g)
{
    constexpr uint32_t lds = kLds;
    if (!dkv_tile<D, false>(s, g, lds)) return;
    if constexpr (D == 128) dkv_tile_again<D>(s, g, lds);
    else dkv_tile<D, true>(s, g, lds);
}

// Sums of the parts: a thread has four channels of a token and key head.  Places of a sequence's first 64 keys stand one sequence after the
// other where nothing else is to be summed, else items are tokens.
template <int D> __device__ __forceinline__ void join_four(const Shape &s, const Back &g, int64_t i)
{
    const int64_t row = i / ((int64_t)D * s.heads_kv), inner = i - row * (int64_t)D * s.heads_kv;
    int64_t index, first;                                    // in the sequence, and the sequence's first token
    int64_t len = s.tokens;
    int seq;
    if (g.heads_only) {
        seq = (int)(row / kTile);
        index = row - (int64_t)seq * kTile;
        first = s.cu ? cu_at(s, seq) : (int64_t)seq * s.tokens;
        if (s.cu) len = cu_at(s, seq + 1) - first;
        if (index >= len) return;
    } else if (s.cu) {
        int lo = 0, hi = s.num_seqs - 1;
        if (row < cu_at(s, 0) || row >= cu_at(s, s.num_seqs)) return;            // owned by no sequence
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (cu_at(s, mid) <= row) lo = mid; else hi = mid - 1;
        }
        seq = lo;
        first = cu_at(s, lo);
        index = row - first;
        len = cu_at(s, lo + 1) - first;
    } else {
        seq = (int)(row / s.tokens);
        first = (int64_t)seq * s.tokens;
        index = row - first;
    }
    f32x4 yk = {0.f, 0.f, 0.f, 0.f}, yv = yk;
    for (int p = 0; p < g.splits; ++p) {
        const int64_t w = p * part_size(s, D) + i;
        yk += *reinterpret_cast<const f32x4 *>(g.part_k + w);
        yv += *reinterpret_cast<const f32x4 *>(g.part_v + w);
    }
    if (g.sink_slots && index < kTile) {
        const int64_t first_slot = s.cu ? first / ((int64_t)kTile * g.sink_tiles) + seq : (int64_t)seq * g.sink_parts;
        const int64_t left = (len + kTile - 1) / kTile - first_walk_tiles(s, (int)len), parts = (left + g.sink_tiles - 1) / g.sink_tiles;
        const int64_t kv = inner / D, step = (int64_t)s.heads_kv * kTile * D;
        const int64_t w = (first_slot * 2 * g.splits * s.heads_kv + kv) * kTile * D + index * D + (inner - kv * D);
#pragma unroll 8
        for (int64_t p = 0; p < parts * 2 * g.splits; ++p) {
            yk += *reinterpret_cast<const f32x4 *>(g.sink_k + w + p * step);
            yv += *reinterpret_cast<const f32x4 *>(g.sink_v + w + p * step);
        }
    }
    const int64_t out = (first + index) * (int64_t)D * s.heads_kv + inner;
    const u32x2 wk = {pack_bf16x2(yk[0], yk[1]), pack_bf16x2(yk[2], yk[3])}, wv = {pack_bf16x2(yv[0], yv[1]), pack_bf16x2(yv[2], yv[3])};
    *reinterpret_cast<u32x2 *>(g.dk + out) = wk;
    *reinterpret_cast<u32x2 *>(g.dv + out) = wv;
}
template <int D>
__global__ __launch_bounds__(256) void kda_attn_join_kernel(const Shape s, const Back g, int64_t rows)
{
    const int64_t all = rows * s.heads_kv * D, step = (int64_t)gridDim.x * 1024;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < all; i += step) join_four<D>(s, g, i);
}

}  // namespace attn

using namespace attn;

// Where things stand in the workspace.
namespace {
struct Plan {
    int32_t splits, sink_slots, sink_tiles, sink_parts;
    bool direct, heads_only;
    int64_t part_rows;
    size_t sink_k, sink_v, part_k, part_v, total;
};
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
int64_t rows_of(const Shape &s) { return s.cu ? s.tokens : s.tokens * s.num_seqs; }

Plan plan_of(const Shape &s, int dim)
{
    Plan p{};
    // Workgroups of the dK / dV walk: two for each place (two a compute unit), so that the second fills in behind walks that end early; more
    // cost their fp32 sums.  Backward pass in us with 512 / 1024 / 2048: 4 x 4096 x 16 heads over 4 causal 1104 / 962 / 985, 32768 x 16 heads
    // over 4, d 64, window 256 342 / 338 / 424.
    const int64_t want = 1024;
    p.splits = 1;
    while (p.splits < s.group && (s.group % p.splits || (int64_t)s.slots * s.heads_kv * p.splits < want)) ++p.splits;
    if (s.sinks) {
        // as many tiles as the window's walk of another workgroup, and 8 at least
        const int64_t tiles = (s.window + kCols) / kTile;
        p.sink_tiles = (int32_t)(tiles < 8 ? 8 : tiles > (1 << 20) ? 1 << 20 : tiles);
        const int64_t per = (int64_t)kTile * p.sink_tiles, parts = (s.tokens + per - 1) / per;
        p.sink_parts = s.cu ? 0 : (int32_t)parts;
        p.sink_slots = (int32_t)(s.cu ? s.tokens / per + s.num_seqs : parts * s.num_seqs);
    }
    p.direct = p.splits == 1 && !s.sinks;
    p.heads_only = p.splits == 1 && s.sinks && (int64_t)s.num_seqs * kTile <= rows_of(s);          // (many short sequences have fewer tokens)
    p.part_rows = p.direct ? 0 : p.heads_only ? (int64_t)s.num_seqs * kTile : rows_of(s);
    size_t at = up256((size_t)rows_of(s) * s.heads_q * 4 * 2);
    const size_t part = up256((size_t)p.splits * p.part_rows * s.heads_kv * dim * 4);
    const size_t sink = up256((size_t)p.sink_slots * 2 * p.splits * s.heads_kv * kTile * dim * 4);
    p.part_k = at;
    p.part_v = at += part;
    p.sink_k = at += part;
    p.sink_v = at += sink;
    p.total = at + sink;
    return p;
}

template <int D> hipError_t launch_bwd(const Shape &s, Back g, const Plan &p, hipStream_t st)
{
    constexpr int kLds = 4 * kTileBytes<D>, kLdsStats = DkvLayout<D>::kBytes;
    static_assert(kLds <= 80 << 10 && kLdsStats <= 80 << 10, "two workgroups a compute unit");
    hipLaunchKernelGGL(kda_attn_dq_kernel<D>, dim3((uint32_t)s.slots * s.heads_q), dim3(kThreads), kLds, st, s, g);
    const uint32_t per_slot = (uint32_t)s.heads_kv * p.splits;
    hipLaunchKernelGGL(kda_attn_dkv_kernel<D>, dim3(((uint32_t)s.slots + p.sink_slots) * per_slot), dim3(kThreads), kLdsStats, st, s, g);
    if (!p.direct) {
        const int64_t threads = p.part_rows * s.heads_kv * (D / 4);
        hipLaunchKernelGGL(kda_attn_join_kernel<D>, dim3((uint32_t)std::min<int64_t>((threads + 255) / 256, 1 << 20)), dim3(256), 0, st, s, g, p.part_rows);
    }
    return hipGetLastError();
}
}  // namespace

size_t attn_bwd_workspace(const Shape &s, int dim) { return plan_of(s, dim).total; }

kda_status attn_bwd_dispatch(const Shape &s, int dim, const void *q, const void *k, const void *v, const void *o, const float *lse, const void *d_o,
                             void *dq, void *dk, void *dv, void *workspace, hipStream_t st)
{
    const Plan p = plan_of(s, dim);
    uint8_t *w = static_cast<uint8_t *>(workspace);
    auto in = [](const void *x) { return static_cast<const uint16_t *>(x); };
    auto at = [&](size_t off) { return reinterpret_cast<float *>(w + off); };
    const Back g = {in(q), in(k), in(v), in(o), in(d_o), lse, at(0), static_cast<uint16_t *>(dq), static_cast<uint16_t *>(dk), static_cast<uint16_t *>(dv),
                    at(p.part_k), at(p.part_v), at(p.sink_k), at(p.sink_v), p.splits, p.sink_slots, p.sink_tiles, p.sink_parts, p.direct, p.heads_only};
    const hipError_t e = dim == 128 ? launch_bwd<128>(s, g, p, st) : launch_bwd<64>(s, g, p, st);
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_window_attn_bwd: %s", hipGetErrorString(e));
}

}  // namespace kda
