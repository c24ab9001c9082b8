// Attention of the newest tokens over a paged cache of e4m3 codes with a scale for each page and head.
//
// A step is 32 keys of one key head for 16 or 32 rows (new tokens x query heads of the group) in one wave and without LDS:
//
//     X^T [key, row] = K Q^T            A: codes widened to bf16 (exact), a lane 8 channels of a key at a time,     B: the rows, in registers
//     O^T [channel, row] += V^T P^T     A: codes of 8 keys' same channel,                                         B: X's accumulators as they stand
//
// 16x16x32 bf16 MFMAs.  A contraction may take its indices in any order that both operands share: keys go to the second product in the
// order in which a lane's accumulators hold them, {4 g + 0..3, 16 + 4 g + 0..3} (g = lane / 16), and channels to the first so that a lane
// reads whole 32-byte pieces of a key.  V is read by rows, 8 channels of 8 keys a lane, and its bytes are regrouped in registers.  Scales
// multiply the 16 logits and numerators of their page, in fp32, so that they may be any numbers.  Statistics as in the prefill: fp32,
// the maximum moved when it is passed by more than 8.  Terms of up to 2^8 times a scale, summed over up to 2^30 keys, leave fp32 where the
// result does not: the logits of a page whose values' scale is 2^64 or more count 64 more to the maximum, so that no term times its scale is
// beyond 2^72.
//
// What bounds it is reading the cache, 2 D bytes a key and head: 256 sequences of 4 096 to 8 192 tokens, 8 heads of 128, in 560 us (5.7 TB/s;
// plain reads of 1 to 4 GiB reach 6.7 to 7.0), 4 sequences of up to 131 072 in 135 us (5.1 TB/s), one of 2 000 in 9.5 us, launches and the
// latency of two steps.  Every wave has a stretch of its own of a sequence's visible keys; the
// next step's codes are in flight while one is worked on.  The four waves of a workgroup join through LDS, the workgroups of a
// sequence and head (as many as fill the device) through the workspace and a second kernel, in a fixed order.
#include "kda_cache.h"
#include "kda_cache_join.h"
#include "kda_tree.h"

namespace kda {
namespace cache {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
constexpr int kStep = 32;            // keys of a step

// A call of kda_cache_tree_attn whose rows are few (a type of its own: its parts are this file's steps).
struct FewRows : TreeAttend {};

// Places that a sequence's tokens take, the new ones among them.
__device__ __forceinline__ int32_t places(const Cache &c, const Attend &, int n) { return c.lens[n]; }
__device__ __forceinline__ int32_t places(const Cache &c, const FewRows &a, int n)
{
    const int32_t held = c.lens[n];
    return held < 0 ? -1 : min(held, 1 << 30) + a.tokens;
}

// The visible keys of a sequence's new tokens as steps: those of the sinks where the window begins behind them, then the window's.
struct Steps {
    int32_t len, low;                // keys; first step of the window
    int32_t sink_steps, count;
};
template <typename A> __device__ __forceinline__ Steps steps_of(const Cache &c, const A &a, int n)
{
    const int32_t most = c.max_pages << c.page_log2, l = places(c, a, n);    // (below 2^31)
    Steps s;
    s.len = l < 0 ? 0 : min(l, most);
    // the first new token's window begins at l - tokens - window + 1
    s.low = a.window && l >= a.tokens && l - a.tokens >= a.window ? (l - a.tokens - a.window + 1) / kStep : 0;
    const int32_t high = (s.len + kStep - 1) / kStep;
    s.low = min(s.low, high);
    s.sink_steps = min(s.low, (a.sinks + kStep - 1) / kStep);
    s.count = high - s.low + s.sink_steps;
    return s;
}
// steps of one wave: as many as the others', and none where it has none left
__device__ __forceinline__ int32_t wave_steps(const Steps &s, int splits) { return (s.count + splits * kWaves - 1) / (splits * kWaves); }

__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t x = i ? b : a;
        w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
        w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true));
    }
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ f32x4 mfma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// value of the lanes 16 and 32 away: reductions over the keys of a row
template <typename F> __device__ __forceinline__ float over_groups(float v, F f)
{
    v = f(v, __shfl_xor(v, 16));
    return f(v, __shfl_xor(v, 32));
}

// RB: blocks of 16 rows.  More than 32 rows go to several workgroups, side by side, which meet in the L2: 64 sequences of up to 8192 tokens,
// 64 rows, 225 us with two of 32, 334 with four of 16; with one of 64 most of its values stand in scratch (1922).
//
// The new tokens of a draft tree (FewRows) see of the places from qfirst on their own lines alone, and stand at the position of their depth.
//
// kFine: the softmax's terms go to the product with V as two bf16, p + rest, of which 2^-16 is left out.  A tree's results in fp32 take that, and of heads of 128 those in bf16
// too, which it costs nothing: 64 sequences of up to 8 000 tokens, 16 rows, 156 us either way, 1.7 10^-3 off in the mean square in place of 2.2; but heads of 64, 32 rows, 93
// with one bf16 and 105 with two.  kda_cache_attn rounds its terms to bf16.
template <int D, int RB, bool kFine, typename A> __device__ __forceinline__ void attend(const Cache &c, const A &a)
{
    constexpr bool kTree = !__is_same(A, Attend);
    constexpr int KW = D / 64;                               // 16-byte pieces of a key that a lane reads
    constexpr int VW = D / 64;                               // dwords of a key's values that a lane reads
    constexpr int CB = D / 16;                               // blocks of 16 channels
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), x = lane & 15, g = lane >> 4;
    uint32_t id = blockIdx.x;
    const int kv = id % c.heads_kv;
    id /= c.heads_kv;
    const int tile = id % a.row_tiles;
    id /= a.row_tiles;
    const int split = id % a.splits, n = id / a.splits;
    const Steps st = steps_of(c, a, n);
    const int32_t per = wave_steps(st, a.splits);
    const int32_t begin0 = (split * kWaves + wave) * per, begin = begin0 < st.count ? begin0 : st.count, end = begin + per < st.count ? begin + per : st.count;
    if (a.splits > 1 && split * kWaves * per >= st.count) return;          // (the join knows)

    // position of the first new token (a sequence of no length has no step)
    const int32_t qfirst = kTree ? max(places(c, a, n) - a.tokens, 0) : max(c.lens[n], 0) - a.tokens;
    // rows of this tile: (token, head of the group)
    bf16x8 qf[RB][D / 32];
    int32_t qpos[RB], row[RB];
    [[maybe_unused]] uint64_t line[RB];
    [[maybe_unused]] bool there[RB];
    [[maybe_unused]] uint64_t mine = 0;                      // lane's token's line
    if constexpr (kTree) mine = tree_line(lane < a.tokens ? a.parents[(int64_t)n * a.tokens + lane] : -2, a.tokens);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        row[r] = (tile * RB + r) * 16 + x;
        const int rr = row[r] < a.rows ? row[r] : a.rows - 1, t = rr / c.group, head = kv * c.group + rr - t * c.group;
        if constexpr (kTree) {
            line[r] = (uint64_t)(uint32_t)__shfl((int)(mine >> 32), t) << 32 | (uint32_t)__shfl((int)mine, t);
            there[r] = line[r] != 0;
            const int32_t depth = __popcll(line[r]) - 1;
            qpos[r] = qfirst + depth;
            if (a.window && a.window < kTreeTokens)
                for (int j = 0; j < a.tokens; ++j) {
                    const int32_t dj = __popcll((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mine, j)) - 1;
                    if (depth - dj >= a.window && qfirst + dj >= a.sinks) line[r] &= ~(1ull << j);
                }
        } else qpos[r] = qfirst + t;
        const uint16_t *from = a.q + ((int64_t)n * a.tokens + t) * a.q_stride + (int64_t)head * D + D / 4 * g;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) qf[r][i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(from + 8 * i));
    }
    const float cs = a.scale * kLog2e;

    f32x4 acc[RB][CB];
    float m[RB], mref[RB], l[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        m[r] = -kInf;
        mref[r] = l[r] = 0.f;
#pragma unroll
        for (int j = 0; j < CB; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // what a lane knows of one 16-key block of the 32 steps at hand: page and scales
    auto first_key = [&](int32_t u) { return (u < st.sink_steps ? u : st.low + u - st.sink_steps) * kStep; };
    int32_t page_l = -1;
    float ks_l = 0.f, vs_l = 0.f;
    auto look_up = [&](int32_t u0) {
        const int32_t u = u0 + lane / 2;
        page_l = -1;
        ks_l = vs_l = 0.f;
        if (u < end) {
            const int32_t key = first_key(u) + 16 * (lane & 1);
            // (a block that no row sees may belong to a page that is another sequence's by now, and its scale be anything)
            const bool hidden = a.window && qfirst - key - 15 >= a.window && key >= a.sinks;
            if (key < st.len && !hidden) page_l = page_at(c, n, key >> c.page_log2);
            if (page_l >= 0) {
                ks_l = c.k_scale[(int64_t)page_l * c.heads_kv + kv];
                vs_l = c.v_scale[(int64_t)page_l * c.heads_kv + kv];
            }
        }
    };
    struct Codes {
        u32x4 k[2][KW];
        u32x2 v[8];                  // (D 64: the first dword alone)
        float ks[2], vs[2];
        int32_t page[2];
    };
    auto fetch = [&](int32_t u, int32_t u0, Codes &w) {
        const int32_t key0 = first_key(u);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int src = 2 * (u - u0) + b;
            w.page[b] = __builtin_amdgcn_readlane(page_l, src);
            const int64_t at = ((int64_t)(w.page[b] < 0 ? 0 : w.page[b]) * c.heads_kv + kv) * c.page_size + ((key0 + 16 * b) & (c.page_size - 1));
            const uint8_t *kp = c.k + (at + x) * D + D / 4 * g;
#pragma unroll
            for (int i = 0; i < KW; ++i) w.k[b][i] = *reinterpret_cast<const u32x4 *>(kp + 16 * i);
            const uint8_t *vp = c.v + (at + 4 * g) * D + D / 16 * x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (VW == 2) w.v[4 * b + i] = *reinterpret_cast<const u32x2 *>(vp + i * D);
                else w.v[4 * b + i][0] = *reinterpret_cast<const uint32_t *>(vp + i * D);
            }
        }
        // (behind the codes' loads, which need the pages alone)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int src = 2 * (u - u0) + b;
            w.ks[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks_l), src));
            w.vs[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs_l), src));
        }
    };
    auto work = [&](int32_t u, Codes &w) {
        const int32_t key0 = first_key(u);
        // some row does not see some key, or there is none
        const bool edge = key0 + kStep - 1 + (kTree ? 1 : 0) > qfirst || (a.window && qfirst + a.tokens - 1 - key0 >= a.window) || w.page[0] < 0 || w.page[1] < 0;
        // logits of all rows, then their terms, then the values: K's and V's widened codes are not held at once
        f32x4 s[RB][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            bf16x8 kf[D / 32];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) kf[i] = widen(w.k[b][i / 2][2 * (i % 2)], w.k[b][i / 2][2 * (i % 2) + 1]);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                s[r][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < D / 32; ++i) s[r][b] = mfma(kf[i], qf[r][i], s[r][b]);
                s[r][b] *= cs * w.ks[b];
            }
        }
        uint32_t seen[RB];
        bool odd = false;                                    // a code that is not a number, on a step that not every row sees whole
        if (edge) {
#pragma unroll
            for (int r = 0; r < RB; ++r) seen[r] = 0;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t key = key0 + 16 * b + 4 * g + i;
                    const bool none = w.page[b] < 0 || key >= st.len;
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        const bool near = a.window == 0 || qpos[r] - key < a.window || key < a.sinks;
                        bool ok;
                        if constexpr (kTree) ok = !none && there[r] && (key < qfirst ? near : (line[r] >> ((key - qfirst) & 63)) & 1);
                        else ok = !none && key <= qpos[r] && near;
                        s[r][b][i] = ok ? s[r][b][i] : -kInf;
                        seen[r] |= (ok ? 1u : 0u) << (4 * b + i);
                    }
#pragma unroll
                    for (int d = 0; d < VW; ++d) {
                        const uint32_t y = none ? 0u : w.v[4 * b + i][d];
                        w.v[4 * b + i][d] = y;
                        odd |= ((((y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0);
                    }
                }
        }
        const bool careful = edge && __any(odd);
        const bool large = (__float_as_uint(w.vs[0]) & 0x7fffffffu) >= kLargeScale || (__float_as_uint(w.vs[1]) & 0x7fffffffu) >= kLargeScale;
        const float lift = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(large ? kLift : 0.f)));
        bf16x8 pb[RB];
        [[maybe_unused]] bf16x8 rest[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float top = s[r][0][0];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[r][b][i]);
            top += lift;
            if (__any(top > m[r] + 8.f)) {
                top = over_groups(top, [](float p, float q) { return fmaxf(p, q); });
                const float mn = fmaxf(m[r], top), f = mn == -kInf ? 1.f : fast_exp2(m[r] - mn);
                m[r] = mn;
                mref[r] = mn == -kInf ? 0.f : mn;
                l[r] *= f;
#pragma unroll
                for (int j = 0; j < CB; ++j) acc[r][j] *= f;
            }
            float p[8];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[4 * b + i] = fast_exp2(s[r][b][i] - mref[r]);
                    l[r] += p[4 * b + i];
                    p[4 * b + i] *= w.vs[b];
                }
            u32x4 pw;
#pragma unroll
            for (int i = 0; i < 4; ++i) pw[i] = pack_bf16x2(p[2 * i], p[2 * i + 1]);
            pb[r] = __builtin_bit_cast(bf16x8, pw);
            if constexpr (kFine) {
#pragma unroll
                for (int i = 0; i < 4; ++i) pw[i] = pack_bf16x2(p[2 * i] - __uint_as_float(pw[i] << 16), p[2 * i + 1] - __uint_as_float(pw[i] & 0xffff0000u));
                rest[r] = __builtin_bit_cast(bf16x8, pw);
            }
        }
        // V^T: channel D/16 x + j of keys 4 g + 0..3 and 16 + 4 g + 0..3, two channels at a time
        auto channels = [&](int d, int half, u32x4 (&two)[2]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t pair = __builtin_amdgcn_perm(w.v[2 * e + 1][d], w.v[2 * e][d], half ? 0x07030602u : 0x05010400u);
                two[0][e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pair, 1.f, false));
                two[1][e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pair, 1.f, true));
            }
        };
        if (!careful) {
#pragma unroll
            for (int j = 0; j < CB; j += 2) {
                u32x4 two[2];
                channels(j / 4, j / 2 & 1, two);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        acc[r][j + i] = mfma(__builtin_bit_cast(bf16x8, two[i]), pb[r], acc[r][j + i]);
                        if constexpr (kFine) acc[r][j + i] = mfma(__builtin_bit_cast(bf16x8, two[i]), rest[r], acc[r][j + i]);
                    }
            }
        } else {
            // such a code leaves the product, and the rows that see it become NaN
#pragma unroll
            for (int j = 0; j < CB; j += 2) {
                u32x4 two[2];
                channels(j / 4, j / 2 & 1, two);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    u32x4 y = two[i], marks;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool lo = (y[e] & 0x7f80u) == 0x7f80u, hi = (y[e] & 0x7f800000u) == 0x7f800000u;
                        marks[e] = (lo ? 0x3f80u : 0u) | (hi ? 0x3f800000u : 0u);
                        y[e] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
                    }
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        u32x4 ones;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            ones[e] = ((seen[r] >> (2 * e)) & 1u ? 0x3f80u : 0u) | ((seen[r] >> (2 * e + 1)) & 1u ? 0x3f800000u : 0u);
                        acc[r][j + i] = mfma(__builtin_bit_cast(bf16x8, y), pb[r], acc[r][j + i]);
                        if constexpr (kFine) acc[r][j + i] = mfma(__builtin_bit_cast(bf16x8, y), rest[r], acc[r][j + i]);
                        const f32x4 count = mfma(__builtin_bit_cast(bf16x8, marks), __builtin_bit_cast(bf16x8, ones), f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[r][j + i][e] = count[e] > 0.f ? __builtin_nanf("") : acc[r][j + i][e];
                    }
                }
            }
        }
    };
    if (begin < end) {
        int32_t u0 = begin;
        look_up(u0);
        Codes w[2];
        fetch(begin, u0, w[0]);
        for (int32_t u = begin; u < end; u += 2) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (u + s >= end) break;
                if (u + s + 1 < end) {
                    if (u + s + 1 - u0 == 32) {
                        u0 += 32;
                        look_up(u0);
                    }
                    fetch(u + s + 1, u0, w[s ^ 1]);
                }
                work(u + s, w[s]);
            }
        }
    }

    if constexpr (kTree) {
        // (rows of nobody, whatever steps that every row sees whole have left in them)
#pragma unroll
        for (int r = 0; r < RB; ++r)
            if (!there[r]) {
                m[r] = -kInf;
                l[r] = 0.f;
#pragma unroll
                for (int j = 0; j < CB; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
    }

    // ---- the four waves' parts: a row's maximum, sum and numerators' sums ----
    constexpr int kPitch = D + 4;
    extern __shared__ __align__(16) float lds[];             // [2][16 RB][D + 4] and [2][16 RB][2]
    float *stats = lds + 2 * 16 * RB * kPitch;
#pragma unroll
    for (int r = 0; r < RB; ++r) l[r] = over_groups(l[r], [](float p, float q) { return p + q; });
    auto leave = [&](int at) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float *to = lds + (at * 16 * RB + 16 * r + x) * kPitch + D / 4 * g;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < CB; j += 4) *reinterpret_cast<f32x4 *>(to + CB * i + j) = f32x4{acc[r][j][i], acc[r][j + 1][i], acc[r][j + 2][i], acc[r][j + 3][i]};
            if (g == 0) {
                stats[(at * 16 * RB + 16 * r + x) * 2] = m[r];
                stats[(at * 16 * RB + 16 * r + x) * 2 + 1] = l[r];
            }
        }
    };
    auto join = [&](int at) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float *from = lds + (at * 16 * RB + 16 * r + x) * kPitch + D / 4 * g;
            const float mo = stats[(at * 16 * RB + 16 * r + x) * 2], lo = stats[(at * 16 * RB + 16 * r + x) * 2 + 1];
            const float mn = fmaxf(m[r], mo), f0 = m[r] == -kInf ? 0.f : fast_exp2(m[r] - mn), f1 = mo == -kInf ? 0.f : fast_exp2(mo - mn);
            // (a part that saw nothing adds nothing; one that is NaN stays so)
            l[r] = l[r] * f0 + lo * f1;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < CB; j += 4) {
                    const f32x4 y = *reinterpret_cast<const f32x4 *>(from + CB * i + j);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][j + e][i] = acc[r][j + e][i] * f0 + y[e] * f1;
                }
            m[r] = mn;
        }
    };
    if (wave >= 2) leave(wave - 2);
    __syncthreads();
    if (wave < 2) join(wave);
    __syncthreads();
    if (wave == 1) leave(0);
    __syncthreads();
    if (wave) return;
    join(0);

#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (row[r] >= a.rows) continue;
        if (a.splits > 1) {
            const int64_t part = (((int64_t)n * c.heads_kv + kv) * a.splits + split) * a.rows + row[r];
            float *to = a.part + part * D + D / 4 * g;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < CB; j += 4) *reinterpret_cast<f32x4 *>(to + CB * i + j) = f32x4{acc[r][j][i], acc[r][j + 1][i], acc[r][j + 2][i], acc[r][j + 3][i]};
            if (g == 0) {
                a.stats[part * 2] = m[r];
                a.stats[part * 2 + 1] = l[r];
            }
            continue;
        }
        const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
        const int t = row[r] / c.group, head = kv * c.group + row[r] - t * c.group;
        const int64_t out = (((int64_t)n * a.tokens + t) * c.heads_q + head) * D + D / 4 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < CB; j += 4) {
                const f32x4 y = f32x4{acc[r][j][i], acc[r][j + 1][i], acc[r][j + 2][i], acc[r][j + 3][i]} * inv;
                if (a.out_bf16) *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.o) + out + CB * i + j) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
                else *reinterpret_cast<f32x4 *>(static_cast<float *>(a.o) + out + CB * i + j) = y;
            }
    }
}

template <int D, int RB> __global__ __launch_bounds__(64 * kWaves, 2) void kda_cache_attn_kernel(const Cache c, const Attend a) { attend<D, RB, false>(c, a); }
template <int D, int RB> __global__ __launch_bounds__(64 * kWaves, 2) void kda_cache_few_kernel(const Cache c, const FewRows a) { attend<D, RB, D == 128>(c, a); }
template <int D, int RB> __global__ __launch_bounds__(64 * kWaves, 2) void kda_cache_few_fine_kernel(const Cache c, const FewRows a) { attend<D, RB, true>(c, a); }

// parts of a sequence and head that hold something
template <typename A> __device__ __forceinline__ int32_t parts_of(const Cache &c, const A &a, int n)
{
    const Steps st = steps_of(c, a, n);
    const int32_t per = wave_steps(st, a.splits) * kWaves;
    return per ? (st.count + per - 1) / per : 0;
}
__device__ __forceinline__ int32_t used_parts(const Cache &c, const Attend &a, int n) { return parts_of(c, a, n); }
__device__ __forceinline__ int32_t used_parts(const Cache &c, const FewRows &a, int n) { return parts_of(c, a, n); }

}  // namespace cache
}  // namespace kda

using namespace kda;
using namespace kda::cache;

namespace kda {

// Workgroups of a sequence and head's keys: enough for two on every compute unit, each of its waves with two steps at least, and one,
// without a join, where six steps do.  us with one / two / four on every compute unit: 8 sequences of 4 096 tokens x 8 heads 17.7 / 17.5 / 20.4,
// 16 of 8 192 x 4 new tokens 31.1 / 25.4 / 24.5, 32 of 4 096 36.4 / 37.8 / 39.0; with one / two / four steps at least: one sequence of 2 000
// 9.6 / 9.9 / 11.2, of 8 192 12.8 / 11.2 / 11.7; with two steps at least / six without a join: of 300 9.8 / 6.9, of 700 10.1 / 9.2.
int32_t cache_attn_splits(const Cache &c, int64_t pairs, int64_t most_keys, int64_t window, int32_t sinks, int32_t tokens)
{
    int64_t keys = most_keys;
    if (window && window + tokens + sinks + 2 * kStep < keys) keys = window + tokens + sinks + 2 * kStep;
    const int64_t steps = (keys + kStep - 1) / kStep, most = steps <= 6 * kWaves ? 1 : (steps + 2 * kWaves - 1) / (2 * kWaves),
                  want = (512 + pairs - 1) / (pairs > 0 ? pairs : 1);
    const int64_t n = want < most ? want : most;
    return (int32_t)(n < 1 ? 1 : n);
}
// Of a tree's few rows; and where that would leave parts of more than 16 384 keys, parts of about 4 096 and up to 2 048 workgroups, as in
// cache_tree_splits.  us without / with that, four new tokens, 32 heads over 8: 64 sequences of 32 000 583 / 579, one in 64 so long and the others of 500 to
// 2 000 269 / 105, one in eight 392 / 190; 16 of 100 000 451 / 473, one in eight 311 / 131.
int32_t cache_few_splits(const Cache &c, int64_t pairs, int64_t most_keys, int64_t window, int32_t sinks, int32_t tokens)
{
    const int64_t n = cache_attn_splits(c, pairs, most_keys, window, sinks, tokens);
    int64_t keys = most_keys;
    if (window && window + tokens + sinks + 2 * kStep < keys) keys = window + tokens + sinks + 2 * kStep;
    if (keys <= 16384 * n || 2048 / pairs <= n) return (int32_t)n;
    const int64_t want = (keys + 4095) / 4096;
    return (int32_t)(want < 2048 / pairs ? want : 2048 / pairs);
}

namespace {
template <int D, int RB> void launch_rows(const Cache &c, const Attend &a, dim3 grid, size_t lds, hipStream_t st)
{
    hipLaunchKernelGGL((kda_cache_attn_kernel<D, RB>), grid, dim3(64 * kWaves), lds, st, c, a);
}
template <int D, int RB> void launch_rows(const Cache &c, const FewRows &a, dim3 grid, size_t lds, hipStream_t st)
{
    if constexpr (D == 64)
        if (!a.out_bf16) {
            hipLaunchKernelGGL((kda_cache_few_fine_kernel<D, RB>), grid, dim3(64 * kWaves), lds, st, c, a);
            return;
        }
    hipLaunchKernelGGL((kda_cache_few_kernel<D, RB>), grid, dim3(64 * kWaves), lds, st, c, a);
}
template <int D, int RB, typename A> hipError_t launch(const Cache &c, const A &a, hipStream_t st)
{
    const uint32_t grid = (uint32_t)c.num_seqs * c.heads_kv * a.row_tiles * a.splits;
    launch_rows<D, RB>(c, a, dim3(grid), 2 * 16 * RB * (D + 4 + 2) * 4, st);
    return hipGetLastError();
}
template <int D, typename A> hipError_t launch(const Cache &c, const A &a, hipStream_t st)
{
    hipError_t e;
    if constexpr (__is_same(A, FewRows) && D == 128) e = launch<D, 1>(c, a, st);           // (cache_few_rows)
    else e = a.row_tiles == 1 && a.rows <= 16 ? launch<D, 1>(c, a, st) : launch<D, 2>(c, a, st);
    if (e == hipSuccess && a.splits > 1) {
        const int64_t items = (int64_t)c.num_seqs * c.heads_kv * a.rows;
        e = launch_join<D>(c, a, items, st);
    }
    return e;
}
}  // namespace

kda_status cache_attn_dispatch(const Cache &c, const Attend &a, int dim, hipStream_t st)
{
    const hipError_t e = dim == 128 ? launch<128>(c, a, st) : launch<64>(c, a, st);
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_cache_attn: %s", hipGetErrorString(e));
}

// Rows of a key head up to which a draft tree's tokens come here, where keys go from memory to registers, and not to tiles that waves share through LDS
// (kda_cache_tree.hip).  us here / there: heads of 64, 32 rows, 64 sequences of up to 8 000 tokens 83 / 124, one of 2 000 11.8 / 11.5, one of 300 8.4 / 11.0; heads of
// 128, 16 rows, the same 155 / 165, 11.9 / 12.6 and 7.8 / 11.8, but 32 rows 173 / 165, 14.5 / 12.8 and 10.9 / 12.0.
int32_t cache_few_rows(int dim) { return dim == 64 ? 32 : 16; }

kda_status cache_few_dispatch(const Cache &c, const TreeAttend &tree, int dim, hipStream_t st)
{
    FewRows a;
    static_cast<TreeAttend &>(a) = tree;
    const hipError_t e = dim == 128 ? launch<128>(c, a, st) : launch<64>(c, a, st);
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_cache_tree_attn: %s", hipGetErrorString(e));
}

}  // namespace kda
