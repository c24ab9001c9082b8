// Softmax attention, forward: o_i = sum_j exp(x_ij - lse_i) v_j over the keys j that query i sees, x_ij = scale q_i . k_j.
//
// One pass over the keys with a running maximum m and sum l per query: a tile of 32 or 64 keys gives X^T = K Q^T, P^T = 2^(X^T c - m)
// (c = scale log2 e, fp32) and O^T = O^T 2^(m_old - m) + V^T P^T, P rounded to bf16 (2^-8 a term at most, the operand type of the
// matrix cores; l sums the unrounded values).  m is moved only when a maximum passes it by more than 8, i.e. terms grow to 2^8 at most,
// which costs no precision and leaves most tiles without the 64 multiplications of O.  Sums of such terms and values of v next to the largest fp32
// leave its range where o does not: the walk is then repeated as for values that are not finite, with P times 2^-38 on its way to the product
// (at most 2^30 terms of at most 2^8: no sum is larger than the largest value).
//
// What bounds it is the matrix cores, at the clock that the power limit leaves them, with the exponentials beside them.  Medians of 7 stretches of 20 runs behind 60
// others (a device that comes from rest takes up to 40 % longer at first): 16 384 tokens x 16 heads of 128 causal in 1 040 us, 1 055 TFLOP/s (a library
// product of 8192^3: 1 251 to 1 304); 4 x 4 096 x 16 heads 275 us (1 000); 65 536 x 16 heads, window 1024, 634 us (860, the visible pairs
// counted); d 64, 8 x 4 096 x 32 heads 661 us (830: as many exponentials for half the product).
// A third buffer of tiles, wave priorities and reads ahead of the products were tried and gave nothing.
#include <type_traits>

#include "kda_attn_tile.h"

namespace kda {
namespace attn {

// Keys of a tile.  At d 64 they are 64, with registers for three waves a SIMD (8 x 4 096 x 32 heads causal 648 us, with two waves 681).  At d 128
// 64 leave two waves, 32 three, whose products and exponentials overlap better, but whose walks have twice the steps.  Side by side, us with 32 / 64: 333
// tokens x 32 heads causal 12.7 / 11.2, 2 000 x 8 53 / 41, 4 x 2 000 x 32 147 / 144, 4 x 4 096 x 16 293 / 295, 16 384 x 16 1 017 / 1 014; with a
// window, whose walks have ends that only some of the waves need, of 512 at 2 000 x 8 22 / 19, at 8 000 x 16 (1 000 workgroups) 55 / 53, at 16 000 x 16 97 /
// 100, of 1 024 at 65 536 x 16 628 / 656, of 2 048 1 085 / 1 112.  So 32 are for a window and more workgroups than this.
constexpr int kMany = 1024;

// o and lse of 128 queries.  Returns true where the walk has to be repeated with care.
template <int D, bool kOutBf16, int kKeys, bool kCareful>
__device__ __forceinline__ bool fwd_tile(const Shape &s, const uint16_t *q, const uint16_t *k, const uint16_t *v, void *o, float *lse, const uint32_t lds)
{
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, x = lane & 31, h = lane >> 5;
    uint32_t slot, kv, sub;
    split_block(blockIdx.x, s.heads_kv, s.group, slot, kv, sub);
    const int head = kv * s.group + sub;
    const Place at = place_of(s, s.slots - 1 - slot, s.window != 0);
    if (at.first >= at.len || at.first < 0) return false;

    const int wq0 = at.first + 32 * wave;                                 // the wave's first query
    const int query = wq0 + x, last = min(at.first + kCols - 1, at.len - 1);
    const int wlast = wq0 > last ? -1 : min(wq0 + 31, last);              // -1: the wave has no query

    TileReader<D> rd;
    rd.init(lane);
    TileLoader<D, kKeys> lk, lv;
    const uint32_t ks_bytes = s.k_stride * 2, vs_bytes = s.v_stride * 2;
    lk.init(wave, lane, ks_bytes);
    lv.init(wave, lane, vs_bytes);
    const uint16_t *kh = k + at.row0 * s.k_stride + (int64_t)kv * D, *vh = v + at.row0 * s.v_stride + (int64_t)kv * D;
    constexpr uint32_t kT = kKeys * D * 2;

    // tiles: that of the sinks, if the window begins behind it, then from the window's first to the last query's
    const int low = s.window && at.first >= s.window ? (at.first - s.window + 1) / kKeys : 0, high = last / kKeys;
    const int sink_steps = min((s.sinks + kKeys - 1) / kKeys, low), steps = high - low + 1 + sink_steps;
    const float c = s.scale * kLog2e;

    auto first_key = [&](int it) { return (it < sink_steps ? it : low + it - sink_steps) * kKeys; };
    // LDS: K and V of one tile, then of another
    auto issue = [&](int it, uint32_t buf) {
        const int k0 = first_key(it);
        lk.issue(lds + 2 * buf * kT, wave, rows_descriptor(kh + k0 * s.k_stride, at.len - k0, ks_bytes));
        lv.issue(lds + (2 * buf + 1) * kT, wave, rows_descriptor(vh + k0 * s.v_stride, at.len - k0, vs_bytes));
    };
    // some query of the wave sees some key of the tile; some does not see some
    auto needed = [&](int k0) { return k0 <= wlast && !(s.window && k0 + kKeys - 1 <= wq0 - s.window && k0 >= s.sinks); };
    auto partial = [&](int k0) { return k0 + kKeys - 1 > wq0 || (s.window && wq0 + 31 - k0 >= s.window); };

    issue(0, 0);
    // Q, B operand: 8 channels 16 s + 8 h .. of the lane's query (a query behind the last reads the last one's)
    bf16x8 qf[D / 16];
    {
        const uint16_t *row = q + (at.row0 + min(query, at.len - 1)) * s.q_stride + (int64_t)head * D + 8 * h;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) qf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(row + 16 * i));
    }
    arrived(qf);

    f32x16 acc[D / 32];
    float m, mref, l;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = zeros16();
    m = -kInf;
    mref = 0.f;
    l = 0.f;
    auto step = [&](int it, auto parity) {
        constexpr int P = decltype(parity)::value;
        tile_barrier();
        if (it + 1 < steps) issue(it + 1, P ^ 1);
        const int k0 = first_key(it);
        const uint32_t kt = lds + 2 * P * kT, vt = kt + kT;
        if (!needed(k0)) return;
        const bool edge = partial(k0);
        f32x16 st[kKeys / 32];
#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b) st[b] = zeros16();
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int b = 0; b < kKeys / 32; ++b) st[b] = mfma(rd.rows(kt, b, i), qf[i], st[b]);
        Seen seen;
        if (edge) {
            seen = seen_keys(query, k0, s.window, s.sinks);
#pragma unroll
            for (int b = 0; b < kKeys / 32; ++b) {
                seen.w[b] >>= 4 * h;
#pragma unroll
                for (int j = 0; j < 16; ++j) st[b][j] = where_seen(seen_bit(seen.w[b], j), st[b][j], -kInf);
            }
        }
        float top = st[0][0];
#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, st[b][j]);
        top = fmaxf(top, other_half(top)) * c;
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
        bf16x8 p[kKeys / 16];
#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b) {
            float e[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                e[j] = fast_exp2(fmaf(st[b][j], c, -mref));
                l += e[j];
                if (kCareful) e[j] *= 0x1p-38f;
            }
            p[2 * b] = pack8(e);
            p[2 * b + 1] = pack8(e + 8);
        }
        if (kCareful && edge) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db) careful_product<D, kKeys / 16>(acc[db], rd, vt, db, 0, p, seen.w);
        } else {
#pragma unroll
            for (int ks = 0; ks < kKeys / 16; ++ks)
#pragma unroll
                for (int db = 0; db < D / 32; ++db) acc[db] = mfma(rd.transposed(vt, db, ks), p[ks], acc[db]);
        }
    };
    int it = 0;
    for (; it + 1 < steps; it += 2) {
        step(it, std::integral_constant<int, 0>{});
        step(it + 1, std::integral_constant<int, 1>{});
    }
    if (it < steps) step(it, std::integral_constant<int, 0>{});

    l += other_half(l);
    // (formed again: held through the walk these would take registers from it)
    int again = tid;
    asm volatile("" : "+v"(again));
    const bool bad = !kCareful && not_finite(acc);
    const int mine = wq0 + (again & 31), half = again & 32;
    if (mine < at.len) {
        const float inv = (l > 0.f ? 1.f / l : l == 0.f ? 0.f : __builtin_nanf("")) * (kCareful ? 0x1p38f : 1.f);
        const int64_t token = at.row0 + mine;
        if (lse && !half) lse[((int64_t)at.batch * (s.heads_q - 1) + head) * s.tokens + token] = l == 0.f ? -kInf : (mref + __log2f(l)) * 0.6931471805599453f;
        const int64_t out = (token * s.heads_q + head) * D + half / 8;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                float e[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) e[j] = acc[db][4 * b + j] * inv;
                const int64_t w = out + 32 * db + 8 * b;
                if constexpr (kOutBf16) {
                    const u32x2 y = {pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3])};
                    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(o) + w) = y;
                } else {
                    const f32x4 y = {e[0], e[1], e[2], e[3]};
                    *reinterpret_cast<f32x4 *>(static_cast<float *>(o) + w) = y;
                }
            }
    }
    return !kCareful && repeat(bad, lds);
}
template <int D, bool kOutBf16, int kKeys>
__device__ __noinline__ void fwd_tile_again(const Shape s, const uint16_t *q, const uint16_t *k, const uint16_t *v, void *o, float *lse, const uint32_t lds)
{
    fwd_tile<D, kOutBf16, kKeys, true>(s, q, k, v, o, lse, lds);
}
template <int D, bool kOutBf16, int kKeys>
__global__ __launch_bounds__(kThreads, D == 128 && kKeys == 64 ? 2 : 3) void kda_attn_fwd_kernel(const Shape s, const uint16_t *q, const uint16_t *k, const uint16_t *v, void *o, float *lse)
{
    constexpr uint32_t lds = kLds;
    if (!fwd_tile<D, kOutBf16, kKeys, false>(s, q, k, v, o, lse, lds)) return;
    fwd_tile_again<D, kOutBf16, kKeys>(s, q, k, v, o, lse, lds);
}

}  // namespace attn
}  // namespace kda

using namespace kda;
using namespace kda::attn;

namespace kda {

template <int D, bool kOutBf16, int kKeys>
static hipError_t launch_fwd(const Shape &s, const void *q, const void *k, const void *v, void *o, float *lse, hipStream_t st)
{
    constexpr int kLds = 4 * kKeys * D * 2;                        // K and V of the tile in work and of the next
    hipLaunchKernelGGL((kda_attn_fwd_kernel<D, kOutBf16, kKeys>), dim3((uint32_t)s.slots * s.heads_q), dim3(kThreads), kLds, st, s,
                       static_cast<const uint16_t *>(q), static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v), o, lse);
    return hipGetLastError();
}
template <bool kOutBf16> static hipError_t launch_fwd(const Shape &s, int dim, const void *q, const void *k, const void *v, void *o, float *lse, hipStream_t st)
{
    if (dim == 64) return launch_fwd<64, kOutBf16, 64>(s, q, k, v, o, lse, st);
    if (s.window && (int64_t)s.slots * s.heads_q > kMany) return launch_fwd<128, kOutBf16, 32>(s, q, k, v, o, lse, st);
    return launch_fwd<128, kOutBf16, 64>(s, q, k, v, o, lse, st);
}

kda_status attn_fwd_dispatch(const Shape &s, int dim, bool out_bf16, const void *q, const void *k, const void *v, void *o, float *lse, hipStream_t st)
{
    const hipError_t e = out_bf16 ? launch_fwd<true>(s, dim, q, k, v, o, lse, st) : launch_fwd<false>(s, dim, q, k, v, o, lse, st);
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_window_attn_fwd: %s", hipGetErrorString(e));
}

}  // namespace kda
