// Appending keys and values to a paged cache of e4m3 codes, with the position rotation of keys (and queries) on the way.
//
//     k'_t = R(p) k_t at position p = len + t: channel pairs (a, b) -> (a cos - b sin, a sin + b cos), angle p f_i
//     s    = max(s_old, the smallest power of two with |x| <= 448 s for every new x of the page and head)
//     code = e4m3(x / s), older codes of the page rounded again where s grew
//
// Scales are powers of two, so that a page that grows costs its older codes only the bits that fall below the smallest step, however
// often it grows, and every cached value is a bf16 number.  Angles are formed as revolutions in 64 bits, p (f / 2 pi) less its nearest
// whole number: at position 2^31 they are still good to 1e-6, where a product in 32 bits would be off by whole turns.  Their sines and cosines are
// in 64 bits as well for keys, whose codes are those of the exact rotation, and the hardware's of the fp32 revolutions for queries.
//
// A workgroup has one page of one sequence and head, keys or values: rows of 8-channel pieces in registers, one pass for the largest
// value, one for the codes.  Further workgroups turn the queries, a token's angles once for several heads.
#include "kda_cache.h"
#include "kda_rotation.h"

namespace kda {
namespace cache {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int64_t cu_at(const Append &a, int n)
{
    const int64_t v = a.cu[n];
    return v < 0 ? 0 : v < a.tokens ? v : a.tokens;
}

// Which channels the 8-channel piece c of a row turns with, and by which frequencies (revolutions a position).
struct Piece {
    bool on, second, interleaved;    // it is rotated; it is the second half's
    int shift;                       // lanes to the piece of the other half
    int first;                       // its first frequency: interleaved four of them, else eight
    __device__ __forceinline__ void init(const Append &a, int c)
    {
        interleaved = a.interleaved;
        on = 8 * c < 2 * a.n_freq;
        second = !interleaved && 8 * c >= a.n_freq;
        shift = interleaved || !on ? 0 : (second ? -1 : 1) * (a.n_freq / 8);
        first = interleaved ? 4 * c : 8 * c - (second ? a.n_freq : 0);
    }
    // revolutions a position of pair e (0: not rotated)
    __device__ __forceinline__ double frequency(const Append &a, int e) const
    {
        return on ? (double)a.inv_freq[first + (interleaved ? e & 3 : e)] * 0.15915494309189535 : 0.0;
    }
    // The pairs that this lane computes angles of: its four, or half of the eight that it shares with the other half's lane.
    __device__ __forceinline__ void own_frequencies(const Append &a, bool wanted, double (&f)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = wanted ? frequency(a, second ? 4 + e : e) : 0.0;
    }
};
// cos and sin of 2 pi r, |r| <= 1/2: Taylor's series about the nearest quarter, to x^14 and x^13 (2^-46 at pi / 4: one code in 2^40 would differ).
struct Angle { double c, s; };
__device__ __forceinline__ Angle angle64(double r)
{
    const double q = __builtin_rint(4.0 * r), x = (r - 0.25 * q) * 6.283185307179586, y = x * x;
    double c = -1.1470745597729725e-11, s = 1.6059043836821613e-10;                          // -1/14!, 1/13!
    c = fma(c, y, 2.08767569878681e-09);
    s = fma(s, y, -2.505210838544172e-08);
    c = fma(c, y, -2.755731922398589e-07);
    s = fma(s, y, 2.7557319223985893e-06);
    c = fma(c, y, 2.48015873015873e-05);
    s = fma(s, y, -0.0001984126984126984);
    c = fma(c, y, -0.001388888888888889);
    s = fma(s, y, 0.008333333333333333);
    c = fma(c, y, 0.041666666666666664);
    s = fma(s, y, -0.16666666666666666);
    c = fma(c, y, -0.5);
    s = fma(s * y, x, x);
    c = fma(c, y, 1.0);
    const int k = (int)q & 3;
    const double cc = k & 1 ? s : c, ss = k & 1 ? c : s;
    return {k == 1 || k == 2 ? -cc : cc, k & 2 ? -ss : ss};
}
__device__ __forceinline__ Angle operator*(const Angle &a, const Angle &b) { return {fma(a.c, b.c, -a.s * b.s), fma(a.c, b.s, a.s * b.c)}; }

__device__ __forceinline__ double from_lane(double v, int byte)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_ds_bpermute(byte, (uint32_t)b), hi = __builtin_amdgcn_ds_bpermute(byte, (uint32_t)(b >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// The angles of a lane's pairs at a position.  (64-bit operations take about three times the others' time: four angles a lane, the rest
// from the lane that has them.  Every lane takes part.)
__device__ __forceinline__ void angles(const Piece &t, const double (&freq)[4], int64_t pos, double (&cs)[8], double (&sn)[8])
{
    const int from = ((int)(threadIdx.x & 63) + t.shift) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const Angle z = angle64(turns(freq[e], pos));
        const double oc = from_lane(z.c, from), os = from_lane(z.s, from);
        cs[e] = t.second ? oc : z.c;
        sn[e] = t.second ? os : z.s;
        cs[4 + e] = t.second ? z.c : oc;
        sn[4 + e] = t.second ? z.s : os;
    }
}

__device__ __forceinline__ void unpack8(const u32x4 &w, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack_bf16x2(w[i], x[2 * i], x[2 * i + 1]);
}
// The other half's piece, from the lane that has it.  (Every lane takes part.)
__device__ __forceinline__ u32x4 partner(const u32x4 &w, int shift)
{
    u32x4 o;
    const int from = ((int)(threadIdx.x & 63) + shift) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_ds_bpermute(from, w[i]);
    return o;
}
// The piece turned by the angles of its pairs, in T and rounded once to fp32.
template <typename T>
__device__ __forceinline__ void turn(const Piece &t, const T (&cs)[8], const T (&sn)[8], const u32x4 &w, float (&x)[8])
{
    unpack8(w, x);
    if (t.interleaved) {
        if (!t.on) return;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const T a = x[e], b = x[e + 1];
            x[e] = (float)(a * cs[e / 2] - b * sn[e / 2]);
            x[e + 1] = (float)(a * sn[e / 2] + b * cs[e / 2]);
        }
    } else {
        float y[8];
        unpack8(partner(w, t.shift), y);
        if (!t.on) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const T own = (T)x[e] * cs[e], other = (T)y[e] * sn[e];
            x[e] = (float)(t.second ? own + other : own - other);
        }
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&x)[8])
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    return w;
}
// e4m3 codes of eight values, round to nearest even; what is not finite becomes NaN.
__device__ __forceinline__ u32x2 codes8(const float (&x)[8], float inv)
{
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
        w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, r, true);
    }
    return w;
}
// The smallest power of two s >= 2^-100 with top <= 448 s (448 = 1.75 * 2^8); top is finite.
__device__ __forceinline__ float scale_for(float top)
{
    const uint32_t b = __float_as_uint(top);
    int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < 27 ? 27 : e;
    return __uint_as_float((uint32_t)e << 23);
}

// Queries: a token's angles, then its heads.
template <int D, int kThreads> __device__ __forceinline__ void turn_queries(const Cache &c, const Append &a, uint32_t block)
{
    constexpr int kPieces = D / 8, kRows = kThreads / kPieces;           // pieces of a row, rows at a time
    const int tid = threadIdx.x, piece = tid % kPieces, row0 = tid / kPieces;
    const int parts = (c.heads_q + a.q_heads - 1) / a.q_heads;
    Piece t;                                                 // (its loads, one after the other, ahead of the tables')
    t.init(a, piece);
    double freq[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) freq[e] = a.q ? t.frequency(a, e) : 0.0;
    const int64_t item = (int64_t)block * kRows + row0;
    const int64_t token = item / parts;
    const int h0 = (int)(item - token * parts) * a.q_heads;
    int64_t pos = -1;
    if (token < a.tokens) {
        if (a.slots_per_seq) {
            const int n = (int)(token / a.per_seq);
            const int64_t len = c.lens[n];
            if (len >= 0) pos = len + token - n * a.per_seq;
        } else if (token >= cu_at(a, 0) && c.num_seqs && token < cu_at(a, c.num_seqs)) {
            int lo = 0, hi = c.num_seqs - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (cu_at(a, mid) <= token) lo = mid; else hi = mid - 1;
            }
            const int64_t len = c.lens[lo];
            if (len >= 0) pos = len + token - cu_at(a, lo);
        }
    }
    if (pos < 0 && token < a.tokens && (a.zero_q || a.zero_k)) {
        const u32x4 zero = {0, 0, 0, 0};
        if (a.zero_q)
            for (int h = h0; h < h0 + a.q_heads && h < c.heads_q; ++h) *reinterpret_cast<u32x4 *>(a.q_out + (token * c.heads_q + h) * D + 8 * piece) = zero;
        if (a.zero_k && h0 == 0)
            for (int h = 0; h < c.heads_kv; ++h) *reinterpret_cast<u32x4 *>(a.k_out + (token * c.heads_kv + h) * D + 8 * piece) = zero;
    }
    if (!a.q) return;
    const bool in = pos >= 0;
    const uint16_t *from = a.q + (in ? token : 0) * a.q_stride + 8 * piece;
    uint16_t *to = a.q_out + (in ? token : 0) * (int64_t)c.heads_q * D + 8 * piece;
    // (no lane leaves early: the pieces of a row exchange their halves.  The loads of the first heads go ahead of the angles.)
    const int last = c.heads_q - 1;
    u32x4 w[4];
    auto fetch = [&](int h) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (u < a.q_heads) w[u] = *reinterpret_cast<const u32x4 *>(from + (int64_t)min(h + u, last) * D);
    };
    fetch(h0);
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float r = (float)turns(freq[e], pos);
        cs[e] = __builtin_amdgcn_cosf(r);                    // (of 2 pi r)
        sn[e] = __builtin_amdgcn_sinf(r);
    }
    for (int h = h0; h < h0 + a.q_heads; h += 4) {
        u32x4 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = w[u];
        if (h + 4 < h0 + a.q_heads) fetch(h + 4);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u >= a.q_heads) break;                       // (the same for every lane)
            float x[8];
            turn(t, cs, sn, y[u], x);
            if (in && h + u <= last) *reinterpret_cast<u32x4 *>(to + (int64_t)(h + u) * D) = pack8(x);
        }
    }
}

// One page of one sequence, keys or values, `heads` heads of it one after the other.
//
// Angles are held in 64 bits, so that the codes are those of the exact rotation (in 32 bits one in 2^21 was another): computed for the
// lane's first row and for the distance to its next, then multiplied, 4 operations a pair instead of 30, down the rows of one head and up
// those of the next.  16 prompts (67 000 tokens, 8 key heads and 32 query heads, pages of 64; 1.8 GB): 604 us with an angle formed for each
// head, 352 so, 5.1 TB/s (a plain copy: 4.8 to 5.2).  256 sequences x 4 tokens: 20 us with a workgroup a page, head and 4 rows, 11 so, and 23
// where every page's scale grows: its older codes are then read and written again, 8 bytes a lane and one round trip after the other.
template <int D, int kThreads, int kIters>
__device__ __forceinline__ void append_page(const Cache &c, const Append &a, const Piece &t, const double (&freq)[4], bool turned, bool values, int head0, int n,
                                            int64_t logical, int64_t len, int64_t count, int64_t first_row)
{
    constexpr int kPieces = D / 8, kRows = kThreads / kPieces;
    const int tid = threadIdx.x, piece = tid % kPieces, row0 = tid / kPieces;
    const int64_t page0 = logical << c.page_log2;
    const int64_t begin = page0 > len ? page0 : len, end = page0 + c.page_size < len + count ? page0 + c.page_size : len + count;
    if (begin >= end) return;
    const int rows = (int)(end - begin), older = (int)(begin - page0);

    const int64_t row = first_row + begin - len;
    const int64_t stride = values ? a.v_stride : a.k_stride;
    const uint16_t *from = (values ? a.v : a.k) + (row + row0) * stride + (int64_t)head0 * D + 8 * piece;
    // a head's new rows, 16 bytes a lane
    auto fetch = [&](int j, u32x4 (&w)[kIters]) {
#pragma unroll
        for (int i = 0; i < kIters; ++i) {
            w[i] = u32x4{0, 0, 0, 0};
            if (i * kRows + row0 < rows) w[i] = *reinterpret_cast<const u32x4 *>(from + i * kRows * stride + (int64_t)j * D);
        }
    };
    u32x4 w[kIters];
    fetch(0, w);
    const int32_t page = page_at(c, n, logical);
    if (page < 0 && (values || !a.k_out)) return;
    float *scale_at = (values ? c.v_scale : c.k_scale) + (int64_t)page * c.heads_kv + head0;
    uint8_t *codes = (values ? c.v : c.k) + ((int64_t)page * c.heads_kv + head0) * c.page_size * D + 8 * piece;
    const bool has_older = page >= 0 && older;
    float scale_next = has_older ? scale_at[0] : 0.f;

    double cs[8], sn[8], nc[8], ns[8];
    if (turned) {
        angles(t, freq, begin + row0, cs, sn);
        if (kIters > 1 && rows > kRows) angles(t, freq, kRows, nc, ns);
    }
    [[maybe_unused]] __shared__ float tops[2][kThreads / 64];
    if constexpr (kThreads > 64) __syncthreads();            // (of the page before)
    for (int j = 0; j < a.page_heads; ++j) {
        const float scale_old = scale_next;
        float x[kIters][8], top = 0.f;
        if (turned) {
            const bool up = j & 1;
            auto one = [&](int i, bool more) {
                turn(t, cs, sn, w[i], x[i]);
                if (more) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const Angle z = Angle{cs[e], sn[e]} * Angle{nc[e], up ? -ns[e] : ns[e]};
                        cs[e] = z.c;
                        sn[e] = z.s;
                    }
                }
            };
            // (the conditions are the same for every lane)
            if (!up) {
#pragma unroll
                for (int i = 0; i < kIters; ++i)
                    if (i * kRows < rows) one(i, (i + 1) * kRows < rows && i + 1 < kIters);
            } else {
#pragma unroll
                for (int i = kIters - 1; i >= 0; --i)
                    if (i * kRows < rows) one(i, i > 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kIters; ++i)
                if (i * kRows < rows) unpack8(w[i], x[i]);
        }
        if (!values && a.k_out) {
            uint16_t *to = a.k_out + ((row + row0) * c.heads_kv + head0 + j) * D + 8 * piece;
#pragma unroll
            for (int i = 0; i < kIters; ++i)
                if (i * kRows + row0 < rows) *reinterpret_cast<u32x4 *>(to + (int64_t)i * kRows * c.heads_kv * D) = pack8(x[i]);
        }
        if (j + 1 < a.page_heads) {
            fetch(j + 1, w);
            scale_next = has_older ? scale_at[j + 1] : 0.f;
        }
        if (page < 0) continue;
#pragma unroll
        for (int i = 0; i < kIters; ++i)
            if (i * kRows < rows) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = fabsf(x[i][e]);
                    top = fmaxf(top, y < __builtin_huge_valf() ? y : 0.f);
                }
            }
#pragma unroll
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        if constexpr (kThreads > 64) {
            if ((tid & 63) == 0) tops[j & 1][tid >> 6] = top;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kThreads / 64; ++i) top = fmaxf(top, tops[j & 1][i]);
        }
        const float scale = fmaxf(scale_old, scale_for(top)), inv = 1.f / scale;
        uint8_t *to = codes + (int64_t)j * c.page_size * D;
        if (scale > scale_old && older) {
            const float again = scale_old * inv;
            for (int r = row0; r < older; r += kRows) {
                u32x2 *at = reinterpret_cast<u32x2 *>(to + r * D);
                const u32x2 y = *at;
                float z[8];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(y[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(y[i], true);
                    z[4 * i] = lo[0];
                    z[4 * i + 1] = lo[1];
                    z[4 * i + 2] = hi[0];
                    z[4 * i + 3] = hi[1];
                }
                *at = codes8(z, again);
            }
        }
#pragma unroll
        for (int i = 0; i < kIters; ++i)
            if (i * kRows + row0 < rows) *reinterpret_cast<u32x2 *>(to + (older + i * kRows + row0) * D) = codes8(x[i], inv);
        if (tid == 0) scale_at[j] = scale;
    }
}

// The pages of a workgroup: its slot's, for some heads.
template <int D, int kThreads, int kIters>
__device__ __forceinline__ void append_pages(const Cache &c, const Append &a, uint32_t block)
{
    constexpr int kPieces = D / 8;
    const int piece = threadIdx.x % kPieces;
    const bool values = block & 1;
    const int groups = c.heads_kv / a.page_heads, head0 = (int)((block >> 1) % groups) * a.page_heads, slot = (int)((block >> 1) / groups);
    const bool turned = !values && a.n_freq;
    Piece t;                                                 // (its loads, one after the other, ahead of the tables')
    t.init(a, piece);
    double freq[4];
    t.own_frequencies(a, turned, freq);
    int n, index;
    int64_t first_row, count;                                // of the sequence's new tokens
    if (a.slots_per_seq) {
        n = slot;                                            // all pages that the sequence's new tokens touch, or a slot a page
        index = 0;
        if (!a.whole) {
            n = slot / a.slots_per_seq;
            index = slot - n * a.slots_per_seq;
        }
        first_row = n * a.per_seq;
        count = a.per_seq;
    } else {
        // slots from cu[n] / page_size + 2 n on are sequence n's: at least as many as the pages it can touch
        int lo = 0, hi = c.num_seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((cu_at(a, mid) >> c.page_log2) + 2 * mid <= slot) lo = mid; else hi = mid - 1;
        }
        n = lo;
        first_row = cu_at(a, n);
        count = cu_at(a, n + 1) - first_row;
        index = slot - (int)((first_row >> c.page_log2) + 2 * n);
    }
    const int64_t len = c.lens[n];
    if (len < 0 || count <= 0 || index < 0) return;
    const int64_t logical = (len >> c.page_log2) + index;
    if constexpr (kIters == 1) {
        const int pages = a.whole ? (int)(((len + count - 1) >> c.page_log2) - logical) + 1 : 1;
        for (int p = 0; p < pages; ++p)
            append_page<D, kThreads, kIters>(c, a, t, freq, turned, values, head0, n, logical + p, len, count, first_row);
    } else {
        append_page<D, kThreads, kIters>(c, a, t, freq, turned, values, head0, n, logical, len, count, first_row);
    }
}

// Pages, and behind them queries.
template <int D, int kThreads, int kIters>
__global__ __launch_bounds__(kThreads, kIters == 1 ? 3 : 2) void kda_cache_append_kernel(const Cache c, const Append a)
{
    if (blockIdx.x < (uint32_t)a.page_blocks) append_pages<D, kThreads, kIters>(c, a, blockIdx.x);
    else turn_queries<D, kThreads>(c, a, blockIdx.x - a.page_blocks);
}

}  // namespace cache

using namespace cache;

template <int D, int kThreads, int kIters>
static hipError_t launch_append(const Cache &c, Append a, hipStream_t st)
{
    constexpr int kRows = kThreads / (D / 8);
    // Heads that share a lane's angles: as many as leave a wave for each SIMD where a workgroup's rows are few, half as many threads where it
    // has a page.  us with half the threads / these / twice: 256 x 4 tokens, 8 heads 14.1 / 11.4 / 12.9; one prompt of 2048 tokens and 32
    // query heads 17.5 / 16.6 / 18.1, four 40.8 / 40.6 / 43.1.
    constexpr int kEnough = kIters == 1 ? 1 << 16 : 1 << 15;
    a.page_heads = c.heads_kv;
    while (a.page_heads > 1 && (c.heads_kv % a.page_heads || (int64_t)a.slots * (c.heads_kv / a.page_heads) * kThreads < kEnough)) --a.page_heads;
    a.page_blocks = a.slots * (c.heads_kv / a.page_heads) * 2;
    int64_t q_blocks = 0;
    if (a.q || a.zero_k) {
        // several heads a thread share its angles once there are threads enough: 2^17 of them (one prompt of 512 tokens 8.2 us, 8.5 with 2^14;
        // of 2048 16.6 and 20.5; with a head a thread 10 and 29)
        a.q_heads = 1;
        while (a.q_heads < 16 && a.tokens * c.heads_q * (D / 8) / a.q_heads > 1 << 17) a.q_heads *= 2;
        const int64_t items = a.tokens * ((c.heads_q + a.q_heads - 1) / a.q_heads);
        q_blocks = (items + kRows - 1) / kRows;
    }
    if (a.page_blocks + q_blocks > 0)
        hipLaunchKernelGGL((kda_cache_append_kernel<D, kThreads, kIters>), dim3((uint32_t)(a.page_blocks + q_blocks)), dim3(kThreads), 0, st, c, a);
    return hipGetLastError();
}

kda_status cache_append_dispatch(const Cache &c, const Append &a, int dim, hipStream_t st)
{
    // Up to 8 new tokens a sequence: a workgroup holds them all, one row a lane group, whatever pages they fall into.  More: a page's rows
    // by 16 or 32.
    Append b = a;
    const bool few = a.slots_per_seq && a.per_seq <= 8;
    if (few) {
        b.whole = 1;
        b.slots = c.num_seqs;
    }
    hipError_t e;
    if (dim == 128)
        e = few ? (a.per_seq <= 4 ? launch_append<128, 64, 1>(c, b, st) : launch_append<128, 128, 1>(c, b, st))
                : c.page_size == 128 ? launch_append<128, 512, 4>(c, b, st)
                : c.page_size == 64  ? launch_append<128, 256, 4>(c, b, st) : launch_append<128, 256, 2>(c, b, st);
    else
        e = few ? launch_append<64, 64, 1>(c, b, st) : c.page_size == 128 ? launch_append<64, 256, 4>(c, b, st) : launch_append<64, 256, 2>(c, b, st);
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_cache_append: %s", hipGetErrorString(e));
}

}  // namespace kda
