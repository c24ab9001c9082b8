// Rotation of queries and keys by positions of one to four axes, forward and inverse.
//
//     (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = p f,  p the position of the pair's axis, f its frequency
//
// Angles are reduced in 64 bits as revolutions, p (f / 2 pi) less its nearest whole number, then less its nearest quarter; sine and cosine of
// what is left, at most pi / 4, are Taylor's series in fp32 to x^9 and x^10 (2^-29 and 2^-33 there: below fp32's own steps).
//
// What bounds it is moving q and k once: 16 384 tokens, 40 heads of 128 in 68 us, 4.9 TB/s (a plain copy: 4.8).  A thread has eight pairs of a
// token, two pieces of eight channels, and forms their angles once for all heads that it turns.
#include "kda_rotation.h"

namespace kda {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Rotate {
    const void *q, *k;
    void *q_out, *k_out;
    const int32_t *positions;
    const float *inv_freq;
    int64_t tokens, q_stride, k_stride;
    uint32_t axis[4];                // two bits a frequency
    int32_t heads_q, heads, axes, n_freq, interleaved, inverse;
    int32_t parts, part_heads;       // workgroups of a block of tokens, and the heads that each of them turns
};

template <typename T> struct Piece;
template <> struct Piece<uint16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t *p) { w = *reinterpret_cast<const u32x4 *>(p); }
    __device__ __forceinline__ void store(uint16_t *p) const { *reinterpret_cast<u32x4 *>(p) = w; }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack_bf16x2(w[i], x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void put(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    }
};
template <> struct Piece<float> {
    f32x4 w[2];
    __device__ __forceinline__ void load(const float *p)
    {
        w[0] = *reinterpret_cast<const f32x4 *>(p);
        w[1] = *reinterpret_cast<const f32x4 *>(p + 4);
    }
    __device__ __forceinline__ void store(float *p) const
    {
        *reinterpret_cast<f32x4 *>(p) = w[0];
        *reinterpret_cast<f32x4 *>(p + 4) = w[1];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = w[i / 4][i % 4];
    }
    __device__ __forceinline__ void put(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4][i % 4] = x[i];
    }
};

// cos and sin of 2 pi r, |r| <= 1/2
__device__ __forceinline__ void angle32(double r, float &c, float &s)
{
    const double q = __builtin_rint(4.0 * r);
    const float x = (float)((r - 0.25 * q) * 6.283185307179586), y = x * x;
    float cc = fmaf(-2.7557319e-07f, y, 2.4801587e-05f), ss = fmaf(2.7557319e-06f, y, -1.9841270e-04f);          // -1/10!, 1/8!; 1/9!, -1/7!
    cc = fmaf(cc, y, -1.3888889e-03f);
    ss = fmaf(ss, y, 8.3333333e-03f);
    cc = fmaf(cc, y, 4.1666667e-02f);
    ss = fmaf(ss, y, -1.6666667e-01f);
    cc = fmaf(cc, y, -0.5f);
    ss = fmaf(ss * y, x, x);
    cc = fmaf(cc, y, 1.0f);
    const int k = (int)q & 3;
    const float a = k & 1 ? ss : cc, b = k & 1 ? cc : ss;
    c = k == 1 || k == 2 ? -a : a;
    s = k & 2 ? -b : b;
}

constexpr int kThreads = 256, kAhead = 4;                    // heads in flight

template <int D, typename T, bool kInterleaved>
__global__ __launch_bounds__(kThreads) void kda_rotate_kernel(const Rotate a)
{
    constexpr int kUnits = D / 16;                           // threads of a token
    const int unit = threadIdx.x % kUnits;
    const uint32_t part = blockIdx.x % a.parts;
    const int64_t token = (int64_t)(blockIdx.x / a.parts) * (kThreads / kUnits) + threadIdx.x / kUnits;
    if (token >= a.tokens) return;
    const int h0 = part * a.part_heads, h1 = min(h0 + a.part_heads, a.heads);
    const bool turned = 16 * unit < 2 * a.n_freq, halves = turned && !kInterleaved;
    const int at0 = halves ? 8 * unit : 16 * unit, at1 = halves ? a.n_freq + 8 * unit : 16 * unit + 8;
    const T *q = static_cast<const T *>(a.q) + token * a.q_stride, *k = static_cast<const T *>(a.k) + token * a.k_stride;
    T *qo = static_cast<T *>(a.q_out) + token * a.heads_q * D, *ko = static_cast<T *>(a.k_out) + token * (a.heads - a.heads_q) * D;
    Piece<T> w[kAhead][2];
    auto fetch = [&](int h) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int hh = min(h + u, h1 - 1);
            const T *from = hh < a.heads_q ? q + (int64_t)hh * D : k + (int64_t)(hh - a.heads_q) * D;
            w[u][0].load(from + at0);
            w[u][1].load(from + at1);
        }
    };
    fetch(h0);
    float cs[8], sn[8];
    if (turned) {
        int32_t pos[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) pos[i] = i < a.axes ? a.positions[i * a.tokens + token] : 0;
        const uint32_t axis = a.axis[unit / 2] >> (16 * (unit & 1));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t x = axis >> (2 * e);
            const int32_t lo = x & 1 ? pos[1] : pos[0], hi = x & 1 ? pos[3] : pos[2];
            angle32(turns((double)a.inv_freq[8 * unit + e] * 0.15915494309189535, x & 2 ? hi : lo), cs[e], sn[e]);
            if (a.inverse) sn[e] = -sn[e];
        }
    }
    for (int h = h0; h < h1; h += kAhead) {
        Piece<T> y[kAhead][2];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            y[u][0] = w[u][0];
            y[u][1] = w[u][1];
        }
        if (h + kAhead < h1) fetch(h + kAhead);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (h + u >= h1) break;
            if (turned) {
                float x[2][8], z[2][8];
                y[u][0].get(x[0]);
                y[u][1].get(x[1]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // pair e: channels e of the two pieces, or the interleaved 2 e and 2 e + 1
                    const int pa = kInterleaved ? e / 4 : 0, pb = kInterleaved ? e / 4 : 1, ia = kInterleaved ? 2 * (e % 4) : e, ib = kInterleaved ? ia + 1 : e;
                    z[pa][ia] = x[pa][ia] * cs[e] - x[pb][ib] * sn[e];
                    z[pb][ib] = x[pa][ia] * sn[e] + x[pb][ib] * cs[e];
                }
                y[u][0].put(z[0]);
                y[u][1].put(z[1]);
            }
            T *to = h + u < a.heads_q ? qo + (int64_t)(h + u) * D : ko + (int64_t)(h + u - a.heads_q) * D;
            y[u][0].store(to + at0);
            y[u][1].store(to + at1);
        }
    }
}

template <int D, typename T> hipError_t launch(const Rotate &a, uint32_t grid, hipStream_t st)
{
    if (a.interleaved) hipLaunchKernelGGL((kda_rotate_kernel<D, T, true>), dim3(grid), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((kda_rotate_kernel<D, T, false>), dim3(grid), dim3(kThreads), 0, st, a);
    return hipGetLastError();
}
bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && na && nb && x < y + nb && y < x + na;
}

}  // namespace
}  // namespace kda

using namespace kda;

extern "C" kda_status kda_rotate(const kda_rotation *r, const void *q, const void *k, const int32_t *positions, void *q_out, void *k_out,
                                 void *hip_stream)
{
    if (!r) return fail(KDA_ERR_INVALID_ARG, "rotation is NULL");
    if (r->batch < 0 || r->seqlen < 0 || r->heads_q < 0 || r->heads_k < 0)
        return fail(KDA_ERR_INVALID_ARG, "negative size (batch %d, seqlen %lld, heads %d and %d)", r->batch, (long long)r->seqlen, r->heads_q, r->heads_k);
    if (r->dim != 64 && r->dim != 128) return fail(KDA_ERR_UNSUPPORTED, "dim must be 64 or 128, got %d", r->dim);
    if (r->dtype != KDA_F32 && r->dtype != KDA_BF16) return fail(KDA_ERR_INVALID_ARG, "dtype %d is not a kda_dtype", (int)r->dtype);
    if (r->heads_q > 65535 || r->heads_k > 65535) return fail(KDA_ERR_UNSUPPORTED, "more than 65535 heads");
    if (r->axes < 1 || r->axes > 4) return fail(KDA_ERR_UNSUPPORTED, "1 to 4 axes, got %d", r->axes);
    if (r->num_freqs < 0 || 2 * (int64_t)r->num_freqs > r->dim || r->num_freqs % 8)
        return fail(KDA_ERR_INVALID_ARG, "num_freqs must be a multiple of 8 up to dim / 2, got %d", r->num_freqs);
    Rotate a = {};
    for (int i = 0; r->axis_of_freq && i < r->num_freqs; ++i) {
        if (r->axis_of_freq[i] >= r->axes) return fail(KDA_ERR_INVALID_ARG, "axis_of_freq[%d] is %d, of %d axes", i, r->axis_of_freq[i], r->axes);
        a.axis[i / 16] |= (uint32_t)r->axis_of_freq[i] << (2 * (i % 16));
    }
    const int64_t row_q = (int64_t)r->heads_q * r->dim, row_k = (int64_t)r->heads_k * r->dim;
    a.q_stride = r->q_stride ? r->q_stride : row_q;
    a.k_stride = r->k_stride ? r->k_stride : row_k;
    if (a.q_stride < row_q || a.q_stride % 8 || a.q_stride > (1 << 24) || a.k_stride < row_k || a.k_stride % 8 || a.k_stride > (1 << 24))
        return fail(KDA_ERR_INVALID_ARG, "strides must be 0 or a multiple of 8 from heads x dim to 2^24, got %lld and %lld", (long long)r->q_stride,
                    (long long)r->k_stride);
    if (r->heads_k && (k == nullptr) != (k_out == nullptr)) return fail(KDA_ERR_INVALID_ARG, "k and k_out come together");
    const int32_t heads_k = k ? r->heads_k : 0;
    if (r->batch && r->seqlen > ((int64_t)1 << 30) / r->batch) return fail(KDA_ERR_UNSUPPORTED, "more than 2^30 tokens");
    a.tokens = r->batch * r->seqlen;
    a.heads_q = r->heads_q;
    a.heads = r->heads_q + heads_k;
    if (a.tokens == 0 || a.heads == 0) return KDA_OK;
    if (r->heads_q && (!q || !q_out)) return fail(KDA_ERR_INVALID_ARG, "q or q_out is NULL");
    if (r->num_freqs && (!positions || !r->inv_freq)) return fail(KDA_ERR_INVALID_ARG, "positions or inv_freq is NULL");
    for (const void *p : {q, k, (const void *)q_out, (const void *)k_out})
        if (!aligned(p, 16)) return fail(KDA_ERR_INVALID_ARG, "kda_rotate: tensors must be 16-byte aligned");
    if (!aligned(positions, 4) || !aligned(r->inv_freq, 4)) return fail(KDA_ERR_INVALID_ARG, "positions or inv_freq is misaligned");
    const size_t size = r->dtype == KDA_BF16 ? 2 : 4, nq = a.tokens * row_q * size, nk = heads_k ? a.tokens * row_k * size : 0;
    const size_t sq = ((a.tokens - 1) * a.q_stride + row_q) * size, sk = heads_k ? ((a.tokens - 1) * a.k_stride + row_k) * size : 0;
    if (overlap(q_out, nq, k_out, nk) || overlap(q_out, nq, k, sk) || overlap(k_out, nk, q, sq) ||
        (overlap(q_out, nq, q, sq) && !(q == q_out && a.q_stride == row_q)) || (overlap(k_out, nk, k, sk) && !(k == k_out && a.k_stride == row_k)))
        return fail(KDA_ERR_INVALID_ARG, "an output overlaps an input that it does not replace, or the other output");
    a.q = q;
    a.k = k;
    a.q_out = q_out;
    a.k_out = k_out;
    a.positions = positions;
    a.inv_freq = r->inv_freq;
    a.axes = r->axes;
    a.n_freq = r->num_freqs;
    a.interleaved = r->interleaved != 0;
    a.inverse = r->inverse != 0;
    // heads of a thread: as many as leave 2048 workgroups, which fill the device
    const int64_t blocks = (a.tokens * (r->dim / 16) + kThreads - 1) / kThreads;
    int64_t per = (blocks * a.heads + 2047) / 2048;
    per = (per + kAhead - 1) / kAhead * kAhead;
    a.part_heads = (int32_t)(per < a.heads ? per : a.heads);
    a.parts = (a.heads + a.part_heads - 1) / a.part_heads;
    // (a launch has fewer than 2^32 threads)
    if (blocks * a.parts > 0xffffff) return fail(KDA_ERR_UNSUPPORTED, "more than 2^24 workgroups");
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const uint32_t grid = (uint32_t)(blocks * a.parts);
    const hipError_t e = r->dim == 128 ? (size == 2 ? launch<128, uint16_t>(a, grid, st) : launch<128, float>(a, grid, st))
                                       : (size == 2 ? launch<64, uint16_t>(a, grid, st) : launch<64, float>(a, grid, st));
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_rotate: %s", hipGetErrorString(e));
}
