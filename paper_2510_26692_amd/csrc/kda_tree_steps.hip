// KDA over a draft tree: a token steps from the state behind its parent (kda_tree_steps), and the accepted path into the states
// (kda_tree_commit).
//
// Written out along a token's line (own derivation: the recurrence unrolled from the state S_0 before the tree).  With P_ij the channelwise product
// of the decays of i and of its ancestors below j, and P_i0 that of all of them,
//
//     u_i = beta_i (v_i - (P_i0 k_i)^T S_0 - sum_{j ancestor of i} (sum_c k_i P_ij k_j) u_j)
//     o_i = scale ((P_i0 q_i)^T S_0 + sum_{j ancestor of i, or i} (sum_c q_i P_ij k_j) u_j)
//
// so that S_0 is read once, whatever the tree, and no token's state is formed.  Products of decays are formed going up a line, one
// multiplication a token and channel, never as the quotient of two long products.  Everything is fp32; the two products with S_0 are
// 16x16x4 fp32 MFMAs.
//
// A workgroup has one sequence and head, a wave 32 columns of its state, held in registers from the start.  What bounds it is reading the
// states, and for large trees the fp32 matrix cores: 4 T dk dv operations a state of 4 dk dv bytes.
#include "kda_tree.h"

namespace kda {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Tree {
    const void *q, *k, *v, *log_alpha, *beta;
    const float *states;
    const int32_t *indices, *parents;
    void *o;
    float scale;
    int32_t heads, tokens, scalar_gate, out_bf16;
};

// four neighbours of a token's row
__device__ __forceinline__ f32x4 load4(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
__device__ __forceinline__ f32x4 load4(const __hip_bfloat16 *p)
{
    const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
    f32x4 x;
    float lo, hi;
    unpack_bf16x2(w[0], lo, hi);
    x[0] = lo;
    x[1] = hi;
    unpack_bf16x2(w[1], lo, hi);
    x[2] = lo;
    x[3] = hi;
    return x;
}
__device__ __forceinline__ f32x2 load2(const float *p) { return *reinterpret_cast<const f32x2 *>(p); }
__device__ __forceinline__ f32x2 load2(const __hip_bfloat16 *p)
{
    float lo, hi;
    unpack_bf16x2(*reinterpret_cast<const uint32_t *>(p), lo, hi);
    return f32x2{lo, hi};
}
// Sum over the sixteen lanes of a row.
template <int kCtrl> __device__ __forceinline__ float add_rotated(float v)
{
    return v + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), kCtrl, 0xf, 0xf, false));
}
__device__ __forceinline__ float over_sixteen(float v) { return add_rotated<0x121>(add_rotated<0x122>(add_rotated<0x124>(add_rotated<0x128>(v)))); }

// LDS: decays, k and q of the tokens, [TM][D + 4] each, the first two replaced by what the products with S_0 give; then for each token and ancestor
// the two sums over channels, beta (sum k P k) and scale (sum q P k).
template <int D, int TM> struct StepLds {
    static constexpr int kPitch = D + 4;
    static constexpr int kRows = TM * kPitch;                // floats
    static constexpr int kSums = 3 * kRows;
    static constexpr int kLines = kSums + 2 * TM * TM;
    static constexpr int kBytes = (kLines + 2 * kTreeTokens) * 4;
};

template <typename Tin, int D, int TM>
__global__ __launch_bounds__(2 * D) void kda_tree_steps_kernel(const Tree a)
{
    using L = StepLds<D, TM>;
    constexpr int kThreads = 2 * D, kGroups = D / 8, kNodes = TM / kGroups > 0 ? TM / kGroups : 1;      // groups of 16 lanes; tokens of one
    constexpr int CH = D / 16;                               // channels of a lane in a group
    constexpr int MT = TM / 16;                              // 16-row blocks of the tokens' products, for k and for q
    extern __shared__ __align__(16) float lds[];
    float *al = lds, *kk = lds + L::kRows, *qq = lds + 2 * L::kRows;
    f32x2 *sums = reinterpret_cast<f32x2 *>(lds + L::kSums);
    uint64_t *lines = reinterpret_cast<uint64_t *>(lds + L::kLines);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, x = lane & 15, g = lane >> 4;
    const int64_t n = blockIdx.x / a.heads;
    const int h = (int)(blockIdx.x - n * a.heads), T = a.tokens;
    const int64_t row0 = n * T * a.heads + h;                // row of token 0; the next is `heads` behind
    const int64_t state = a.indices ? a.indices[n] : n;
    auto put = [&](int t, int col, float v) {
        const int64_t at = (row0 + (int64_t)t * a.heads) * D + col;
        if (a.out_bf16) static_cast<uint16_t *>(a.o)[at] = (uint16_t)pack_bf16x2(v, 0.f);
        else static_cast<float *>(a.o)[at] = v;
    };
    if (state < 0) {
        for (int i = tid; i < T * D; i += kThreads) put(i / D, i % D, 0.f);
        return;
    }
    // ---- the state: columns 32 wave + 2 x, and the next; rows 16 s + 4 g + i ----
    f32x2 s0[D / 16][4];
    {
        const float *from = a.states + (state * a.heads + h) * (D * D) + (4 * g) * D + 32 * wave + 2 * x;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) s0[s][i] = __builtin_nontemporal_load(reinterpret_cast<const f32x2 *>(from + (16 * s + i) * D));
    }
    if (wave == 0) lines[lane] = tree_line(a.parents + n * T, T);
    __syncthreads();

    // ---- tokens (one that is not there: no key, no query, no decay) ----
    {
        const Tin *q = static_cast<const Tin *>(a.q), *k = static_cast<const Tin *>(a.k), *la = static_cast<const Tin *>(a.log_alpha);
        for (int i = tid; i < TM * (D / 4); i += kThreads) {
            const int t = i / (D / 4), c = 4 * (i % (D / 4));
            f32x4 qv = {0.f, 0.f, 0.f, 0.f}, kv = qv, av = {1.f, 1.f, 1.f, 1.f};
            if (t < T && lines[t]) {
                const int64_t row = row0 + (int64_t)t * a.heads;
                qv = load4(q + row * D + c);
                kv = load4(k + row * D + c);
                if (a.scalar_gate) av = f32x4{1.f, 1.f, 1.f, 1.f} * load_as_float(la + row);
                else av = load4(la + row * D + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) av[e] = fast_exp2(av[e] * kLog2e);
            }
            *reinterpret_cast<f32x4 *>(al + t * L::kPitch + c) = av;
            *reinterpret_cast<f32x4 *>(kk + t * L::kPitch + c) = kv;
            *reinterpret_cast<f32x4 *>(qq + t * L::kPitch + c) = qv;
        }
    }
    __syncthreads();

    // ---- up every token's line: the sums over channels, and the product of all decays ----
    float all[kNodes][CH];
    const int group = tid >> 4;
    auto channels = [&](const float *rows, int t, float (&v)[CH]) {
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
            const f32x4 w = *reinterpret_cast<const f32x4 *>(rows + t * L::kPitch + CH * x + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i + e] = w[e];
        }
    };
#pragma unroll
    for (int r = 0; r < kNodes; ++r) {
        const int t = group + kGroups * r;
#pragma unroll
        for (int i = 0; i < CH; ++i) all[r][i] = 1.f;
        if (t >= T) continue;
        uint64_t line = lines[t];
        if (!line) continue;
        const float beta = load_as_float(static_cast<const Tin *>(a.beta) + row0 + (int64_t)t * a.heads);
        float kt[CH], qt[CH];
        channels(kk, t, kt);
        channels(qq, t, qt);
        while (line) {
            const int j = 63 - __builtin_clzll(line);
            line &= ~(1ull << j);
            float kj[CH], aj[CH], dk = 0.f, dq = 0.f;
            channels(kk, j, kj);
            channels(al, j, aj);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const float w = all[r][i] * kj[i];
                dk = fmaf(kt[i], w, dk);
                dq = fmaf(qt[i], w, dq);
                all[r][i] *= aj[i];
            }
            dk = over_sixteen(dk);
            dq = over_sixteen(dq);
            if (x == 0) sums[t * TM + j] = f32x2{beta * dk, a.scale * dq};
        }
    }
    __syncthreads();
    // ---- P_i0 k_i and scale P_i0 q_i ----
#pragma unroll
    for (int r = 0; r < kNodes; ++r) {
        const int t = group + kGroups * r;
        if (t >= TM) continue;
        float v[CH];
        channels(kk, t, v);
#pragma unroll
        for (int i = 0; i < CH; i += 4)
            *reinterpret_cast<f32x4 *>(kk + t * L::kPitch + CH * x + i) = f32x4{v[i] * all[r][i], v[i + 1] * all[r][i + 1], v[i + 2] * all[r][i + 2], v[i + 3] * all[r][i + 3]};
        channels(qq, t, v);
#pragma unroll
        for (int i = 0; i < CH; i += 4)
            *reinterpret_cast<f32x4 *>(qq + t * L::kPitch + CH * x + i) = f32x4{v[i] * all[r][i], v[i + 1] * all[r][i + 1], v[i + 2] * all[r][i + 2], v[i + 3] * all[r][i + 3]} * a.scale;
    }
    __syncthreads();

    // ---- their products with S_0; lane's rows 16 m + 4 g + e, columns 32 wave + 2 x + j ----
    f32x4 acc[2][MT][2];
    f32x2 vv[MT][4];
    float beta[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = 16 * m + 4 * g + e;
            vv[m][e] = f32x2{0.f, 0.f};
            beta[m][e] = 0.f;
            if (t < T && lines[t]) {
                const int64_t row = row0 + (int64_t)t * a.heads;
                vv[m][e] = load2(static_cast<const Tin *>(a.v) + row * D + 32 * wave + 2 * x);
                beta[m][e] = load_as_float(static_cast<const Tin *>(a.beta) + row);
            }
        }
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            acc[w][m][0] = acc[w][m][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (16 * m >= T) continue;
            const float *rows = (w ? qq : kk) + (16 * m + x) * L::kPitch + 4 * g;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                const f32x4 r = *reinterpret_cast<const f32x4 *>(rows + 16 * s);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[w][m][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(r[i], s0[s][i][j], acc[w][m][j], 0, 0, 0);
            }
        }
    __syncthreads();
    float *u = lds, *os = lds + L::kRows;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = 16 * m + 4 * g + e, at = t * L::kPitch + 32 * wave + 2 * x;
            *reinterpret_cast<f32x2 *>(u + at) = f32x2{beta[m][e] * (vv[m][e][0] - acc[0][m][0][e]), beta[m][e] * (vv[m][e][1] - acc[0][m][1][e])};
            *reinterpret_cast<f32x2 *>(os + at) = f32x2{acc[1][m][0][e], acc[1][m][1][e]};
        }
    __syncthreads();

    // ---- corrections and outputs, a column a thread, down the tree ----
    if (tid >= D) return;
    for (int t = 0; t < T; ++t) {
        const uint64_t mine = lines[t];
        const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(mine >> 32)), lo = __builtin_amdgcn_readfirstlane((uint32_t)mine);
        uint64_t line = (uint64_t)hi << 32 | lo;
        if (!line) {
            put(t, tid, 0.f);
            continue;
        }
        line &= ~(1ull << t);
        float ut = u[t * L::kPitch + tid], ot = os[t * L::kPitch + tid];
        while (line) {
            const int j = __builtin_ctzll(line);
            line &= line - 1;
            const f32x2 w = sums[t * TM + j];
            const float uj = u[j * L::kPitch + tid];
            ut = fmaf(-w[0], uj, ut);
            ot = fmaf(w[1], uj, ot);
        }
        u[t * L::kPitch + tid] = ut;
        put(t, tid, fmaf(sums[t * TM + t][1], ut, ot));
    }
}

struct Commit {
    const void *k, *v, *log_alpha, *beta;
    float *states;
    const int32_t *indices, *kept;
    int32_t heads, tokens, most, scalar_gate;
};
constexpr int kAtOnce = 8;           // tokens in LDS

// The accepted tokens, as the decode kernel steps (kda_step.hip): a wave has 32 columns of a state, 8 row groups by 8 groups of four columns, in
// registers from the first token to the last.
template <typename Tin, int D>
__global__ __launch_bounds__(2 * D) void kda_tree_commit_kernel(const Commit a)
{
    constexpr int ROWS = D / 8, kThreads = 2 * D;
    __shared__ float s_alpha[kAtOnce][D], s_k[kAtOnce][D], s_v[kAtOnce][D], s_beta[kAtOnce];
    __shared__ int32_t s_path[kTreeTokens];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, cg = lane & 7, rg = lane >> 3, col = wave * 32 + cg * 4;
    const int64_t n = blockIdx.x / a.heads;
    const int h = (int)(blockIdx.x - n * a.heads);
    const int64_t state = a.indices ? a.indices[n] : n;
    if (state < 0) return;
    const int32_t x = lane < a.most ? a.kept[n * a.most + lane] : -1, before = __shfl_up(x, 1);
    const uint64_t bad = ~__ballot(x >= 0 && x < a.tokens && (lane == 0 || x > before));
    const int count = bad ? __builtin_ctzll(bad) : 64;
    if (count == 0) return;
    if (wave == 0) s_path[lane] = x;

    f32x4 *Sp = reinterpret_cast<f32x4 *>(a.states + (state * a.heads + h) * (D * D) + (int64_t)rg * D + col);
    f32x4 s[ROWS];
#pragma unroll
    for (int m = 0; m < ROWS; ++m) s[m] = __builtin_nontemporal_load(Sp + (int64_t)m * (8 * D / 4));
    const Tin *k = static_cast<const Tin *>(a.k), *v = static_cast<const Tin *>(a.v), *la = static_cast<const Tin *>(a.log_alpha);
    for (int t0 = 0; t0 < count; t0 += kAtOnce) {
        const int some = min(kAtOnce, count - t0);
        __syncthreads();
        for (int i = tid; i < some * D; i += kThreads) {
            const int t = i / D, c = i - t * D;
            const int64_t row = (n * a.tokens + s_path[t0 + t]) * a.heads + h;
            s_alpha[t][c] = fast_exp2(load_as_float(la + (a.scalar_gate ? row : row * D + c)) * kLog2e);
            s_k[t][c] = load_as_float(k + row * D + c);
            s_v[t][c] = load_as_float(v + row * D + c);
            if (c == 0) s_beta[t] = load_as_float(static_cast<const Tin *>(a.beta) + row);
        }
        __syncthreads();
        for (int t = 0; t < some; ++t) {
            f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < ROWS; ++m) {
                const float kr = s_k[t][rg + 8 * m];
                s[m] *= s_alpha[t][rg + 8 * m];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = fmaf(kr, s[m][e], p[e]);
            }
#pragma unroll
            for (int d = 8; d < 64; d <<= 1)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] += __shfl_xor(p[e], d);
            const float b = s_beta[t];
            const f32x4 vt = *reinterpret_cast<const f32x4 *>(&s_v[t][col]);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = b * (vt[e] - p[e]);
#pragma unroll
            for (int m = 0; m < ROWS; ++m) {
                const float kr = s_k[t][rg + 8 * m];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[m][e] = fmaf(kr, p[e], s[m][e]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < ROWS; ++m) __builtin_nontemporal_store(s[m], Sp + (int64_t)m * (8 * D / 4));
}

template <typename Tin, int D, int TM> hipError_t launch_steps(const Tree &a, int64_t pairs, hipStream_t st)
{
    constexpr int kBytes = StepLds<D, TM>::kBytes;
    if (kBytes > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kda_tree_steps_kernel<Tin, D, TM>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((kda_tree_steps_kernel<Tin, D, TM>), dim3((uint32_t)pairs), dim3(2 * D), kBytes, st, a);
    return hipGetLastError();
}
template <typename Tin, int D> hipError_t launch_steps(const Tree &a, int64_t pairs, hipStream_t st)
{
    return a.tokens <= 16 ? launch_steps<Tin, D, 16>(a, pairs, st) : a.tokens <= 32 ? launch_steps<Tin, D, 32>(a, pairs, st) : launch_steps<Tin, D, 64>(a, pairs, st);
}
template <typename Tin, int D> hipError_t launch_commit(const Commit &a, int64_t pairs, hipStream_t st)
{
    hipLaunchKernelGGL((kda_tree_commit_kernel<Tin, D>), dim3((uint32_t)pairs), dim3(2 * D), 0, st, a);
    return hipGetLastError();
}

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
kda_status check(const kda_dims *d, uint32_t flags)
{
    if (!d) return fail(KDA_ERR_INVALID_ARG, "dims is NULL");
    if (d->batch < 0 || d->seqlen < 0 || d->heads < 0 || d->num_seqs < 0)
        return fail(KDA_ERR_INVALID_ARG, "negative size (batch %d, seqlen %lld, heads %d, num_seqs %d)", d->batch, (long long)d->seqlen, d->heads, d->num_seqs);
    if (d->in_dtype != KDA_F32 && d->in_dtype != KDA_BF16) return fail(KDA_ERR_INVALID_ARG, "in_dtype %d is not a kda_dtype", (int)d->in_dtype);
    if (d->out_dtype != KDA_F32 && d->out_dtype != KDA_BF16) return fail(KDA_ERR_INVALID_ARG, "out_dtype %d is not a kda_dtype", (int)d->out_dtype);
    if (!(d->dk == d->dv && (d->dk == 64 || d->dk == 128)))
        return fail(KDA_ERR_UNSUPPORTED, "head dims must satisfy dk == dv in {64,128}, got %d x %d", d->dk, d->dv);
    if (d->heads > 65535) return fail(KDA_ERR_UNSUPPORTED, "heads > 65535");
    if (d->num_seqs != d->batch) return fail(KDA_ERR_INVALID_ARG, "fixed-length batches need num_seqs == batch");
    if (d->seqlen > kTreeTokens) return fail(KDA_ERR_UNSUPPORTED, "at most %d drafted tokens a sequence, got %lld", kTreeTokens, (long long)d->seqlen);
    if (!(d->scale == d->scale)) return fail(KDA_ERR_INVALID_ARG, "scale is NaN");
    if (flags & ~(uint32_t)KDA_STEPS_SCALAR_GATE) return fail(KDA_ERR_INVALID_ARG, "unknown flags %u", (unsigned)flags);
    // (a launch has fewer than 2^32 threads)
    if ((int64_t)d->num_seqs * d->heads > 0xffffff) return fail(KDA_ERR_UNSUPPORTED, "more than 2^24 sequences and heads");
    return KDA_OK;
}

}  // namespace
}  // namespace kda

using namespace kda;

extern "C" kda_status kda_tree_steps(const kda_dims *dims, const void *q, const void *k, const void *v, const void *log_alpha, const void *beta,
                                     const float *S_pool, const int32_t *state_indices, const int32_t *parents, void *o, uint32_t flags,
                                     void *hip_stream)
{
    if (const kda_status st = check(dims, flags); st != KDA_OK) return st;
    const int64_t pairs = (int64_t)dims->num_seqs * dims->heads;
    if (pairs == 0 || dims->seqlen == 0) return KDA_OK;
    if (!q || !k || !v || !log_alpha || !beta || !S_pool || !parents || !o)
        return fail(KDA_ERR_INVALID_ARG, "q, k, v, log_alpha, beta, S_pool, parents and o must be non-NULL");
    const bool scalar = flags & KDA_STEPS_SCALAR_GATE, bf = dims->in_dtype == KDA_BF16;
    const uintptr_t size = bf ? 2 : 4;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(log_alpha, scalar ? size : 16) || !aligned(beta, size) || !aligned(S_pool, 16) ||
        !aligned(o, 16) || !aligned(state_indices, 4) || !aligned(parents, 4))
        return fail(KDA_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned (state_indices and parents: 4)");
    const Tree a = {q, k, v, log_alpha, beta, S_pool, state_indices, parents, o, dims->scale, dims->heads, (int32_t)dims->seqlen, scalar,
                    dims->out_dtype == KDA_BF16};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = dims->dk == 128 ? (bf ? launch_steps<__hip_bfloat16, 128>(a, pairs, st) : launch_steps<float, 128>(a, pairs, st))
                                         : (bf ? launch_steps<__hip_bfloat16, 64>(a, pairs, st) : launch_steps<float, 64>(a, pairs, st));
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_tree_steps: %s", hipGetErrorString(e));
}

extern "C" kda_status kda_tree_commit(const kda_dims *dims, const void *k, const void *v, const void *log_alpha, const void *beta, float *S_pool,
                                      const int32_t *state_indices, const int32_t *kept, int32_t max_kept, uint32_t flags, void *hip_stream)
{
    if (const kda_status st = check(dims, flags); st != KDA_OK) return st;
    if (max_kept < 0) return fail(KDA_ERR_INVALID_ARG, "negative size (max_kept %d)", max_kept);
    if (max_kept > kTreeTokens) return fail(KDA_ERR_UNSUPPORTED, "at most %d kept tokens a sequence, got %d", kTreeTokens, max_kept);
    const int64_t pairs = (int64_t)dims->num_seqs * dims->heads;
    if (pairs == 0 || dims->seqlen == 0 || max_kept == 0) return KDA_OK;
    if (!k || !v || !log_alpha || !beta || !S_pool || !kept) return fail(KDA_ERR_INVALID_ARG, "k, v, log_alpha, beta, S_pool and kept must be non-NULL");
    const bool scalar = flags & KDA_STEPS_SCALAR_GATE, bf = dims->in_dtype == KDA_BF16;
    const uintptr_t size = bf ? 2 : 4;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(log_alpha, scalar ? size : 16) || !aligned(beta, size) || !aligned(S_pool, 16) ||
        !aligned(state_indices, 4) || !aligned(kept, 4))
        return fail(KDA_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned (state_indices and kept: 4)");
    const Commit a = {k, v, log_alpha, beta, S_pool, state_indices, kept, dims->heads, (int32_t)dims->seqlen, max_kept, scalar};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = dims->dk == 128 ? (bf ? launch_commit<__hip_bfloat16, 128>(a, pairs, st) : launch_commit<float, 128>(a, pairs, st))
                                         : (bf ? launch_commit<__hip_bfloat16, 64>(a, pairs, st) : launch_commit<float, 64>(a, pairs, st));
    return e == hipSuccess ? KDA_OK : fail(KDA_ERR_LAUNCH, "kda_tree_commit: %s", hipGetErrorString(e));
}
