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
// 16x16x4 fp32 MFMAs for trees of up to 16 tokens.  For larger ones their factors are written as three bf16 each, x = h + m + l exactly, and six
// products of those, the largest, are summed in fp32 by 16x16x32 MFMAs: what is left out is below 2^-22 of a term and of either sign, the result as near as
// with fp32 MFMAs (1.6 10^-7 in the mean square, 2.0 with those), in 3/8 of their time.  (Pieces below 2^-126 may be lost: of states below 2^-110 that is more than
// fp32's own steps.)  A large tree's q goes to the lanes that need it without LDS, so that two workgroups share a compute unit in fp32 too.
//
// A workgroup has one sequence and head, a wave 32 columns of its state, held in registers from the start.  The sums over channels make a lower
// triangular matrix N = -beta (sum k P k), zero but at ancestors, whose 16x16 blocks take the u of one block of tokens to the next:
//
//     r_m = beta (v - P k S_0) + sum_{n < m} N_mn u_n,     u_m = (I - N_mm)^-1 r_m,     o_m = scale P q S_0 + sum_{n <= m} (scale sum q P k)_mn u_n
//
// all of them fp32 MFMAs whose accumulators are the operands of the next, so u never leaves its registers.
//
// A sum over channels may leave fp32 where u and the scale would bring it back, and entries of an inverse that do would make NaN of tokens beside their line (0 times
// infinity).  So what is not finite is kept out of the matrices and of r, and remembered: the rows that it belongs to, and whatever rows are not finite at the end,
// are worked through again from state to state, as kda_recurrent_steps does, a line at a time.  Only those are written again: a row is the same
// whatever its neighbours hold.  (Looking for them costs 0.3 us of 132.  The pass itself is slow: 64 chains of 64 tokens with keys 22 long 1.5 ms for 230 us.)
//
// What bounds it is reading the states, and for large trees no part alone: vector instructions are 54 % busy, half of them the sums up the lines, the matrix cores
// 31 %.  256 trees of up to 16 tokens, 32 heads: 132 to 134 us (0.68 GB, 5.1 TB/s); 64 of 64 tokens: 128 to 134, in fp32 150; 64 chains of 64: 230; 128 trees of 20: 99.
// With fp32 MFMAs and q in LDS these were 170, 271, 320 and 126.  A step up a line is some 65 vector instructions for a group: scales and what is not finite
// are looked at behind it (chains 278 -> 230).  (Pieces for trees of 16, too: the same time in bf16, 172 for 156 in fp32.  With a column a thread and a loop
// over each token's ancestors in place of the blocks: 231 and 474.)
#include "kda_tree.h"

namespace kda {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Tree {
    const void *q, *k, *v, *log_alpha, *beta;
    const float *states;
    const int32_t *indices, *parents;
    void *o;
    float scale;
    int32_t heads, tokens, scalar_gate, out_bf16;
};

// four neighbours of a token's row, as they come and in fp32
template <typename T> struct FourOf;
template <> struct FourOf<float> { typedef f32x4 type; };
template <> struct FourOf<__hip_bfloat16> { typedef u32x2 type; };
template <typename T> using Four = typename FourOf<T>::type;
__device__ __forceinline__ f32x4 widened(const f32x4 &w) { return w; }
__device__ __forceinline__ f32x4 widened(const u32x2 &w)
{
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
template <typename T> __device__ __forceinline__ f32x4 load4(const T *p) { return widened(*reinterpret_cast<const Four<T> *>(p)); }
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

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
// x = h + m + l in bf16, exactly: h what bf16's bits have of x, m and l the rest rounded, for two values each
__device__ __forceinline__ void three_of(float x0, float x1, uint32_t &h, uint32_t &m, uint32_t &l)
{
    const uint32_t b0 = __float_as_uint(x0) & 0xffff0000u, b1 = __float_as_uint(x1) & 0xffff0000u;
    h = b0 >> 16 | b1;
    float r0 = x0 - __uint_as_float(b0), r1 = x1 - __uint_as_float(b1), m0, m1;
    m = pack_bf16x2(r0, r1);
    unpack_bf16x2(m, m0, m1);
    l = pack_bf16x2(r0 - m0, r1 - m1);
}
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f32x4 mfma16(const f32x4 &a, const f32x4 &b, f32x4 acc)      // a 16 x 16 x 16 product: slot g of step i is index 4 g + i
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    return acc;
}

// LDS: decays of the tokens in fp32, then their k and, of small trees, q as they came, [TM][D + 4] each; in the same place P_i0 k_i and scale P_i0 q_i in fp32, or of
// larger trees their pieces; and then the two matrices of sums over channels, [TM][TM + 4] each.  Behind them the lines, parents, v and beta.
template <typename Tin, int D, int TM> struct StepLds {
    static constexpr int kPitch = D + 4, kSumPitch = TM + 4;
    static constexpr int kRows = TM * kPitch;
    // (the products with S_0 are of bf16 pieces: three planes of half the channels of P_i0 k_i, three of scale P_i0 q_i, [TM][D / 2 + 8] each)
    static constexpr bool kPlanes = TM >= 32;
    static constexpr int kPlanePitch = D / 2 + 8, kPlane = TM * kPlanePitch * 2;
    static constexpr int kTokens = kRows * (4 + (kPlanes ? 1 : 2) * (int)sizeof(Tin)),
                         kProducts = kPlanes ? 6 * kPlane : 2 * kRows * 4, kSums = 2 * TM * kSumPitch * 4;
    static constexpr int kMost = kTokens > kProducts ? kTokens : kProducts, kLines = kMost > kSums ? kMost : kSums;
    // (values and betas of trees of up to 32 tokens; a large tree's would leave one workgroup a compute unit)
    static constexpr bool kHasValues = TM < 64;
    static constexpr int kParents = kLines + kTreeTokens * 8, kValues = kParents + kTreeTokens * 4, kBetas = kValues + (kHasValues ? kRows * (int)sizeof(Tin) : 0);
    static constexpr int kLost = kBetas + (kHasValues ? TM * 4 : 0), kBytes = kLost + 16;    // tokens with a sum that is not finite, of k and of q: 64 bits each
};

// The rows of a wave's 32 columns that are not finite in o, from state to state along their lines: eight columns at a time, sixteen lanes with D / 16 channels
// each to two of them, so that the registers of what comes before are not added to.
template <typename Tin, int D>
__device__ __forceinline__ void step_again(const Tree &a, const uint64_t *lines, int64_t row0, int64_t state_at)
{
    constexpr int CH = D / 16;                               // channels of a lane
    const int lane = threadIdx.x & 63, x = lane & 15, T = a.tokens;
    auto row_of = [&](int t) { return (uint32_t)(t * a.heads); };
    auto uniform = [](uint64_t w) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(w >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)w);
    };
    auto joined = [](uint64_t w, int lanes) { return w | (uint64_t)(uint32_t)__shfl_xor((int)(w >> 32), lanes) << 32 | (uint32_t)__shfl_xor((int)w, lanes); };
    __threadfence_block();                                   // (o is read here as this wave has left it)
#pragma unroll 1
    for (int col = 32 * (threadIdx.x >> 6) + 2 * (lane >> 4), end = col + 32; col < end; col += 8) {
        uint64_t odd[2] = {0, 0};                            // tokens, of the lane's columns
#pragma unroll 1
        for (int t = x; t < T; t += 16) {
            if (!lines[t]) continue;
            const int64_t at = row0 * D + (row_of(t) * D + (uint32_t)col);
            const f32x2 o = a.out_bf16 ? load2(static_cast<const __hip_bfloat16 *>(a.o) + at) : load2(static_cast<const float *>(a.o) + at);
#pragma unroll
            for (int j = 0; j < 2; ++j) odd[j] |= finite(o[j]) ? 0ull : 1ull << t;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 1; i < 16; i <<= 1) odd[j] = joined(odd[j], i);
        uint64_t left = uniform(joined(joined(odd[0] | odd[1], 16), 32)), above = 0;          // above: the line of the token whose state is at hand
        float S[2][CH];
#pragma unroll 1
        for (bool begin = true; left; begin = false) {
            const int t = __builtin_ctzll(left);
            left &= left - 1;
            const uint64_t line = uniform(lines[t]);
            if (begin || (above & ~line)) {
                above = 0;
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const f32x2 w = load2(a.states + state_at + (CH * x + i) * D + col);
                    S[0][i] = w[0];
                    S[1][i] = w[1];
                }
            }
            uint64_t ahead = line & ~above;
            above = line;
#pragma unroll 1
            while (ahead) {
                const int n = __builtin_ctzll(ahead);
                ahead &= ahead - 1;
                const uint32_t row = row_of(n), at = row * D + CH * x;
                const Tin *la = static_cast<const Tin *>(a.log_alpha) + row0 * (a.scalar_gate ? 1 : D);
                float k[CH], w[2] = {0.f, 0.f};
#pragma unroll
                for (int i = 0; i < CH; i += 4) {
                    const f32x4 kf = load4(static_cast<const Tin *>(a.k) + row0 * D + (at + i));
                    f32x4 af = f32x4{1.f, 1.f, 1.f, 1.f} * (a.scalar_gate ? load_as_float(la + row) : 0.f);
                    if (!a.scalar_gate) af = load4(la + (at + i));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        k[i + e] = kf[e];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            S[j][i + e] *= fast_exp2(af[e] * kLog2e);
                            w[j] = fmaf(kf[e], S[j][i + e], w[j]);
                        }
                    }
                }
                const float b = load_as_float(static_cast<const Tin *>(a.beta) + row0 + row);
                const f32x2 v = load2(static_cast<const Tin *>(a.v) + row0 * D + (row * D + (uint32_t)col));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float u = b * (v[j] - over_sixteen(w[j]));
#pragma unroll
                    for (int i = 0; i < CH; ++i) S[j][i] = fmaf(k[i], u, S[j][i]);
                }
            }
            float y[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < CH; i += 4) {
                const f32x4 q = load4(static_cast<const Tin *>(a.q) + row0 * D + (row_of(t) * D + (uint32_t)(CH * x + i)));
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < 2; ++j) y[j] = fmaf(q[e], S[j][i + e], y[j]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float out = a.scale * over_sixteen(y[j]);
                if (x != 0 || !(odd[j] >> t & 1)) continue;
                const int64_t to = row0 * D + (row_of(t) * D + (uint32_t)(col + j));
                if (a.out_bf16) static_cast<uint16_t *>(a.o)[to] = (uint16_t)pack_bf16x2(out, 0.f);
                else static_cast<float *>(a.o)[to] = out;
            }
        }
    }
}

template <typename Tin, int D, int TM>
__global__ __launch_bounds__(2 * D, TM == 16 ? 4 : 2) void kda_tree_steps_kernel(const Tree a)
{
    using L = StepLds<Tin, D, TM>;
    constexpr int kThreads = 2 * D, kGroups = D / 8, kNodes = TM / kGroups > 0 ? TM / kGroups : 1;      // groups of 16 lanes; tokens of one
    constexpr int CH = D / 16;                               // channels of a lane in a group
    constexpr int MT = TM / 16;                              // 16-token blocks
    extern __shared__ __align__(16) uint8_t lds[];
    float *al = reinterpret_cast<float *>(lds);
    Tin *kk = reinterpret_cast<Tin *>(al + L::kRows), *qq = kk + L::kRows;
    uint64_t *lines = reinterpret_cast<uint64_t *>(lds + L::kLines);
    int32_t *parents = reinterpret_cast<int32_t *>(lds + L::kParents);       // (of tokens that are there: -1 ends a line)
    [[maybe_unused]] Tin *vs = reinterpret_cast<Tin *>(lds + L::kValues);
    [[maybe_unused]] float *betas = reinterpret_cast<float *>(lds + L::kBetas);
    uint32_t *lost = reinterpret_cast<uint32_t *>(lds + L::kLost);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, x = lane & 15, g = lane >> 4;
    int seq = (int)(blockIdx.x / (uint32_t)a.heads);
    asm("" : "+s"(seq));                                     // (a division's result stands in vector registers, and all that is made of it)
    const int64_t n = seq;
    const int h = (int)(blockIdx.x - n * a.heads), T = a.tokens;
    const int64_t row0 = n * T * a.heads + h;                // row of token 0; the next is `heads` behind
    // a token's row behind that: below 2^22, and so a channel's place below 2^29
    auto row_of = [&](int t) { return (uint32_t)(min(t, T - 1) * a.heads); };
    const int64_t state = a.indices ? a.indices[n] : n;
    const int col = 32 * wave + 2 * x;                       // the lane's columns are this and the next
    auto put = [&](int t, float lo, float hi) {
        const uint32_t at = row_of(t) * D + col;
        if (a.out_bf16) *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(a.o) + row0 * D + at) = pack_bf16x2(lo, hi);
        else *reinterpret_cast<f32x2 *>(static_cast<float *>(a.o) + row0 * D + at) = f32x2{lo, hi};
    };
    if (state < 0) {
        for (int t = g; t < T; t += 4) put(t, 0.f, 0.f);
        return;
    }
    // ---- everything is asked for at once: parents and tokens, which are needed first, then the state ----
    int32_t up = -2;
    if (wave == 0 && lane < T) up = a.parents[n * T + lane];
    constexpr int kPieces = TM * (D / 4) / kThreads;         // fours of a thread
    const int group = tid >> 4;
    auto own = [&](int i) { return L::kPlanes ? D / CH * i + 4 * x : CH * x + i; };      // a lane's channels in a group: four from here on
    [[maybe_unused]] Four<Tin> queries[kNodes][CH / 4];      // of large trees, of the group's own tokens
    [[maybe_unused]] Four<Tin> qv[kPieces];
    Four<Tin> kv[kPieces], lv[kPieces];
    Tin lh[kPieces];
    {
        const Tin *q = static_cast<const Tin *>(a.q) + row0 * D, *k = static_cast<const Tin *>(a.k) + row0 * D;
        const Tin *la = static_cast<const Tin *>(a.log_alpha) + (a.scalar_gate ? row0 : row0 * D);
        const uint32_t c = 4 * (tid % (D / 4));
#pragma unroll
        for (int r = 0; r < kPieces; ++r) {
            const uint32_t row = row_of((tid + kThreads * r) / (D / 4));
            kv[r] = *reinterpret_cast<const Four<Tin> *>(k + (row * D + c));
            if constexpr (!L::kPlanes) qv[r] = *reinterpret_cast<const Four<Tin> *>(q + (row * D + c));
            if (a.scalar_gate) lh[r] = la[row];
            else lv[r] = *reinterpret_cast<const Four<Tin> *>(la + (row * D + c));
        }
        if constexpr (L::kPlanes) {
#pragma unroll
            for (int r = 0; r < kNodes; ++r)
#pragma unroll
                for (int i = 0; i < CH; i += 4)
                    queries[r][i / 4] = *reinterpret_cast<const Four<Tin> *>(q + (row_of(group + kGroups * r) * D + (uint32_t)own(i)));
        }
    }
    [[maybe_unused]] Four<Tin> values[kPieces];
    [[maybe_unused]] float own_beta = 0.f;
    if constexpr (L::kHasValues) {
#pragma unroll
        for (int r = 0; r < kPieces; ++r) {
            const uint32_t c = 4 * (tid % (D / 4)), row = row_of((tid + kThreads * r) / (D / 4));
            values[r] = *reinterpret_cast<const Four<Tin> *>(static_cast<const Tin *>(a.v) + row0 * D + (row * D + c));
        }
        own_beta = load_as_float(static_cast<const Tin *>(a.beta) + row0 + row_of(tid));
    }
    // the state's rows 16 s + 4 g + i
    f32x2 s0[D / 16][4];
    {
        const float *from = a.states + (state * a.heads + h) * (D * D) + (4 * g) * D + col;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) s0[s][i] = __builtin_nontemporal_load(reinterpret_cast<const f32x2 *>(from + (16 * s + i) * D));
    }
    if (wave == 0) {
        lines[lane] = tree_line(up, T);
        parents[lane] = up;
        if (lane < 4) lost[lane] = 0u;
    }
    __syncthreads();
    // ---- tokens (one that is not there: no key, no query, no decay) ----
#pragma unroll
    for (int r = 0; r < kPieces; ++r) {
        const int t = (tid + kThreads * r) / (D / 4), c = 4 * (tid % (D / 4));
        const bool there = t < T && lines[t];
        f32x4 av = f32x4{1.f, 1.f, 1.f, 1.f} * (a.scalar_gate ? load_as_float(&lh[r]) : 0.f);
        if (!a.scalar_gate) av = widened(lv[r]);
#pragma unroll
        for (int e = 0; e < 4; ++e) av[e] = there ? fast_exp2(av[e] * kLog2e) : 1.f;
        *reinterpret_cast<f32x4 *>(al + t * L::kPitch + c) = av;
        *reinterpret_cast<Four<Tin> *>(kk + t * L::kPitch + c) = there ? kv[r] : Four<Tin>{};
        if constexpr (!L::kPlanes) *reinterpret_cast<Four<Tin> *>(qq + t * L::kPitch + c) = there ? qv[r] : Four<Tin>{};
        if constexpr (L::kHasValues) *reinterpret_cast<Four<Tin> *>(vs + t * L::kPitch + c) = values[r];
    }
    if (L::kHasValues && tid < TM) betas[tid] = own_beta;
    __syncthreads();

    // ---- up every token's line: the sums over channels, column j with lane j % 16, and the product of all decays ----
    float all[kNodes][CH], nk[kNodes][MT], nq[kNodes][MT];
    auto channels = [&](const auto *rows, int t, float (&v)[CH]) {
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
            const f32x4 w = load4(rows + t * L::kPitch + own(i));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i + e] = w[e];
        }
    };
    auto block_of = [](int r) constexpr { return (kGroups * r + kGroups - 1) / 16; };       // of a group's token r, and so of its ancestors the last
    auto query = [&](int r, int t, float (&v)[CH]) {
        if constexpr (!L::kPlanes) channels(qq, t, v);
        else
#pragma unroll
            for (int i = 0; i < CH; i += 4) {
                const f32x4 w = widened(queries[r][i / 4]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i + e] = lines[t] ? w[e] : 0.f;
            }
    };
#pragma unroll
    for (int r = 0; r < kNodes; ++r) {
        const int t = group + kGroups * r;
#pragma unroll
        for (int i = 0; i < CH; ++i) all[r][i] = 1.f;
#pragma unroll
        for (int c = 0; c < MT; ++c) nk[r][c] = nq[r][c] = 0.f;
        float b = 0.f, kt[CH], qt[CH];
        int j = -1;
        if (t < TM) {
            channels(kk, t, kt);
            query(r, t, qt);
            if (lines[t]) {
                b = L::kHasValues ? betas[t] : load_as_float(static_cast<const Tin *>(a.beta) + row0 + row_of(t));
                j = t;
            }
        }
        while (j >= 0) {
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
#pragma unroll
            for (int c = 0; c < MT; ++c) {
                if (c > block_of(r)) continue;
                const bool here = x == j - 16 * c;
                nk[r][c] = here ? dk : nk[r][c];
                nq[r][c] = here ? dq : nq[r][c];
            }
            j = parents[j];
        }
        bool lost_k = false, lost_q = false;
#pragma unroll
        for (int c = 0; c < MT; ++c) {
            if (c > block_of(r)) continue;
            const float dk = x + 16 * c == t ? 0.f : -b * nk[r][c], dq = a.scale * nq[r][c];
            // (zero here, one that is not finite stays out of the others' rows)
            lost_k |= !finite(dk);
            lost_q |= !finite(dq);
            nk[r][c] = finite(dk) ? dk : 0.f;
            nq[r][c] = finite(dq) ? dq : 0.f;
        }
        if (lost_k) atomicOr(lost + (t >> 5), 1u << (t & 31));
        if (lost_q) atomicOr(lost + 2 + (t >> 5), 1u << (t & 31));
    }
    __syncthreads();
    f32x2 vv[MT][4];
    float beta[MT][4];
    // (what of v and beta is not in LDS is asked for when there are registers for it)
    auto ask = [&]() {
        if constexpr (!L::kHasValues) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t row = row_of(16 * m + 4 * g + e);
                    vv[m][e] = load2(static_cast<const Tin *>(a.v) + row0 * D + (row * D + (uint32_t)col));
                    beta[m][e] = load_as_float(static_cast<const Tin *>(a.beta) + row0 + row);
                }
        }
    };
    f32x4 acc[2][MT][2];
    // ---- P_i0 k_i and scale P_i0 q_i, where the tokens stood, and their products with S_0: tokens 16 m + 4 g + e ----
    if constexpr (L::kPlanes) {
        float kt[kNodes][CH], qt[kNodes][CH];
#pragma unroll
        for (int r = 0; r < kNodes; ++r) {
            const int t = group + kGroups * r;
            channels(kk, t, kt[r]);
            query(r, t, qt[r]);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                kt[r][i] *= all[r][i];
                qt[r][i] *= all[r][i] * a.scale;
            }
        }
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[w][m][0] = acc[w][m][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        // a pass has half of the channels; channel 32 s + 16 i + 4 g + e of it stands at 32 s + 8 g + 4 i + e
        const int at = 32 * (D == 128 ? x >> 3 : 0) + 8 * (x & 3) + 4 * ((x >> 2) & 1);
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
            __syncthreads();
            if (D == 128 || x >> 3 == pass)
#pragma unroll
                for (int r = 0; r < kNodes; ++r)
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const float *from = (w ? qt[r] : kt[r]) + (D == 128 ? 4 * pass : 0);
                        uint32_t p[2][3];
#pragma unroll
                        for (int i = 0; i < 2; ++i) three_of(from[2 * i], from[2 * i + 1], p[i][0], p[i][1], p[i][2]);
#pragma unroll
                        for (int i = 0; i < 3; ++i)
                            *reinterpret_cast<u32x2 *>(lds + (3 * w + i) * L::kPlane + 2 * ((group + kGroups * r) * L::kPlanePitch + at)) = u32x2{p[0][i], p[1][i]};
                    }
            __syncthreads();
#pragma unroll
            for (int s = 0; s < D / 64; ++s) {
                bf16x8 b[2][3];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    u32x4 p[3];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x2 *of = s0[D / 32 * pass + 2 * s + i / 2] + 2 * (i % 2);
                        uint32_t hi, mid, lo;
                        three_of(of[0][j], of[1][j], hi, mid, lo);
                        p[0][i] = hi;
                        p[1][i] = mid;
                        p[2][i] = lo;
                    }
#pragma unroll
                    for (int i = 0; i < 3; ++i) b[j][i] = __builtin_bit_cast(bf16x8, p[i]);
                }
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        if (16 * m >= T) continue;
                        bf16x8 r[3];
#pragma unroll
                        for (int i = 0; i < 3; ++i)
                            r[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(lds + (3 * w + i) * L::kPlane + 2 * ((16 * m + x) * L::kPlanePitch + 32 * s + 8 * g)));
                        // small ones first; what is left out is below 2^-22 of a product
#pragma unroll
                        for (int i = 2; i >= 0; --i)
#pragma unroll
                            for (int k = 0; k <= i; ++k)
#pragma unroll
                                for (int j = 0; j < 2; ++j) acc[w][m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r[k], b[j][i - k], acc[w][m][j], 0, 0, 0);
                    }
                if (pass == 1 && s == 0) ask();
            }
        }
    } else {
        float *pk = reinterpret_cast<float *>(lds), *pq = pk + L::kRows;
        float kt[kNodes][CH], qt[kNodes][CH];
#pragma unroll
        for (int r = 0; r < kNodes; ++r) {
            const int t = min(group + kGroups * r, TM - 1);
            channels(kk, t, kt[r]);
            channels(qq, t, qt[r]);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                kt[r][i] *= all[r][i];
                qt[r][i] *= all[r][i] * a.scale;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kNodes; ++r) {
            const int t = group + kGroups * r;
            if (t >= TM) continue;
#pragma unroll
            for (int i = 0; i < CH; i += 4) {
                *reinterpret_cast<f32x4 *>(pk + t * L::kPitch + CH * x + i) = f32x4{kt[r][i], kt[r][i + 1], kt[r][i + 2], kt[r][i + 3]};
                *reinterpret_cast<f32x4 *>(pq + t * L::kPitch + CH * x + i) = f32x4{qt[r][i], qt[r][i + 1], qt[r][i + 2], qt[r][i + 3]};
            }
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                acc[w][m][0] = acc[w][m][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (16 * m >= T) continue;
                const float *rows = (w ? pq : pk) + (16 * m + x) * L::kPitch + 4 * g;
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    const f32x4 r = *reinterpret_cast<const f32x4 *>(rows + 16 * s);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) acc[w][m][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(r[i], s0[s][i][j], acc[w][m][j], 0, 0, 0);
                }
            }
    }
    __syncthreads();
    // ---- the matrices, and the inverses of the first one's diagonal blocks in their places ----
    float *sk = reinterpret_cast<float *>(lds), *sq = sk + TM * L::kSumPitch;
#pragma unroll
    for (int r = 0; r < kNodes; ++r) {
        const int t = group + kGroups * r;
        if (t >= TM) continue;
#pragma unroll
        for (int c = 0; c < MT; ++c) {
            sk[t * L::kSumPitch + 16 * c + x] = c > block_of(r) ? 0.f : nk[r][c];
            sq[t * L::kSumPitch + 16 * c + x] = c > block_of(r) ? 0.f : nq[r][c];
        }
    }
    if constexpr (L::kHasValues) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                vv[m][e] = load2(vs + (16 * m + 4 * g + e) * L::kPitch + col);
                beta[m][e] = betas[16 * m + 4 * g + e];
            }
    }
    // r, but for what is not finite, which the descendants of its token see and no others
    uint32_t odd = 0;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = beta[m][e] * (vv[m][e][j] - acc[0][m][j][e]);
                const bool ok = finite(v) || !lines[16 * m + 4 * g + e];
                acc[0][m][j][e] = finite(v) ? v : 0.f;
                odd |= (ok ? 0u : 1u) << (8 * m + 4 * j + e);
            }
    __syncthreads();
    if (group < MT) {
        // lane x has column x of the inverse: row by row, v_i = [i == x] + sum_{k < i} N_ik v_k
        float *block = sk + 16 * group * L::kSumPitch + 16 * group;
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float sum = i == x ? 1.f : 0.f;
#pragma unroll
            for (int k = 0; k < i; k += 4) {
                const f32x4 w = *reinterpret_cast<const f32x4 *>(block + i * L::kSumPitch + k);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k + e < i) sum = fmaf(w[e], v[k + e], sum);
            }
            v[i] = sum;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 16; ++i) block[i * L::kSumPitch + x] = v[i];
    }
    __syncthreads();

    // ---- down the blocks of tokens ----
    auto part = [&](const float *s, int m, int k) { return *reinterpret_cast<const f32x4 *>(s + (16 * m + x) * L::kSumPitch + 16 * k + 4 * g); };
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (16 * m >= T) continue;
#pragma unroll
        for (int k = 0; k <= m; ++k) {
            const f32x4 w = part(sk, m, k);
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[0][m][j] = k < m ? mfma16(w, acc[0][k][j], acc[0][m][j]) : mfma16(w, acc[0][m][j], f32x4{0.f, 0.f, 0.f, 0.f});
        }
#pragma unroll
        for (int k = 0; k <= m; ++k) {
            const f32x4 w = part(sq, m, k);
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[1][m][j] = mfma16(w, acc[0][k][j], acc[1][m][j]);
        }
    }
    const uint64_t lost_k = lost[0] | (uint64_t)lost[1] << 32, lost_q = lost[2] | (uint64_t)lost[3] << 32;
    if (__any(odd != 0 || (lost_k | lost_q) != 0)) {
        // of how many tokens of each line r, or a sum of k, was taken out
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const uint64_t line = lines[16 * m + x];
            f32x4 seen[2] = {};
#pragma unroll
            for (int k = 0; k <= m; ++k) {
                f32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (line >> (16 * k + 4 * g + e)) & 1 ? 1.f : 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    f32x4 marks;
#pragma unroll
                    for (int e = 0; e < 4; ++e) marks[e] = ((odd >> (8 * k + 4 * j + e)) | (uint32_t)(lost_k >> (16 * k + 4 * g + e))) & 1 ? 1.f : 0.f;
                    seen[j] = mfma16(w, marks, seen[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[1][m][j][e] = seen[j][e] > 0.f || (lost_q >> (16 * m + 4 * g + e)) & 1 ? __builtin_nanf("") : acc[1][m][j][e];
        }
    }
    bool some = false;                                       // not finite, of a row that may be nobody's
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = 16 * m + 4 * g + e;
            if (t >= T) continue;
            const bool there = lines[t] != 0;
            some |= !finite(acc[1][m][0][e]) || !finite(acc[1][m][1][e]);
            put(t, there ? acc[1][m][0][e] : 0.f, there ? acc[1][m][1][e] : 0.f);
        }
    if (!__any(some)) return;

    step_again<Tin, D>(a, lines, row0, (state * a.heads + h) * (D * D));
}

struct Commit {
    const void *k, *v, *log_alpha, *beta;
    float *states;
    const int32_t *indices, *kept;
    int32_t heads, tokens, most, scalar_gate;
};
constexpr int kAtOnce = 8;           // tokens in LDS

// The accepted tokens, as the decode kernel steps (kda_step.hip): a wave has 32 columns of a state, 8 row groups by 8 groups of four columns, in
// registers from the first token to the last.  256 x 32 states of 64 KiB through paths of up to 16 tokens in 192 us, 5.6 TB/s.
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
    constexpr int kBytes = StepLds<Tin, D, TM>::kBytes;
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
