/*
 * kda.h -- C ABI of libkda: Kimi Delta Attention (KDA), forward and backward, on one MI355X.
 *
 * KDA is the gated delta rule of the paper's Section 3, Eq. (1):
 *
 *     S_t = (I - beta_t k_t k_t^T) Diag(alpha_t) S_{t-1} + beta_t k_t v_t^T,
 *     o_t = scale * S_t^T q_t,          alpha_t = exp(log_alpha_t) in (0,1]^dk
 *
 * with one dk x dv state S per (sequence, head).  Two entry points compute it:
 * kda_chunk_fwd with the chunkwise WY / UT-transform algorithm of Section 3.1
 * (prefill), kda_recurrent_step with one literal step of Eq. (1) (decode,
 * Section 6.3 "Inference strategy").
 *
 * Conventions shared by every call
 *   - All tensor pointers are DEVICE pointers to contiguous row-major arrays,
 *     16-byte aligned.  The caller owns every buffer, including the workspace.
 *     The library allocates nothing, frees nothing, creates no stream or event
 *     and keeps no state between calls (beyond per-device caches of constant
 *     device attributes).
 *   - Calls are asynchronous on `hip_stream` (a hipStream_t passed as void*,
 *     NULL = default stream): every kernel of a call is launched on that stream,
 *     no host synchronisation happens inside (kda_chunk_fwd_check, which exists to
 *     wait, aside), and a call may be captured into a graph.  The current device has to
 *     be that of the tensors and of the stream (the Python binding sees to it).
 *   - Concurrency: calls may be issued from several host threads and on several
 *     streams at once, each with its own workspace (a workspace belongs to one call
 *     until that call has completed).  The bf16 prefill runs its per-chunk stage and
 *     its sequential stage as workgroups of ONE kernel: the sequential workgroups (one
 *     per (sequence, head), or a few for calls with few pairs and long sequences, each
 *     on half a compute unit, never more than half of the device's such places at a
 *     time) wait for the slots that the per-chunk workgroups behind them
 *     in the same grid produce.  The producers wait for nothing and are dispatched as
 *     soon as any half compute unit is free, so every wait ends; each wait is bounded
 *     all the same (about two seconds).  Should other work on the device starve the
 *     producers that long, the waiting workgroup gives up: the outputs it had still
 *     to write for that (sequence, head), to the end of the sequence (a call that scans
 *     ranges of a long sequence side by side: at least to the end of the range), and the
 *     final state if the stretch reaches it, are NaN, never stale data, and
 *     kda_chunk_fwd_check reports it.
 *   - Element offsets are 64-bit; tensors with more than 2^31 elements are fine.
 *   - Errors: a non-zero kda_status is returned and kda_last_error() holds a
 *     thread-local description.  For KDA_ERR_INVALID_ARG, KDA_ERR_UNSUPPORTED
 *     and KDA_ERR_WORKSPACE nothing has been launched.  No exception crosses
 *     the ABI.
 *   - log_alpha must be finite and <= 0 (alpha = 0 is not representable);
 *     alpha = 1 (log_alpha = 0) is allowed.  Values are never clamped.
 */
#ifndef KDA_H_
#define KDA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    KDA_OK = 0,
    KDA_ERR_INVALID_ARG = 1,   /* null pointer, negative size, bad combination   */
    KDA_ERR_UNSUPPORTED = 2,   /* head dim / chunk / dtype outside the built set */
    KDA_ERR_WORKSPACE = 3,     /* workspace missing, misaligned or too small     */
    KDA_ERR_LAUNCH = 4         /* the HIP runtime refused a launch               */
} kda_status;

typedef enum { KDA_F32 = 0, KDA_BF16 = 1 } kda_dtype;

/*
 * Problem description.
 *   Fixed-length batch : cu_seqlens == NULL, num_seqs == batch, every batch row
 *                        is one sequence of `seqlen` tokens.
 *   Packed batch       : cu_seqlens != NULL, batch == 1, `seqlen` is the total
 *                        number of packed tokens, sequence n owns tokens
 *                        [cu_seqlens[n], cu_seqlens[n+1]).
 * Supported: dk == dv in {64, 128}, chunk == 64, in_dtype KDA_F32 or KDA_BF16
 * (bf16 inputs with head dim 64 are processed by the fp32 kernels: exact
 * widening, fp32 arithmetic, fp32 o).  out_dtype KDA_F32 always; KDA_BF16 with
 * in_dtype KDA_BF16 and head dim 128 (o is computed in fp32 and rounded to
 * nearest even once, when it is stored; states stay fp32).
 */
typedef struct {
    int32_t   batch;       /* B                                                  */
    int64_t   seqlen;      /* T per batch row, or total packed tokens            */
    int32_t   heads;       /* H                                                  */
    int32_t   dk, dv;      /* key / value head dimension                         */
    int32_t   chunk;       /* C of Section 3.1; must be 64                       */
    int32_t   num_seqs;    /* N                                                  */
    kda_dtype in_dtype;    /* q, k, v, log_alpha, beta all share it              */
    kda_dtype out_dtype;   /* dtype of o                                         */
    float     scale;       /* multiplies o; 1.0f gives Eq. (1), dk^-0.5 gives    */
                           /* the App. C listing                                 */
    int64_t   max_seqlen;  /* packed batches only: upper bound on the longest    */
                           /* sequence, 0 = unknown (seqlen is assumed)          */
} kda_dims;

/*
 * Workspace, in bytes, with which kda_chunk_fwd runs `dims` in a single
 * segment (fastest).  kda_chunk_fwd also accepts any workspace of at least
 * kda_chunk_fwd_min_workspace_size(dims) bytes and then walks the time axis
 * in several segments, carrying the state between them.  Both return 0 for an
 * unsupported or malformed `dims`, and for problems that need no workspace.
 * KDA_F32 inputs: the minimum is 0 (one sequential kernel per sequence, head and
 * 32 state columns); with kda_chunk_fwd_workspace_size(dims) bytes (per chunk and
 * head three 64 x dk fp32 operand tiles, the lower triangles of two 64 x 64
 * matrices, dk + 64 floats, and 13 KiB that the size has always held and nothing
 * uses) a parallel per-chunk kernel and a matrix-core walk run instead, some thirty
 * times faster at 4 x 4096 tokens x 16 heads; anything in between runs the
 * sequential kernel.
 */
size_t kda_chunk_fwd_workspace_size(const kda_dims *dims);
size_t kda_chunk_fwd_min_workspace_size(const kda_dims *dims);

/*
 * Chunkwise prefill (Section 3.1: chunk expansion, WY representation, UT
 * transform, chunk state update, inter/intra-chunk output; the decay products
 * follow the reading gamma^{i->r} = exp(G^r - G^i), G the inclusive running
 * sum of log_alpha inside a chunk).  Each sequence is cut into chunks of 64
 * tokens starting at its own first token; a shorter last chunk is legal.
 *
 *   q, k       [B,T,H,dk]      in_dtype
 *   v          [B,T,H,dv]      in_dtype
 *   log_alpha  [B,T,H,dk]      in_dtype, natural log of the per-channel decay
 *   beta       [B,T,H]         in_dtype
 *   h0         [N,H,dk,dv]     fp32 initial states, or NULL for zeros
 *   cu_seqlens [N+1]           int32, device memory, non-decreasing, starts at
 *                              0, last entry <= T; or NULL (fixed length)
 *   o          [B,T,H,dv]      out_dtype; rows of tokens owned by no sequence
 *                              are left untouched
 *   hT         [N,H,dk,dv]     fp32 final states (state after the last token of
 *                              each sequence; equals h0 for an empty sequence),
 *                              or NULL if not wanted.  May alias h0.
 *   workspace                  device scratch, 256-byte aligned (may be NULL
 *                              when the required size is 0)
 * o must not alias any input.  Arithmetic: KDA_F32 inputs are processed in fp32
 * throughout; KDA_BF16 inputs use fp16 matrix-core operands with fp32
 * accumulation, fp32 cumulative decay and an fp32 state.  Domain of the KDA_BF16
 * path: |k_t| <= 4 and entries of q within +-3.9 (the paper's q and k are
 * L2-normalised, Section 4), and states, values, pseudo-values and k_t^T S (what the
 * key of a token reads of the state that its chunk starts from) small enough for
 * fp16 (below 65504 in magnitude).  bf16 inputs convert to fp16 exactly while their magnitude is
 * zero or within [2^-14, 65504]; smaller ones lose bits or flush, larger ones
 * become infinite.  Beyond the domain an fp16 operand overflows to infinity and
 * the affected outputs and states come back as Inf or NaN; kda_chunk_fwd_check
 * reports a key beyond the domain and a state that is not finite.
 */
kda_status kda_chunk_fwd(const kda_dims *dims,
                         const void *q, const void *k, const void *v,
                         const void *log_alpha, const void *beta,
                         const float *h0, const int32_t *cu_seqlens,
                         void *o, float *hT,
                         void *workspace, size_t workspace_bytes,
                         void *hip_stream);

/*
 * kda_chunk_fwd for callers that cannot allocate device memory and have no workspace to bring: code
 * under graph capture, tight serving loops, harnesses that forbid hipMalloc.  The workspace is a
 * static device array inside the library, kda_static_scratch_size() bytes (64 MiB) per GPU that the
 * library runs on, held until the process ends.  Everything else (arguments, results, arithmetic) is
 * that of kda_chunk_fwd given a workspace of that size: long inputs are walked in time segments with
 * the state carried between them.  The call allocates nothing and frees nothing.  A call whose
 * smallest workspace (kda_chunk_fwd_min_workspace_size) exceeds the array is refused with
 * KDA_ERR_WORKSPACE and launches nothing: at dk = dv = 128 that is beyond about 190 (sequence, head)
 * pairs per call.  All calls on one GPU share that GPU's array, which keeps the last call's contents
 * (each call clears what it needs at zero itself): calls that overlap in time on one GPU, from any
 * stream or thread, race on it and must not be made.  kda_chunk_fwd_check does not apply.
 */
size_t kda_static_scratch_size(void);
kda_status kda_chunk_fwd_static_scratch(const kda_dims *dims,
                                        const void *q, const void *k, const void *v,
                                        const void *log_alpha, const void *beta,
                                        const float *h0, const int32_t *cu_seqlens,
                                        void *o, float *hT, void *hip_stream);

/*
 * Backward pass of kda_chunk_fwd: gradients of  sum(o . d_o) + sum(hT . d_hT)  with respect to
 * every input.  The paper motivates a training kernel (Section 3.1 compares the chunkwise form
 * with the general DPLR one for exactly that purpose) but derives no backward algorithm; what
 * is computed here is the chain rule applied to Eq. (1), organised chunk by chunk through the
 * quantities of Section 3.1 (A_kk, A_qk, the UT transform, the chunk state update), in fp32
 * throughout.  Some products are formed from three bf16 pieces of their fp32 operands, which
 * hold them exactly, and accumulated in fp32: what is left out is at most 1.01 * 2^-24 of a
 * product, and the 2-norm errors of sums are smaller than with fp32 products (1.6e-7 against
 * 2.05e-7 at 128 terms).  That holds for values of d_o, the states and what is formed from them
 * down to 2^-110 (7.7e-34); smaller ones are rounded to multiples of 2^-133 there.  An infinity
 * in d_o, h0 or d_hT comes back as NaN in the gradients of its (sequence, head).
 * A decay between two tokens of a chunk is the product of two or three factors, each within
 * 2^(+-60), so that nothing overflows; a channel that decays by more than 2^-60 within 8 tokens
 * is added pair by pair where it still counts.
 *
 *   q, k, v, log_alpha, beta, h0, cu_seqlens   as for kda_chunk_fwd (in_dtype KDA_F32 or
 *                              KDA_BF16, dk == dv in {64, 128})
 *   d_o        [B,T,H,dv]      gradient of o in out_dtype, i.e. the dtype o had: fp32, or bf16
 *                              with bf16 inputs (rows of tokens owned by no sequence are not
 *                              read)
 *   d_hT       [N,H,dk,dv]     fp32 gradient of the final states, or NULL for zeros
 *   dq, dk, dlog_alpha [B,T,H,dk], dv [B,T,H,dv], dbeta [B,T,H]    fp32, written; rows of
 *                              tokens owned by no sequence are left untouched
 *   dh0        [N,H,dk,dv]     fp32 gradient of the initial states (equals d_hT for an empty
 *                              sequence), or NULL if not wanted
 *   workspace                  at least kda_chunk_bwd_workspace_size(dims) bytes, 256-byte
 *                              aligned: the state at the start of every chunk and the
 *                              gradient of the state at its end (2 * dk * dv floats per chunk
 *                              and head), two [tokens, H, dv] arrays, the decay-scaled
 *                              operands and two triangular C x C matrices per chunk and head,
 *                              and a fifth that is spare (the size is part of the interface:
 *                              callers keep it with their plans and buffers); it is not
 *                              bounded by time segments
 * No gradient may alias an input or another gradient.  Sequences of more than 65535 * 64
 * tokens are KDA_ERR_UNSUPPORTED.  Everything runs on `hip_stream`.
 */
size_t kda_chunk_bwd_workspace_size(const kda_dims *dims);
kda_status kda_chunk_bwd(const kda_dims *dims,
                         const void *q, const void *k, const void *v,
                         const void *log_alpha, const void *beta,
                         const float *h0, const int32_t *cu_seqlens,
                         const void *d_o, const float *d_hT,
                         float *dq, float *dk, float *dv, float *dlog_alpha, float *dbeta,
                         float *dh0,
                         void *workspace, size_t workspace_bytes,
                         void *hip_stream);

/*
 * Fused input prologue (Section 4, "Neural Parameterization").  With a kda_prologue the kernels
 * take the raw projections and apply, in fp32 and before anything else,
 *     q <- q / sqrt(sum_c q_c^2 + l2norm_eps),   k likewise            (L2Norm over dk)
 *     beta <- 1 / (1 + exp(-beta))                                       (Sigmoid)
 *     log_alpha[c] <- -a_scale[h] * log(1 + exp(gate[c] + dt_bias[h][c]))
 * The paper does not print its decay function f; this is the softplus form of the two models
 * it names as its pattern, with the constants exposed (a_scale = NULL means 1, dt_bias = NULL
 * means 0, which gives log_alpha = -softplus(gate)).  The short convolution, Swish and the
 * projections themselves stay with the caller.
 */
typedef struct {
    float        l2norm_eps;   /* >= 0                                            */
    const float *a_scale;      /* [H]     fp32, device memory, or NULL            */
    const float *dt_bias;      /* [H,dk]  fp32, device memory, or NULL            */
} kda_prologue;

/*
 * Fused output gate (Section 4): with a kda_epilogue the kernels replace each o (one vector of
 * dv values per token and head) by
 *     o <- Sigmoid(gate) * o / sqrt(mean_j o_j^2 + rms_eps) * norm_weight
 * in fp32 before they store it (`scale` is applied to o first; the prefill carries the factor
 * norm_weight * Sigmoid(gate) from its per-chunk stage to its sequential stage as fp16, the decode
 * kernel evaluates it in fp32).  The paper gives neither the epsilon nor the shape of the learned
 * RMSNorm weight: one vector of dv values shared by all heads is taken (NULL = ones).  The gate's
 * and the output's projections stay with the caller.
 */
typedef struct {
    float        rms_eps;      /* >= 0                                                       */
    const void  *gate;         /* gate logits, same shape and dtype as v ([..,H,dv]), device  */
    const float *norm_weight;  /* [dv] fp32, device memory, or NULL                           */
} kda_epilogue;

/*
 * Workspace sizes for kda_chunk_fwd_fused: as kda_chunk_fwd_workspace_size and
 * kda_chunk_fwd_min_workspace_size, plus, when `epilogue` is not NULL, room for the gate factors that
 * the per-chunk stage leaves for the sequential stage (16 KiB per chunk and head held at once).
 * With epilogue == NULL they equal the plain functions.  A fused call whose workspace is smaller
 * than the first figure still runs, in more segments.
 */
size_t kda_chunk_fwd_fused_workspace_size(const kda_dims *dims, const kda_epilogue *epilogue);
size_t kda_chunk_fwd_fused_min_workspace_size(const kda_dims *dims, const kda_epilogue *epilogue);

/*
 * kda_chunk_fwd with the fused stages: `prologue` (or NULL: q, k, gate = log_alpha and beta are
 * taken as kda_chunk_fwd takes them) and `epilogue` (or NULL: o is stored as it is).  Everything
 * else is as for kda_chunk_fwd.  Built for KDA_BF16 inputs with dk == dv == 128.
 */
kda_status kda_chunk_fwd_fused(const kda_dims *dims, const kda_prologue *prologue,
                               const kda_epilogue *epilogue,
                               const void *q_raw, const void *k_raw, const void *v,
                               const void *gate, const void *beta_logit,
                               const float *h0, const int32_t *cu_seqlens,
                               void *o, float *hT,
                               void *workspace, size_t workspace_bytes,
                               void *hip_stream);

/*
 * kda_chunk_fwd for the scalar-gate special case of Eq. (1) (Section 2.2: alpha_t = a_t I, one
 * decay per token and head): log_alpha_head is [B,T,H] in in_dtype, everything else as for
 * kda_chunk_fwd.  The result equals kda_chunk_fwd on that decay repeated over the dk channels; the
 * per-chunk kernel is cheaper (the decay leaves the matrix-core operands and multiplies the fp32
 * tiles instead, so no range handling is needed whatever the decay).  Built for KDA_BF16 inputs with
 * dk == dv == 128; workspace sizes as for kda_chunk_fwd.
 */
kda_status kda_chunk_fwd_scalar_gate(const kda_dims *dims,
                                     const void *q, const void *k, const void *v,
                                     const void *log_alpha_head, const void *beta,
                                     const float *h0, const int32_t *cu_seqlens,
                                     void *o, float *hT,
                                     void *workspace, size_t workspace_bytes,
                                     void *hip_stream);

/*
 * Optional check after a bf16 kda_chunk_fwd: waits for `hip_stream` and reads
 * the status word that the call left in `workspace` (same dims, workspace and
 * size as that call).  The sequential workgroups of the prefill wait, for a
 * bounded time, for each workspace slot; if such a wait ever ran out, the call
 * has written NaN to o from that point of the (sequence, head) on (see the
 * conventions above) and this returns KDA_ERR_LAUNCH.  If a state of the call ended
 * up not finite (an fp16 operand overflowed) or a key was beyond the domain
 * stated at kda_chunk_fwd it returns KDA_ERR_INVALID_ARG.  KDA_OK otherwise (also for
 * calls that keep no status word: fp32 inputs).
 */
kda_status kda_chunk_fwd_check(const kda_dims *dims, const void *workspace, size_t workspace_bytes,
                               void *hip_stream);

/*
 * One decode step of Eq. (1) for N = dims->num_seqs sequences (Section 6.3):
 *     S <- Diag(alpha) S;  r = v - S^T k;  S <- S + beta k r^T;  o = scale S^T q.
 * dims->seqlen must be 1 and dims->batch == dims->num_seqs.
 *
 *   q, k, log_alpha [N,H,dk]   in_dtype
 *   v               [N,H,dv]   in_dtype
 *   beta            [N,H]      in_dtype
 *   S               [N,H,dk,dv] fp32, read and written IN PLACE
 *   o               [N,H,dv]   out_dtype
 * All arithmetic is fp32.  No workspace.
 */
kda_status kda_recurrent_step(const kda_dims *dims,
                              const void *q, const void *k, const void *v,
                              const void *log_alpha, const void *beta,
                              float *S, void *o, void *hip_stream);

/*
 * Decode over a state pool (serving-shaped variant of kda_recurrent_step, same
 * Eq. (1) and Section 6.3): sequence n works on the state S_pool[state_indices[n]]
 * and takes Tq = dims->seqlen new tokens (1 <= Tq <= 8) through it in order, e.g.
 * the draft tokens of a speculative-decoding verification step.  The state is read
 * once and written once per call, whatever Tq is.  dims->batch == dims->num_seqs = N.
 *
 *   q, k, log_alpha [N,Tq,H,dk]   in_dtype
 *   v               [N,Tq,H,dv]   in_dtype
 *   beta            [N,Tq,H]      in_dtype
 *   S_pool          [P,H,dk,dv]   fp32 pool of P states; only the addressed ones are
 *                                 read and written, in place
 *   state_indices   [N]           int32, device memory; entry n in [0,P) names the state
 *                                 of sequence n, a negative entry skips the sequence
 *                                 (its rows of o are left untouched); NULL = 0,1,..,N-1.
 *                                 Entries are not range-checked against P, and two
 *                                 sequences naming the same state race.
 *   o               [N,Tq,H,dv]   out_dtype; o of token t reads the state after token t
 * All arithmetic is fp32.  No workspace.
 */
kda_status kda_recurrent_steps_pooled(const kda_dims *dims,
                                      const void *q, const void *k, const void *v,
                                      const void *log_alpha, const void *beta,
                                      float *S_pool, const int32_t *state_indices,
                                      void *o, void *hip_stream);

/* kda_recurrent_steps_pooled with one decay per token and head: log_alpha_head is [N,Tq,H]. */
kda_status kda_recurrent_steps_pooled_scalar_gate(const kda_dims *dims,
                                                  const void *q, const void *k, const void *v,
                                                  const void *log_alpha_head, const void *beta,
                                                  float *S_pool, const int32_t *state_indices,
                                                  void *o, void *hip_stream);

/*
 * kda_recurrent_steps_pooled with the fused stages (either may be NULL; see kda_prologue and
 * kda_epilogue); q_raw, k_raw, gate [N,Tq,H,dk], beta_logit [N,Tq,H], epilogue->gate [N,Tq,H,dv].
 */
kda_status kda_recurrent_steps_fused(const kda_dims *dims, const kda_prologue *prologue,
                                     const kda_epilogue *epilogue,
                                     const void *q_raw, const void *k_raw, const void *v,
                                     const void *gate, const void *beta_logit,
                                     float *S_pool, const int32_t *state_indices,
                                     void *o, void *hip_stream);

/*
 * The decode entry points above in one, with two choices in `flags`: KDA_STEPS_SCALAR_GATE, log_alpha is [N,Tq,H] (prologue and
 * epilogue must then be NULL); KDA_STEPS_ZERO_SKIPPED, the rows of o of a skipped sequence are written as zeros instead of left
 * untouched, for callers that want all of a fresh o defined.
 */
enum { KDA_STEPS_SCALAR_GATE = 1, KDA_STEPS_ZERO_SKIPPED = 2 };
kda_status kda_recurrent_steps(const kda_dims *dims, const kda_prologue *prologue, const kda_epilogue *epilogue,
                               const void *q, const void *k, const void *v, const void *log_alpha, const void *beta,
                               float *S_pool, const int32_t *state_indices, void *o, uint32_t flags, void *hip_stream);

/*
 * Zeros in the rows [0, cu_seqlens[0]) and [cu_seqlens[num_seqs], tokens) of up to eight arrays of `tokens` rows of
 * row_bytes[i] bytes each (a multiple of 4; arrays 16-byte aligned): the tokens of a packed batch that belong to no sequence,
 * which kda_chunk_fwd leaves untouched in o and kda_chunk_bwd in the per-token gradients.  For callers that want them defined.
 */
kda_status kda_clear_unowned_rows(const int32_t *cu_seqlens, int32_t num_seqs, int64_t tokens, int32_t num_arrays,
                                  void *const *arrays, const size_t *row_bytes, void *hip_stream);

/*
 * ---- Softmax attention: the other layers of a hybrid stack ----
 *
 * The paper's model interleaves KDA with layers of softmax attention (Section 4, "Hybrid model architecture").  These entry points
 * compute them: causal attention with grouped heads over fixed or packed batches, forward and backward, for local layers with a
 * sliding window and a few first tokens (sinks) that stay visible; and its serving form over a paged cache held in 8 bits
 * (kda_cache_append, kda_cache_attn).
 *
 * Query i of a sequence sees key j of it when  j <= i  and  (window == 0  or  i - j < window  or  j < sinks).
 * heads_q is a multiple of heads_kv; query head h reads key head h / (heads_q / heads_kv).
 */
typedef struct {
    int32_t   batch;       /* B                                                                        */
    int64_t   seqlen;      /* T per batch row, or total packed tokens (as in kda_dims), at most 2^30    */
    int32_t   heads_q, heads_kv;
    int32_t   dim;         /* head dimension of q, k and v: 64 or 128                                   */
    int32_t   num_seqs;    /* N: == batch, or the sequences of a packed batch                           */
    kda_dtype in_dtype;    /* KDA_BF16                                                                  */
    kda_dtype out_dtype;   /* dtype of o (kda_window_attn_bwd: KDA_BF16)                                */
    float     scale;       /* multiplies q . k; in [1e-30, 1e30], usually dim^-0.5                      */
    int64_t   window;      /* visible tokens before a query, itself included; 0: all                    */
    int32_t   sinks;       /* first tokens of a sequence visible beyond the window, 0..64               */
    int64_t   q_stride, k_stride, v_stride;    /* elements from a token to the next: 0 = contiguous     */
                           /* (heads x dim), else at least that, a multiple of 8, at most 2^24          */
                           /* (q, k and v may be slices of one projection's output)                     */
} kda_attn_dims;

/*
 *   q          [B,T,heads_q,dim]   k, v [B,T,heads_kv,dim]    bf16, 16-byte aligned
 *   cu_seqlens [N+1]               int32, device memory, as for kda_chunk_fwd, or NULL
 *   o          [B,T,heads_q,dim]   out_dtype; rows of tokens owned by no sequence are left untouched
 *   lse        [B,heads_q,T]       fp32: log sum_j exp(scale q_i . k_j) over the keys that i sees, or NULL
 * Products on the bf16 matrix cores with fp32 accumulation, softmax statistics in fp32, its terms rounded to bf16 ahead of the
 * product with v.  o must not alias an input.  Values that are not finite reach the outputs of the queries that see them and no others: a query that sees a
 * value of v that is not finite gets NaN or an infinity there, in every channel concerned, one that sees a key that is not
 * finite, or is not finite itself, NaN; but for a logit of minus infinity, whose term is zero, so that the key is as one that is not seen (a query
 * with no other logits gets zeros, and lse minus infinity).  (Such a tile is worked through twice.)  o is finite for values of v up to 2^127; the products
 * q . k, ahead of the scale, have to stay within fp32.  No workspace.
 */
kda_status kda_window_attn_fwd(const kda_attn_dims *dims, const void *q, const void *k, const void *v, const int32_t *cu_seqlens,
                               void *o, float *lse, void *hip_stream);

/*
 * Gradients of sum(o . d_o) with respect to q, k and v.
 *   o, lse     what kda_window_attn_fwd gave for the same dims and inputs, o in bf16
 *   d_o        [B,T,heads_q,dim]   bf16
 *   dq         [B,T,heads_q,dim]   dk, dv [B,T,heads_kv,dim]    bf16, contiguous, written; rows of tokens owned by no sequence are
 *                                  left untouched.  No gradient may alias an input or another gradient.
 *   workspace                      at least kda_window_attn_bwd_workspace_size(dims) bytes, 256-byte aligned
 * Sums in fp32 in an order that depends on the sizes alone (no atomics: the same call gives the same bits); the softmax's terms and
 * their gradients are rounded to bf16 ahead of the products, and each gradient once when it is stored.  What is not finite
 * reaches the gradients that depend on it and no others.
 */
size_t kda_window_attn_bwd_workspace_size(const kda_attn_dims *dims);
kda_status kda_window_attn_bwd(const kda_attn_dims *dims, const void *q, const void *k, const void *v, const int32_t *cu_seqlens,
                               const void *o, const float *lse, const void *d_o, void *dq, void *dk, void *dv,
                               void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ---- The serving form: a paged cache of keys and values held in 8 bits ----
 *
 * Keys and values of heads_kv heads stand in pages of page_size tokens as e4m3 codes (OCP: no infinities, 448 the largest), with one
 * fp32 scale for each page and head: value = code * scale.
 *   k, v           [num_pages,heads_kv,page_size,dim]   codes, 16-byte aligned
 *   k_scale, v_scale [num_pages,heads_kv]               fp32
 *   block_table    [num_seqs,max_pages]   int32: token t of sequence n stands in page block_table[n][t / page_size], at t % page_size.
 *                                         An entry outside [0, num_pages) is no page: what would be appended there is dropped, and
 *                                         its tokens are not visible.  Sequences may share pages that they only read.
 *   kv_lens        [num_seqs]             int32: see the calls
 */
typedef struct {
    int32_t  num_seqs;
    int32_t  heads_q, heads_kv;    /* heads_q a multiple of heads_kv                                          */
    int32_t  dim;                  /* 64 or 128                                                               */
    int32_t  page_size;            /* 16, 32, 64 or 128                                                       */
    int64_t  num_pages;
    int32_t  max_pages;            /* columns of block_table; max_pages * page_size at most 2^30              */
    void    *k, *v;
    float   *k_scale, *v_scale;
    const int32_t *block_table, *kv_lens;
} kda_cache;

/*
 * Position rotation: channel pair i of a token at position p turns by the angle p * inv_freq[i].  Pairs are (i, i + num_freqs)
 * or, interleaved, (2 i, 2 i + 1); channels from 2 * num_freqs on stay as they are.
 */
typedef struct {
    const float *inv_freq;         /* [num_freqs] fp32, device memory                                         */
    int32_t      num_freqs;        /* a multiple of 8, at most dim / 2                                        */
    int32_t      interleaved;
} kda_rope;

/*
 * Appends new tokens to the cache: sequence n holds kv_lens[n] tokens before the call (a negative entry skips the sequence), and its
 * new ones take the positions from there on.  kv_lens is not changed: the caller adds to it.
 *   seqlen, cu_seqlens   tokens of each sequence, at most 2^30, or with cu_seqlens [num_seqs+1] (as for kda_chunk_fwd) all of a packed batch's
 *   k, v           [..,heads_kv,dim]   bf16, [num_seqs,seqlen] or packed rows; strides in elements from a token to the next as in kda_attn_dims
 *   rope           rotation of k (and q), or NULL: as they are
 *   k_out          [..,heads_kv,dim]   bf16: the rotated keys, for a prefill that follows, or NULL
 *   q, q_out       [..,heads_q,dim]    bf16: queries to be rotated at their tokens' positions, and where to; NULL both or neither.  k_out may
 *                  be k and q_out q, where those are contiguous
 * Scales: powers of two.  A page and head's scale is the smallest (2^-100 at least) with which its largest new value is at most 448 codes'
 * steps, or the one it has, if that is larger and the page holds older tokens; where it grows, the older tokens' codes are rounded again
 * to the new scale.  Codes are rounded to nearest even from the fp32 rotation; values that are not finite are stored as NaN and leave the
 * scale alone.  Whatever stands in a page behind the sequence's last token is left as it is.  A page that is appended to must belong to
 * one sequence.
 *   flags          rows of q_out (KDA_APPEND_ZERO_Q) and k_out (KDA_APPEND_ZERO_K) of skipped sequences and of tokens owned by none are
 *                  written as zeros instead of left untouched
 */
enum { KDA_APPEND_ZERO_Q = 1, KDA_APPEND_ZERO_K = 2 };
kda_status kda_cache_append(const kda_cache *cache, int64_t seqlen, const void *k, const void *v, int64_t k_stride, int64_t v_stride,
                            const int32_t *cu_seqlens, const kda_rope *rope, void *k_out, const void *q, int64_t q_stride, void *q_out,
                            uint32_t flags, void *hip_stream);

/* A call of kda_cache_attn. */
typedef struct {
    int32_t   tokens;              /* new tokens of every sequence: 0..8                                      */
    int64_t   q_stride;            /* elements from a token of q to the next, as in kda_attn_dims             */
    int64_t   window;              /* as in kda_attn_dims                                                     */
    int32_t   sinks;               /* 0..64                                                                   */
    float     scale;               /* in [1e-30, 1e30]                                                        */
    int64_t   max_kv_len;          /* upper bound of kv_lens, 0 = unknown (max_pages * page_size): it sets how */
                                   /* far the keys are split, and is not needed for correctness               */
    kda_dtype out_dtype;
} kda_cache_query;

/*
 * Attention of each sequence's newest tokens over the cache: kv_lens[n] counts the tokens it holds, the new ones (appended before) among
 * them, so that new token t stands at position kv_lens[n] - tokens + t and sees what it sees of kda_window_attn_fwd.  A token that sees
 * nothing (kv_lens[n] <= 0, a position below zero: a batch of sequences with fewer new tokens is padded in front) gets zeros.
 *   q [num_seqs,tokens,heads_q,dim] bf16      o [num_seqs,tokens,heads_q,dim] out_dtype
 *   workspace   at least kda_cache_attn_workspace_size bytes (0 for some calls), 256-byte aligned
 * Products in fp32, the softmax's terms rounded to bf16 ahead of the product with v, as in kda_window_attn_fwd, whatever out_dtype is.
 * Scales may be any finite numbers here, so that scale * k_scale is finite and, for full precision, v_scale is 2^-110 at least and within a factor
 * of 2^100 of the sequence and head's largest: results are finite for values up to 2^127.  What is not finite reaches the rows that see it and no
 * others, whatever stands behind the last token of a page or in pages that no row sees.
 */
size_t kda_cache_attn_workspace_size(const kda_cache *cache, const kda_cache_query *query);
kda_status kda_cache_attn(const kda_cache *cache, const kda_cache_query *query, const void *q, void *o, void *workspace,
                          size_t workspace_bytes, void *hip_stream);

/*
 * ---- Draft trees: several tokens of a sequence verified at once, of which any path from the root may be accepted ----
 *
 * A sequence has up to 64 drafted tokens.  parents[n][t] is the index of the token that token t follows, below t, or -1 where it follows what
 * the sequence holds.  Any other entry means that there is no token t (sequences of a batch may have fewer than others), and a token whose
 * parent is not there is not there either.  depth(t): 0 for a token that follows what the sequence holds, else its parent's and one.
 * A token's ancestors are its parent and its parent's ancestors.
 *
 * A step of a hybrid stack: kda_rotate turns queries and keys by the positions of their depths, kda_cache_append (without rope) puts
 * token t's key and value at place kv_lens[n] + t of the cache, kda_cache_tree_attn and kda_tree_steps read cache and states without changing
 * them, and once the accepted path is known kda_cache_keep and kda_tree_commit make its tokens what the sequence holds.
 */

/*
 * Position rotation by positions of one to four axes (time, height and width of an image's token; one axis: a text's).
 *   q [B,T,heads_q,dim]   k [B,T,heads_k,dim]   dtype, 16-byte aligned; k may be NULL (heads_k 0)
 *   positions [axes,B,T]  int32
 * Channel pair i, (i, i + num_freqs) or interleaved (2 i, 2 i + 1), turns by the angle positions[axis_of_freq[i]][b][t] * inv_freq[i];
 * channels from 2 * num_freqs on stay as they are.  inverse: by the angle's negative, which is the gradient of the rotation as well: dq, dk from
 * the gradients of q_out, k_out.  q_out and k_out are contiguous; q_out may be q and k_out k, where those are contiguous; no other
 * outputs may overlap inputs or one another.  Angles are reduced in 64 bits, products in fp32, each output rounded once.  What is not finite
 * reaches its own pair alone.
 */
typedef struct {
    int32_t        batch;
    int64_t        seqlen;
    int32_t        heads_q, heads_k;
    int32_t        dim;                /* 64 or 128                                                               */
    kda_dtype      dtype;              /* of q, k and what is written                                             */
    int64_t        q_stride, k_stride; /* elements from a token to the next, as in kda_attn_dims                  */
    int32_t        axes;               /* 1..4                                                                    */
    int32_t        num_freqs;          /* a multiple of 8, at most dim / 2                                        */
    const float   *inv_freq;           /* [num_freqs] fp32, device memory                                         */
    const uint8_t *axis_of_freq;       /* [num_freqs], HOST memory, read during the call: below axes; NULL: all 0 */
    int32_t        interleaved, inverse;
} kda_rotation;
kda_status kda_rotate(const kda_rotation *rotation, const void *q, const void *k, const int32_t *positions, void *q_out, void *k_out,
                      void *hip_stream);

/*
 * Attention of every sequence's drafted tokens over the cache, like kda_cache_attn but for whom a token sees: kv_lens[n] (0 or more; a negative
 * one skips the sequence, whose rows of o become zeros) counts what the sequence holds without the drafted tokens, whose keys and values
 * stand at places kv_lens[n] + t.  Token t is at position kv_lens[n] + depth(t), and sees of what is held, of its ancestors and itself
 * what is at position j with  window == 0  or  its position - j < window  or  j < sinks.  Rows of tokens that are not there are zeros.
 *   query       tokens 0..64, the rest as for kda_cache_attn; max_kv_len: upper bound of kv_lens[n] + tokens
 *   parents     [num_seqs,tokens] int32
 *   workspace   at least kda_cache_tree_attn_workspace_size bytes (0 for some calls), 256-byte aligned
 * The softmax's terms go to the product with v rounded to bf16 where o is bf16 (to 2^-16 of themselves for heads of 128 and up to 16 rows, tokens x heads_q / heads_kv), and
 * to 2^-16 of themselves where it is fp32, which takes about 1.3 times as long.
 * Scales and what is not finite: as for kda_cache_attn.  o must not alias an input.
 */
size_t kda_cache_tree_attn_workspace_size(const kda_cache *cache, const kda_cache_query *query);
kda_status kda_cache_tree_attn(const kda_cache *cache, const kda_cache_query *query, const void *q, const int32_t *parents, void *o,
                               void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The accepted tokens of a tree become the end of what the sequence holds: the keys and values at places kv_lens[n] + kept[n][i] of the cache move
 * to kv_lens[n] + i, in all of `layers` caches that lie one behind the other (k, v [layers,num_pages,heads_kv,page_size,dim], k_scale, v_scale
 * [layers,num_pages,heads_kv]) and share block_table and kv_lens.  kv_lens is not changed: the caller adds to it.
 *   kept        [num_seqs,max_kept] int32, max_kept up to 64: indices of drafted tokens, increasing.  An entry that is negative or not above the
 *               one before ends the path.  A sequence with kv_lens[n] < 0 is skipped.
 * A page and head's scale becomes the largest of those of the tokens that move into it and, where older tokens stand in it, its own; codes
 * whose scale grows are rounded to it once.  Scales are positive, as kda_cache_append makes them.  What stands behind the kept tokens is left
 * as it is.  A token without a page, there or where it would go, is dropped.  Pages that are written must belong to one sequence.
 */
kda_status kda_cache_keep(const kda_cache *cache, int32_t layers, const int32_t *kept, int32_t max_kept, void *hip_stream);

/*
 * KDA over a draft tree: token t steps from the state behind its parent, or from the sequence's own, and its output reads the state behind it,
 *     S_t = (I - beta_t k_t k_t^T) Diag(alpha_t) S_parent(t) + beta_t k_t v_t^T,      o_t = scale * S_t^T q_t.
 * The states are read once and not changed.  dims as for kda_recurrent_steps_pooled, seqlen 0..64 tokens of every sequence;
 *   q, k, log_alpha [N,Tq,H,dk]   v [N,Tq,H,dv]   beta [N,Tq,H]   S_pool [P,H,dk,dv] fp32   state_indices [N] int32 or NULL, all as there, but
 *                  that sequences may read the same state; rows of o of skipped sequences and of tokens that are not there become zeros
 *   parents        [N,Tq] int32
 *   o              [N,Tq,H,dv]   out_dtype, either with either in_dtype
 *   flags          KDA_STEPS_SCALAR_GATE: log_alpha is [N,Tq,H]
 * All arithmetic is of fp32's precision (of states, and of keys and queries with a line's decays, below 2^-110: to 2^-126; sums over channels of two
 * tokens' vectors, with the scale, to 2^-126 ahead of the values that they weigh).  Where such sums or what they weigh leave fp32's range, the rows
 * concerned are formed from state to state, as kda_recurrent_steps forms them along a line (but for the order of sums), and in a time that grows with the lines.  What is not
 * finite in a token, or becomes so on the way, reaches its own row and its descendants' alone.  o must not alias an input.  No workspace.
 */
kda_status kda_tree_steps(const kda_dims *dims, const void *q, const void *k, const void *v, const void *log_alpha, const void *beta,
                          const float *S_pool, const int32_t *state_indices, const int32_t *parents, void *o, uint32_t flags, void *hip_stream);

/*
 * Takes the states through the accepted tokens of a tree, in place: sequence n's through tokens kept[n][0], kept[n][1], ... of the k, v,
 * log_alpha and beta that kda_tree_steps had (dims->seqlen: their tokens a sequence).  kept [N,max_kept] as for kda_cache_keep; an entry of seqlen
 * or more ends the path too.  A state without an accepted token is not touched.  Two sequences naming the same state race.
 */
kda_status kda_tree_commit(const kda_dims *dims, const void *k, const void *v, const void *log_alpha, const void *beta, float *S_pool,
                           const int32_t *state_indices, const int32_t *kept, int32_t max_kept, uint32_t flags, void *hip_stream);

/*
 * ---- Pages that several sequences share ----
 *
 * block_table as in kda_cache; page_refs [num_pages] int32: how many of its entries name a page.  A page with none is free.
 * Entries outside [0, num_pages) are no page and not counted.  Counts are the caller's to begin with (zeros beside a table of -1) and kept by these calls;
 * they are 16-byte aligned.
 */

/*
 * Rows of the table become copies of other rows, in place: row n what row source[n] was (source[n] == n or >= num_seqs: it stays), or
 * empty (-1) where source[n] < 0, which frees what it alone had.  Beams that are carried on, dropped or doubled, prompts that are shared,
 * and sequences that end.  page_refs follows.  num_seqs at most 8192, max_pages below 2^24.
 */
kda_status kda_pages_fork(int32_t *block_table, int32_t num_seqs, int32_t max_pages, int32_t *page_refs, int64_t num_pages,
                          const int32_t *source, void *hip_stream);

/*
 * Makes every sequence the only owner of the pages that it writes next, when it grows from kv_lens[n] to new_lens[n] tokens (one that does not
 * grow, or has a negative length, is skipped): entries of the columns kv_lens[n] / page_size up to that of its last token that are no page,
 * or a page with more than one reference when the call begins, become free pages, the lowest-numbered first, in the order of rows and then
 * columns; a page that is replaced loses a reference.  Tokens behind the table's columns get no page.
 *   copies      [num_seqs,2] int32, written: (from, to) for a sequence whose page of column kv_lens[n] / page_size is replaced and holds older
 *               tokens, for kda_cache_copy_pages; else (-1, -1)
 *               (a page whose last reference goes is free from then on: the copies have to be made before anything else takes or writes it)
 *   missing     [1] int32, written: 0, or by how many pages the free ones fall short: then nothing else is changed, and copies are all (-1, -1)
 * num_seqs at most 8192, num_seqs * max_pages below 2^31 - 1024.  workspace: kda_pages_reserve_workspace_size bytes, 256-byte aligned.
 */
size_t kda_pages_reserve_workspace_size(int32_t num_seqs, int32_t max_pages, int64_t num_pages);
kda_status kda_pages_reserve(int32_t *block_table, int32_t num_seqs, int32_t max_pages, int32_t page_size, int32_t *page_refs, int64_t num_pages,
                             const int32_t *kv_lens, const int32_t *new_lens, int32_t *copies, int32_t *missing, void *workspace,
                             size_t workspace_bytes, void *hip_stream);

/*
 * Moves the pages in use to the front of the pool: with U of them, those at U and above take the free places below, the lowest first, in
 * order.  Table and counts are changed; the pages themselves are the caller's to move:
 *   moves       [num_pages / 2,2] int32, written: (from, to), and (-1, -1) behind the last
 * for kda_cache_copy_pages, before anything else writes them.  workspace: 4 * num_pages + 256 bytes, 256-byte aligned.
 */
kda_status kda_pages_compact(int32_t *block_table, int32_t num_seqs, int32_t max_pages, int32_t *page_refs, int64_t num_pages, int32_t *moves,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Copies pages, codes and scales, in all of `layers` caches that lie one behind the other (as for kda_cache_keep): pairs [num_pairs,2] int32, device
 * memory, (from, to).  A pair with an entry outside [0, num_pages) is skipped.  No page may be written by two pairs, or written by one and read by
 * another.  Of `cache`, heads_kv, dim, page_size, num_pages and the four arrays are read.
 */
kda_status kda_cache_copy_pages(const kda_cache *cache, int32_t layers, const int32_t *pairs, int64_t num_pairs, void *hip_stream);

/* Static description of a status code (never NULL). */
const char *kda_status_string(kda_status status);

/* Detail of the last error raised on the calling thread ("" if none). */
const char *kda_last_error(void);

/* Library version string, e.g. "kda-gfx950 0.1". */
const char *kda_version(void);

#ifdef __cplusplus
}
#endif
#endif /* KDA_H_ */
