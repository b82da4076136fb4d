/*
 * sgd_kernels.h — kernel-level entry points of libsgd, one per hot-path kernel of
 * the scheduled denoiser step.  They exist so that every kernel can be checked
 * against the CPU oracle on its own; sgd_step launches the same kernels with the
 * same launch configurations.
 *
 * Paper passages (Algorithm 2, "Jagged-Stream Execution"):
 *   - an active unit computes Delta_{l,s} = F_l(h_{l-1,s}; c_s), refreshes its cache
 *     and sets h_{l,s} = h_{l-1,s} + Delta   -> sgd_kernel_gemm with SGD_EPI_DELTA
 *     (the branch's last projection, its epilogue stores the cache and adds to h);
 *   - the branch body F_l (norm, projections, attention, MLP activation)
 *                                          -> sgd_kernel_norm, sgd_kernel_gemm,
 *                                             sgd_kernel_attention;
 *   - a frozen unit reads its cached Delta_{l, r_l(s)} and adds it to the current
 *     residual stream                        -> sgd_kernel_frozen_run (one pass over h
 *     for a run of consecutive frozen units).
 *
 * Beside them stand operators on what a token model's step writes, its logits, for programs that turn them
 * into tokens or compare two evaluations: sgd_kernel_logprobs, sgd_kernel_sample and sgd_kernel_distill (and sgd.h's
 * sgd_sampler_reveal); and, for programs that train a token model's ends on that gradient, its embedding with the table's
 * gradient and the norms' backward pass.
 *
 * Where an output must not overlap an argument, matrices may lie between one another's rows if they have one row stride.
 *
 * All pointers are device pointers; all calls are asynchronous on `stream`
 * (a cudaStream_t) and return an sgd_status (sgd.h).  Arguments are validated on
 * the host (SGD_ERR_ARG / SGD_ERR_SHAPE); nothing is launched on a validation error.
 */
#ifndef SGD_KERNELS_H
#define SGD_KERNELS_H

#include <stdint.h>

#ifndef SGD_API
#if defined(__GNUC__)
#define SGD_API __attribute__((visibility("default")))
#else
#define SGD_API
#endif
#endif

#ifdef __cplusplus
extern "C" {
#endif

/* Epilogue applied to the fp32 accumulator tile of C = A B^T. */
/* acc = alpha * (A B^T), fp32.  fp16 outputs saturate at +-65504. */
typedef enum {
  SGD_EPI_F16 = 0,    /* out fp16 [M, N] = acc                                          */
  SGD_EPI_F32 = 1,    /* out fp32 [M, N] = acc                                          */
  SGD_EPI_DELTA = 2,  /* Delta = gate * acc; h fp32 [M, N] += Delta; cache fp16 = Delta   */
  SGD_EPI_GATED = 3,  /* B has 2f rows; out fp16 [M, f] = act(acc[:, :f], acc[:, f:])   */
  SGD_EPI_GELU = 4,   /* out fp16 [M, N] = gelu(acc)                                    */
  SGD_EPI_ROPE = 5    /* out fp16 [M, N] = acc with rotate-half RoPE on columns < rope_cols */
} sgd_epilogue_kind;

typedef struct {
  int kind;                      /* sgd_epilogue_kind                                        */
  float alpha;                   /* accumulator scale (0 is read as 1)                        */
  void* out; int ldo;            /* output (elements); unused by SGD_EPI_DELTA               */
  float* h; int ldh;             /* DELTA: fp32 residual updated in place                   */
  void* cache; int ld_cache;     /* DELTA: optional fp16 copy of Delta (NULL: not stored)    */
  const float* gate;             /* DELTA: optional fp32 gate [B, ld_gate], row r uses sample r / rows_per_batch */
  int ld_gate, rows_per_batch;
  int act;                       /* GATED: 0 = silu(a) * b (SwiGLU), 1 = a * gelu_erf(b) (GEGLU);
                                    GELU: 0 = tanh form, 1 = erf form                           */
  const float* rope_cos;         /* ROPE: fp32 [rope_tokens, d_head / 2] tables, row = token % rope_tokens */
  const float* rope_sin;
  int rope_tokens, d_head, rope_cols;
  /* Pre-norm folded into the GEMM (Algorithm 2, an active branch's Norm before its first
   * projection): A holds the un-normalised rows x (fp16), B = W diag(g) (the norm gain
   * folded into the weight), and before its epilogue each accumulator value of row r, B
   * row j becomes
   *   SGD_FNORM_RMS (1): rstd_r acc,  rstd_r = rsqrt(sum_p sq[p][r] / K + norm_eps);
   *   SGD_FNORM_LN  (2): rstd_r (acc - mean_r colsum[j]) + colbias[j], with mean_r =
   *                      sum_p s[p][r] / K and rstd_r = rsqrt(sum_p sq[p][r] / K - mean_r^2 + eps),
   * where sq[p][r] = rstat[p * stat_ld + r] and s[p][r] = rstat[(64 + p) * stat_ld + r] are
   * the partial row sums of x^2 and x in stat_slots (1..64) slots, added in slot order.
   * colsum[j] = alpha sum_k B[j, k] and colbias[j] = sum_k b_k W[j, k] (b the LayerNorm shift),
   * fp32 with at least 512 entries of padding past the last B row.  Not with SGD_EPI_DELTA. */
  int norm;
  const float* rstat;
  int stat_slots, stat_ld;
  float norm_eps;
  const float* colsum;
  const float* colbias;
  /* Writer of the residual stream (SGD_EPI_DELTA, or SGD_EPI_F32 writing h): with h16 set,
   * also stores fp16(new h) in h16 (row stride ldh, or ldo for F32) and, per row, the partial
   * sums of its new values' squares and values over the columns of each half of each output
   * tile in slot 2 t + half of stat_out (same layout as rstat, stat_out_ld >= M): the
   * statistics a following SGD_FNORM_* GEMM reads.  The slot count is 2 ceil(N / tile
   * width); sgd_kernel_gemm_stat_slots returns it. */
  void* h16;
  float* stat_out;
  int stat_out_ld;
  /* Optional, with h16: the CTA that completes the last column tile of a 128-row block
   * (tickets in stat_cnt, one int per row block, zero before the launch and left zero after
   * it; no CTA waits for another) adds that block's slots in slot order and stores each row's
   * totals in slot 0 of stat_final (same layout as rstat, 256-byte aligned like any device
   * allocation), so that a following SGD_FNORM_* GEMM reads stat_slots = 1 of stat_final. */
  int* stat_cnt;
  float* stat_final;
} sgd_epilogue_args;

/* Kernel launches the calling thread has made so far with programmatic dependent launch (steps
 * launched op by op, and the capture of their graphs in sgd_set_schedule). */
SGD_API int sgd_kernel_dependent_launches(int64_t* launches);

/* The tile sgd_kernel_gemm takes for these arguments on the current device: CTAs of a group per tile
 * (1 or 2; 0: the one-CTA kernel of the forced forms and folded norms, or the SIMT kernel) and
 * the tile's columns of B. */
SGD_API int sgd_kernel_gemm_tile(int M, int N, int K, const sgd_epilogue_args* epi, int variant,
                                 int* group, int* columns);

/* Partial-sum slots a residual writer with these arguments fills (see h16 above). */
SGD_API int sgd_kernel_gemm_stat_slots(int M, int N, int K, const sgd_epilogue_args* epi,
                                       int variant, int* slots);

/*
 * C = alpha A B^T.  A fp16 [M, K] (row stride lda elements), B fp16 [N or 2N, K]
 * (row stride ldb).  K, lda, ldb multiples of 8; N multiple of 8; pointers 16-byte
 * aligned.  use_simt = 1 runs the plain SIMT kernel (reference / debugging); the others are
 * tcgen05 + TMA kernels (fp32 accumulators in TMEM).  0 runs the CTA-group kernel, whose tiles of
 * 128 x 64 to 128 x 256 (one CTA) or 256 x 128 to 256 x 256 (a cluster of two CTAs, M = 256
 * instructions; M > 128) it chooses by their cost.  With a folded norm or the residual writer
 * below, and in the forms 3 and 5 to 12, the one-CTA kernel (M = 128, N = 256, K = 16
 * instructions, 64-element K-blocks) runs, choosing by itself 128 x 256 or 128 x 128 tiles, 4 or 8
 * epilogue warps, and whether the tiles left over after the last full wave of CTAs are
 * split along K over all SMs ("stream-K": fp32 partial tiles in a workspace, summed in a
 * fixed order by the CTA that finishes a tile last, so results are deterministic).  3: with
 * 32-element K-blocks (64-byte swizzle); 2 and 4 are not defined and are
 * rejected with SGD_ERR_ARG; 5, 6, 7 force 128 x 256 tiles with 4 epilogue warps, 128 x 256 with 8, and
 * 128 x 128 with 8 and no stream-K (128 x 128 applies to plain, GELU and DELTA epilogues
 * only); 8 is without stream-K, 9 with stream-K whenever the last wave is partial;
 * 10 forces 128 x 224 tiles (5 pipeline stages, no stream-K; plain, GELU and DELTA only);
 * 11 and 12 have the tiles visited M-fastest, and in groups of 16 row-blocks (each
 * group column by column, every other group backwards), instead of by choice
 * (groups where there are at least two groups and two waves).
 * The stream-K workspace is owned by the library, one per (device, stream), allocated
 * or grown by the first call that needs it (after synchronising that stream).
 */
SGD_API int sgd_kernel_gemm(const void* A, int lda, const void* B, int ldb, int M, int N, int K,
                    const sgd_epilogue_args* epi, int use_simt, void* stream);

/*
 * sgd_kernel_gemm without any device memory allocation.  The paper has no counterpart:
 * this is an interface for callers that cannot let the library allocate, such as a
 * process whose device memory is all reserved by its own pool allocator, or one that
 * cannot take the device-wide synchronisation that cudaMalloc / cudaFree may imply while
 * its other streams run.  Same arguments, variant codes (`variant` = use_simt above),
 * kernels and results bit for bit as sgd_kernel_gemm; the only difference is where a
 * stream-K split keeps its partial tiles and tile tickets: in one fixed array compiled
 * into the library (32 MiB of fp32 partial tiles, then 1024 tickets) instead of a
 * workspace the library allocates.
 * Limit: a problem whose stream-K split (that of the one-CTA kernel, whichever kernel variant 0
 * runs) needs more than the array holds is rejected with SGD_ERR_SHAPE before anything is
 * launched (variant 8, or sgd_kernel_gemm, runs it).
 * The tickets are cleared (cudaMemsetAsync on `stream`) before each stream-K launch; the
 * partial tiles need no clearing (each is written before it is read within one launch).
 * Every call on a device uses the same array: calls that can overlap in time (launched
 * on different streams without ordering, or from several host threads at once) race on
 * it and can produce wrong results, so order them on one stream or with events.
 */
SGD_API int sgd_kernel_gemm_static_ws(const void* A, int lda, const void* B, int ldb, int M, int N,
                              int K, const sgd_epilogue_args* epi, int variant, void* stream);

/*
 * O = softmax(Q K^T / sqrt(d_head)) V per (sample, head), non-causal, keys beyond n_kv
 * masked.  Row r = b * n_q + i of q / o, row b * n_kv + j of k / v; head h occupies
 * columns [h d_head, (h+1) d_head).  fp16 in and out; d_head in {64, 72, 128};
 * leading dimensions in elements, multiples of 8.  impl = 0: tcgen05 for d_head 64 / 128
 * (S, P and O in TMEM; by shape two 128-query tiles per CTA, whose softmax warpgroups alternate
 * with each other's MMAs, or one per CTA and several CTAs per SM), the mma.sync kernel for 72
 * (see sgd_kernel_attention_hs for 72 on tcgen05); 1: the mma.sync kernel for every d_head;
 * 2: tcgen05 with one query tile per CTA and P in shared memory; 3: tcgen05 with two query tiles
 * per CTA for every shape.
 */
SGD_API int sgd_kernel_attention(const void* q, int ldq, const void* k, const void* v, int ldkv,
                         void* o, int ldo, int batch, int n_q, int n_kv, int n_heads,
                         int d_head, int impl, void* stream);

/*
 * sgd_kernel_attention with the input heads `head_stride` columns apart (head h of q, k, v
 * at columns [h head_stride, h head_stride + d_head); head_stride >= d_head, a multiple of
 * 8); o keeps d_head columns per head.  With d_head 72, impl 0 / 3 run the tcgen05 kernel
 * when head_stride >= 80: each head is read as 80 columns (one 64-column and one
 * 16-column block), so columns [72, 80) after every Q head must be zero and those after
 * every K and V head finite (a layout whose gaps are zero, as sgd_step uses, satisfies
 * both); with head_stride 72 they fall back to the mma.sync kernel.
 */
SGD_API int sgd_kernel_attention_hs(const void* q, int ldq, const void* k, const void* v, int ldkv,
                                    int head_stride, void* o, int ldo, int batch, int n_q, int n_kv,
                                    int n_heads, int d_head, int impl, void* stream);

/*
 * out fp16 [rows, d] = norm(h fp32 [rows, d]); kind = sgd_norm_kind.  g, b: bf16 [d]
 * (NULL allowed for LN_PLAIN).  shift/scale: optional fp32 AdaLN modulation
 * [B, ld_mod]: out = norm(h) * (1 + scale[r / rows_per_batch]) + shift[...].
 * h 16-byte and out 8-byte aligned (else SGD_ERR_ARG).
 */
SGD_API int sgd_kernel_norm(const float* h, void* out, int rows, int d, int kind, const void* g,
                    const void* b, const float* shift, const float* scale, int ld_mod,
                    int rows_per_batch, float eps, void* stream);

/*
 * h fp32 [n] += sum_{i < n_caches} caches[i] (fp16 [n]), summed in order i = 0, 1, ...
 * in fp32.  caches_host: host array of n_caches (<= 96) device pointers.  n multiple
 * of 8, pointers 16-byte aligned.
 */
SGD_API int sgd_kernel_frozen_run(float* h, const void* const* caches_host, int n_caches, int64_t n,
                          void* stream);

/* Element type of a row of logits or of its gradient. */
typedef enum { SGD_F16 = 0, SGD_BF16 = 1, SGD_F32 = 2 } sgd_dtype;

/*
 * Log-probabilities of given tokens, entropy and the likeliest tokens of rows of logits (such as a
 * step of a SGD_HEAD_LOGITS model writes).  With p = softmax(scale * logits[r, :]), ln p
 * computed in fp32 whatever the logits' type:
 *   token_logprobs fp32 [rows, n_tokens] = ln p of tokens int32 [rows, n_tokens]; 0 where the token is
 *     negative (padding), NaN where it is not below vocab;
 *   entropy fp32 [rows] = - sum p ln p (0 ln 0 = 0);
 *   top_ids int32 [rows, top_k], top_logprobs fp32 [rows, top_k]: the tokens of the largest logits, in
 *     descending order, equal logits (-0 and +0 are equal) in the order of the token.
 * Any of the outputs may be NULL (tokens with n_tokens = 0), but not all.  With rows = 0 nothing is done, and every
 * pointer may be NULL (so in sgd_kernel_distill).
 * logits [rows, vocab] of type dtype, rows ld elements apart, aligned to their elements alone.
 * 0 < scale <= 2e38 (1 / temperature).  row_ids int32 [rows]: where given, only rows with row_ids[r] == row_id
 * (positions that are still masked, say) are read, and what the others' outputs held stays.
 * -inf masks a token: its ln p is -inf.  Finite logits may be of any magnitude (masks of the type's lowest value, of
 * -1e10), at any scale: what fp32 does not hold of their ln p is -inf.  A row of -inf alone has ln p = -inf, entropy 0 and the
 * top tokens 0, 1, ...; a row that holds NaN or +inf has NaN for every ln p and for the entropy,
 * and NaN ranks with -inf.
 * 0 <= top_k <= 64 and <= vocab (else SGD_ERR_ARG); vocab * element size <= 3 MiB (else SGD_ERR_SHAPE).
 * No output may overlap an input or another output.  No workspace:
 * calls on several streams and replays of captured ones may overlap.  Results are the same on
 * every run.
 */
SGD_API int sgd_kernel_logprobs(const void* logits, int dtype, int64_t ld, int rows, int vocab, float scale,
                                const int32_t* row_ids, int row_id, const int32_t* tokens, int n_tokens,
                                float* token_logprobs, float* entropy, int top_k, int32_t* top_ids,
                                float* top_logprobs, void* stream);

/* What a teacher's list says of the tokens that are not in it (sgd_kernel_distill). */
typedef enum {
  SGD_TAIL_RENORM = 0,  /* nothing: the list's probabilities are divided by their sum          */
  SGD_TAIL_BUCKET = 1   /* together they have what is left of 1: one more outcome, "any other" */
} sgd_tail_kind;

/*
 * Divergence of rows of logits from a teacher's likeliest tokens, with its gradient (the full
 * model's lists from sgd_kernel_logprobs against a scheduled model's logits, say).  With
 * p = softmax(scale * logits[r, :]), the list's tokens S and q_i = exp(teacher_logprobs_i), Q = sum q_i:
 *   SGD_TAIL_RENORM: L = sum_S (q_i / Q) (ln (q_i / Q) - ln p_i); only differences of teacher_logprobs count, which
 *                    may be any scores;
 *   SGD_TAIL_BUCKET: L = sum_S q_i (ln q_i - ln p_i) + q_T (ln q_T - ln p_T), q_T = max(0, 1 - Q),
 *                    p_T = sum of p outside S; the second term is left out where q_T or p_T is 0.  Lists are meant
 *                    to have Q <= 1; where it is more, grad is that of Q = 1 (scale w_r (p - q) in S, scale w_r p
 *                    outside) and not L's derivative;
 *   loss fp32 [rows] = w_r L;  grad [rows, vocab] = w_r dL / dlogits (NULL: the loss alone).
 * top_k = 1 with teacher_logprobs 0 and SGD_TAIL_RENORM is the cross entropy of the listed token.
 * logits [rows, vocab] of type dtype, rows ld elements apart; teacher_ids int32 and teacher_logprobs
 * fp32 [rows, top_k].  An id outside [0, vocab) pads the list; of ids that are equal the first counts.
 * row_weight fp32 [rows] (NULL: 1): the logits of rows of weight 0 are not read, their loss and
 * gradient are 0; so are those of a row whose list has no token (SGD_TAIL_RENORM: or none that is above -inf).
 * -inf masks a token (p = 0): the loss is +inf where the list gives it weight, the gradient finite.
 * NaN in a row, or +inf, makes its loss and gradient NaN.
 * grad of type grad_dtype, rows ld_grad elements apart, each value rounded once from fp32 (out of
 * fp16's range: inf).  grad may be logits itself (same type and ld); it must not overlap it
 * otherwise (SGD_ERR_ARG), and nothing else may overlap.  1 <= top_k <= 64 (else SGD_ERR_ARG); vocab * element
 * size of logits <= 3 MiB (else SGD_ERR_SHAPE).
 * No workspace: calls on several streams and replays of captured ones may overlap.  Results are
 * the same on every run.
 */
SGD_API int sgd_kernel_distill(const void* logits, int dtype, int64_t ld, int rows, int vocab, float scale,
                               const int32_t* teacher_ids, const float* teacher_logprobs, int top_k,
                               const float* row_weight, int tail, float* loss, void* grad, int grad_dtype,
                               int64_t ld_grad, void* stream);

/* Tokens of a block of the vocabulary (sgd_kernel_sample). */
#define SGD_SAMPLE_BLOCK 512

/*
 * A token drawn from each row of logits.  With x = scale * logits[r, :], w = exp(x - max x) and the tokens in the order
 * (logit descending, token ascending; -0 and +0 are equal), the tokens that may be drawn are
 *   K1: of the first top_k of the order (0, or vocab and more: of all) those with w >= min_p (0: all);
 *   K: the shortest prefix of K1, in the order, whose mass (sum of w) is at least top_p times K1's (1: all of K1).
 * Two numbers u0, u1 in [0, 1) a row (uniforms fp32 [rows, 2]; what lies outside is taken as 0 or 1, NaN as 0) choose
 *   b, the first block of SGD_SAMPLE_BLOCK neighbouring tokens whose cumulative mass (of K's tokens, blocks ascending) is above
 *     u0 mass(K), and the first token of K in b whose cumulative mass inside b (tokens ascending) is above u1 mass(b);
 *     the last one of positive mass where rounding leaves none.
 * With independent uniform numbers that is a draw from w over K, with the resolution of both.  Masses are compared as
 * sums of whole multiples of 2^-43 of the largest weight, each within 2^-29 of its value and half of one (tokens below 2^-44 have none).
 *   ids int32 [rows] = the token;  logprobs fp32 [rows] (NULL: not wanted) = its ln p, p = softmax(x) over all tokens.
 * scale = 1 / temperature, 0 < scale <= 2e38.  top_k >= 0, 0 < top_p <= 1, 0 <= min_p <= 1 (else SGD_ERR_ARG).
 * row_ids, row_id, the rows of logits and their limits as in sgd_kernel_logprobs.  -inf masks a token.  A row without a
 * distribution takes the first token of the order: one of -inf alone token 0 with ln p = -inf, one that holds NaN
 * (which ranks with -inf) or +inf its ln p = NaN.
 * No output may overlap an input or the other output (SGD_ERR_ARG).  No workspace: calls on several streams and replays of captured
 * ones may overlap.  Results are the same on every run.
 */
SGD_API int sgd_kernel_sample(const void* logits, int dtype, int64_t ld, int rows, int vocab, float scale, int top_k, double top_p,
                              double min_p, const float* uniforms, const int32_t* row_ids, int row_id, int32_t* ids,
                              float* logprobs, void* stream);

/*
 * out[r, :] = scale * table[ids[r], :], rounded once from fp32 (out of fp16's range: inf); zeros where ids[r] is not in [0, vocab)
 * (padding; a model's own stem, SGD_STEM_EMBED, takes the table's first or last row there).  table [vocab, d] of type dtype, rows
 * ld elements apart; ids int32 [rows]; out [rows, d] of type out_dtype, rows ld_out elements apart; both aligned to their
 * elements alone.  1 <= d <= 2^20.  out must not overlap the table or the ids (SGD_ERR_ARG).
 */
SGD_API int sgd_kernel_embedding(const void* table, int dtype, int64_t ld, int vocab, int d, const int32_t* ids, int rows, float scale,
                                 void* out, int out_dtype, int64_t ld_out, void* stream);

/* Bytes of workspace of sgd_kernel_embedding_grad. */
SGD_API int sgd_kernel_embedding_grad_workspace(int rows, int vocab, int d, int64_t* bytes);

/*
 * Gradient of sgd_kernel_embedding's table: with S[t] = scale * sum of grad[r, :] over the rows r with ids[r] = t, in fp32 and in
 * one order (that of the rows, and of groups of 8 to 32 rows sorted by token for tokens with many),
 *   accumulate = 0: dtable[t, :] = S[t] for every t in [0, vocab), zeros for tokens without a row;
 *   accumulate = 1: dtable[t, :] += S[t] for the tokens that have rows; the others are neither read nor written;
 * each rounded once from fp32.  Rows whose id is not in [0, vocab) are left out, and not read.
 * grad [rows, d] of type grad_dtype, rows ld_grad elements apart; dtable [vocab, d] of type dtable_dtype, rows ld
 * elements apart; both aligned to their elements alone.  1 <= d <= 2^20.  workspace: 16-byte aligned, of the size that
 * sgd_kernel_embedding_grad_workspace gives (else SGD_ERR_ARG); what it holds before and after means nothing.  Calls
 * and replays that may overlap need one each.  dtable must not overlap another argument (SGD_ERR_ARG).  Results are the same
 * on every run.
 */
SGD_API int sgd_kernel_embedding_grad(const void* grad, int grad_dtype, int64_t ld_grad, const int32_t* ids, int rows, int vocab,
                                      int d, float scale, int accumulate, void* dtable, int dtable_dtype, int64_t ld,
                                      void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes of workspace of sgd_kernel_norm_grad (rows_per_batch: 0 without a modulation). */
SGD_API int sgd_kernel_norm_grad_workspace(int rows, int d, int rows_per_batch, int64_t* bytes);

/*
 * Backward pass of sgd_kernel_norm.  With xhat = (h - mean) rstd of a row (no mean for SGD_NORM_RMS), n = xhat g + b and
 * out = n (1 + scale) + shift as there, and dout = dL / dout:
 *   dn = dout (1 + scale), dx = dn g,
 *   dh fp32 [rows, d] = rstd (dx - mean(dx) - xhat mean(dx xhat)) + residual, without mean(dx) for SGD_NORM_RMS
 *     (residual fp32 [rows, d], NULL: 0: what reaches h past the branch; dh may be residual itself);
 *   dg fp32 [d] = sum over the rows of dn xhat, db fp32 [d] = sum of dn;
 *   dshift, dscale fp32 [samples, ld_dmod] = sums over a sample's rows of dout and of dout n.
 * Any of the outputs may be NULL, but not all; dg needs g, db needs b, dshift and dscale need scale, residual needs dh.
 * h fp32 [rows, d], dout [rows, d] of type dtype, g, b bf16 [d] or NULL, scale fp32 [samples, ld_mod] or NULL, row r of sample
 * r / rows_per_batch.  d a multiple of 4, 4 <= d <= 4096; h, dh, residual, dg, db and fp32 dout 16-byte aligned, other dout,
 * g and b 8-byte aligned.  Sums are fp32 (over a share of the rows at a time, then over the shares) and the same on every run.
 * With rows = 0, dg and db are zeros.  workspace as in sgd_kernel_embedding_grad; none is needed where dh is the only
 * output.  Otherwise no output, nor the workspace, may overlap another argument (SGD_ERR_ARG).
 */
SGD_API int sgd_kernel_norm_grad(const float* h, const void* dout, int dtype, int rows, int d, int kind, const void* g,
                                 const void* b, const float* scale, int ld_mod, int rows_per_batch, float eps,
                                 const float* residual, float* dh, float* dg, float* db, float* dshift, float* dscale,
                                 int ld_dmod, void* workspace, int64_t workspace_bytes, void* stream);

/* Device status word shared by all kernels (bounded-wait expiry); returns and clears it. */
SGD_API int sgd_kernel_status(int* status_host);

/* *clamped_host = 1 if any kernel stored an fp16 value that it had to clamp to +-65504
 * (the value was out of fp16's range, or NaN) since the last call, else 0; clears the
 * flags.  A reading aid for fp16 operands, which the paper (bf16) does not use. */
SGD_API int sgd_kernel_f16_clamped(int* clamped_host);

/*
 * Failure-path self-test (no counterpart in the paper): launches on `stream` one kernel
 * whose thread waits, with the same bounded wait every kernel uses, on an mbarrier that
 * nothing completes.  After the wait limit (2 s) it records SGD_SELFTEST_TIMEOUT_CODE in
 * the device status word (read and cleared by sgd_kernel_status) and returns, leaving the
 * context usable.  Nothing faults, traps or hangs.
 */
#define SGD_SELFTEST_TIMEOUT_CODE 99
SGD_API int sgd_selftest_wait_timeout(void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SGD_KERNELS_H */
