/*
 * hydra_ops.h -- C entry points of the individual device operations the trainer is built from.
 *
 * They exist so that every kernel can be checked and timed on its own.  All data pointers are
 * DEVICE pointers owned by the caller; the pointer tables themselves (X, W, ...) are HOST arrays of
 * G entries.  `stream` is a hipStream_t (NULL = the default stream).  Calls enqueue work and return;
 * they neither allocate nor synchronise.  Return value: 0 on success, otherwise a hydra_status
 * (HYDRA_ERR_INVALID_ARG for shapes/alignments the kernel does not accept, HYDRA_ERR_DEVICE for a
 * launch failure); hydra_ops_last_error() gives the text.
 *
 * The operations are the ones a forward pass, a backward pass and a gradient update of a shard
 * consist of (paper, Introduction, "Motivation": features flow layer to layer forward, gradients
 * backward; Approach, "Desiderata": gradient updates must be exactly those of unsharded training),
 * written for G same-shaped problems of different models at once (Approach: shards of different
 * models are independent units of parallel work).
 */
#ifndef HYDRA_OPS_H
#define HYDRA_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { HYDRA_OPS_F32 = 0, HYDRA_OPS_BF16 = 1 };                  /* operand dtype                    */
enum { HYDRA_EPI_NONE = 0, HYDRA_EPI_RELU = 1, HYDRA_EPI_GELU = 2 };

/* out_g[M,N] = epilogue( sum_k X_g(m,k) * W_g(n,k) ), fp32 accumulation.
 *   epilogue: v = acc + bias[n] (if bias); pre[m,n] = v (if pre);
 *             v = gate ? v * act'(gate[m,n]) : act(v);  v += resid[m,n] (if resid); out[m,n] = v.
 * x_kmajor = 1: X_g stored [M, ldx], k contiguous; 0: stored [K, ldx], m contiguous.
 * w_kmajor = 1: W_g stored [N, ldw], k contiguous; 0: stored [K, ldw], n contiguous.
 * Forward Linear: X = input, W = weight[out,in], both k-major.  Input gradient: X = dY (k-major),
 * W = weight (k is its slow index).  Weight gradient: X = dY, W = input, both with k slow.
 * Leading dimensions count elements; ldx, ldw multiples of 16 bytes and >= the contiguous extent
 * rounded up to 16 bytes; ldo, ldg, ldr multiples of 8 and >= N.  bias is fp32 [N].  out is fp32
 * when out_f32, else the operand dtype; pre, gate, resid have the operand dtype.  Optional tables
 * may be NULL.  tile: 0 = automatic, 1 = 256x256, 2 = 128x128, 3 = 32x128 workgroup tiles, 4 = 256x256 with
 * operands staged through registers (1 loads bf16 k-contiguous operands straight into LDS).  All give the
 * same bits. */
typedef struct {
  int dtype, M, N, K, x_kmajor, w_kmajor, ldx, ldw, ldo, ldg, ldr, act, out_f32, tile, G;
  const void* const* X;
  const void* const* W;
  const float* const* bias;
  void* const* out;
  void* const* pre;
  const void* const* gate;
  const void* const* resid;
  float* const* rowsum; /* optional, weight-gradient layout (x_kmajor = w_kmajor = 0) only: rowsum_g[m] =
                           sum_k X_g(m,k) in fp32, M floats each; with X = dY this is the bias gradient */
  void* const* ws;      /* optional device scratch, 32-byte aligned, ws_bytes each: a bf16 weight-gradient problem
                           (x_kmajor = w_kmajor = 0, out_f32, no bias/pre/gate/resid, no activation) with
                           hydra_op_gemm_split_k(M, N, K) = S > 1 then sums S contiguous ranges of k separately and
                           adds the partial sums in ascending order in a second launch.  S depends on the shape
                           alone.  Without scratch (or with too little) the sum runs in one chain */
  size_t ws_bytes;
} hydra_gemm_desc;
int hydra_op_gemm_split_k(int M, int N, int K);                   /* 1 = this shape is never split   */
size_t hydra_op_gemm_split_ws_bytes(int M, int N, int K, int ldo);  /* scratch bytes per problem, 0 if S = 1 */
int hydra_op_gemm(const hydra_gemm_desc* d, void* stream);

/* out_g[n] = sum_{m<M} src_g[m,n]; src has the operand dtype and leading dimension ld, out is fp32.
 * part_g: scratch of hydra_op_colsum_part_floats(M, N) floats (0 for M <= 256: the table may then be NULL). */
int hydra_op_colsum(int dtype, int M, int N, int ld, int G, const void* const* src, float* const* out,
                    float* const* part, void* stream);
size_t hydra_op_colsum_part_floats(int M, int N);

/* hydra_op_colsum for callers that cannot allocate device memory or hand over scratch: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same kernels, same order of additions and therefore the same
 * bits as hydra_op_colsum; the partial sums live in an array built into the library (one copy per GPU, held until the
 * process ends) of hydra_op_colsum_noalloc_max_floats() = 1048576 floats (4 MiB).  A call needs
 * G * hydra_op_colsum_part_floats(M, N) of them; more returns HYDRA_ERR_INVALID_ARG and nothing is launched.  The
 * call allocates and frees nothing and does not synchronise.  Every call on a GPU uses that GPU's one array: calls
 * whose kernels may overlap on one GPU (different streams, or different threads) race; calls on one stream do not. */
int hydra_op_colsum_noalloc(int dtype, int M, int N, int ld, int G, const void* const* src, float* const* out,
                            void* stream);
size_t hydra_op_colsum_noalloc_max_floats(void);

/* Softmax cross-entropy over fp32 logits [M, ldz] with C classes and int32 labels [M] (shared by the
 * group): rowloss_g[m] = logsumexp(z_m) - z_m[y_m]; dz_g[m,c] = (softmax(z_m)[c] - [c==y_m]) * inv_n
 * in the operand dtype with leading dimension lddz (columns [C,lddz) are zeroed);
 * loss_g[0] = inv_n * sum_m rowloss_g[m]. */
int hydra_op_softmax_ce(int dtype, int M, int C, int ldz, int lddz, float inv_n, int G, const float* const* logits,
                        const int32_t* labels, void* const* dz, float* const* rowloss, float* const* loss, void* stream);

/* Optimizer step over flat fp32 blocks of n elements (n % 4 == 0).  opt 0 = SGD (m, v ignored),
 * 1 = Adam with bias-correction factors bc1 = 1/(1-b1^t), bc2 = 1/(1-b2^t) given per problem.
 * w16 (optional) receives the bf16 rounding of the updated parameters.  hp: G rows of
 * {lr, b1, b2, eps, bc1, bc2} in double (host); they are rounded to fp32 once, as is 1-b. */
int hydra_op_optim(int opt, size_t n, int G, float* const* p, const float* const* g, float* const* m, float* const* v,
                   void* const* w16, const double* hp, void* stream);

/* Weight gradient with the optimizer step in its epilogue (paper, Approach, "Desiderata": the update
 * is the one a separate optimizer pass would apply, bit for bit).  d describes the gradient GEMM
 * dW_g[M,N] = sum_k X_g(m,k) W_g(n,k) with x_kmajor = w_kmajor = 0, out_f32 = 1, no bias/pre/gate/resid
 * and act = HYDRA_EPI_NONE; element [m,n] of the gradient updates p_g[m*ldo + n] (and m_g, v_g, w16_g
 * at the same index) as hydra_op_optim would.  d->out may be NULL (the gradient is then never
 * stored) or a table of fp32 [M, ldo] buffers that also receive it.  p, m, v 32-byte aligned, w16 16-byte;
 * hp as for hydra_op_optim.  Errors: HYDRA_ERR_INVALID_ARG for shapes or tables the kernel cannot take. */
int hydra_op_gemm_update(const hydra_gemm_desc* d, int opt, float* const* p, float* const* m, float* const* v,
                         void* const* w16, const double* hp, void* stream);

/* dst[i] = u_i * 2a - a with u_i the 24-bit uniform of the counter generator (SplitMix64 keyed by
 * (seed, stream_id)); the values a model's tensor `stream_id = (model << 20) | tensor` is initialised with. */
int hydra_op_init_uniform(float* dst, size_t n, uint64_t seed, uint64_t stream_id, float a, void* stream);

/* dst[i] = bf16(src[i]) (round to nearest even), i < n. */
int hydra_op_cast_bf16(const float* src, void* dst, size_t n, void* stream);

/* LayerNorm over rows of width d (d % 8 == 0, d <= 4096, ld % 8 == 0): per row mu = mean, var = biased
 * variance, y = (x-mu)/sqrt(var+eps)*gamma + beta.  x, y have the operand dtype; gamma, beta, mean, rstd fp32. */
int hydra_op_layernorm_fwd(int dtype, int rows, int d, int ld, float eps, int G, const void* const* x, void* const* y,
                           const float* const* gamma, const float* const* beta, float* const* mean,
                           float* const* rstd, void* stream);
/* Adjoint: dx = rstd*(g - mean(g) - xhat*mean(g*xhat)) + add, g = dy*gamma (add optional: NULL table);
 * dgamma = sum_rows dy*xhat; dbeta = sum_rows dy.  part_g: scratch of hydra_op_layernorm_part_floats(rows, d) floats.
 * dx_g may be x_g, dy_g or add_g itself (the same bits as with a buffer of its own); it may not overlap them otherwise. */
int hydra_op_layernorm_bwd(int dtype, int rows, int d, int ld, int G, const void* const* x, const void* const* dy,
                           const void* const* add, void* const* dx, const float* const* gamma,
                           const float* const* mean, const float* const* rstd, float* const* part,
                           float* const* dgamma, float* const* dbeta, void* stream);
size_t hydra_op_layernorm_part_floats(int rows, int d);

/* Attention, bf16, head width DH in {64,128}.  qkv_g [B*S, ld_qkv]: q of head h at columns [h*DH,(h+1)*DH),
 * k at H*DH + the same, v at 2*H*DH + the same.  o_g [B*S, ld_o].  P = softmax(q k^T * scale (+ causal mask)),
 * o = P v, lse_g [B*H*S] = log-sum-exp of the scaled scores.  qkv_g (and dout_g below) 16-byte aligned, ld_qkv and ld_o
 * multiples of 8, 64 rows (or S, if fewer) of either below 2 GiB. */
int hydra_op_attention_fwd(int B, int S, int H, int DH, int ld_qkv, int ld_o, int causal, float scale, int G,
                           const void* const* qkv, void* const* o, float* const* lse, void* stream);
/* Adjoint given dout_g [B*S, ld_o] (gradient w.r.t. o): dqkv_g in the layout of qkv; delta_g [B*H*S] scratch.
 * o_g may lie in the query columns of dqkv_g, which then overwrites it; nothing else may overlap dqkv_g or delta_g. */
int hydra_op_attention_bwd(int B, int S, int H, int DH, int ld_qkv, int ld_o, int causal, float scale, int G,
                           const void* const* qkv, const void* const* o, const void* const* dout,
                           const float* const* lse, float* const* delta, void* const* dqkv, void* stream);

/* x_g[t,:] = tok_g[ids[t],:] + pos_g[t mod S,:]; ids int32 [tokens] shared by the group; tables in the operand dtype. */
int hydra_op_embed_fwd(int dtype, int tokens, int S, int d, int ld, int G, const int32_t* ids, const void* const* tok,
                       const void* const* pos, void* const* x, void* stream);
/* dtok_g[v,:] = sum of dx_g[t,:] over tokens with id v, listed by the CSR (row_ptr [V+1], positions [B*S], both
 * int32 device arrays); dpos_g[s,:] = sum_b dx_g[b*S+s,:] for s < S, zero for S <= s < S_table.  Outputs fp32. */
int hydra_op_embed_bwd(int dtype, int V, int S, int S_table, int B, int d, int ld, int G, const int32_t* row_ptr,
                       const int32_t* positions, const void* const* dx, float* const* dtok, float* const* dpos,
                       void* stream);

/* ---- A decoder's next tokens: keys and values in a paged cache of 8-bit codes, attention over it, drawing a token -----------------
 *
 * The cache of one layer of each of G models.  A pool k_g (and v_g) has n_pages pages, page_bytes from one to the next; a page is
 * [HKV, page, DH] codes of one byte, its scale of head h is k_scale_g[p*HKV + h], and a code stands for code * scale.  HYDRA_CACHE_INT8:
 * -127..127; HYDRA_CACHE_E4M3: 1 sign, 4 exponent, 3 fraction bits, largest 448, no infinities.  Tokens [i*page, (i+1)*page) of sequence b
 * lie in page page_table[b*max_pages + i] of every model's pool; entries past its last page are not used, and a page id outside [0, n_pages)
 * holds nothing: nothing is stored there, and its tokens are masked.
 * lens[b]: tokens of sequence b with those of the call; the call's n tokens of b are the last n of them, at positions lens[b]-n .. lens[b]-1, and
 * are rows q_ptr[b] .. q_ptr[b+1]-1 of the call's matrices.  q_ptr NULL: one token per sequence, row b.  A sequence may have no tokens in a call,
 * and no tokens at all.  The host's bounds: n_tok = q_ptr[B] rows, max_q rows of one sequence, max_len tokens in one (at most
 * max_pages*page); the kernels hold what the device arrays say to these bounds.  page_table, lens and q_ptr are device arrays that the
 * group shares.  page 16, 32, 64 or 128; DH 64 or 128; pools 16-byte aligned, page_bytes 0 (HKV*page*DH) or a multiple of 16 of at
 * least that, for pools that several layers or k and v share. */
enum { HYDRA_CACHE_INT8 = 0, HYDRA_CACHE_E4M3 = 1 };
enum { HYDRA_ROT_NONE = 0, HYDRA_ROT_HALVES = 1, HYDRA_ROT_NEIGHBOURS = 2 };
typedef struct {
  int kind, B, HKV, DH, page, n_pages, max_pages, G;
  int n_tok, max_q, max_len;
  size_t page_bytes;
  const int32_t* page_table;
  const int32_t* lens;
  const int32_t* q_ptr;
  void* const* k;
  void* const* v;
  float* const* k_scale;
  float* const* v_scale;
} hydra_cache_desc;

/* The call's keys and values into the cache.  qkv_g [n_tok, ld_qkv] bf16: H query heads of DH columns, then HKV key heads, then HKV value heads;
 * 16-byte aligned, ld_qkv a multiple of 8.  The position rotation turns the first rot_dim columns (a multiple of 16) of every query and key head:
 * with c, s = cos_sin[position*rot_dim + i], cos_sin[position*rot_dim + rot_dim/2 + i] and a, b = columns i and i + rot_dim/2
 * (HYDRA_ROT_HALVES) or 2i and 2i + 1 (HYDRA_ROT_NEIGHBOURS): a' = a c - b s, b' = b c + a s.  cos_sin: fp32 device array of max_len rows, 16-byte
 * aligned, shared by the group.  HYDRA_ROT_NONE: rot_dim and cos_sin are not looked at.
 * q_g [n_tok, ld_q] (table NULL: queries are left alone) receives the query heads, rotated, in bf16; it may be qkv_g with ld_q = ld_qkv.
 * A page's scale of a head is max(scale before, largest |x| of the new tokens / Q, 2^-126), Q = 127 or 448; a page whose first slot is new
 * has no scale before.  Where it grows, codes that the page holds become round(code * (before / scale)); new codes are
 * round(x * (1 / scale)), to nearest even.  Infinities become the largest code and do not count for a scale, NaN becomes 0.  Slots past a
 * sequence's last token keep what they have.  A page may belong to one sequence of the call only, unless nothing is appended to it.
 * Tokens at positions below 0 (lens[b] less than the tokens of the call) are dropped. */
typedef struct {
  hydra_cache_desc cache;
  int H, ld_qkv, ld_q, rot, rot_dim;
  const float* cos_sin;
  const void* const* qkv;
  void* const* q;
} hydra_cache_append_desc;
int hydra_op_cache_append(const hydra_cache_append_desc* d, void* stream);

/* o_i = sum_t softmax_t(scale * q_i . k_t) v_t over the tokens t that the cache holds of the row's sequence, with causal those up to the
 * row's own position.  q_g [n_tok, ld_q] and o_g [n_tok, ld_o] bf16, H heads of DH columns; query head i reads key/value head i / (H/HKV).
 * lse_g (table NULL: not wanted) [n_tok, H] fp32: log-sum-exp of the scaled scores.  A row that sees no token gets o = 0 and lse = -inf, a row of no
 * sequence (past q_ptr[B], or past the max_q that one may have) is left alone.
 * o_g may be q_g with the same leading dimension.  q, o 16-byte aligned, ld_q and ld_o multiples of 8.  What slots past a sequence's
 * length hold does not matter; codes of its tokens are numbers (hydra_op_cache_append stores no NaN).  Scales of values below 2^-64 of a
 * sequence's largest count as that.
 * ws_g: device scratch of hydra_op_cache_attention_ws_bytes bytes, 16-byte aligned, so that a sequence's tokens can be split over
 * workgroups whose results are joined in ascending order; it need not be initialised.  Without it (or with too little) nothing is split.
 * The size and the split depend on the descriptor's sizes and H alone. */
typedef struct {
  hydra_cache_desc cache;
  int H, ld_q, ld_o, causal;
  float scale;
  const void* const* q;
  void* const* o;
  float* const* lse;
  void* const* ws;
  size_t ws_bytes;
} hydra_cache_attention_desc;
int hydra_op_cache_attention(const hydra_cache_attention_desc* d, void* stream);
size_t hydra_op_cache_attention_ws_bytes(const hydra_cache_desc* cache, int H);
/* How a call of these sizes with enough scratch is launched: plan = {rows of a key/value head that one workgroup has, its waves, runs that a sequence's
 * tokens are split into}.  16 rows: the kernel for few rows, more: the one for prompts. */
int hydra_op_cache_attention_plan(const hydra_cache_desc* cache, int H, int32_t plan[3]);

/* One token per row of logits_g [rows, ldz] (fp32 or bf16, V columns, 262144 at most), drawn from given uniforms u_g [rows, ldu] in [0, 1), one per token.
 * temperature, top_k, top_p, min_p: device arrays of `rows` entries, shared by the group.  With tokens in order of falling logits (the lower index
 * first among equals) and w_i = exp((z_i - max z) / temperature), kept are the first top_k (0: all); of those the shortest run from the first on
 * whose sum of w reaches top_p times the sum over all of them (top_p >= 1: all, at least one token always); of those the tokens with w_i >= min_p
 * times the largest.  token_g[row] = argmax over the kept of z_i / temperature - log(-log u_i), which draws i with probability proportional to
 * w_i; temperature <= 0: the largest logit.  logprob_g[row] (table NULL: not wanted) = log softmax(z)[token], over all tokens at temperature 1.
 * Logits of -inf or NaN are never drawn, +inf counts as the largest number of the logits' dtype; a row without a token to draw gets -1 and -inf. */
int hydra_op_sample(int dtype, int rows, int V, int ldz, int ldu, int G, const void* const* logits, const float* const* u,
                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, int32_t* const* token,
                    float* const* logprob, void* stream);

/* Measurement aid: enqueues n launches of a kernel that does nothing (one wave) on `stream`.  The time per launch of
 * a long run of them is the floor under any step that is a chain of dependent launches, which is what bounds the
 * smallest workload (its whole step is microseconds of arithmetic). */
int hydra_op_empty_launches(int n, void* stream);

const char* hydra_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* HYDRA_OPS_H */
