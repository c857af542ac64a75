/*
 * trevs.h - C ABI of the TReVS visual-token pruning library for MI355X (gfx950).
 *
 * TReVS ("Integrating Textual Relevance and Visual Saliency for Efficient
 * Vision-Language Model Token Pruning", arxiv 2609.37581) prunes the visual
 * tokens of a vision-language model in two stages:
 *   Stage 1, before the LLM (Sec. 4.1, Eq. (2)-(7)): fuse the vision
 *     encoder's [CLS] attention saliency with the textual relevance of each
 *     visual token, take a stable top-K_1, and gather the kept tokens.
 *   Stage 2, inside the LLM at one layer (Sec. 4.2, Eq. (8)-(9)): compute the
 *     text->vision attention, keep the high-variance heads, score each visual
 *     token by its max-over-text attention averaged over those heads, take a
 *     stable top-K_2, and compact hidden states, position ids and K/V rows.
 *
 * The pruned sequence then goes to a serving cache: rotary positions, a paged
 * K/V cache in 8 bits with the attention that reads it, and its pages.
 *
 * Conventions for every entry point:
 *   - Tensor pointers are DEVICE pointers to dense row-major tensors.  Float
 *     tensors share one element type per call (trevs_dtype).  Pointers that
 *     are read or written as 16-byte vectors (named below) must be 16-byte
 *     aligned; every other tensor must be aligned to its element size.
 *   - The caller owns every buffer, including the workspace; the library
 *     never allocates, frees or keeps state between calls.  Calls are
 *     reentrant and thread-safe.
 *   - Work is enqueued asynchronously on `stream` (a hipStream_t; NULL means
 *     the default stream); the host never waits for the device.
 *   - Arguments are validated on the host before anything is launched;
 *     invalid arguments return an error and launch nothing.  Values that live
 *     in device memory (text lengths) cannot be checked without a device
 *     synchronisation: the kernels clamp a text length into 1..M_max (or
 *     1..T_max), so an out-of-range length computes with the nearest valid
 *     one and never reads or writes outside the buffers.
 *   - Inputs must be finite.  Output buffers must not overlap the inputs or
 *     each other.  Outputs are undefined when an error is returned.
 *   - Index lists are int32, ascending and unique.  Top-K order is score
 *     descending with ties going to the lower index.
 *   - Optional `events`: NULL, or an array of 2*TREVS_*_NUM_KERNELS
 *     hipEvent_t handles (entries may be NULL).  Event 2k is recorded on the
 *     stream right before kernel k of the call and event 2k+1 right after
 *     it, for per-kernel timing by the caller.  Kernels that a call does not
 *     launch (see the limits below) leave both events next to each other.
 */
#ifndef TREVS_H
#define TREVS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum trevs_status {
  TREVS_OK = 0,
  TREVS_ERR_INVALID_ARG = 1, /* a size, ratio, pointer or alignment is invalid */
  TREVS_ERR_UNSUPPORTED = 2, /* valid, but beyond this implementation's limits */
  TREVS_ERR_WORKSPACE = 3,   /* workspace NULL, misaligned or too small */
  TREVS_ERR_HIP = 4          /* a HIP launch or event call failed */
} trevs_status;

typedef enum trevs_dtype { TREVS_F32 = 0, TREVS_BF16 = 1 } trevs_dtype;

/* Implementation limits (TREVS_ERR_UNSUPPORTED beyond them). */
#define TREVS_MAX_SELECT_N 65536 /* tokens ranked per sample by one top-K */
#define TREVS_MAX_FPS_N 32768    /* tokens per sample with a diversity set (k_div > 0) */
/* prep (none on small grids: the relevance launch does it), relevance, robust stats, fuse+top-K
 * (+ diversity set), gather */
#define TREVS_PRELLM_NUM_KERNELS 5
#define TREVS_INLLM_NUM_KERNELS 5  /* t2v stats (+ causal rest keys), head variance, head set+token score, top-K, compaction */
#define TREVS_SENSITIVITY_NUM_KERNELS 7 /* both questions: t2v stats, head variance, profile; three without a launch; Eq. (1) */

/* ------------------------------------------------------------------------
 * Stage 1 (pre-LLM), Sec. 4.1.  Per sample b:
 *   s^v_i  = (1/H_v) sum_h softmax(cls_logits[b,h,segment(i)])[i]   Eq. (2)-(3)
 *            the softmax runs over the N/n_seg patch logits of the segment
 *            (image tile or video frame) holding patch i.
 *   s^t_i  = sqrt((1/M_b) sum_{j<M_b} max(tbar_j . zbar_i, 0)^2)     Eq. (4)-(5)
 *            zbar, tbar: rows of vis_feats / text_emb over their L2 norm
 *            (norm floored at 1e-12); M_b = text_len[b].
 *   shat^c = max((s^c - Med(s^c)) / (MAD(s^c) + eps), 0) / tau_c     Eq. (6)
 *            Med = lower median (0-based rank floor((N-1)/2)), MAD = lower
 *            median of |s^c - Med|.
 *   s_i    = max(a_i, b_i) + lambda sqrt(a_i b_i),                   Eq. (7)
 *            a = 2(1-rho) shat^v, b = 2 rho shat^t  (rho = textual_ratio;
 *            rho = 0.5 is Eq. (7) exactly, rho = 0 is [CLS]-only saliency).
 *   kept_idx[b]   = TopK(s, k_keep) in ascending order
 *   kept_feats[b] = vis_feats[b, kept_idx[b], :]  (bit copy)
 * With k_div = K_d > 0 the top-K above keeps K_r = k_keep - K_d pivots, and
 * K_d more tokens are added by farthest point sampling (context
 * preservation, Sec. 4.1 after Eq. (7)): one at a time, the token outside
 * the selected set whose cosine distance 1 - zbar_i . zbar_j to its nearest
 * selected token is largest (ties to the lower index).  Tokens whose distance
 * is not a number (the squares of a row overflow fp32) follow after all others,
 * in index order.  The workspace has
 * room for a Gram matrix of every sample, beyond the k_div = 0 size: of all N
 * tokens (85 MB at B = 64, N = 576), or, where the picks are made in rounds over
 * pools of tokens, of those that are no pivots, for what the rounds leave, and
 * for lists, a few words a token and a bit for each pair of a pool (2.8 GB at
 * B = 4, N = 16,384, K_r = 3072; 0.37 GB at B = 16, N = 2880, K_r = 480);
 * trevs_prellm_workspace_size includes it, and the call itself allocates
 * nothing.
 * With ratio_mode = TREVS_RATIO_BUDGET the textual ratio is instead the
 * share of the token budget given to textual relevance (the reading of the
 * preliminary analysis, Sec. 3): K_t = floor(rho * k_keep + 1/2) tokens with
 * the highest s^t, then the k_keep - K_t tokens with the highest s^v among
 * the others; Eq. (6)-(7) are not used, and score_out and norm_stats must
 * be NULL.  Every top-K is stable (score descending, lower index first).
 * ---------------------------------------------------------------------- */
typedef enum trevs_ratio_mode {
  TREVS_RATIO_WEIGHTS = 0, /* branch weights 2(1-rho), 2rho inside Eq. (7) */
  TREVS_RATIO_BUDGET = 1   /* budget split between s^t and s^v */
} trevs_ratio_mode;

typedef struct trevs_prellm_args {
  uint32_t struct_size;      /* sizeof(trevs_prellm_args) */
  int32_t B;                 /* samples */
  int32_t N;                 /* visual tokens per sample, 1..TREVS_MAX_SELECT_N */
  int32_t n_seg;             /* [CLS] softmax segments; N % n_seg == 0 */
  int32_t H_v;               /* vision-encoder heads, >= 1 */
  int32_t d;                 /* projected width d'; d * elem_size % 16 == 0 */
  int32_t M_max;             /* padded text rows, >= 1 */
  int32_t k_keep;            /* K_1 = K_r + K_d, 1..N */
  int32_t k_div;             /* K_d farthest-point diversity tokens, 0..k_keep-1; N <= TREVS_MAX_FPS_N when > 0 */
  float textual_ratio;       /* rho in [0, 1]; 0.5 reproduces Eq. (7) */
  float tau_v, tau_t;        /* temperatures > 0 (paper: 1.4, 1.0) */
  float lambda_;             /* consistency reward weight >= 0 (paper: 1.0) */
  float eps;                 /* MAD stabiliser >= 0 (default 1e-8) */
  int32_t dtype;             /* trevs_dtype of cls_logits, vis_feats, text_emb, kept_feats */
  const void* cls_logits;    /* [B,H_v,N] pre-softmax [CLS]->patch logits, scaled by 1/sqrt(d_h) */
  const void* vis_feats;     /* [B,N,d] projected visual features Z (16-byte aligned) */
  const void* text_emb;      /* [B,M_max,d] text embeddings (16-byte aligned) */
  const int32_t* text_len;   /* [B] valid text rows M_b in 1..M_max, or NULL (= M_max) */
  int32_t* kept_idx;         /* OUT [B,k_keep] ascending */
  void* kept_feats;          /* OUT [B,k_keep,d] gathered rows (16-byte aligned) */
  float* score_out;          /* OPTIONAL OUT [B,N] fused score s */
  float* sal_out;            /* OPTIONAL OUT [B,N] s^v */
  float* rel_out;            /* OPTIONAL OUT [B,N] s^t */
  float* norm_stats;         /* OPTIONAL OUT [B,4] Med(s^v), MAD(s^v), Med(s^t), MAD(s^t) */
  void* const* events;       /* OPTIONAL [2*TREVS_PRELLM_NUM_KERNELS] hipEvent_t */
  int32_t ratio_mode;        /* trevs_ratio_mode */
  int32_t* div_idx;          /* OPTIONAL OUT [B,k_div] diversity tokens in pick order */
} trevs_prellm_args;

/* ------------------------------------------------------------------------
 * Stage 2 (in-LLM, at the pruning layer), Sec. 4.2.  Sequence layout per
 * sample: rows [0,P) prefix, [P,P+K_in) visual, [P+K_in, P+K_in+T_max) text,
 * then any further rows up to S.  Per sample b with G = H_q/H_kv and
 * T_b = text_len[b]:
 *   x[h,q,i] = scale * q[b,P+K_in+q,h,:] . k[b,P+i,h/G,:]   (q < T_b, i < K_in)
 *   A[h,q,:] = exp(x[h,q,:] - LSE[h,q]) over the visual columns, where the
 *              softmax domain (trevs_softmax) sets LSE[h,q]:
 *              VISUAL: logsumexp_i x[h,q,i] over the K_in visual keys; when
 *                lse_rest is given, logaddexp(that, lse_rest[b,h,q]), the
 *                full-row softmax with the non-visual part supplied by the
 *                caller;
 *              CAUSAL: the log-sum-exp of the row's whole causal attention
 *                row at this layer, computed from q and k: the prefix keys
 *                [0,P), the visual keys, and the text keys P+K_in .. P+K_in+q
 *                (the row's own position and those before it); every key
 *                uses the row's KV head h/G.  A thus holds the visual columns
 *                of the layer's own attention matrix (Sec. 4.2).
 *   u_h      = (1/T_b) sum_q Var_i A[h,q,i]  (population variance)    Eq. (8)
 *              (with row_stats: (1/T_b) sum_q [S2/K_in - (S1/K_in)^2] from the
 *              caller's per-row sums S1 = sum_i A, S2 = sum_i A^2, and the
 *              row log-sum-exp from row_stats as well)
 *   H*       = the n_keep_heads heads first under (u desc, h asc)
 *   p_i      = max_{q<T_b} (1/|H*|) sum_{h in H*} A[h,q,i]            Eq. (9)
 *   kept_idx = TopK(p, k_keep) ascending, relative to the visual block
 *   rows     = [0,P) ++ (P + kept_idx) ++ [P+K_in, S);  S' = S - K_in + k_keep
 *   hidden_out[b] = hidden[b,rows], k_out[b] = k[b,rows], v_out[b] = v[b,rows],
 *   pos_out[p,b]  = pos[p,b,rows]   (bit copies; position ids are not renumbered)
 * ---------------------------------------------------------------------- */
typedef enum trevs_softmax {
  TREVS_SOFTMAX_VISUAL = 0,  /* softmax over the visual keys (plus lse_rest, if given) */
  TREVS_SOFTMAX_CAUSAL = 1   /* softmax over each text row's causal row of the sequence */
} trevs_softmax;

typedef struct trevs_inllm_args {
  uint32_t struct_size;      /* sizeof(trevs_inllm_args) */
  int32_t B;                 /* samples */
  int32_t S;                 /* sequence rows at the pruning layer */
  int32_t P;                 /* prefix rows before the visual block, >= 0 */
  int32_t K_in;              /* visual rows K_1, 1..TREVS_MAX_SELECT_N */
  int32_t T_max;             /* padded text rows; P + K_in + T_max <= S */
  int32_t H_q, H_kv;         /* query / key-value heads; H_q % H_kv == 0 */
  int32_t d_head;            /* 64, 128 or 256 */
  int32_t D;                 /* hidden size; D * elem_size % 16 == 0 */
  int32_t n_pos;             /* position-id planes (1, or 3 for M-RoPE), >= 1 */
  int32_t n_keep_heads;      /* |H*|, 1..H_q (paper: H_q / 2) */
  int32_t k_keep;            /* K_2, 1..K_in */
  float scale;               /* logit scale > 0, normally 1/sqrt(d_head) */
  int32_t dtype;             /* trevs_dtype of q, k, v, hidden and their outputs */
  const void* q;             /* [B,S,H_q,d_head] (16-byte aligned) */
  const void* k;             /* [B,S,H_kv,d_head] (16-byte aligned) */
  const void* v;             /* [B,S,H_kv,d_head] (16-byte aligned) */
  const void* hidden;        /* [B,S,D] (16-byte aligned) */
  const int64_t* pos;        /* [n_pos,B,S] */
  const int32_t* text_len;   /* [B] T_b in 1..T_max, or NULL (= T_max) */
  const float* lse_rest;     /* OPTIONAL [B,H_q,T_max] log-sum-exp of each text row's non-visual
                                logits (natural log); VISUAL softmax only, NULL with CAUSAL */
  int32_t* kept_idx;         /* OUT [B,k_keep] ascending, relative to the visual block */
  void* hidden_out;          /* OUT [B,S',D] (16-byte aligned) */
  void* k_out;               /* OUT [B,S',H_kv,d_head] (16-byte aligned) */
  void* v_out;               /* OUT [B,S',H_kv,d_head] (16-byte aligned) */
  int64_t* pos_out;          /* OUT [n_pos,B,S'] */
  int32_t* head_sel;         /* OPTIONAL OUT [B,n_keep_heads] H*, ascending */
  float* head_var;           /* OPTIONAL OUT [B,H_q] u_h */
  float* score_out;          /* OPTIONAL OUT [B,K_in] p_i */
  void* const* events;       /* OPTIONAL [2*TREVS_INLLM_NUM_KERNELS] hipEvent_t */
  int32_t softmax;           /* trevs_softmax: domain of the attention softmax (0 = VISUAL) */
  const float* row_stats;    /* OPTIONAL [B,H_q,T_max,3] per text row, from the layer's own
                                attention pass: (log-sum-exp of the row's logits over its
                                softmax domain, natural log; sum and sum of squares of A over
                                the K_in visual columns).  When given, u_h is formed from them
                                and the row log-sum-exp is taken from them instead of being
                                recomputed from q and k (softmax is then ignored and lse_rest
                                must be NULL); the token score still recomputes the logits of
                                the H* heads.  Rows q >= T_b are not read for u_h. */
} trevs_inllm_args;

/* ------------------------------------------------------------------------
 * Diagnostics of the preliminary analysis (Sec. 3), computed on the same
 * tensors as the pruning stages.
 *
 * Text sensitivity of the attention heads (Eq. (1)).  One image paired with
 * two questions gives two stage-2 inputs of one shape, each laid out as for
 * trevs_inllm_prune (visual rows [P,P+K_in), text rows after them).  For
 * question c in {0,1} with T^c_b = text_len[c][b] valid text rows:
 *   A^c[h,q,:]  = the text->vision attention of trevs_inllm_prune, in the
 *                 same softmax domain (VISUAL, with lse_rest[c] if given, or
 *                 CAUSAL computed from q[c] and k[c])
 *   s^c_h       = (1/T^c_b) sum_{q<T^c_b} A^c[h,q,:]   the head's attention
 *                 distribution over the visual tokens for that question
 *   ts[b,h]     = 1 - cos(s^0_h, s^1_h)                                 Eq. (1)
 * head_var[c] optionally receives u_h of Eq. (8) for question c, so that the
 * heads can be ranked by attention variance as in the analysis.
 * ---------------------------------------------------------------------- */
typedef struct trevs_sensitivity_args {
  uint32_t struct_size;      /* sizeof(trevs_sensitivity_args) */
  int32_t B, S, P, K_in, T_max;  /* as in trevs_inllm_args; P + K_in + T_max <= S */
  int32_t H_q, H_kv;         /* query / key-value heads; H_q % H_kv == 0 */
  int32_t d_head;            /* 64, 128 or 256 */
  float scale;               /* logit scale > 0 */
  int32_t dtype;             /* trevs_dtype of q and k */
  const void* q[2];          /* per question [B,S,H_q,d_head] (16-byte aligned) */
  const void* k[2];          /* per question [B,S,H_kv,d_head] (16-byte aligned); may be one buffer */
  const int32_t* text_len[2];  /* per question [B] in 1..T_max, or NULL (= T_max) */
  const float* lse_rest[2];  /* OPTIONAL per question [B,H_q,T_max] non-visual log-sum-exp
                                (VISUAL softmax only) */
  float* ts;                 /* OUT [B,H_q] text sensitivity */
  float* profile[2];         /* OPTIONAL OUT per question [B,H_q,K_in] s^c_h */
  float* head_var[2];        /* OPTIONAL OUT per question [B,H_q] u_h */
  void* const* events;       /* OPTIONAL [2*TREVS_SENSITIVITY_NUM_KERNELS] hipEvent_t */
  int32_t softmax;           /* trevs_softmax, as in trevs_inllm_args (0 = VISUAL) */
} trevs_sensitivity_args;

size_t trevs_sensitivity_workspace_size(const trevs_sensitivity_args* args);
trevs_status trevs_text_sensitivity(const trevs_sensitivity_args* args, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* Spearman rank correlation between visual saliency and textual relevance
 * within the top-K saliency set (Sec. 3).  sv, st [B,N] are s^v and s^t
 * (device, finite fp32; e.g. sal_out and rel_out of trevs_prellm_prune).
 * Per sample b: the K tokens first under (sv desc, index asc), the same
 * stable top-K as the pruning; the 1-based ranks of sv and of st over those
 * K tokens, tied values sharing the mean of the ranks they span; rho[b] =
 * the Pearson correlation of the two rank vectors, NaN when either is
 * constant (always for K = 1).  The rank sums are exact integers, so rho is
 * correctly rounded up to one division and one square root in double.
 * kept_idx: OPTIONAL OUT [B,K] the set, ascending.  N in
 * 1..TREVS_MAX_SELECT_N, K in 1..N. */
size_t trevs_spearman_workspace_size(int32_t B, int32_t N, int32_t K);
trevs_status trevs_topk_spearman(const float* sv, const float* st, int32_t B, int32_t N, int32_t K,
                                 double* rho, int32_t* kept_idx, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Workspace bytes the call needs for these arguments (0 on invalid args).
 * The workspace must be 256-byte aligned; its contents need no initialisation
 * and are garbage afterwards. */
size_t trevs_prellm_workspace_size(const trevs_prellm_args* args);
size_t trevs_inllm_workspace_size(const trevs_inllm_args* args);
size_t trevs_topk_workspace_size(int32_t B, int32_t N, int32_t K);

/* Stage 1 (Sec. 4.1, Eq. (2)-(7) and the pivot Top-K). */
trevs_status trevs_prellm_prune(const trevs_prellm_args* args, void* workspace,
                                size_t workspace_bytes, void* stream);

/* Stage 2 (Sec. 4.2, Eq. (8)-(9), Top-K_2 and compaction). */
trevs_status trevs_inllm_prune(const trevs_inllm_args* args, void* workspace,
                               size_t workspace_bytes, void* stream);

/* Stage 2 exactly as trevs_inllm_prune, for callers that cannot allocate
 * device memory: code under HIP graph capture, tight serving loops, and
 * harnesses that forbid allocation.  The caller passes inputs and outputs
 * only; the workspace is a static device array of
 * TREVS_NOALLOC_SCRATCH_BYTES inside the library, one per GPU, held from the
 * first call on that GPU until the process ends.  The call allocates and
 * frees nothing.
 *   - Runs on the calling thread's current device, which must be the
 *     stream's device.  The first call on a device looks up the array's
 *     address there (hipGetSymbolAddress); make that first call before
 *     capturing a graph.
 *   - Arguments whose workspace (trevs_inllm_workspace_size) exceeds
 *     TREVS_NOALLOC_SCRATCH_BYTES return TREVS_ERR_WORKSPACE before any
 *     launch; invalid arguments return the status trevs_inllm_prune gives.
 *   - Every call on a GPU shares that GPU's array: calls that overlap on one
 *     GPU (different streams, or host threads) race and give undefined
 *     results.  Serialise them, e.g. on one stream.  Calls in order on one
 *     stream are safe; no state carries from one call to the next. */
#define TREVS_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)
trevs_status trevs_inllm_prune_noalloc(const trevs_inllm_args* args, void* stream);

/* Stable top-K of each row of scores [B,N] (device, finite fp32): writes the
 * K kept indices of row b, ascending, to kept_idx [B,K].  N in
 * 1..TREVS_MAX_SELECT_N, K in 1..N.  Needs no workspace (pass NULL, 0). */
trevs_status trevs_topk_select(const float* scores, int32_t B, int32_t N, int32_t K,
                               int32_t* kept_idx, void* workspace, size_t workspace_bytes,
                               void* stream);

/* ------------------------------------------------------------------------
 * Rotary positions of query and key rows (the positions that stage 2 compacts
 * without renumbering them).  For token (b,s), pair i < R/2 of the first
 * R = rot_dim values of every head, with a, b the pair's values:
 *   w  = 2 pi * pos[plane(i)][b][s] * freqs[i]
 *   a' = attn_factor (a cos w - b sin w),  b' = attn_factor (b cos w + a sin w)
 * A pair is values (i, i + R/2) of the head, or (2i, 2i+1) with `interleaved`.
 * plane(i) deals the pairs to the n_pos position planes in order: the first
 * section[0] pairs use plane 0, the next section[1] plane 1, and so on.
 * Values past R are copied.  `inverse` turns by -w instead (with the same
 * attn_factor): the gradient of the rotation, and with attn_factor 1 its undoing.
 * The fractions of a turn are formed in 64 bits, and so are their sine and
 * cosine, times attn_factor, for fp32 tensors, rounded once to 32 (for bf16
 * ones in 32); positions are exact up to 2^53.
 * ---------------------------------------------------------------------- */
#define TREVS_MAX_POS_PLANES 4
typedef struct trevs_rope_args {
  uint32_t struct_size;      /* sizeof(trevs_rope_args) */
  int32_t B, S;              /* samples, rows of each */
  int32_t H_q, H_k;          /* heads of q and k; 0 leaves that tensor out (not both) */
  int32_t d_head;            /* 64, 128 or 256 */
  int32_t rot_dim;           /* R: a multiple of 16, 16..d_head */
  int32_t n_pos;             /* position planes, 1..TREVS_MAX_POS_PLANES */
  int32_t section[TREVS_MAX_POS_PLANES]; /* pairs of each plane, >= 0; the first n_pos sum to R/2 */
  int32_t interleaved;       /* 0: pairs (i, i + R/2); 1: pairs (2i, 2i+1) */
  int32_t inverse;           /* 1: turn by -w */
  int32_t dtype;             /* trevs_dtype of q, k and their outputs */
  float attn_factor;         /* finite; normally 1 */
  const double* freqs;       /* [R/2] turns per position, on the device (trevs_rope_frequencies) */
  const int64_t* pos;        /* [n_pos,B,S] */
  const void* q;             /* [B,S,H_q,d_head], rows q_ld elements apart (16-byte aligned) */
  const void* k;             /* [B,S,H_k,d_head], rows k_ld elements apart (16-byte aligned) */
  void* q_out;               /* OUT as q, rows q_out_ld apart; may be q itself (in place) */
  void* k_out;               /* OUT as k, rows k_out_ld apart; may be k itself (in place) */
  int64_t q_ld, k_ld;        /* elements from one row to the next, 0 = H * d_head; row bytes % 16 == 0 */
  int64_t q_out_ld, k_out_ld;
} trevs_rope_args;

trevs_status trevs_rope(const trevs_rope_args* args, void* stream);

/* The frequencies of trevs_rope, computed on the host into freqs [rot_dim/2]
 * (host memory): f_i = base^(-2i/rot_dim) / (2 pi) turns per position, for
 * contexts longer than the model's own divided by `factor`
 *   NONE    not at all
 *   LINEAR  in every pair (the positions are interpolated)
 *   PARTS   by parts (arxiv 2309.00071, Sec. 3.2): with r = original_len * f_i
 *           turns over the original context, pairs with r >= beta_fast not at
 *           all, with r <= beta_slow in full, between them in proportion. */
typedef enum trevs_rope_scaling {
  TREVS_ROPE_NONE = 0,
  TREVS_ROPE_LINEAR = 1,
  TREVS_ROPE_PARTS = 2
} trevs_rope_scaling;
trevs_status trevs_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                                    double original_len, double beta_fast, double beta_slow,
                                    double* freqs);

/* ------------------------------------------------------------------------
 * A paged K/V cache held in 8 bits: what the layers after the pruning, and
 * the decode steps, attend to.  Tokens live in pages of page_tokens; every
 * page holds, for each layer and KV head, one block of keys and one of
 * values as OCP e4m3 numbers with one scale each:
 *   key   of token t, channel c = k[layer][page][h][t][c] * k_scale[layer][page][h]
 *   value of token t, channel c = v[layer][page][h][c][t] * v_scale[layer][page][h]
 * (values are stored with the token last).  A scale is a power of two,
 * 2^-126..2^120: the smallest s with |x| <= 448 s over the block when its rows
 * were written, so that dividing by it is exact and a value is rounded once,
 * to the nearest e4m3 (ties to even); rows hold magnitudes up to 2^127.  Rows
 * should be finite: an infinity or NaN is stored as NaN and does not count for
 * the scale, so the block's other values are as without it.  Rows appended to
 * a block that already holds tokens keep its scale or raise it; when it rises,
 * the block's earlier values are rounded again to the new scale (exact above
 * its subnormals).
 *
 * One page table serves every layer: sequence slot i < n_slots holds len[i]
 * tokens, token t in page table[i][t / page_tokens].  ref[p] counts the slots
 * that hold page p; 0 means free.  Slots may share pages (trevs_pages_fork);
 * a shared page is only read: trevs_pages_reserve gives a slot its own copy
 * of a shared last page before rows are appended to it.
 * An empty table is: len and ref all 0 (table entries past a slot's pages
 * are not read; the page operations leave -1 there).  All arrays are the
 * caller's, in device memory.  Table entries outside 0..n_pages-1 are taken
 * as absent (read as masked, never written), slots outside 0..n_slots-1 as
 * empty, and lengths are clamped into 0..max_pages * page_tokens.
 * ---------------------------------------------------------------------- */
typedef struct trevs_kv8_cache {
  uint32_t struct_size;      /* sizeof(trevs_kv8_cache) */
  int32_t n_layers;          /* >= 1 */
  int32_t n_pages;           /* >= 1 */
  int32_t page_tokens;       /* 16, 32 or 64 */
  int32_t H_kv;              /* KV heads */
  int32_t d_head;            /* 64, 128 or 256 */
  int32_t n_slots;           /* sequences */
  int32_t max_pages;         /* pages of the longest sequence; max_pages * page_tokens <= 2^30 */
  uint8_t* k;                /* [n_layers,n_pages,H_kv,page_tokens,d_head] e4m3 (16-byte aligned) */
  uint8_t* v;                /* [n_layers,n_pages,H_kv,d_head,page_tokens] e4m3 (16-byte aligned) */
  float* k_scale;            /* [n_layers,n_pages,H_kv] */
  float* v_scale;            /* [n_layers,n_pages,H_kv] */
  int32_t* table;            /* [n_slots,max_pages] */
  int32_t* len;              /* [n_slots] */
  int32_t* ref;              /* [n_pages] */
} trevs_kv8_cache;

/* Page operations.  Every list below has n entries, n in
 * 1..TREVS_MAX_PAGE_REQUESTS, in device memory; a list of slots that is NULL
 * stands for 0..n-1 (n <= n_slots).  Results are those of serving the
 * requests in order.  A request that names a slot out of range, or the slot
 * that an earlier request of the call names (as its destination, in a fork),
 * does nothing.  The calls only change table, len and ref; a call must not run
 * beside another one on the same cache. */
#define TREVS_MAX_PAGE_REQUESTS 1024

/* Room for n_new[i] more tokens in slots[i]: its length grows by that and its
 * table by the pages needed, the lowest free ones first, in ascending order.
 * When the slot's last page is shared and not full, the first of them
 * replaces it: copy_src[i] and copy_dst[i] are then the shared page and its
 * replacement, for trevs_kv8_copy_pages, else both are -1.  A request that
 * the free pages or max_pages do not cover, or with n_new[i] < 1, changes
 * nothing; granted[i] is n_new[i] or 0. */
trevs_status trevs_pages_reserve(const trevs_kv8_cache* cache, int32_t n, const int32_t* slots,
                                 const int32_t* n_new, int32_t* granted, int32_t* copy_src,
                                 int32_t* copy_dst, void* stream);

/* Slot dst[i], which must be empty, shares the pages of the first n_tokens[i]
 * tokens (clamped into 0..len) of slot src[i], or of all of them with n_tokens
 * NULL.  A source that is a destination of the same call is refused.  done[i]
 * is 1, or 0 when the request did nothing. */
trevs_status trevs_pages_fork(const trevs_kv8_cache* cache, int32_t n, const int32_t* src, const int32_t* dst,
                              const int32_t* n_tokens, int32_t* done, void* stream);

/* Slot slots[i] keeps its first keep[i] tokens (clamped into 0..len), or none
 * with keep NULL, and gives up its other pages; pages that no slot holds any
 * more are free. */
trevs_status trevs_pages_free(const trevs_kv8_cache* cache, int32_t n, const int32_t* slots,
                              const int32_t* keep, void* stream);

/* Pages src[i] copied to pages dst[i] in every layer, keys, values and scales
 * (bit copies); pairs with an entry out of range are skipped.  No page may be
 * the destination of two pairs, nor of one and the source of another.  n is at
 * most 2^24 - 1. */
trevs_status trevs_kv8_copy_pages(const trevs_kv8_cache* cache, int32_t n, const int32_t* src,
                                  const int32_t* dst, void* stream);

/* Rows written to one layer of the cache: the last n_new[b] tokens of slot
 * slots[b] (their room reserved before), token len - n_new + t from row t.
 * n_new is clamped into 0..min(T_max, len).  The pages written must be held
 * by that slot alone. */
typedef struct trevs_kv8_write_args {
  uint32_t struct_size;      /* sizeof(trevs_kv8_write_args) */
  int32_t B;                 /* sequences */
  int32_t T_max;             /* padded rows, >= 1 */
  int32_t layer;             /* 0..n_layers-1 */
  int32_t dtype;             /* trevs_dtype of k and v */
  const void* k;             /* [B,T_max,H_kv,d_head], rows k_ld elements apart (16-byte aligned) */
  const void* v;             /* [B,T_max,H_kv,d_head], rows v_ld elements apart (16-byte aligned) */
  int64_t k_ld, v_ld;        /* 0 = H_kv * d_head; row bytes % 16 == 0 */
  const int32_t* n_new;      /* [B], or NULL (= T_max) */
  const int32_t* slots;      /* [B], or NULL (= 0..B-1, B <= n_slots); no slot twice */
} trevs_kv8_write_args;

trevs_status trevs_kv8_write(const trevs_kv8_cache* cache, const trevs_kv8_write_args* args, void* stream);

/* Attention of query rows over one layer of the cache.  With L = len[slot],
 * query row t < q_len[b] of head h sees the keys j of KV head h/G, G = H_q/H_kv,
 *   causal: j <= L - q_len[b] + t (the rows are the sequence's last ones)
 *   else:   every j < L
 *   out[b,t,h,:] = sum_j softmax_j(scale q . k_j) v_j
 *   lse[b,h,t]   = logsumexp_j(scale q . k_j), natural log
 * A row that sees no key gives zeros and -inf.  A stored NaN makes the rows that
 * see it NaN, a key's everywhere, a value's in its channel; others are as
 * without it.  Rows t >= q_len[b] are left as they were.  Products run on the
 * matrix cores with 32-bit sums: bf16 queries and attention weights as bf16
 * (which adds a tenth to a quarter to the rounding error of bf16 outputs), fp32
 * ones as three bf16 parts each. */
typedef struct trevs_kv8_attention_args {
  uint32_t struct_size;      /* sizeof(trevs_kv8_attention_args) */
  int32_t B;                 /* sequences */
  int32_t T_max;             /* padded query rows, >= 1 */
  int32_t H_q;               /* query heads; H_q % H_kv == 0 */
  int32_t layer;             /* 0..n_layers-1 */
  int32_t dtype;             /* trevs_dtype of q and out */
  int32_t causal;            /* 0 or 1 */
  int32_t kv_max;            /* no sequence of the call is longer (longer ones are cut there);
                                0 = max_pages * page_tokens.  Sizes the launch and the workspace. */
  float scale;               /* logit scale > 0, normally 1/sqrt(d_head) */
  const void* q;             /* [B,T_max,H_q,d_head], rows q_ld elements apart (16-byte aligned) */
  int64_t q_ld;              /* 0 = H_q * d_head; row bytes % 16 == 0 */
  const int32_t* q_len;      /* [B], clamped into 0..T_max, or NULL (= T_max) */
  const int32_t* slots;      /* [B], or NULL (= 0..B-1, B <= n_slots) */
  void* out;                 /* OUT [B,T_max,H_q,d_head] (16-byte aligned) */
  float* lse;                /* OPTIONAL OUT [B,H_q,T_max] */
} trevs_kv8_attention_args;

/* About 68 MB at most, and 256 bytes for calls whose tiles of rows fill the GPU by
 * themselves (0 on invalid args); contents as for the other workspaces. */
size_t trevs_kv8_attention_workspace_size(const trevs_kv8_cache* cache, const trevs_kv8_attention_args* args);
trevs_status trevs_kv8_attention(const trevs_kv8_cache* cache, const trevs_kv8_attention_args* args,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* The compaction of trevs_inllm_prune inside the cache, in every layer: with
 * L = len[src_slots[b]], rows [0,P) ++ (P + kept_idx[b]) ++ [P+K_in, L) of slot
 * src_slots[b] become the first L - K_in + n_kept tokens of slot dst_slots[b], in
 * that order, their blocks rounded to scales of their own.  Rows past
 * len[dst_slots[b]] are dropped (room is reserved before), and a sample with
 * L < P + K_in, or one slot as both, is skipped.  No destination twice, and the
 * slots' pages must not meet: a destination is filled from pages that no
 * destination of the call holds. */
typedef struct trevs_kv8_compact_args {
  uint32_t struct_size;      /* sizeof(trevs_kv8_compact_args) */
  int32_t B;                 /* sequences */
  int32_t P, K_in;           /* prefix rows and visual rows, as in trevs_inllm_args */
  int32_t n_kept;            /* 1..K_in */
  const int32_t* kept_idx;   /* [B,n_kept] (clamped into 0..K_in-1) */
  const int32_t* src_slots;  /* [B] */
  const int32_t* dst_slots;  /* [B] */
} trevs_kv8_compact_args;

trevs_status trevs_kv8_compact(const trevs_kv8_cache* cache, const trevs_kv8_compact_args* args, void* stream);

/* Static description of a status code. */
const char* trevs_status_string(trevs_status status);

/* Budget bookkeeping: floor(ratio * n + 1/2) clamped to [1, n] (0 if n < 1). */
int32_t trevs_keep_count(float ratio, int32_t n);

/* sizeof() of the argument structs as compiled into the library, for
 * bindings that mirror them. */
size_t trevs_prellm_args_size(void);
size_t trevs_inllm_args_size(void);
size_t trevs_sensitivity_args_size(void);
size_t trevs_rope_args_size(void);
size_t trevs_kv8_cache_size(void);
size_t trevs_kv8_write_args_size(void);
size_t trevs_kv8_attention_args_size(void);
size_t trevs_kv8_compact_args_size(void);

#ifdef __cplusplus
}
#endif

#endif /* TREVS_H */
