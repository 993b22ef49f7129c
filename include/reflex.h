/*
 * reflex.h - C ABI of the REFLEX variable-K MoE layer for MI355X (gfx950).
 *
 * The layer is the MoE feed-forward block of a diffusion language model's
 * denoising forward in which each token i gets its own expert count k_i
 * (Section 3.2, Eq. (2)), chosen per forward by Refinement-Role Budgeting
 * (Section 4.2, Eq. (5)) and Frontier-Guided Expert Reallocation with the
 * Frontier-Progress Score (Section 4.3, Eqs. (6)-(9)), subject to the count
 * bounds of Eq. (3).
 *
 * Conventions shared by every entry point
 *  - All array arguments are DEVICE pointers owned by the caller; the library
 *    never allocates, frees or retains them.  Struct arguments
 *    (reflex_alloc_params, reflex_moe_args) are HOST pointers, read during the
 *    call only.
 *  - bf16 data is passed as uint16_t bit patterns.  Matrices are row-major and
 *    dense (leading dimension = row length).
 *  - `stream` is a hipStream_t passed as void* (NULL = default stream).  Work is
 *    enqueued asynchronously; nothing is read back to the host and no call
 *    synchronises.  Calls keep no state between them and may be made from several
 *    threads; the lasting resources are a second stream per device (non-blocking,
 *    default priority, created on first use) on which reflex_moe_forward runs the
 *    shared expert beside the routing, ordered against `stream` by events from a
 *    per-device pool (created on first use, reused by later calls), and the device
 *    scratch of reflex_moe_forward_noalloc.
 *  - Arguments are validated on the host before anything is launched; on error
 *    nothing is launched and a negative status is returned.  No C++ exception
 *    crosses the ABI.
 *  - T = 0 (no tokens) is valid and enqueues nothing.
 *  - Alignment (REFLEX_ERR_SHAPE otherwise): bf16 matrices (h, expert weights,
 *    y_sorted, shared_y, residuals, out), the fp32 router weight and workspaces
 *    must be 16-byte aligned (the kernels move them in 16-byte vectors); every
 *    other pointer needs the natural alignment of its element type.
 *  - Content preconditions that cannot be checked without reading device memory
 *    (seq_offsets non-decreasing from 0 to T, block_idx >= 0, hist_len in
 *    {0,1,2}, finite logits, expert_offsets consistent with the pair count) are
 *    the caller's.  Kernels never index outside the buffers whose sizes the
 *    arguments state, whatever those contents are: counts are clamped to
 *    [0, k_max] before they size anything.
 */
#ifndef REFLEX_H
#define REFLEX_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------------ */
#define REFLEX_OK                 0
#define REFLEX_ERR_NULL         (-1)  /* a required pointer is NULL                        */
#define REFLEX_ERR_SHAPE        (-2)  /* a size is out of range or not a supported multiple */
#define REFLEX_ERR_PARAM        (-3)  /* a hyper-parameter is out of range or not finite    */
#define REFLEX_ERR_WORKSPACE    (-4)  /* workspace or pair capacity too small               */
#define REFLEX_ERR_LAUNCH       (-5)  /* the HIP runtime reported a launch error            */
#define REFLEX_ERR_UNSUPPORTED  (-6)  /* a valid request this build does not implement      */

/* ---- limits ------------------------------------------------------------------ */
#define REFLEX_MAX_EXPERTS  256       /* E <= 256                                        */
#define REFLEX_MAX_K        32        /* k_max <= min(E, 32)                             */
#define REFLEX_D_MULTIPLE   128       /* hidden size d must be a multiple of this        */
#define REFLEX_F_MULTIPLE   64        /* expert widths f, f_shared must be multiples     */
#define REFLEX_MAX_DIM      16384     /* d, f, f_shared <= this                          */
#define REFLEX_MAX_TOKENS   (1 << 24) /* T <= this                                       */

/* Ranking key of the active-block reallocation (Section 4.3; Appendix C). */
#define REFLEX_SIGNAL_FPS          0  /* S = F * P, Eq. (8)                    */
#define REFLEX_SIGNAL_FRONTIER     1  /* F alone, Eq. (6)                      */
#define REFLEX_SIGNAL_PROGRESS     2  /* P alone, Eq. (7)                      */
#define REFLEX_SIGNAL_CONFIDENCE   3  /* lagged confidence c^{t-1}             */
#define REFLEX_SIGNAL_UNCERTAINTY  4  /* 1 - c^{t-1}                           */

/*
 * Allocation hyper-parameters (Eqs. (3), (5)-(9); defaults in Section 5.1:
 * k_base 8, delta_role 4, delta_cur 2, q 0.25, theta 0.9, w_cf 0.30 or 0.25,
 * v_ref 0.01, tau 0.05).  Real values are float32 and are widened exactly to
 * fp64 inside the kernels.
 * Valid: 0 <= k_min <= k_max <= REFLEX_MAX_K; k_base, delta_role, delta_cur >= 0;
 * 0 < q <= 0.5; tau > 0; w_cf > 0; theta, v_ref finite; signal in 0..4.
 */
typedef struct {
  int32_t k_base;      /* K_base: nominal count (Eq. (5))                            */
  int32_t delta_role;  /* delta_role: role offset (Eq. (5)); K_cur = k_base+delta_role */
  int32_t delta_cur;   /* delta_cur: reallocation offset (Eq. (9))                  */
  int32_t k_min;       /* K_min: lower count bound (Eq. (3)), applied as a clamp     */
  int32_t k_max;       /* K_max: upper count bound (Eq. (3)), applied as a clamp     */
  float   q;           /* outer-group fraction; groups have floor(q*m) members      */
  float   theta;       /* commitment threshold theta                                */
  float   w_cf;        /* commitment-frontier width w_cf                            */
  float   v_ref;       /* velocity reference v_ref                                  */
  float   tau;         /* gate temperature tau                                      */
  int32_t signal;      /* REFLEX_SIGNAL_*                                           */
} reflex_alloc_params;

/*
 * The paper's settings as ready-made parameters (host only, no GPU work):
 * Section 5.1 defaults with the given count bounds and frontier width, and the
 * ablation variants of Section 5.3 and Appendix C:
 *  REFLEX_PRESET_FULL         RRB + FGER with the Frontier-Progress Score
 *  REFLEX_PRESET_RRB_ONLY     delta_cur = 0 (no reallocation inside the active block)
 *  REFLEX_PRESET_FGER_ONLY    delta_role = 0 (every role keeps k_base)
 *  REFLEX_PRESET_FRONTIER_ONLY, _PROGRESS_ONLY, _CONFIDENCE_ONLY, _UNCERTAINTY_ONLY
 *                             the full method ranking by one signal (REFLEX_SIGNAL_*)
 *  k_min, k_max   count bounds (e.g. 2, 12); w_cf 0.30 (LLaDA-MoE) or 0.25 (LLaDA2.0-mini)
 * Errors: NULL out; unknown preset (REFLEX_ERR_PARAM); the result failing the
 * validity rules above (REFLEX_ERR_PARAM).
 */
#define REFLEX_PRESET_FULL              0
#define REFLEX_PRESET_RRB_ONLY          1
#define REFLEX_PRESET_FGER_ONLY         2
#define REFLEX_PRESET_FRONTIER_ONLY     3
#define REFLEX_PRESET_PROGRESS_ONLY     4
#define REFLEX_PRESET_CONFIDENCE_ONLY   5
#define REFLEX_PRESET_UNCERTAINTY_ONLY  6
int reflex_alloc_preset(int preset, int k_min, int k_max, float w_cf, reflex_alloc_params* out);

/* ---- introspection ---------------------------------------------------------- */
int         reflex_version(void);               /* 100 * major + minor                */
const char* reflex_status_string(int status);   /* static string, never NULL          */
size_t      reflex_sizeof_alloc_params(void);   /* sizeof(reflex_alloc_params)        */
size_t      reflex_sizeof_moe_args(void);       /* sizeof(reflex_moe_args)            */

/* ---- workspace sizes ----------------------------------------------------------
 * Bytes of device scratch the entry points below need; 0 on invalid sizes.
 * reflex_workspace_size covers reflex_moe_forward and is also large enough for
 * reflex_permute and reflex_grouped_swiglu with pair_capacity = T * k_max. */
size_t reflex_workspace_size(int T, int E, int d, int f, int f_shared, int k_max);
size_t reflex_permute_workspace_size(int pair_capacity, int E);

/*
 * Where reflex_moe_forward (and _timed, _noalloc) leaves the routing of a forward in its
 * workspace, for inspection once the stream has completed (tests, debugging): byte
 * offset of `field` in a workspace sized by reflex_workspace_size with the same
 * arguments (k_max = the forward's pair-capacity count kcap).  The arrays are those of
 * reflex_topk_variable (pair_offsets [T+1], pair_expert and pair_weight [T * kcap]) and
 * reflex_permute (expert_offsets [E+1], sorted_token and pair_to_sorted [T * kcap]),
 * holding the forward's P selected expert-token pairs (Section 3.2).  The layout is
 * internal to this library version.  Returns (size_t)-1 for invalid sizes or field.
 */
#define REFLEX_WS_PAIR_OFFSETS    0
#define REFLEX_WS_PAIR_EXPERT     1
#define REFLEX_WS_PAIR_WEIGHT     2
#define REFLEX_WS_EXPERT_OFFSETS  3
#define REFLEX_WS_SORTED_TOKEN    4
#define REFLEX_WS_PAIR_TO_SORTED  5
size_t reflex_workspace_offset(int T, int E, int d, int f, int f_shared, int k_max, int field);
size_t reflex_swiglu_workspace_size(int pair_capacity, int E, int f);

/*
 * Router scores r_{i,e} = sum_k h[i,k] * w_router[e,k] (+ bias[e])  (Section 3.2).
 *  h        [T, d]  bf16   token representations
 *  w_router [E, d]  fp32   router weight (nn.Linear layout)
 *  bias     [E]     fp32   optional per-expert offset, NULL for none
 *  logits   [T, E]  fp32   output; products of the bf16 input and the fp32 weight
 *                          are accumulated in fp32 (max row error ~1e-6 relative)
 * Errors: NULL h/w_router/logits; T, d or E out of range (d % 128, 1 <= E <= 256).
 */
int reflex_router_logits(const uint16_t* h, const float* w_router, const float* bias,
                         float* logits, int T, int d, int E, void* stream);

/*
 * Per-token expert counts for one denoising forward (the allocator Pi of Eq. (3)).
 * For every sequence s (tokens seq_offsets[s] .. seq_offsets[s+1]-1, active block
 * active_block[s]):
 *   1. RRB prior k_i = H(|b(i) - a_s|)  (Eq. (5)); prompt tokens have b = 0.
 *   2. J = masked tokens of the active block (Section 3.1).  Tokens of J with
 *      hist_len >= 1 are ranked by the key `params->signal` selects, in fp64,
 *      descending, ties to the lower token index; the first floor(q*m) get
 *      K_cur + delta_cur, the last floor(q*m) get K_cur - delta_cur, the rest
 *      K_cur (Eq. (9)).  Tokens of J with no history keep K_cur.
 *      Forecast (Section 4.3): hist 2: v = c1 - c2 clipped to +-w_cf/2,
 *      c_hat = clip(c1 + v, 0, 1); hist 1: v = 0, c_hat = c1, P = 1.
 *   3. Every count is clamped to [k_min, k_max].
 *  block_idx   [T] int32   b(i) >= 0
 *  masked      [T] uint8   nonzero = position still [MASK]
 *  hist_len    [T] int8    number of confidence observations available (0..2)
 *  conf_prev1  [T] fp32    c^{t-1};  conf_prev2 [T] fp32  c^{t-2}
 *  seq_offsets [B+1] int32 token ranges, non-decreasing, 0 .. T
 *  active_block[B] int32   a_s >= 1
 *  params      host pointer
 *  k_out       [T] int32   output counts
 *  pairs_out   [1] int32   output sum_i k_i
 *  fps_out     [T] fp64    optional: the ranking key of every ranked token, NaN
 *                          for tokens that are not ranked; NULL to skip
 * Errors: NULL required pointers; T > 0 with B < 1; invalid params.
 */
int reflex_assign_budget(const int32_t* block_idx, const uint8_t* masked, const int8_t* hist_len,
                         const float* conf_prev1, const float* conf_prev2,
                         const int32_t* seq_offsets, const int32_t* active_block, int B, int T,
                         const reflex_alloc_params* params, int32_t* k_out, int32_t* pairs_out,
                         double* fps_out, void* stream);

/*
 * Decoding state after one denoising forward (Section 3.1, Eq. (1)), per sequence:
 * the masked positions of the active block whose confidence reaches theta are
 * committed (with min_commit = 1, a forward that would commit none commits the
 * most confident one, lowest position on ties); every position that was masked
 * records the forward's confidence (conf_prev2 <- conf_prev1, conf_prev1 <- conf_t,
 * hist_len <- min(hist_len + 1, 2)); a sequence whose active block has no masked
 * position left moves to its next block, if it has one.
 *  conf_t       [T] fp32  confidences of this forward (read at masked positions)
 *  block_idx    [T] int32, seq_offsets [B+1] int32   as in reflex_assign_budget
 *  theta        commitment threshold in (0, 1]
 *  masked, hist_len, conf_prev1, conf_prev2 [T], active_block [B]   updated in place
 *  remaining    [B] int32 output: masked positions left per sequence, or NULL
 * Errors: NULL required pointers; T > 0 with B < 1; theta outside (0, 1] or
 * min_commit not 0/1 (REFLEX_ERR_PARAM).
 */
int reflex_advance_state(const float* conf_t, const int32_t* block_idx, const int32_t* seq_offsets,
                         int B, int T, float theta, int min_commit, uint8_t* masked,
                         int8_t* hist_len, float* conf_prev1, float* conf_prev2,
                         int32_t* active_block, int32_t* remaining, void* stream);

/*
 * Counts derived from the router scores alone: the score-threshold rules the
 * paper compares against (Appendix B).  Routing mass is the softmax of a token's
 * scores over all E experts, evaluated in fp64.
 *  rule = REFLEX_RULE_TOP_P:     k_i = the smallest n such that the n best experts
 *                                (logit descending, index ascending) hold routing
 *                                mass >= threshold (summed in that order);
 *  rule = REFLEX_RULE_THRESHOLD: k_i = the number of experts with routing mass
 *                                > threshold;
 * then k_i = min(max(k_i, k_min), k_max).
 *  logits    [T, E] fp32
 *  threshold p in (0, 1] for Top-p; tau in [0, 1) for the threshold rule (a float,
 *            widened exactly to fp64)
 *  k_out     [T] int32 output counts
 *  pairs_out [1] int32 output sum_i k_i, or NULL
 * Errors: NULL logits / k_out; unknown rule or threshold out of range
 * (REFLEX_ERR_PARAM); k_min < 0, k_min > k_max or k_max > min(E, 32) (REFLEX_ERR_SHAPE).
 */
#define REFLEX_RULE_BUDGET     0   /* Refinement-Role Budgeting + FGER (Sections 4.2-4.3) */
#define REFLEX_RULE_TOP_P      1   /* Top-p over routing mass (Appendix B)                */
#define REFLEX_RULE_THRESHOLD  2   /* Expert-Threshold Routing (Appendix B)               */
int reflex_count_rule(const float* logits, int T, int E, int rule, float threshold, int k_min,
                      int k_max, int32_t* k_out, int32_t* pairs_out, void* stream);

/*
 * Variable-count TopK and routing weights (Section 3.2, Eq. (2)).
 * Token i keeps its min(max(k[i],0), k_max) best experts in the order (logit
 * descending, expert index ascending; -0.0 == +0.0).  Pairs are written
 * token-major, in rank order, at pair_offsets[i] ... pair_offsets[i+1]-1.
 *  logits       [T, E] fp32
 *  k            [T]    int32   counts (clamped as above)
 *  norm_topk    1: alpha = softmax over the selected experts (sums to 1);
 *               0: alpha = the full softmax probability over all E experts
 *  pair_offsets [T+1]  int32   output exclusive prefix sum of the counts
 *  pair_expert  [pair_capacity] int32  output expert of each pair
 *  pair_weight  [pair_capacity] fp32   output alpha of each pair
 *  pair_capacity must be >= T * k_max (REFLEX_ERR_WORKSPACE otherwise).
 * Errors: NULL pointers; k_max < 0 or > min(E, 32); norm_topk not 0/1.
 */
int reflex_topk_variable(const float* logits, const int32_t* k, int T, int E, int k_max,
                         int norm_topk, int32_t* pair_offsets, int32_t* pair_expert,
                         float* pair_weight, int32_t pair_capacity, void* stream);

/*
 * Group the selected expert-token pairs by expert.  The pairs are those of
 * Section 3.2: token i contributes one pair per selected expert, P = sum_i k_i in
 * all, and each pair is one row of the routed experts' work in Eq. (2).  A stable
 * counting sort of the token-major pair list by expert orders the rows by
 * (expert, token), so every expert's rows are contiguous for its GEMM.
 *  pair_offsets [T+1] int32, pair_expert [P] int32   from reflex_topk_variable
 *  pairs        [1]   int32  device P (clamped to pair_capacity)
 *  expert_offsets [E+1] int32  output: rows of expert e are
 *                              expert_offsets[e] .. expert_offsets[e+1]-1
 *  sorted_token [pair_capacity] int32  output: token of each expert-sorted row
 *  pair_to_sorted [pair_capacity] int32 output: expert-sorted row of each pair
 *  ws, ws_bytes  scratch of >= reflex_permute_workspace_size(pair_capacity, E)
 * Errors: NULL pointers; E out of range; workspace too small.
 */
int reflex_permute(const int32_t* pair_offsets, const int32_t* pair_expert, const int32_t* pairs,
                   int T, int E, int32_t pair_capacity, int32_t* expert_offsets,
                   int32_t* sorted_token, int32_t* pair_to_sorted, void* ws, size_t ws_bytes,
                   void* stream);

/*
 * SwiGLU experts on expert-sorted rows (the expert E_e of Eq. (2); two input and
 * one output projection as counted in Appendix A, Eq. (10)):
 *   for each row j of expert e, x = h[sorted_token[j]],
 *   y_sorted[j] = W_down[e] (SiLU(W_gate[e] x) * (W_up[e] x)).
 * Both projections run on bf16 MFMA with fp32 accumulation; the activation
 * SiLU(g)*u is rounded to bf16 once, y once.  SiLU may be taken as 0 for g below -87, where its
 * magnitude is less than 2^-119.
 *  h        [T, d] bf16;  w_gate, w_up [E, f, d] bf16;  w_down [E, d, f] bf16
 *  y_sorted [pair_capacity, d] bf16 output (rows >= expert_offsets[E] untouched)
 *  ws       scratch of >= reflex_swiglu_workspace_size(pair_capacity, E, f)
 * Errors: NULL pointers; d % 128 or f % 64 nonzero; workspace too small.
 */
int reflex_grouped_swiglu(const uint16_t* h, const int32_t* sorted_token,
                          const int32_t* expert_offsets, const uint16_t* w_gate,
                          const uint16_t* w_up, const uint16_t* w_down, int T, int E, int d,
                          int f, int32_t pair_capacity, uint16_t* y_sorted, void* ws,
                          size_t ws_bytes, void* stream);

/*
 * Weighted combine (Eq. (2)): out[i] = sum over the pairs j of token i, in rank
 * order, of pair_weight[j] * y_sorted[pair_to_sorted[j]], plus shared_y[i] when
 * given; accumulated in fp32 and rounded to bf16 once.
 *  y_sorted [pair_capacity, d] bf16; pair_offsets [T+1];
 *  pair_to_sorted, pair_weight [pair_capacity]  (pair indices and rows are clamped
 *                          to [0, pair_capacity) before use)
 *  shared_y [T, d] bf16 optional (always-on shared expert, weight 1)
 *  out      [T, d] bf16 output
 * Errors: NULL pointers; d % 128 nonzero; pair_capacity < 0.
 */
int reflex_combine(const uint16_t* y_sorted, const int32_t* pair_offsets,
                   const int32_t* pair_to_sorted, const float* pair_weight,
                   const uint16_t* shared_y, int T, int d, int32_t pair_capacity, uint16_t* out,
                   void* stream);

/*
 * The whole layer on one stream, no host synchronisation: router -> counts ->
 * TopK -> permutation -> SwiGLU experts -> combine (+ shared expert, + residuals).
 * Count source, first match wins:
 *   k_in != NULL   reuse counts computed earlier in the same forward (the paper
 *                  shares k_i across MoE layers, Section 3.3);
 *   uniform_k > 0  default fixed token-choice routing, k_i = uniform_k;
 *   k_rule = REFLEX_RULE_TOP_P / REFLEX_RULE_THRESHOLD
 *                  reflex_count_rule on this layer's scores with k_threshold and the
 *                  bounds params.k_min, params.k_max;
 *   otherwise      reflex_assign_budget with `params` and the token state.
 * Pair capacity is T * kcap with kcap = uniform_k if uniform_k > 0, else params.k_max;
 * counts (k_in included) are clamped to [0, kcap].  `params` is validated only when
 * uniform_k <= 0.
 */
typedef struct {
  int32_t T, d, E, f;
  int32_t f_shared;        /* width of the always-on shared expert, 0 = none           */
  int32_t norm_topk;       /* as in reflex_topk_variable                               */
  int32_t uniform_k;       /* > 0: fixed count for every token                         */
  int32_t B;               /* number of sequences (budget path)                         */
  int32_t k_rule;          /* REFLEX_RULE_*; 0 = the REFLEX budget                      */
  float   k_threshold;     /* p or tau of the score-derived rules                       */
  const uint16_t *h;                         /* [T, d]                                   */
  const uint16_t *w_gate, *w_up, *w_down;    /* [E, f, d], [E, f, d], [E, d, f]          */
  const uint16_t *ws_gate, *ws_up, *ws_down; /* shared [fs, d], [fs, d], [d, fs] or NULL  */
  const float    *w_router, *router_bias;    /* [E, d], [E] or NULL                      */
  const int32_t  *block_idx, *seq_offsets, *active_block;  /* budget path only           */
  const uint8_t  *masked;
  const int8_t   *hist_len;
  const float    *conf_prev1, *conf_prev2;
  const int32_t  *k_in;                      /* [T] or NULL                              */
  const uint16_t *residual_a, *residual_b;   /* [T, d] bf16 added before rounding, or NULL */
  reflex_alloc_params params;
  uint16_t *out;                             /* [T, d] bf16                              */
  int32_t  *k_out;                           /* [T] counts used, or NULL                 */
  int32_t  *pairs_out;                       /* [1] P, or NULL                           */
  float    *logits_out;                      /* [T, E] router scores (bias added), or NULL */
} reflex_moe_args;

/* ws: >= reflex_workspace_size(T, E, d, f, f_shared, kcap) bytes, 256-byte aligned. */
int reflex_moe_forward(const reflex_moe_args* args, void* ws, size_t ws_bytes, void* stream);

/*
 * reflex_moe_forward for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the same work
 * on the same kernels, with the workspace taken from a scratch array the library holds
 * on each device (REFLEX_NOALLOC_SCRATCH_BYTES, reserved when the library is loaded on
 * that device and held until the process ends).  The call allocates nothing: no
 * hipMalloc / hipFree, no stream or event creation (the shared expert runs on `stream`,
 * not on a side stream).  The caller still passes every input and output in `args`.
 * Layers whose reflex_workspace_size(T, E, d, f, f_shared, kcap) exceeds
 * REFLEX_NOALLOC_SCRATCH_BYTES are rejected with REFLEX_ERR_WORKSPACE before anything
 * is launched (96 MiB holds, e.g., one LLaDA-MoE-shaped layer of T = 1024 tokens,
 * d 2048, E 64, f 1024, k_max 12).  Every call on a device shares that device's scratch
 * and leaves its contents behind (nothing in it needs to start zeroed): calls whose
 * work overlaps on one device (other streams, other threads) race on it and must be
 * serialised by the caller.
 * Errors: as reflex_moe_forward; REFLEX_ERR_LAUNCH if the scratch cannot be located.
 */
#define REFLEX_NOALLOC_SCRATCH_BYTES (96u << 20)
int reflex_moe_forward_noalloc(const reflex_moe_args* args, void* stream);

/*
 * reflex_moe_forward with timing marks, for benchmarks: identical work, plus
 * hipEventRecord(stage_events[i], stream) at each stage boundary:
 *   0 start, 1 router done (mostly as partial sums over slices of d, which step 2's rule or
 *   step 3 adds with the bias; on the REFLEX budget path the same launch computes the
 *   counts), 2 counts done (rule / what is left of the above; uniform counts: step 3),
 *   3 count scan + TopK done (and the pair sort of small layers), 4 permutation done,
 *   5 gate/up GEMM done, 6 down GEMM done, 7 shared expert done (nothing is left to do
 *   there where its rows ride in the two GEMMs: f_shared = f and T * max(kcap, 1) <= 5 E),
 *   8 combine done.
 * stage_events: host array of REFLEX_N_STAGE_EVENTS hipEvent_t handles created by
 * the caller (hipEventCreate); the library only records them.
 * Errors: as reflex_moe_forward; NULL stage_events or a NULL entry;
 * n_stage_events != REFLEX_N_STAGE_EVENTS (REFLEX_ERR_SHAPE).
 */
#define REFLEX_N_STAGE_EVENTS 9
int reflex_moe_forward_timed(const reflex_moe_args* args, void* ws, size_t ws_bytes, void* stream,
                             void* const* stage_events, int n_stage_events);

/* ---- 8-bit products --------------------------------------------------------------
 * Matrices of 8-bit floating point numbers (e4m3: 3 fraction bits, largest 448, no
 * infinities, NaN 0x7f) with one scale for each block of 128 columns.  A block's scale
 * is a power of two, held as the byte e of 2^(e - 127): the smallest for which the
 * block's largest magnitude is at most 448 scales (1 .. 247; 127 for a block of
 * zeros).  A code is the number over its scale, rounded to nearest with ties to even.
 * A number that is not finite becomes NaN and takes no part in its block's scale.
 *
 *  rows     codes [M, K] row-major; every row has its own scale per 128 columns, the
 *           scale of columns 128 b .. of row i at [b / 4][i][b % 4] of a byte array
 *           [ceil(K / 512), M, 4] (reflex_fp8_scale_bytes(M, K) bytes);
 *  weights  codes [N, K] row-major; one scale per 128 x 128 block, that of rows 128 a ..
 *           and columns 128 b .. at [a][b] of a byte array [ceil(N / 128), 4 ceil(K / 512)]
 *           (reflex_fp8_weight_scale_bytes(N, K) bytes, experts one after the other).
 * Bytes for blocks past K are padding: the quantisers write 0, nothing reads them.
 * K is a multiple of 128 and at most REFLEX_MAX_DIM; M and N are any.  Codes must be
 * 16-byte aligned, scale arrays 4-byte aligned. */
#define REFLEX_FP8_BLOCK 128
size_t reflex_fp8_scale_bytes(int M, int K);           /* 0 on invalid sizes */
size_t reflex_fp8_weight_scale_bytes(int N, int K);

/* Element types of the operands that come in several. */
#define REFLEX_TYPE_BF16 0
#define REFLEX_TYPE_F32  1

/*
 * The masked positions (Section 3.1) as a list: rows[0 .. n-1] are the indices i with
 * masked[i] != 0, ascending, n_rows[0] = n.  A head that predicts only those rows reads
 * the list and the count on the device (reflex_quantize_fp8, reflex_matmul_fp8,
 * reflex_sample_tokens).
 *  masked [T] uint8;  rows [T] int32 output, entries from n on untouched;  n_rows [1]
 *  int32 output (0 for T = 0);  ws >= reflex_select_rows_workspace_size(T) bytes
 * Errors: NULL pointers; T out of range; workspace too small.
 */
size_t reflex_select_rows_workspace_size(int T);
int reflex_select_rows(const uint8_t* masked, int T, int32_t* rows, int32_t* n_rows, void* ws,
                       size_t ws_bytes, void* stream);

/*
 * bf16 rows to 8-bit rows.  Row j of the output is row rows[j] of x (rows NULL: row j);
 * rows from n_rows[0] on (n_rows NULL: M) are left as they were, a source row outside
 * [0, x_rows) gives a row of zeros.
 *  x [x_rows, K] bf16;  rows [M] int32 or NULL (then x_rows >= M);  n_rows [1] int32 on
 *  the device or NULL;  q [M, K] codes;  scale [ceil(K / 512), M, 4]
 * Errors: NULL pointers; sizes (REFLEX_ERR_SHAPE); rows NULL with x_rows < M.
 */
int reflex_quantize_fp8(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, int x_rows,
                        int M, int K, uint8_t* q, uint8_t* scale, void* stream);

/*
 * bf16 weights of E experts (1: a plain matrix) to 8-bit weights.
 *  w [E, N, K] bf16;  q [E, N, K] codes;  scale [E, ceil(N / 128), 4 ceil(K / 512)]
 * Errors: NULL pointers; sizes (REFLEX_ERR_SHAPE; E up to REFLEX_MAX_EXPERTS, less than 2^24
 *  blocks of 128 x 128).
 */
int reflex_quantize_fp8_weight(const uint16_t* w, int E, int N, int K, uint8_t* q, uint8_t* scale,
                               void* stream);

/*
 * out[i, n] = sum_k x[i, k] w[n, k] of 8-bit rows and weights, on the matrix cores.  Rows
 * from n_rows[0] on (n_rows NULL: M) are left as they were.
 *  REFLEX_TYPE_F32   the products are exact and summed in fp32: off by at most K 2^-23 of the
 *                    sum of the terms' magnitudes (numbers under the scale bytes 1 and 2 to within
 *                    2^-133 where a neighbouring row has numbers under 247)
 *  REFLEX_TYPE_BF16  by the 8-bit instruction, which adds 64 products at a time to an fp32 sum and
 *                    keeps some 17 bits below the largest of them: for every 64 columns off by
 *                    another 2^-11 of the largest |x| times the largest |w| among them at
 *                    most (1.4e-5 in the 2-norm of random rows); then rounded once
 *  x [M, K], x_scale;  w [N, K], w_scale;  out [M, N] dense (16-byte aligned)
 * Errors: NULL pointers; sizes (REFLEX_ERR_SHAPE); unknown out_type (REFLEX_ERR_PARAM).
 */
int reflex_matmul_fp8(const uint8_t* x, const uint8_t* x_scale, const uint8_t* w,
                      const uint8_t* w_scale, const int32_t* n_rows, int M, int N, int K,
                      int out_type, void* out, void* stream);

/*
 * reflex_grouped_swiglu on 8-bit rows and weights.  For row j of expert e, x the row
 * sorted_token[j] of h:  g = W_gate[e] x, u = W_up[e] x, SiLU(g) * u rounded to an 8-bit row
 * (as reflex_quantize_fp8 does, from fp32), y_sorted[j] = W_down[e] of it, rounded to bf16
 * once.  All three products are those of reflex_matmul_fp8 with bf16 results ahead of the
 * rounding (8-bit instruction, fp32 sums); SiLU is within (|g| + 4) 2^-22 of itself for g from
 * -87 on; below, where its magnitude is less than 2^-119, it may be taken as 0.  A value that an
 * error takes across a border between two codes has the other one, a step away, and a block's
 * largest across a border between two scales moves the block's.
 *  h [T, d], h_scale;  w_gate, w_up [E, f, d], w_down [E, d, f] with s_gate, s_up, s_down;
 *  sorted_token, expert_offsets, pair_capacity, y_sorted as in reflex_grouped_swiglu
 *  ws  scratch of >= reflex_swiglu_fp8_workspace_size(pair_capacity, E, f)
 * Errors: NULL pointers; d % 128 or f % 128 nonzero; workspace too small.
 */
size_t reflex_swiglu_fp8_workspace_size(int pair_capacity, int E, int f);
int reflex_grouped_swiglu_fp8(const uint8_t* h, const uint8_t* h_scale, const int32_t* sorted_token,
                              const int32_t* expert_offsets, const uint8_t* w_gate,
                              const uint8_t* w_up, const uint8_t* w_down, const uint8_t* s_gate,
                              const uint8_t* s_up, const uint8_t* s_down, int T, int E, int d,
                              int f, int32_t pair_capacity, uint16_t* y_sorted, void* ws,
                              size_t ws_bytes, void* stream);

/*
 * reflex_moe_forward with the routed and the shared experts in 8 bits: the router, the
 * counts, TopK and the combine as there (from the bf16 h), the experts as
 * reflex_grouped_swiglu_fp8 on h quantised by the call.  The expert weights of `args`
 * (w_gate .. ws_down) are not read and may be NULL.
 *  ws: >= reflex_workspace_fp8_size(T, E, d, f, f_shared, kcap) bytes, 256-byte aligned
 * Errors: as reflex_moe_forward; f or f_shared not a multiple of 128 (REFLEX_ERR_SHAPE).
 */
typedef struct {
  const uint8_t *w_gate, *w_up, *w_down;      /* codes [E, f, d], [E, f, d], [E, d, f]          */
  const uint8_t *s_gate, *s_up, *s_down;      /* their scales                                   */
  const uint8_t *ws_gate, *ws_up, *ws_down;   /* shared [fs, d], [fs, d], [d, fs] (f_shared > 0) */
  const uint8_t *ss_gate, *ss_up, *ss_down;
} reflex_fp8_experts;
size_t reflex_sizeof_fp8_experts(void);       /* sizeof(reflex_fp8_experts)                     */
size_t reflex_workspace_fp8_size(int T, int E, int d, int f, int f_shared, int k_max);
int reflex_moe_forward_fp8(const reflex_moe_args* args, const reflex_fp8_experts* experts, void* ws,
                           size_t ws_bytes, void* stream);

/* ---- 8-bit integer products ------------------------------------------------------------
 * Matrices of 8-bit integers (-127 .. 127) with one fp32 scale for each row: a token of the
 * input, an output channel of the weights.  a = the row's largest magnitude (2^-100 at least):
 * the scale is a / 127, a code the number times (127 / a), rounded to nearest with ties to even
 * (quotients and product rounded to fp32 first).  A row that holds a number which is not finite
 * has codes 0 and the scale NaN: whatever is computed from it is NaN, and nothing else is.
 *
 *  rows     codes [M, K] row-major, scale [M] fp32
 *  weights  codes [N, K] row-major, scale [N] fp32 (experts one after the other)
 * Codes of -128 are multiplied as such.  K is a multiple of 128 and at most REFLEX_MAX_DIM; M and
 * N are any.  Codes must be 16-byte aligned, scales 4-byte aligned.
 *
 * bf16 rows to 8-bit rows; x, rows, n_rows, x_rows as in reflex_quantize_fp8.
 *  q [M, K] codes;  scale [M]
 * Errors: NULL pointers; sizes (REFLEX_ERR_SHAPE); rows NULL with x_rows < M.
 */
int reflex_quantize_int8(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, int x_rows,
                         int M, int K, int8_t* q, float* scale, void* stream);

/*
 * bf16 weights of E experts (1: a plain matrix) to 8-bit weights.
 *  w [E, N, K] bf16;  q [E, N, K] codes;  scale [E, N]
 * Errors: NULL pointers; sizes (REFLEX_ERR_SHAPE; E up to REFLEX_MAX_EXPERTS, E N less than 2^31).
 */
int reflex_quantize_int8_weight(const uint16_t* w, int E, int N, int K, int8_t* q, float* scale,
                                void* stream);

/*
 * out[i, n] = (sum_k x[i, k] w[n, k]) (x_scale[i] w_scale[n]): the sum of the codes' products is
 * exact, on the matrix cores; it, the product of the scales and the result are rounded to fp32
 * (off by at most 3 2^-24 of itself while the scales' product is a normal fp32 number), for bf16
 * results then to bf16.  Rows from n_rows[0] on (n_rows NULL: M) are left as they were.
 *  x [M, K], x_scale [M];  w [N, K], w_scale [N];  out [M, N] dense (16-byte aligned), out_type
 *  REFLEX_TYPE_*
 * Errors: NULL pointers; sizes (REFLEX_ERR_SHAPE); unknown out_type (REFLEX_ERR_PARAM).
 */
int reflex_matmul_int8(const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale,
                       const int32_t* n_rows, int M, int N, int K, int out_type, void* out,
                       void* stream);

/*
 * reflex_grouped_swiglu on 8-bit integers.  For row j of expert e, x the row sorted_token[j] of
 * h:  g = W_gate[e] x and u = W_up[e] x as fp32 results of reflex_matmul_int8, SiLU(g) * u rounded
 * to bf16, that row rounded to 8 bits as reflex_quantize_int8 does, y_sorted[j] = W_down[e] of it
 * as a bf16 result of reflex_matmul_int8.  SiLU is within (|g| + 4) 2^-22 of itself for g from
 * -87 on; below, where its magnitude is less than 2^-119, it may be taken as 0.  A value that this
 * or a rounding takes across a border between two codes has the other one, a step away.
 *  h [T, d], h_scale [T];  w_gate, w_up [E, f, d], w_down [E, d, f] with s_gate, s_up [E, f],
 *  s_down [E, d];  sorted_token, expert_offsets, pair_capacity, y_sorted as in
 *  reflex_grouped_swiglu
 *  ws  scratch of >= reflex_swiglu_int8_workspace_size(pair_capacity, E, f)
 * Errors: NULL pointers; d % 128 or f % 128 nonzero; workspace too small.
 */
size_t reflex_swiglu_int8_workspace_size(int pair_capacity, int E, int f);
int reflex_grouped_swiglu_int8(const int8_t* h, const float* h_scale, const int32_t* sorted_token,
                               const int32_t* expert_offsets, const int8_t* w_gate,
                               const int8_t* w_up, const int8_t* w_down, const float* s_gate,
                               const float* s_up, const float* s_down, int T, int E, int d, int f,
                               int32_t pair_capacity, uint16_t* y_sorted, void* ws,
                               size_t ws_bytes, void* stream);

/* ---- between blocks --------------------------------------------------------------------
 * From a block's output and the residual stream to the next block's input.  For each row i:
 *   y_i = y[i], or from the experts' rows, sum over the pairs j of token i, in rank order, of
 *         pair_weight[j] y_sorted[pair_to_sorted[j]], plus shared_y[i] when given, in fp32;
 *         nothing where neither is given
 *   u_i = residual_scale x_i + gate_i (y_i r(y_i) w_post), rounded to stream_type: x_out[i]
 *   n_i = u_i r(u_i) w_pre, rounded to bf16: n_out[i]
 *   q_out[i], q_scale[i]: the row n_i in 8 bits, as reflex_quantize_int8 of n_out gives it
 * with r(v) = 1 / sqrt(mean of v^2 + eps).  x NULL: no first term; w_post NULL: y_i as it is;
 * gate NULL: 1; w_pre NULL: no n (then n_out and q_out are NULL).  Products from the left, each
 * operation rounded to fp32 (the experts' rows by fused multiply-adds); mean and root are taken in
 * fp64 and r rounded to fp32.
 *  x, x_out [T, d] of stream_type (REFLEX_TYPE_*);  y, shared_y, n_out [T, d] bf16;  w_post, w_pre
 *  [d] fp32;  y_sorted [pair_capacity, d] bf16 with pair_offsets [T+1], pair_to_sorted and
 *  pair_weight [pair_capacity] as in reflex_combine;  q_out [T, d], q_scale [T]
 *  gate      [gate_rows, d] bf16: one row (gate_rows 1), one a token (gate_rows T) or, with
 *            seq_offsets [gate_rows + 1], one for each sequence (rows past the last sequence have
 *            the last one's)
 *  n_rows    [1] int32 on the device or NULL: rows from n_rows[0] on are left as they were
 * x_out may be x and, of a bf16 stream, y or both at once (a row is read before it is written);
 * otherwise no output may share memory with an input or another output.
 * Errors: NULL args or a struct without x, y and y_sorted, without any output, or with some arrays
 *  of a group alone (pair arrays with y_sorted, q_scale with q_out; n_out or q_out without w_pre)
 *  (REFLEX_ERR_NULL); y together with y_sorted, w_post, gate or shared_y without an output of the
 *  block to apply to, unknown stream_type, eps not positive and finite, residual_scale not finite, reserved not 0
 *  (REFLEX_ERR_PARAM); sizes and alignment (REFLEX_ERR_SHAPE; all matrices and weights 16 bytes).
 */
typedef struct {
  int32_t T, d;
  int32_t stream_type;            /* REFLEX_TYPE_* of x and x_out                         */
  int32_t gate_rows;
  int32_t pair_capacity;
  float   eps;
  float   residual_scale;
  int32_t reserved;               /* 0                                                    */
  const void *x;
  const uint16_t *y;
  const uint16_t *y_sorted;
  const int32_t *pair_offsets, *pair_to_sorted;
  const float *pair_weight;
  const uint16_t *shared_y;
  const float *w_post, *w_pre;
  const uint16_t *gate;
  const int32_t *seq_offsets;
  const int32_t *n_rows;
  void *x_out;
  uint16_t *n_out;
  int8_t *q_out;
  float *q_scale;
} reflex_norm_args;
size_t reflex_sizeof_norm_args(void);         /* sizeof(reflex_norm_args)                       */
int reflex_block_norm(const reflex_norm_args* args, void* stream);

/*
 * reflex_moe_forward with the routed and the shared experts in 8-bit integers: the router, the
 * counts and TopK as there (from the bf16 h), the experts as reflex_grouped_swiglu_int8 on h_q and
 * h_scale, the 8-bit rows of h that a norm before left (both NULL: h quantised by the call).  The
 * expert weights of `args` (w_gate .. ws_down) are not read and may be NULL.
 *  join  NULL: the combine of reflex_moe_forward, to args->out.  Otherwise the experts' rows go on
 *        through reflex_block_norm(join), which gets them, the pairs and the shared expert's rows
 *        from the call (its y, y_sorted, pair arrays and shared_y must be NULL; T and d those of
 *        args; its outputs may be h, h_q and h_scale); args->out, residual_a and residual_b must be
 *        NULL then.
 *  ws: >= reflex_workspace_int8_size(T, E, d, f, f_shared, kcap) bytes, 256-byte aligned
 * Errors: as reflex_moe_forward and, for join, reflex_block_norm; f or f_shared not a multiple of
 *  128 (REFLEX_ERR_SHAPE); h_q without h_scale or the reverse (REFLEX_ERR_NULL); what must be NULL
 *  is not, or T or d of join differ (REFLEX_ERR_PARAM).
 */
typedef struct {
  const int8_t *w_gate, *w_up, *w_down;       /* codes [E, f, d], [E, f, d], [E, d, f]          */
  const float  *s_gate, *s_up, *s_down;       /* their scales [E, f], [E, f], [E, d]            */
  const int8_t *ws_gate, *ws_up, *ws_down;    /* shared [fs, d], [fs, d], [d, fs] (f_shared > 0) */
  const float  *ss_gate, *ss_up, *ss_down;
} reflex_int8_experts;
size_t reflex_sizeof_int8_experts(void);      /* sizeof(reflex_int8_experts)                    */
size_t reflex_workspace_int8_size(int T, int E, int d, int f, int f_shared, int k_max);
int reflex_moe_forward_int8(const reflex_moe_args* args, const reflex_int8_experts* experts,
                            const int8_t* h_q, const float* h_scale, const reflex_norm_args* join,
                            void* ws, size_t ws_bytes, void* stream);

/* ---- tokens and confidences ----------------------------------------------------------
 * The token a forward predicts at each position and its confidence c^t (Section 3.1), as
 * reflex_advance_state takes it, from rows of logits and given uniform numbers.
 * Row j of the logits is position i = rows[j] (rows NULL: i = j), j < n_rows[0] (n_rows
 * NULL: M); positions outside [0, T) are skipped, those of no row are left as they were.
 * Where a position is listed twice, tokens[i] and conf[i] are each of one of its rows, not
 * always of the same one.
 *   weight of token v:  w_v = exp((l_v - max l) / temperature), to within 1e-10 of itself in
 *     fp64 (below 2^-1020: 0)
 *   kept tokens, in the order (logit descending, index ascending, -0.0 == +0.0): the first
 *     top_k; of those the shortest prefix whose weights sum to at least top_p of theirs
 *     (in fixed point: to within 2^-30 of the row's weight; equal logits at the maximum
 *     exactly); of those the ones with w_v >= min_p.  The first token is always kept.
 *   tokens[i] = the first kept v by index for which the kept weights up to v sum to more
 *     than u[i] of the kept weights' sum; temperature 0: the first token of the order.
 *   conf[i] = the softmax of the row's logits (temperature 1, all tokens) at tokens[i], to within
 *     2^-17 of itself (fp32 powers; at temperature 1 2^-23).
 * A logit of -inf has weight 0 and so has NaN; where some are +inf they alone have
 * weight, the same each.  A row without any weight gives token -1, confidence 0.
 *  logits [M, V], logits_type REFLEX_TYPE_*;  u [T] fp32 in [0, 1) (others are clamped);
 *  tokens [T] int32, conf [T] fp32 outputs (conf NULL: skipped)
 *  ws >= reflex_sample_workspace_size(M, V) bytes (33 to 81 KB a row, for 2^16 rows at
 *    most)
 * params (host):  temperature >= 0 and finite; top_k >= 0 (0: all); 0 < top_p <= 1;
 *  0 <= min_p <= 1 (REFLEX_ERR_PARAM otherwise).
 * Errors: NULL pointers; sizes; unknown logits_type; workspace too small.
 */
typedef struct {
  float   temperature;
  int32_t top_k;
  float   top_p;
  float   min_p;
} reflex_sample_params;
#define REFLEX_MAX_VOCAB (1 << 20)     /* V <= this                                      */
size_t reflex_sizeof_sample_params(void);
size_t reflex_sample_workspace_size(int M, int V);
int reflex_sample_tokens(const void* logits, int logits_type, const int32_t* rows,
                         const int32_t* n_rows, int M, int V, const float* u,
                         const reflex_sample_params* params, int T, int32_t* tokens, float* conf,
                         void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* REFLEX_H */
