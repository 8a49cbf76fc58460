/*
 * libmot — Mixture-of-Translators KV-cache translation on AMD Instinct MI355X
 * (gfx950).  Plain C ABI: device pointers, host structs of sizes, status codes.
 *
 * Operation (paper Sec. 2.1 "Problem Setup", paragraphs "Translation" and
 * "Communication"; Sec. 3, Definition "Mixture-of-Translators", Eq.
 * mot_definition; translator activation phi = GELU, App. C.2):
 *
 *   A source model's context KV cache is translated into the target model's
 *   cache space.  A channel (i, j) connects source layer i to target layer j;
 *   layer_map[j] = i lists the channels (App. C.3 "Depth-Ratio Mapping" gives
 *   the default map, mot_depth_ratio_map below).  For every channel, for keys
 *   and for values separately, every context token row z (the source cache row
 *   of one token, flattened head-major: index h*D_src + d) is translated as
 *
 *       g      = softmax(Wr z + br)                   (E nonnegative gates)
 *       Tr_m z = W2_m GELU(W1_m z + b1_m) + b2_m     (m = 0..E-1)
 *       S      = the top_k largest g_m (ties: lower index), 1 <= top_k <= E
 *       out    = sum_{m in S} (g_m / sum_{r in S} g_r) Tr_m z
 *
 *   and written into target layer j, un-flattened as (h', d') =
 *   (o / D_tgt, o % D_tgt).  top_k = E is the dense mixture.  GELU is
 *   x * Phi(x) with the exact erf in MOT_F32; every MOT_BF16 kernel evaluates
 *   the tanh form of GELU (Hendrycks & Gimpel), whose largest deviation from
 *   the erf form is 4.7e-4 absolute (at |x| ~ 2.7), well below the bf16
 *   rounding of the hidden activation that follows it.
 *
 * Terms.  d_in = H_src*D_src, d_out = H_tgt*D_tgt, N_tok = B*T.  A "unit" is
 * one (target layer j, X in {K, V}) with layer_map[j] >= 0.
 */
#ifndef MOT_H
#define MOT_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MOT_ABI_VERSION 5
#define MOT_MAX_LAYERS 256   /* L_src, L_tgt <= MOT_MAX_LAYERS               */
#define MOT_MAX_EXPERTS 16   /* E <= MOT_MAX_EXPERTS                         */

typedef enum {
    MOT_OK = 0,
    MOT_ERR_NULL_ARG = 1,            /* a required pointer is NULL                */
    MOT_ERR_BAD_SHAPE = 2,           /* a size is <= 0, too large, or inconsistent */
    MOT_ERR_BAD_LAYER_MAP = 3,       /* layer_map[j] >= L_src or < -1             */
    MOT_ERR_UNSUPPORTED = 4,         /* valid but not implemented (see below)     */
    MOT_ERR_MISALIGNED = 5,          /* a device pointer is not 16-byte aligned   */
    MOT_ERR_WORKSPACE_TOO_SMALL = 6, /* caller workspace below the minimum        */
    MOT_ERR_HIP = 7                  /* a HIP runtime call or launch failed       */
} mot_status;

typedef enum { MOT_F32 = 0, MOT_BF16 = 1 } mot_dtype;
typedef enum { MOT_LAYOUT_BTHD = 0, MOT_LAYOUT_BHTD = 1 } mot_layout;
typedef enum { MOT_ACT_GELU = 0, MOT_ACT_IDENTITY = 1 } mot_act;
typedef enum { MOT_ALGO_AUTO = 0, MOT_ALGO_UNFUSED = 1, MOT_ALGO_FUSED = 2, MOT_ALGO_ROUTED = 3 } mot_algo;

/*
 * Problem sizes and options (host struct, read during the call only).
 *   L_src, L_tgt   source / target layer counts (1..MOT_MAX_LAYERS)
 *   B, T           batch and context tokens (B*T >= 0; 0 is a no-op)
 *   H_src, D_src   source KV heads and head dim
 *   H_tgt, D_tgt   target KV heads and head dim
 *   E              translators per unit (1..MOT_MAX_EXPERTS)
 *   top_k          translators used per token, 1..E: the top_k largest softmax
 *                  scores are kept and renormalised to sum to one, the others
 *                  are zero (ties go to the lower translator index); top_k = E
 *                  is the dense mixture.  MOT_ALGO_ROUTED runs each translator
 *                  only on the tokens that selected it; MOT_ALGO_FUSED and
 *                  MOT_ALGO_UNFUSED evaluate every translator and give the
 *                  unselected ones a gate of exactly zero.
 *   hidden         translator hidden width
 *   dtype          MOT_F32: fp32 storage and math (erf GELU, expf softmax).
 *                  Where hidden % 64 == 0 and d_in % 16 == 0 the products are
 *                  formed on the bf16 matrix cores from exact three-way splits
 *                  of their operands, to 2^-33 of a product, and summed in fp32;
 *                  results for which parts of operands or products leave bf16's
 *                  or fp32's range (infinities, NaN, values near the least or
 *                  the largest ones) are computed on the fp32 matrix cores.
 *                  MOT_BF16: bf16 storage; fp32 accumulation; fp32 gates;
 *                  tanh-form GELU (within 4.7e-4 absolute of the erf form);
 *                  the gate-scaled hidden activation is rounded to bf16
 *                  before the second translator layer; outputs rounded to
 *                  nearest even.
 *   src_layout     layout of each source layer: BTHD [B][T][H][D] or BHTD
 *   dst_layout     layout of each target layer, same encoding
 *   act            MOT_ACT_GELU (the method) or MOT_ACT_IDENTITY (tests)
 *   algo           kernel path: MOT_ALGO_AUTO picks (bf16: ROUTED when
 *                  top_k < E, else FUSED when the fused kernel fits, else
 *                  UNFUSED; fp32: UNFUSED); MOT_ALGO_FUSED = one kernel per
 *                  token tile over every translator (bf16 only; d_in and d_out
 *                  in {128, 256, 512}; no workspace); MOT_ALGO_ROUTED = Top-K
 *                  sparse (bf16 only): a router pass writes each token's top_k
 *                  translators, a per-unit counting sort groups the (token,
 *                  translator) pairs by translator, each translator runs only
 *                  on its tokens (the fused kernel over translator tiles where
 *                  it fits, else the two GEMMs over translator tiles of up to
 *                  256 pairs), and for top_k > 1 a combine sums each token's
 *                  top_k rows (workspace needed); MOT_ALGO_UNFUSED = router,
 *                  then two grouped GEMMs over every translator through a
 *                  hidden-activation workspace (the fp32 GEMMs on the matrix
 *                  cores, see dtype, compute the router in the first one's
 *                  launch).  Requesting an impossible path
 *                  returns MOT_ERR_UNSUPPORTED.  All paths compute the same
 *                  function.
 *   streams        2 (or 0): keys and values, each with its own translators;
 *                  1: one activation stream per layer (the MoT-h variant,
 *                  paper App. C.5): src_k -> dst_k with translators indexed
 *                  [L_tgt][1][E]...; src_v and dst_v are ignored (may be
 *                  NULL).  mot_restore_kv then forms K and V from it.
 *   workspace      optional device scratch; NULL = library-owned buffer
 *   workspace_bytes size of `workspace` in bytes
 *   usage          optional device uint32 [L_tgt][streams][E], 4-byte aligned:
 *                  translator usage (paper Sec. 4, "MoT Architecture
 *                  Ablation": I_m, the cumulative selection count of
 *                  translator m).  For every mapped unit (j, x) and every
 *                  context token, usage[j][x][m] is incremented once for each
 *                  translator m of the token's Top-K set, so each call adds
 *                  top_k * B * T to a unit's row (B * T per translator when
 *                  top_k = E).  Counts accumulate over calls (zero the array
 *                  to start; they wrap at 2^32); rows of unmapped layers are
 *                  not touched; NULL = not counted.  mot_usage_stats turns
 *                  the counts into the paper's usage imbalance and entropy.
 *
 * Supported sizes (others return MOT_ERR_UNSUPPORTED):
 *   MOT_BF16: D_src, D_tgt multiples of 8; d_in multiple of 64;
 *             hidden multiple of 64; d_out multiple of 32.
 *   MOT_F32:  D_src, D_tgt multiples of 4; d_in, hidden multiples of 4.
 */
typedef struct {
    int32_t L_src, L_tgt;
    int32_t B, T;
    int32_t H_src, D_src;
    int32_t H_tgt, D_tgt;
    int32_t E, top_k, hidden;
    int32_t dtype, src_layout, dst_layout, act, algo;
    int32_t streams;
    void* workspace;
    size_t workspace_bytes;
    uint32_t* usage;
} mot_shapes;

/*
 * Translator weights: host struct of device pointers, element type = dtype,
 * nn.Linear layout ([out][in]); index 1 of every array is 0 = keys, 1 = values.
 *   w1 [L_tgt][2][E][hidden][d_in]     b1 [L_tgt][2][E][hidden]   (may be NULL)
 *   w2 [L_tgt][2][E][d_out][hidden]    b2 [L_tgt][2][E][d_out]    (may be NULL)
 * Weights are indexed by TARGET layer: two target layers that read the same
 * source layer still have their own translators.
 */
typedef struct {
    const void* w1;
    const void* b1;
    const void* w2;
    const void* b2;
} mot_translator_weights;

/* Router (gate) weights, element type = dtype:
 *   w [L_tgt][2][E][d_in]    b [L_tgt][2][E] (may be NULL)                   */
typedef struct {
    const void* w;
    const void* b;
} mot_router_weights;

/*
 * mot_translate — translate the source context cache into the target layout.
 *
 *   src_k, src_v  device, [L_src] x (src_layout) of dtype
 *   layer_map     HOST int32[L_tgt]; layer_map[j] in [0, L_src) reads that
 *                 source layer, -1 leaves target layer j untouched
 *   tw, rw        translator / router weights (above)
 *   dst_k, dst_v  device, [L_tgt] x (dst_layout) of dtype; only mapped layers
 *                 are written
 *   shapes        sizes and options (above)
 *   stream        HIP stream the work is enqueued on (0 = default stream)
 *
 * B*T == 0 is a valid no-op that inspects no pointer.
 *
 * Asynchronous with respect to the host; results are ready when `stream`
 * reaches this point.  All argument checks run before anything is enqueued:
 * on any error nothing is launched and the outputs are untouched.  Device
 * pointers must be 16-byte aligned; dst must not overlap src, weights or the
 * workspace.  With workspace == NULL the library uses a per-device buffer it
 * owns (grown with hipMalloc on first need, kept until process exit); calls
 * that overlap in time on different streams of one device must then pass
 * their own workspaces.  No call retains any pointer after it returns.
 */
mot_status mot_translate(const void* src_k, const void* src_v, const int32_t* layer_map,
                         const mot_translator_weights* tw, const mot_router_weights* rw,
                         void* dst_k, void* dst_v, const mot_shapes* shapes,
                         hipStream_t stream);

/*
 * Workspace bytes mot_translate needs for `shapes` (its dtype, sizes and
 * options; the workspace fields are ignored).  0 when the chosen kernels need
 * none.  A smaller caller workspace that is still >= the per-unit minimum is
 * accepted and processed in smaller unit groups.  Returns SIZE_MAX when the
 * shapes are invalid or unsupported (mot_last_error() says why).
 */
size_t mot_workspace_bytes(const mot_shapes* shapes);

/*
 * mot_translate with optional scratch for the fused dense path, whose own need
 * is zero.  A launch whose token tiles do not fill whole rounds of the chip (a
 * short context above all) then cuts its last tiles along the expert-hidden
 * axis over several workgroups each, which leave fp32 partial rows in
 * `scratch` that a second kernel sums.  Same results up to the order of those
 * fp32 sums: which tiles are cut depends on the whole call, so a token's row may
 * differ in its last bit from its row in a call with other tokens (mot_translate's
 * fused path gives it the same bits in both).  scratch: device memory used by this call only (calls that overlap
 * in time need their own).  With at least mot_translate_scratch_bytes (and those
 * not 0) it must be 16-byte aligned (else MOT_ERR_MISALIGNED) and those bytes must
 * not overlap a cache, the weights, the router or usage (else MOT_ERR_BAD_SHAPE).
 * With fewer, or NULL, or where mot_translate_scratch_bytes is 0 (as on every other
 * path), the call is exactly mot_translate and scratch is not looked at.
 */
mot_status mot_translate_scratch(const void* src_k, const void* src_v, const int32_t* layer_map,
                                 const mot_translator_weights* tw, const mot_router_weights* rw,
                                 void* dst_k, void* dst_v, const mot_shapes* shapes, void* scratch,
                                 size_t scratch_bytes, hipStream_t stream);

/*
 * Scratch bytes with which mot_translate_scratch splits a call of these shapes
 * over layer_map (host int32[L_tgt]); 0 when it would not (the tiles fill the
 * chip, another path, or a splitting that would not pay) or when an argument
 * is invalid.
 */
size_t mot_translate_scratch_bytes(const mot_shapes* shapes, const int32_t* layer_map);

/*
 * Depth-ratio channel map (paper App. C.3, "Depth-Ratio Mapping"): target
 * layer j reads source layer floor(j * L_src / L_tgt), in exact integer
 * arithmetic.  out: host int32[L_tgt].
 */
mot_status mot_depth_ratio_map(int32_t L_src, int32_t L_tgt, int32_t* out);

/*
 * Translator usage statistics (paper Sec. 4, "MoT Architecture Ablation",
 * Table "mot_analysis") of n rows of selection counts I[n][E] (as written
 * by mot_translate's usage output; device uint32):
 *     cv2[r]     = Var_m(I[r][m]) / Mean_m(I[r][m])^2   (population variance
 *                  over the E translators: the usage imbalance CV^2)
 *     entropy[r] = -sum_m p_m ln p_m,  p_m = I[r][m] / sum_m I[r][m]
 *                  (natural log, 0 ln 0 = 0: the usage entropy)
 * in double precision; both are NaN for a row of zeros.  cv2 and entropy:
 * device double [n], 8-byte aligned, not overlapping the counts.  1 <= E <=
 * MOT_MAX_EXPERTS; n = 0 is a no-op.  Asynchronous on `stream`; every check
 * runs before the launch.
 */
mot_status mot_usage_stats(const uint32_t* counts, int32_t n, int32_t E, double* cv2, double* entropy,
                           hipStream_t stream);

/* Static text for a status code. */
const char* mot_status_string(mot_status status);

/* Detail of the last error raised on the calling thread ("" if none). */
const char* mot_last_error(void);

/*
 * Key/value restoration for the activation-translation variant MoT-h (paper
 * App. C.5): the target's key and value projections applied to a translated
 * intermediate activation a (as written by mot_translate with streams = 1):
 *     K[l][t] = W^K[l] a[l][t] + b^K[l],    V[l][t] = W^V[l] a[l][t] + b^V[l]
 * for every layer l with layer_map[l] >= 0 (NULL: every layer).
 *
 *   act        device bf16 [L][B][T][d_act]
 *   wk, wv     device bf16 [L][d_kv][d_act], d_kv = H_tgt * D_tgt (nn.Linear layout)
 *   bk, bv     device bf16 [L][d_kv] or NULL (zero)
 *   dst_k/v    device bf16 [L] x dst_layout ([B][T][H_tgt][D_tgt] or [B][H_tgt][T][D_tgt])
 *   layer_map  HOST int32[L] or NULL; layers with a negative entry are not written
 * Requires dtype MOT_BF16, d_act a multiple of 64, D_tgt a multiple of 8
 * (MOT_ERR_UNSUPPORTED otherwise).  Same error discipline as mot_translate:
 * every check runs before anything is enqueued.
 */
typedef struct {
    int32_t L, B, T;
    int32_t d_act;
    int32_t H_tgt, D_tgt;
    int32_t dtype, dst_layout;
} mot_restore_shapes;

mot_status mot_restore_kv(const void* act, const int32_t* layer_map, const void* wk, const void* bk,
                          const void* wv, const void* bv, void* dst_k, void* dst_v,
                          const mot_restore_shapes* shapes, hipStream_t stream);

/*
 * Context replay after translation (paper App. C.4, "Post-Translation Phase:
 * Cache Replay", Top-S source-guided sparse attention).  Query position u of
 * a target layer attends only to the S context positions that the source
 * model attended to most at the guiding source layer (head-averaged map A),
 * or, in the bottom L_Full layers, to every position 0..u.
 *
 *   B, T       batch rows, context tokens
 *   H_q, H_kv  target query heads and KV heads (H_q a multiple of H_kv; query
 *              head h reads KV head h / (H_q / H_kv), at most 16 per KV head;
 *              H_kv * D below 2^20)
 *   D          head dim: 64 or 128
 *   S          Top-S budget: a multiple of 32, 32 .. 256 (at most 192 when
 *              D = 128); the paper uses 128
 *   kv_layout  K and V in MOT_LAYOUT_BTHD ([B][T][H_kv][D]) or MOT_LAYOUT_BHTD
 *   workspace, workspace_bytes
 *              optional device scratch of mot_replay_attention without key
 *              sets (16-byte aligned, at least mot_replay_workspace_bytes);
 *              NULL = the library's per-device buffer (see below)
 */
typedef struct {
    int32_t B, T;
    int32_t H_q, H_kv, D;
    int32_t S;
    int32_t kv_layout;
    void* workspace;
    size_t workspace_bytes;
} mot_replay_shapes;

/*
 * mot_replay_attention for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same operation, arguments and checks, but the full causal
 * path (idx = NULL) stages V in a static 32 MiB array that the library holds
 * on each device it runs on until the process ends, instead of a workspace
 * or a library-allocated buffer; it calls no hipMalloc, hipFree or
 * allocating routine.  shapes->workspace and workspace_bytes are ignored.
 * Shapes whose staged V (mot_replay_workspace_bytes) exceeds 32 MiB return
 * MOT_ERR_WORKSPACE_TOO_SMALL before anything is launched.  All calls on one
 * device share that array (its contents after a call are unspecified): calls
 * that overlap in time on one device race.  With key sets (idx != NULL) no
 * scratch is used.
 */
mot_status mot_replay_attention_noalloc(const void* q, const void* k, const void* v, const int32_t* idx, void* o,
                                        const mot_replay_shapes* shapes, hipStream_t stream);

/* Scratch bytes mot_replay_attention needs for `shapes` with idx = NULL (V
 * staged transposed: B * H_kv * D * T rounded up to 64, bf16); 0 with key
 * sets; SIZE_MAX for invalid or unsupported shapes. */
size_t mot_replay_workspace_bytes(const mot_replay_shapes* shapes, int with_sets);

/*
 * Top-S key sets (App. C.4, N(u) = Top-S of A[u, 1:u]): for every b and u,
 * the S positions v <= u with the largest A[b][u][v] (ties: lower v), written
 * in ascending order to idx[b][u][0..S) and padded with -1 (all of 0..u when
 * u < S).  A: device fp32 [B][T][T] head-averaged source attention (entries
 * v > u have no influence; up to three of them, inside the row, may be read);
 * idx: device int32 [B][T][S].  Only B, T and S of `shapes` are used (T at most
 * 65536).  Both pointers 4-byte aligned and non-overlapping.
 */
mot_status mot_topS_select(const float* A, int32_t* idx, const mot_replay_shapes* shapes, hipStream_t stream);

/*
 * Replay attention of one target layer: for every b, u and query head h,
 *     o[b][u][h] = sum_{v in N(u)} softmax_v(q[b][u][h] . k[v] / sqrt(D)) v[v]
 * with N(u) = the entries of idx[b][u] that lie in 0..u (others, such as the
 * -1 padding, are skipped; a set with none gives zeros), or the full causal
 * set 0..u when idx is NULL.  q, o: device bf16 [B][T][H_q][D]; k, v: device
 * bf16 in kv_layout; idx: device int32 [B][T][S] or NULL.  Softmax and
 * accumulation in fp32; o rounded to bf16.  All pointers 16-byte aligned; o
 * must not overlap an input.  With idx NULL the call stages V transposed
 * (mot_replay_workspace_bytes) in shapes->workspace, or, when that is NULL,
 * in the per-device buffer that mot_translate uses without a workspace (so
 * such calls and those of mot_translate or mot_backbone_translate without
 * workspaces that overlap in time on one device race; calls with their own
 * workspaces do not).  A workspace below the need returns
 * MOT_ERR_WORKSPACE_TOO_SMALL; it must not overlap q, k, v or o.  With idx
 * NULL, (T + 64) * row stride * 2 bytes must stay under 2^31 (row stride:
 * H_kv * D in BTHD, D in BHTD), else MOT_ERR_UNSUPPORTED.
 */
mot_status mot_replay_attention(const void* q, const void* k, const void* v, const int32_t* idx, void* o,
                                const mot_replay_shapes* shapes, hipStream_t stream);

/*
 * The backbone translator body (paper App. C.2, "Backbone Translator") as the
 * experts of the mixture, over channel windows of N = dims->n_slots slots (0
 * or 1: one slot per unit).  Window w covers target layers wN .. wN+N-1 (so
 * L_tgt must be a multiple of N); its slot r reads source layer
 * layer_map[wN + r], and a window is either fully mapped or fully -1
 * (skipped).  Keys and values are translated separately; one unit is a
 * (window, K or V).  For each batch row, over the context positions t,
 * expert m computes
 *     z_r = GELU(W_in LN_in(x_r[t]) + b_in)                     r = 1..N (d_h)
 *     h_0 = z_1;  for r = 1..N (block CAB_r, its own parameters):
 *       h~  = h_{r-1} + Wo CausalMHA(Wq LN_Q(h_{r-1}) + bq, Wk LN_C(z_r) + bk,
 *                                    Wv LN_C(z_r) + bv) + bo
 *       h_r = h~ + W_f2 GELU(W_f1 LN_F(h~) + b_f1) + b_f2
 *     y_t = GELU(W_out LN_out(Concat(h_1..h_N)) + b_out)          (N d_out)
 * (n_heads heads of width d_h / n_heads, softmax(q.k / sqrt(width)) over the
 * positions s <= t of the same batch row; LN with population variance,
 * eps 1e-5); the output row is sum_m g~_m y_t^(m) with Top-K gates from a
 * router over the window's concatenated source rows, and its slice
 * [r d_out, (r+1) d_out) is written to target layer wN + r.  One translator
 * stage (one scan) per expert.
 *
 *   params   device bf16 [L_tgt/N][2][E][P], P = mot_backbone_param_count():
 *            per expert, in order: ln_in_g[d_in] ln_in_b[d_in] w_in[d_h][d_in]
 *            b_in[d_h]; then for each slot r = 1..N: ln_q_g[d_h] ln_q_b[d_h]
 *            ln_c_g[d_h] ln_c_b[d_h] wq[d_h][d_h] bq[d_h] wk[d_h][d_h] bk[d_h]
 *            wv[d_h][d_h] bv[d_h] wo[d_h][d_h] bo[d_h] ln_f_g[d_h] ln_f_b[d_h]
 *            w_f1[d_ff][d_h] b_f1[d_ff] w_f2[d_h][d_ff] b_f2[d_h]; then
 *            ln_out_g[N d_h] ln_out_b[N d_h] w_out[N d_out][N d_h]
 *            b_out[N d_out]
 *   router   w [L_tgt/N][2][E][N d_in], b [L_tgt/N][2][E] (bias optional);
 *            with N = 1 the layout of mot_translate's router
 *   shapes   as for mot_translate (including the optional usage counts of
 *            the Top-K selections, here [L_tgt/N][2][E]: one row per
 *            window and K/V); dtype MOT_BF16, both layouts
 *            MOT_LAYOUT_BTHD, streams 2; hidden, act and algo are not used.
 *            workspace: device scratch of at least
 *            mot_backbone_workspace_bytes (16-byte aligned, not overlapping
 *            any other argument), or NULL for the per-device buffer that
 *            mot_translate uses without a workspace (calls of either that
 *            overlap in time on one device then race)
 * Requires d_in and d_h multiples of 64 up to 4096, N d_h up to 4096, d_ff a
 * multiple of 64, D_tgt a multiple of 8, head width d_h / n_heads of 64 or
 * 128, N <= 8, (T + 64) d_h 2 < 2^31 (MOT_ERR_UNSUPPORTED / MOT_ERR_BAD_SHAPE
 * otherwise; a window mixing mapped and unmapped slots is
 * MOT_ERR_BAD_LAYER_MAP).  Every check runs before any enqueue.
 */
typedef struct {
    int32_t d_h;       /* translator width                               */
    int32_t n_heads;   /* attention heads                                */
    int32_t d_ff;      /* feed-forward width                             */
    int32_t n_slots;   /* channel-window slots N (0 or 1: one per unit)  */
} mot_backbone_dims;

/* Elements per expert of the packed parameters (0 for invalid arguments). */
size_t mot_backbone_param_count(const mot_shapes* shapes, const mot_backbone_dims* dims);

/* Scratch bytes mot_backbone_translate needs (the router's gates for every
 * unit, one unit's activations and the attention's staged V); SIZE_MAX for
 * invalid or unsupported arguments. */
size_t mot_backbone_workspace_bytes(const mot_shapes* shapes, const mot_backbone_dims* dims);

mot_status mot_backbone_translate(const void* src_k, const void* src_v, const int32_t* layer_map,
                                  const void* params, const mot_router_weights* router, void* dst_k, void* dst_v,
                                  const mot_shapes* shapes, const mot_backbone_dims* dims, hipStream_t stream);

/*
 * The paged cache: where the target model goes on from its translated context.
 * A layer's keys and values lie in pools of pages of page_size positions; a
 * row of the page table names the pages of a sequence in order, so sequences
 * of different lengths share a pool, grow by a page at a time and share the
 * pages of a common prefix.
 *
 *   k_pages, v_pages  device, dtype: [L][n_pages] x [page_size][H_kv][D]
 *                (page_layout MOT_LAYOUT_BTHD) or [H_kv][page_size][D] (BHTD)
 *   table        device int32 [B][max_pages]: entry j of row b is the page
 *                of positions j * page_size .. + page_size - 1 of sequence b.
 *                An entry outside 0 .. n_pages - 1 (-1, say) is a hole: its
 *                positions are neither read nor written
 *   kv_len       device int32 [B]: positions of each sequence, the new tokens
 *                of the call among them (cut to 0 .. max_pages * page_size)
 *   new_start    device int32 [B + 1] or NULL: the new tokens of sequence b
 *                are the rows new_start[b] .. new_start[b + 1] - 1 of the
 *                call's row tensors (cut to 0 .. n_new).  They ascend; where
 *                they do not, what the outputs' new rows hold is unspecified.
 *                NULL: every sequence has max_new of them, at batch row b
 *
 * New token i of the c of sequence b is at position kv_len[b] - c + i.  Rows
 * of no sequence are left as they are, and so are, of a sequence with more
 * than max_new new tokens, those from the max_new-th on.  A call takes at most
 * 2^26 - 32 new tokens.
 *
 *   L            layers of the pools (1..MOT_MAX_LAYERS)
 *   n_pages      pages of a layer's pool
 *   page_size    positions per page: a power of two, 16 .. 1024
 *   H_kv, D      KV heads and head dim
 *   B, max_pages rows and entries per row of the table (max_pages * page_size
 *                at most 2^30, B at most 65535)
 *   dtype        MOT_F32 or MOT_BF16
 *   page_layout  MOT_LAYOUT_BTHD or MOT_LAYOUT_BHTD, see above
 * A page of a layer is under 2 GiB.
 */
typedef struct {
    int32_t L, n_pages, page_size;
    int32_t H_kv, D;
    int32_t B, max_pages;
    int32_t dtype, page_layout;
} mot_cache_shapes;

/* Elements from one layer, batch row, token and head of a row tensor to the
 * next; a head's D elements are contiguous.  With new_start the tokens of all
 * sequences are in one axis and `batch` is not used.  Multiples of 8 (bf16)
 * or 4 (fp32), not negative; the rows of an output share no element. */
typedef struct {
    int64_t layer, batch, token, head;
} mot_strides;

/*
 * Attention of new tokens over the paged cache of one layer (L = 1; pass the
 * layer's pools): for the new token at position u of sequence b and query
 * head h, which reads KV head h / (H_q / H_kv),
 *     o = sum_{v in N} softmax_v(scale q . k[v]) v[v]
 *     N = { 0 <= v <= u, v > u - window (when window > 0), v in no hole }
 * and zeros where N is empty.  One new token per sequence is a decoding step,
 * many are a chunk of a prompt over what is already cached.  Softmax and
 * accumulation in fp32, o rounded once to dtype.  The second product takes the
 * probabilities of MOT_BF16 as two bf16 terms (16 bits) where a sequence's rows
 * are few: max_new H_q / H_kv at most 32, or n_new H_q / H_kv at most 32 B;
 * elsewhere rounded to bf16, as replay attention does.
 * Positions from kv_len on and holes are not looked at, whatever they hold;
 * a NaN or infinite value reaches the tokens that see it and no others.  A row
 * that sees positions, all with the score -inf, is NaN.
 *
 *   q, o         device, dtype: rows of the new tokens, strides below (head
 *                pitch and all); o must not overlap q, the pools or the tables
 *   n_new        rows of q and o over all sequences (B * max_new without
 *                new_start)
 *   max_new      most new tokens of a sequence (packed: n_new will do, a close
 *                bound is a little faster)
 *   H_q          query heads, a multiple of H_kv
 *   window       0: every position up to u; else that many, u among them
 *   max_kv       0, or a bound on kv_len that is better than max_pages *
 *                page_size (a hint for how work is cut; longer sequences are
 *                still attended in full)
 *   scale        0: 1 / sqrt(D); positive, scale log2(e) finite in fp32
 *   q, o strides of q and o (layer not used)
 *   workspace, workspace_bytes
 *                optional device scratch of this call (16-byte aligned, not
 *                overlapping its arrays; calls that overlap in time need their
 *                own).  With at least mot_attend_workspace_bytes, and those not
 *                0, long sequences are cut along their positions over several
 *                workgroups, whose partial sums a second kernel joins in a
 *                fixed order; with less, or NULL, no sequence is cut (same
 *                results up to the order of fp32 sums)
 * D is 64 or 128 (else MOT_ERR_UNSUPPORTED, as are more tiles of query rows
 * than a launch holds: from 2^28 rows of a sequence in fp32).  n_new = 0 and
 * B = 0 are no-ops.
 * No allocation, no synchronisation; can be captured into a graph.
 */
typedef struct {
    int32_t n_new, max_new;
    int32_t H_q;
    int32_t window;
    int32_t max_kv;
    float scale;
    mot_strides q, o;
    void* workspace;
    size_t workspace_bytes;
} mot_attend_shapes;

mot_status mot_paged_attention(const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                               const int32_t* kv_len, const int32_t* new_start, void* o,
                               const mot_cache_shapes* cache, const mot_attend_shapes* shapes, hipStream_t stream);

/* Scratch bytes with which mot_paged_attention cuts calls of these shapes
 * (0: it would not); SIZE_MAX for invalid or unsupported shapes.  Does not go
 * by any data. */
size_t mot_attend_workspace_bytes(const mot_cache_shapes* cache, const mot_attend_shapes* shapes);

/*
 * New tokens into the paged cache, in one pass over q, k and v: for every new
 * token and layer l
 *     x' = gain x / sqrt(mean_d x_d^2 + eps)      (queries with q_gain, keys
 *                                                  with k_gain, where given)
 *     each pair (x'_i, x'_j) turned by the angle position * inv_freq[r]
 *     q_out = queries,  key and value -> the token's place in its page
 * Pair r of the first rotary_dim elements is (r, r + rotary_dim / 2), or
 * (2 r, 2 r + 1) when interleaved; the others stay.  Norms, angles and turns
 * are computed in fp32 (angles in fp64 until they are reduced to one turn) and
 * rounded once; values are copied.  A token at a negative position or in a
 * hole is not stored; its query is written all the same.
 * Without norms and rotation the call stores a translated cache (all layers
 * at once) into pages.  Tokens of one call must not share a place: a page in
 * which several rows grow is made several by mot_cache_reorder first.
 *
 *   q, q_out     device or NULL (both): [L] rows of H_q heads; q_out may be q
 *                (same strides), else it must not overlap q, k or v
 *   k, v         device or NULL (both): [L] rows of H_kv heads
 *   rope         NULL, or the arrays of
 *     q_gain, k_gain  device, dtype [L][D], or NULL: no norm
 *     inv_freq        device float [rotary_dim / 2] or NULL: no rotation
 *     positions       device int32 [n_new] (packed, or [B][max_new]) or NULL:
 *                     the position each row is turned by, where it is not the
 *                     position of its place
 *   H_q          query heads (not used without q)
 *   rotary_dim   a multiple of 16, at most D (0: D)
 *   eps          >= 0
 * D is a multiple of 16 up to 256.  Same error discipline as mot_translate.
 */
typedef struct {
    const void* q_gain;
    const void* k_gain;
    const float* inv_freq;
    const int32_t* positions;
} mot_rope;

typedef struct {
    int32_t n_new, max_new;
    int32_t H_q;
    int32_t rotary_dim, interleaved;
    float eps;
    mot_strides q, q_out, k, v;
} mot_append_shapes;

mot_status mot_cache_append(const void* q, const void* k, const void* v, void* q_out, void* k_pages, void* v_pages,
                            const int32_t* table, const int32_t* kv_len, const int32_t* new_start,
                            const mot_rope* rope, const mot_cache_shapes* cache, const mot_append_shapes* shapes,
                            hipStream_t stream);

/*
 * The next table of the sequences, made from the present one: forking,
 * copying, cutting back, freeing and growing, for every row at once.  New row
 * b (of n_rows) takes the first keep[b] positions of row source[b] and has
 * room for want[b]:
 *   - pages that the kept positions fill are shared with every other new row
 *     that keeps them;
 *   - a last page that they fill in part stays with the lowest row that keeps
 *     it, unless some row keeps it whole.  The others get a page of their own
 *     with a copy of the kept positions, in every layer's keys and values;
 *   - want[b] beyond that is met with pages of unspecified content.
 * New pages are the lowest-numbered ones that no new row takes over, given out
 * in the order of rows and of positions within a row; all other pages are
 * free: a page is in use when the table names it, nothing else is kept.
 *
 *   table        device int32 [B][max_pages], read
 *   source       device int32 [n_rows]; outside 0 .. B - 1: an empty row, which
 *                keeps nothing (keep is not looked at) but still gets room for
 *                want: a new prompt's pages
 *   keep, want   device int32 [n_rows], cut to 0 .. max_pages * page_size;
 *                want below keep means keep.  keep is at most what the source
 *                row holds; holes among the kept pages stay holes
 *   new_table    device int32 [n_rows][max_pages], written whole (-1 past the
 *                pages of a row); not overlapping any other array
 *   missing      device int32 [1]: pages that could not be had (their entries
 *                are holes); 0 when the pool sufficed
 *   workspace    device scratch of this call, at least mot_cache_workspace_bytes
 *                (16-byte aligned, not overlapping its arrays; calls that
 *                overlap in time need their own); not looked at where that is 0
 * Beam search sets source to the parents and want = keep + 1; a row that ends
 * (a finished beam or sequence) has source -1 and want 0, else it would take
 * want's pages anew.  n_rows at most 4096 (0: a no-op that writes nothing).  The
 * data of pages that new rows take over does not move.
 */
mot_status mot_cache_reorder(void* k_pages, void* v_pages, const int32_t* table, const int32_t* source,
                             const int32_t* keep, const int32_t* want, int32_t* new_table, int32_t* missing,
                             const mot_cache_shapes* cache, int32_t n_rows, void* workspace, size_t workspace_bytes,
                             hipStream_t stream);

/*
 * The pages in use (those that the table names) moved together to the lowest
 * numbers, in every layer: with n of them, those numbered n and up go to the
 * free pages under n, the lowest to the lowest.  new_table: the table with the
 * new numbers (holes -1), not overlapping any other array; used: device int32
 * [1], n.  The pool can then be cut to its first n pages.  Moved pages keep
 * their old content too.  workspace as for mot_cache_reorder.  B = 0 is a no-op
 * that writes nothing.
 */
mot_status mot_cache_compact(void* k_pages, void* v_pages, const int32_t* table, int32_t* new_table, int32_t* used,
                             const mot_cache_shapes* cache, void* workspace, size_t workspace_bytes,
                             hipStream_t stream);

/* Scratch bytes of mot_cache_reorder for n_rows new rows (n_rows 0: of
 * mot_cache_compact); 0 for small pools and tables; SIZE_MAX for invalid
 * shapes. */
size_t mot_cache_workspace_bytes(const mot_cache_shapes* cache, int32_t n_rows);

/* MOT_ABI_VERSION of the loaded library. */
int mot_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* MOT_H */
