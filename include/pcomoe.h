/*
 * pcomoe.h -- C ABI of the path-compositional MoE layer (PCoMoE, arXiv 2609.01024)
 * on AMD Instinct MI355X (gfx950).
 *
 * One layer, per token h with router logits l (Section 2, vanilla MoE; Section 4):
 *   1. route          top-k experts e_0..e_{k-1} of l (logit descending, ties to the lower
 *                     id) and weights p_a = softmax over the k selected logits.
 *   2. build paths    Pi(h) = {(a, b) : m[e_a][e_b] = 1 or a == b} over the token's slots,
 *                     with the diagonal of the compatibility mask forced to 1 (Section 4.2,
 *                     m_ii = 1; Section 4.3, fallback to vanilla); path weights beta_ab;
 *                     the grouped dispatch layout (rows sorted by expert, then token).
 *   3. expand         U_(t,a) = SiLU(W_gate[e_a] x_t) * (W_up[e_a] x_t), once per
 *                     (token, source) pair (Section 4.1 U_e; Section 4.3 source-grouped reuse).
 *   4. project and    y_t = sum_{(a,b) in Pi} beta_ab W_down[e_b] U_(t,a)  (Section 4.1 path
 *      combine        aggregation, Section 4.3 source-grouped form), computed as
 *                     y_t = sum_b W_down[e_b] z_(t,b) with z_(t,b) = sum_a beta_ab U_(t,a),
 *                     which is the same sum because W_down is linear (Section 4.1 D_e).
 *
 * Conventions for every call:
 *   - Pointers named as device pointers must be device memory of the current HIP device,
 *     16-byte aligned; arrays are dense and row-major. The caller owns every buffer; the
 *     library never allocates or frees memory and holds no mutable global state (except
 *     pcm_project_combine_noalloc's per-GPU scratch array and its looked-up addresses).
 *   - `stream` is a hipStream_t (NULL = the default stream). Work is enqueued and the call
 *     returns without synchronising. Device-side faults surface at the caller's next sync.
 *   - Arguments are validated on the host before anything is enqueued. On error nothing
 *     is enqueued and outputs are untouched. T = 0 is a successful no-op.
 *   - Limits: 1 <= k <= min(n, 8); n <= 256; H and F multiples of 64; T*k < 2^31.
 *   - Logits must be finite. Index arrays passed back in (topk_ids, the pcm_paths layout)
 *     must be what the library produced; other values give undefined results, but every
 *     gathered index is clamped, so memory outside the buffers is never touched.
 */
#ifndef PCOMOE_H
#define PCOMOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum pcm_status {
    PCM_OK = 0,
    PCM_ERR_ARG = 1,          /* null pointer, misaligned pointer, negative size, k > n ... */
    PCM_ERR_UNSUPPORTED = 2,  /* outside the limits above */
    PCM_ERR_WORKSPACE = 3,    /* ws_bytes smaller than pcm_workspace_bytes(...) */
    PCM_ERR_HIP = 4           /* a launch failed (hipGetLastError) */
} pcm_status;

typedef enum pcm_dtype {
    PCM_F32 = 0,   /* x and weights float32; FMA on the vector ALUs */
    PCM_BF16 = 1,  /* x and weights bfloat16; float32 accumulate throughout. The expansion
                      runs on bf16 MFMA and keeps u in float32; the projection input z is
                      carried as row-scaled float16 (11 significant bits) and the bf16
                      projection weights are widened to float16 in registers, so the
                      projection runs on f16 MFMA. Precondition on the projection weights
                      (w_down, and the shared expert's): |w| <= 65504, float16's largest value
                      (larger values become inf). Values with |w| >= 2^-17 widen exactly (a
                      bfloat16 there has at most 8 significant bits, all of which float16's
                      normal and upper subnormal range keep); smaller values round to the nearest
                      multiple of 2^-24 (float16's subnormal spacing; absolute error <= 2^-25),
                      so that magnitudes of 2^-25 or less become 0 */
    PCM_BF16_F16DOWN = 2  /* a PCM_BF16 layer whose projection weights (w_down, and the shared
                      expert's w_down) are passed as float16, widened once from the bf16
                      weights by pcm_widen_f16: the projection then uses them as read instead
                      of widening every fragment it loads, with bit-identical results. Every
                      other operand is as for PCM_BF16; calls that take no projection weights
                      treat this value as PCM_BF16. */
} pcm_dtype;

/* Path weights beta_ab for (a, b) in Pi (p = the renormalised router weights).
 * The paper names beta without a formula; the default is the reading under which a
 * diagonal-only mask reproduces the vanilla layer exactly (beta_aa = p_a, as Section 4.1
 * requires) and an all-pairs mask gives the product p_a p_b:
 *   SRC_COND: beta_ab = p_a p_b / sum_{b' : (a,b') in Pi} p_b'   (sum over Pi is 1)
 *   PRODUCT:  beta_ab = p_a p_b
 *   GLOBAL:   beta_ab = p_a p_b / sum_{(a',b') in Pi} p_a' p_b'                       */
typedef enum pcm_beta_mode {
    PCM_BETA_SRC_COND = 0,
    PCM_BETA_PRODUCT = 1,
    PCM_BETA_GLOBAL = 2
} pcm_beta_mode;

typedef enum pcm_op {
    PCM_OP_BUILD_PATHS = 0,
    PCM_OP_EXPAND = 1,
    PCM_OP_PROJECT_COMBINE = 2,
    PCM_OP_DENSE_SWIGLU = 3,
    PCM_OP_ROUTE_SCORED = 4,
    PCM_OP_LAYER_PER_PATH = 5,
    PCM_OP_ROUTE_LOGITS = 6,
    PCM_OP_ROUTE_PATHS = 7,
    PCM_OP_GROUPED_DX = 8,
    PCM_OP_GROUPED_DW = 9,
    PCM_OP_GRAD_NORM = 10
} pcm_op;

/* Path table and grouped dispatch layout of T tokens (caller-owned device buffers).
 * A "row" is one (token, slot) pair; rows are ordered by (expert ascending, token
 * ascending), so the rows of expert e are [expert_offsets[e], expert_offsets[e+1]). */
typedef struct pcm_paths {
    uint64_t* path_bits;       /* [T]      bit a*k+b set iff (a, b) in Pi(token)            */
    float* beta;               /* [T,k,k]  beta[t][a][b]; exactly 0 where the bit is clear   */
    int32_t* expert_offsets;   /* [n+1]    first row of each expert; [n] = T*k              */
    int32_t* row_token;        /* [T*k]    token of each row                                 */
    int32_t* row_slot;         /* [T*k]    slot a of each row                                */
    int32_t* row_of;           /* [T*k]    row of pair (t, a) at index t*k + a               */
} pcm_paths;

/* Route (Section 2's top-k selection; Section 4.3's fused indexing starts here).
 * logits [T,n] f32 (device). Outputs (device): topk_ids [T,k] i32, experts of slots
 * 0..k-1 by logit descending with ties to the lower id (signed zeros are equal);
 * topk_w [T,k] f32, softmax over the k selected logits. */
pcm_status pcm_route(const float* logits, int64_t T, int n, int k, int32_t* topk_ids,
                     float* topk_w, void* stream);

/* The router's own GEMM fused with the routing above: logits[t, e] = x_t . W_r[e]
 * (the scores the router computes from the hidden state, Section 2), float32 accumulation
 * (bf16: products on the matrix cores), then pcm_route's top-k and softmax on those float32
 * values. x [T,H] and w_router [n,H] of `dtype` (device); logits [T,n] f32 is written when
 * not NULL; topk_ids / topk_w as pcm_route. H must be a multiple of 64. The bf16 path splits
 * K into slices whose partial sums are added in a fixed order (deterministic).
 * ws: pcm_workspace_bytes(PCM_OP_ROUTE_LOGITS, T, H, 0, n, k, dtype) bytes. */
pcm_status pcm_route_logits(pcm_dtype dtype, const void* x, const void* w_router, int64_t T,
                            int H, int n, int k, float* logits, int32_t* topk_ids, float* topk_w,
                            void* ws, size_t ws_bytes, void* stream);

/* Build the path table and dispatch layout (Section 4.2's mask with m_ii = 1, applied
 * before any weighting; Section 4.3's source-grouped dispatch metadata).
 * topk_ids/topk_w [T,k] from pcm_route; mask [n,n] u8 (device), row = expansion source
 * expert i, column = projection target expert j, nonzero = allowed; its diagonal is
 * ignored (treated as 1). Fills every array of *out (the struct itself is host memory).
 * Deterministic: integer outputs are bit-identical from run to run.
 * ws: device workspace of pcm_workspace_bytes(PCM_OP_BUILD_PATHS, T, 0, 0, n, k, 0). */
pcm_status pcm_build_paths(const int32_t* topk_ids, const float* topk_w, const uint8_t* mask,
                           int64_t T, int n, int k, pcm_beta_mode beta_mode,
                           const pcm_paths* out, void* ws, size_t ws_bytes, void* stream);

/* Offline per-layer layout of the compatibility mask for pcm_route_paths (Section 4.3's
 * indexing reads a mask fixed per layer, Section 4.2 with m_ii = 1). mask [n,n] u8 (device),
 * as pcm_build_paths; packed [n, ceil(n/64)] u64 (device, caller-owned): bit j % 64 of word
 * [i][j / 64] is set iff mask[i][j] != 0 or i == j; bits at j >= n are 0. One launch. */
pcm_status pcm_mask_pack(const uint8_t* mask, int n, uint64_t* packed, void* stream);

/* Section 4.3's fused indexing operation: pcm_route's top-k and softmax, pcm_build_paths's
 * path bits and beta, and the grouped dispatch layout, from the logits and a packed mask.
 * One launch when T <= 64 (one token per wavefront; the last workgroup to finish builds the
 * dispatch layout); otherwise a launch that routes, forms the path table and counts rows
 * per (32-token block, expert), then one that places the rows. Outputs are
 * bit-identical to pcm_route followed by pcm_build_paths with the mask that packed_mask
 * was packed from, and deterministic. logits [T,n] f32 (device); packed_mask from
 * pcm_mask_pack; topk_ids [T,k] i32 and topk_w [T,k] f32 (device) as pcm_route; *out as
 * pcm_build_paths (all of its arrays written). Limits and errors as pcm_build_paths.
 * ws: pcm_workspace_bytes(PCM_OP_ROUTE_PATHS, T, 0, 0, n, k, 0) bytes (device, 16-byte
 * aligned; 256 when T <= 64). Its first 256 bytes hold a completion counter of the
 * single-launch case: they must be zero before the first call that uses this workspace,
 * and every call leaves them zero (the rest needs no initialisation). Calls that overlap
 * in time must not share a workspace. */
pcm_status pcm_route_paths(const float* logits, const uint64_t* packed_mask, int64_t T, int n,
                           int k, pcm_beta_mode beta_mode, int32_t* topk_ids, float* topk_w,
                           const pcm_paths* out, void* ws, size_t ws_bytes, void* stream);

/* Expansion side, once per (token, source) row (Section 4.1 U_e; Section 4.3 reuse):
 * u[r,:] = SiLU(x[row_token[r]] W_gate[e]^T) * (x[row_token[r]] W_up[e]^T) for the rows r
 * of expert e. x [T,H] and w_gate/w_up [n,F,H] of `dtype`; u [T*k,F] float32 (device).
 * bf16: MFMA products accumulate in float32; SiLU and the product are float32 and u is
 * stored unrounded. ws: pcm_workspace_bytes(PCM_OP_EXPAND, ...) bytes (0; may be NULL). */
pcm_status pcm_expand(pcm_dtype dtype, const void* x, const void* w_gate, const void* w_up,
                      const pcm_paths* paths, int64_t T, int H, int F, int n, int k, void* u,
                      void* ws, size_t ws_bytes, void* stream);

/* Projection side and combine (Section 4.1 D_e and path aggregation; Section 4.3):
 * z_(t,b) = sum_{a : (a,b) in Pi} beta_ab u_(t,a)   (float32),
 * o_(t,b) = W_down[e_b] z_(t,b)                     (float32 accumulate),
 * y_t = [y_t if accumulate] + sum_{b ascending} o_(t,b).
 * For bf16 layers each z row is multiplied by a power of two that puts its largest
 * element just below 2^14 and stored as float16; the down GEMM multiplies its output row
 * by the inverse (exact), so any activation magnitude stays inside float16's range.
 * u [T*k,F] f32 from pcm_expand, w_down [n,H,F] of `dtype`, y [T,H] f32 (device).
 * ws: pcm_workspace_bytes(PCM_OP_PROJECT_COMBINE, ...) bytes (holds z and o). */
pcm_status pcm_project_combine(pcm_dtype dtype, const void* u, const void* w_down,
                               const pcm_paths* paths, int64_t T, int H, int F, int n, int k,
                               float* y, int accumulate, void* ws, size_t ws_bytes,
                               void* stream);

/* pcm_project_combine for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops such as a decode step, harnesses that forbid allocation): the
 * same computation, kernels and result, with z, its scales and o kept in a scratch array
 * inside the library instead of a caller workspace. It allocates nothing. The array holds
 * PCM_NOALLOC_SCRATCH_BYTES (16 MiB) per GPU, is reserved on every GPU the library runs on
 * until the process ends, and its address on a device is looked up on the first call made
 * with that device current. Sizes whose workspace
 * (pcm_workspace_bytes(PCM_OP_PROJECT_COMBINE, T, H, F, n, k, dtype)) exceeds the array give
 * PCM_ERR_UNSUPPORTED (a decode-shaped layer, T = 32, H = 7168, F = 2048, k = 8, needs
 * 8.0 MiB). All calls on one GPU share its array and each leaves its intermediates there:
 * calls that overlap on one GPU (other streams, other host threads) race and must be
 * serialised by the caller. Arguments as pcm_project_combine. */
#define PCM_NOALLOC_SCRATCH_BYTES (16u << 20)
pcm_status pcm_project_combine_noalloc(pcm_dtype dtype, const void* u, const void* w_down,
                                      const pcm_paths* paths, int64_t T, int H, int F, int n,
                                      int k, float* y, int accumulate, void* stream);

/* A dense SwiGLU FFN applied to every token with weight 1 (Section 2's expert F_e), for an
 * always-on shared expert that sits beside the routed experts and outside the path
 * space: y_t = [y_t if accumulate] + W_down (SiLU(W_gate x_t) * (W_up x_t)).
 * The SwiGLU output is kept in float32 and, for bf16 layers, enters the down projection
 * as row-scaled float16 like pcm_project_combine's z.
 * x [T,H], w_gate/w_up [Fs,H], w_down [H,Fs] of `dtype`; y [T,H] f32 (device).
 * ws: pcm_workspace_bytes(PCM_OP_DENSE_SWIGLU, T, H, Fs, 1, 1, dtype) bytes. */
pcm_status pcm_dense_swiglu(pcm_dtype dtype, const void* x, const void* w_gate,
                            const void* w_up, const void* w_down, int64_t T, int H, int Fs,
                            float* y, int accumulate, void* ws, size_t ws_bytes, void* stream);

/* Residual connection around the layer in a stack of layers (each MoE layer's output is
 * added to the hidden state it read): h = h + y elementwise, rounded to h's dtype (bf16:
 * round to nearest even). h [T,H] of `dtype`, y [T,H] f32 (device); H a multiple of 64. */
pcm_status pcm_residual_add(pcm_dtype dtype, void* h, const float* y, int64_t T, int H,
                            void* stream);

/* Offline weight layout for PCM_BF16_F16DOWN (projection weights are fixed per layer, like the
 * packed mask of pcm_mask_pack): w_f16[i] = w_bf16[i] rounded to float16, to nearest even,
 * exactly as the projection kernels widen each bf16 weight fragment for PCM_BF16 (so the
 * PCM_BF16 precondition on w_down applies). w_bf16 and w_f16 are device arrays of `count`
 * 16-bit values (count >= 0; 16-byte aligned; they must not overlap). One launch. */
pcm_status pcm_widen_f16(const void* w_bf16, int64_t count, void* w_f16, void* stream);

/* Per-path execution of the layer, a baseline for the target-mixed projection above: the
 * path-level aggregation of Section 4.1 evaluated one projection per path, as in Section
 * 4.3's source-grouped form, with no mixing of paths that share a target:
 *   reuse = 1: U_(t,a) once per (token, source) (Section 4.3's reuse);
 *   reuse = 0: U recomputed for every path (no reuse at all);
 *   o_(t,a,b) = W_down[e_b] U_(t,a) for every (a, b) in Pi,
 *   y_t = [y_t if accumulate] + sum_{(a,b) in Pi, a-major} beta_ab o_(t,a,b).
 * Same inputs, path table and result (to rounding) as pcm_expand + pcm_project_combine; bf16
 * layers project row-scaled float16 U rows. Sized for at most T*k*k paths.
 * ws: pcm_workspace_bytes(PCM_OP_LAYER_PER_PATH, T, H, F, n, k, dtype) bytes. */
pcm_status pcm_layer_per_path(pcm_dtype dtype, const void* x, const void* w_gate,
                              const void* w_up, const void* w_down, const pcm_paths* paths,
                              int64_t T, int H, int F, int n, int k, int reuse, float* y,
                              int accumulate, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------- scored routing
 * The router the paper runs at inference (Section 4.2's compatibility-aware path score
 * and Section 4.3's TopK over the active path set):
 *   s_ij = g_base_i + b_ij + lambda g_tgt_j over A = {(i, j) : m_ij = 1}, m_ii = 1;
 *   Pi = the K best paths (ties to the lower i*n + j), beta = softmax of their scores;
 *   S = the distinct sources, each expanded once; T_i = the targets of source i;
 *   y = sum_{i in S} sum_{j in T_i} beta_ij D_j(U_i(h)).
 * The score is formed in float32 as fmaf(lambda, g_tgt_j, g_base_i + b_ij). K <= min(n, 8). */

/* Active pairs of one layer, materialised once (Section 4.3's offline path layout).
 * Caller-owned device buffers: count [1] i32; pair [n*n] u32 ((i << 16) | j of each active
 * pair in ascending i*n + j); bias [n*n] f32 (b_ij of each active pair). */
typedef struct pcm_path_layout {
    int32_t* count;
    uint32_t* pair;
    float* bias;
} pcm_path_layout;

/* Selected paths, groups and the two dispatch layouts of T tokens (caller-owned device
 * buffers). Source slots a < n_src[t] index the token's distinct sources and target slots
 * b < n_tgt[t] its distinct targets, both in ascending expert order. Expansion rows
 * (one per (token, source)) and projection rows (one per (token, target)) are each
 * ordered by (expert ascending, token ascending); at most T*K of each are used. */
typedef struct pcm_scored_paths {
    int32_t* sel_pair;         /* [T,K]    i*n + j of each selected path, selection order     */
    float* sel_score;          /* [T,K]    its score                                           */
    int32_t* n_src;            /* [T]      distinct sources                                    */
    int32_t* src_expert;       /* [T,K]    ascending; -1 from n_src on                         */
    int32_t* n_tgt;            /* [T]      distinct targets                                    */
    int32_t* tgt_expert;       /* [T,K]    ascending; -1 from n_tgt on                         */
    uint64_t* path_bits;       /* [T]      bit a*K+b: path src_expert[a] -> tgt_expert[b]      */
    float* beta;               /* [T,K,K]  weight of path (a, b); 0 where the bit is clear     */
    int32_t* src_offsets;      /* [n+1]    expansion rows of each expert                       */
    int32_t* src_row_token;    /* [T*K]    token of each expansion row                         */
    int32_t* src_row_slot;     /* [T*K]    source slot of each expansion row                   */
    int32_t* src_row_of;       /* [T*K]    expansion row of (t, a); -1 from n_src on           */
    int32_t* tgt_offsets;      /* [n+1]    projection rows of each expert                      */
    int32_t* tgt_row_token;    /* [T*K]                                                         */
    int32_t* tgt_row_slot;     /* [T*K]                                                         */
    int32_t* tgt_row_of;       /* [T*K]    projection row of (t, b); -1 from n_tgt on          */
} pcm_scored_paths;

/* Build the active-pair layout of a layer from mask [n,n] u8 (row = source i, column =
 * target j; the diagonal is treated as 1) and the compatibility bias [n,n] f32 (device). */
pcm_status pcm_path_layout_build(const uint8_t* mask, const float* bias, int n,
                                 const pcm_path_layout* out, void* stream);

/* Route T tokens over the layer's active pairs: selection, source / target groups,
 * weights and both dispatch layouts in one call (Section 4.3's fused indexing).
 * g_base, g_tgt [T,n] f32 (device); lambda finite. Deterministic.
 * ws: pcm_workspace_bytes(PCM_OP_ROUTE_SCORED, T, 0, 0, n, K, 0) bytes. */
pcm_status pcm_route_scored(const float* g_base, const float* g_tgt, float lambda,
                            const pcm_path_layout* layout, int64_t T, int n, int K,
                            const pcm_scored_paths* out, void* ws, size_t ws_bytes, void* stream);

/* pcm_expand over the expansion rows of scored routing: one row per (token, distinct
 * source). u [T*K,F] f32; rows from src_offsets[n] on are not written. */
pcm_status pcm_expand_scored(pcm_dtype dtype, const void* x, const void* w_gate,
                             const void* w_up, const pcm_scored_paths* paths, int64_t T, int H,
                             int F, int n, int K, void* u, void* ws, size_t ws_bytes,
                             void* stream);

/* pcm_project_combine for scored routing: z_(t,b) = sum_{a : (a,b) in Pi} beta_ab u_(t,a)
 * over the token's source and target slots, o_(t,b) = W_down[tgt_expert[b]] z_(t,b),
 * y_t = [y_t] + sum_{b ascending} o_(t,b); the same float16 projection input as
 * pcm_project_combine. ws: pcm_workspace_bytes(PCM_OP_PROJECT_COMBINE, T, H, F, n, K,
 * dtype) bytes. */
pcm_status pcm_project_combine_scored(pcm_dtype dtype, const void* u, const void* w_down,
                                      const pcm_scored_paths* paths, int64_t T, int H, int F,
                                      int n, int K, float* y, int accumulate, void* ws,
                                      size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------- experts' products on their own
 * The matrix products of the layer without what is fused around them, with their gradients, and in
 * 8-bit floating point: for training, and for experts whose weights are held in 8 bits.
 *
 * Rows and groups are those of the path tables: row r belongs to group e where
 * offsets[e] <= r < offsets[e+1] (offsets [n+1] i32, ascending from offsets[0] >= 0; empty groups are
 * allowed), and comes from row s(r) = row_token[r] of x, or r where row_token is NULL (then T = R).
 * offsets = NULL: one group (n = 1) of all R rows, row_token NULL: a plain product. R counts the rows of
 * the row buffers: rows from offsets[n] on are neither read nor written. Offsets are held inside [0, R]
 * and gathered indices inside [0, T), so no value of theirs reaches outside the buffers.
 * Limits: K and N multiples of 16, at most 2^31 - 128; n <= 256; R and T below 2^30. Sums are float32. Deterministic. */

/* y[r, :] = x[s(r), :] W[e]^T for the rows r of group e. x [T,K] and w [n,N,K] of `dtype` (PCM_F32 or
 * PCM_BF16), y [R,N] of out_dtype: PCM_F32, or for bf16 operands also PCM_BF16 (each float32 sum rounded
 * once, to nearest even). */
pcm_status pcm_grouped_gemm(pcm_dtype dtype, pcm_dtype out_dtype, const void* x, const void* w,
                            const int32_t* offsets, const int32_t* row_token, int64_t T, int64_t R,
                            int K, int N, int n, void* y, void* stream);

/* Gradient by x of pcm_grouped_gemm. dy [R,N] and w [n,N,K] of `dtype`. row_of = NULL: dx [R,K],
 * dx[r, :] = dy[r, :] W[e] (T = R, k = 1). row_of [T,k] i32 (the rows that read each row of x, as in
 * pcm_paths; a number outside [offsets[0], offsets[n]), or [0, R) without offsets: none): dx [T,K], the
 * sum of those rows' gradients, slots ascending, in float32, rounded once; every row of dx is written.
 * k is at most 8 and R at most T*k.
 * ws: pcm_workspace_bytes(PCM_OP_GROUPED_DX, T, K, 0, n, k, dtype) bytes where row_of is given. */
pcm_status pcm_grouped_gemm_dx(pcm_dtype dtype, pcm_dtype out_dtype, const void* dy, const void* w,
                               const int32_t* offsets, const int32_t* row_of, int64_t T, int k,
                               int64_t R, int K, int N, int n, void* dx, void* ws, size_t ws_bytes,
                               void* stream);

/* Gradient by w of pcm_grouped_gemm: dw[e] = [dw[e] +] sum over the rows r of group e of
 * dy[r, :]^T x[s(r), :]. x [T,K], dy [R,N] of `dtype`, dw [n,N,K] of out_dtype. accumulate adds into dw
 * (PCM_F32 only: a sum over calls is held in 32 bits); otherwise an empty group's dw is zero.
 * ws: pcm_workspace_bytes(PCM_OP_GROUPED_DW, R, K, N, n, 1, dtype) bytes (0 but for many rows and a
 * small dw, whose rows are summed in parts). */
pcm_status pcm_grouped_gemm_dw(pcm_dtype dtype, pcm_dtype out_dtype, const void* x, const void* dy,
                               const int32_t* offsets, const int32_t* row_token, int64_t T, int64_t R,
                               int K, int N, int n, void* dw, int accumulate, void* ws, size_t ws_bytes,
                               void* stream);

/* 8-bit values (OCP e4m3: sign, 4 exponent bits, 3 mantissa bits, largest 448, NaN but no infinity) with
 * a float32 scale for each block of 128: the value stands for code * scale. A block whose largest finite
 * magnitude is m has a = max(m, 2^-100), scale = a / 448, code = e4m3(v * (448 / a)), all float32
 * operations, the code to nearest even. Infinities and NaN become NaN codes and leave the scale alone.
 *
 * Rows, blocks of 128 along a row (the last one shorter where K is no multiple): x [R,K] of `dtype`,
 * q [R,K] u8, scale [R, ceil(K/128)] f32. count: device pointer to the number of rows to do (such as
 * offsets + n; rows from there on are left as they were), NULL: all R. */
pcm_status pcm_quant_fp8_rows(pcm_dtype dtype, const void* x, const int32_t* count, int64_t R, int K,
                              uint8_t* q, float* scale, void* stream);

/* The same for SiLU(gate) * up (Section 4.1's expansion, float32 in between): gate_up [R, 2F], a row's
 * gate values before its up values; q [R,F], scale [R, ceil(F/128)]. */
pcm_status pcm_swiglu_quant_fp8(pcm_dtype dtype, const void* gate_up, const int32_t* count, int64_t R,
                                int F, uint8_t* q, float* scale, void* stream);

/* Weights in blocks of 128 x 128: w [n,N,K] of `dtype`, q [n,N,K] u8, scale [n, ceil(N/128),
 * ceil(K/128)] f32. q_t [n,K,N] and scale_t [n, ceil(K/128), ceil(N/128)] (both or neither): the same
 * codes and scales of every W^T, with which pcm_grouped_gemm_fp8 gives the gradient by its input. */
pcm_status pcm_quant_fp8_weights(pcm_dtype dtype, const void* w, int n, int N, int K, uint8_t* q,
                                 float* scale, uint8_t* q_t, float* scale_t, void* stream);

/* pcm_grouped_gemm of 8-bit operands: y[r, c] = sum over the blocks b of K of
 * x_scale[s(r), b] w_scale[e, c / 128, b] sum over k in b of x[s(r), k] w[e, c, k].
 * x [T,K] u8 with x_scale [T, ceil(K/128)], w [n,N,K] u8 with w_scale [n, ceil(N/128), ceil(K/128)], y [R,N]
 * of out_dtype. A block's two scales are multiplied with each other first, in float32, then with its sum. Their
 * product has to be a normal float32 number (2^-126 up to below 2^128): a smaller one loses bits and from 2^-150
 * down the whole block, a larger one is infinite, which makes NaN of a block that adds up to 0. (Quantised blocks
 * keep to it where their largest magnitudes multiply to 2^-108 at least and below 2^128.)
 * The scaled blocks are added in float32. PCM_F32: so are a block's
 * products (as bf16 values, exactly, at half the rate). PCM_BF16: on the 8-bit matrix cores, which cut
 * products below 2^-13 of the largest among their neighbours (1.3e-5 of the result's norm on normal
 * values; the rounding to bf16 is 1.7e-3).
 * Backward: the gradient by the input is this call with dy quantised by rows and W^T's codes; the weight
 * gradient's sum runs over rows, along which these scales are not shared: pcm_grouped_gemm_dw. */
pcm_status pcm_grouped_gemm_fp8(pcm_dtype out_dtype, const uint8_t* x, const float* x_scale,
                                const uint8_t* w, const float* w_scale, const int32_t* offsets,
                                const int32_t* row_token, int64_t T, int64_t R, int K, int N, int n,
                                void* y, void* stream);

/* ---------------------------------------------------------------- training around the experts' products
 * What a training step does between the products above, with its gradients. `dtype` is that of the inputs,
 * `out_dtype` that of the result, each PCM_F32 or PCM_BF16; computed in float32, rounded once, to nearest even.
 * Limits: widths (H, F) multiples of 16, at most 2^28; k <= 8; n <= 256; T and R below 2^30. Outputs must not
 * overlap inputs (but for the gradients clipped in place). Deterministic. */

/* Rows of tokens. row_of [T,k] i32: the row of pair (t, a), as in pcm_paths; a number outside [offsets[0],
 * offsets[n]) (offsets [n+1] i32, which may be a part of a table's: a rank that holds some of the experts), or
 * [0, R) without offsets (then n = 1), is no row and has no part. No two pairs have the same row. R counts the rows
 * of the row buffers. weights [T,k] f32, or NULL: 1.
 *
 * Tokens to rows: y[r, :] = weights[t, a] x[t, :] for r = row_of[t, a]. x [T,H], y [R,H]; rows of no pair are left
 * as they were. */
pcm_status pcm_dispatch_rows(pcm_dtype dtype, pcm_dtype out_dtype, const void* x, const int32_t* row_of,
                             const float* weights, const int32_t* offsets, int64_t T, int k, int64_t R,
                             int H, int n, void* y, void* stream);

/* Its gradients: dx[t, :] = sum over a (ascending) of weights[t, a] dy[r, :], every row written; dweights[t, a] =
 * sum over the columns of dy[r, :] x[t, :], 0 for a pair without a row. dy [R,H] of `dtype`, x [T,H] of x_dtype, dx [T,H]
 * of out_dtype, dweights [T,k] f32. dx or dweights may be NULL: not wanted; x may be NULL without dweights. */
pcm_status pcm_dispatch_rows_grad(pcm_dtype dtype, pcm_dtype x_dtype, pcm_dtype out_dtype, const void* dy, const void* x,
                                  const int32_t* row_of, const float* weights, const int32_t* offsets,
                                  int64_t T, int k, int64_t R, int H, int n, void* dx, float* dweights,
                                  void* stream);

/* Rows back to tokens: y[t, :] = [y[t, :] +] sum over a (ascending) of weights[t, a] o[r, :], every row written.
 * o [R,H], y [T,H]. accumulate adds into y (PCM_F32 only). */
pcm_status pcm_combine_rows(pcm_dtype dtype, pcm_dtype out_dtype, const void* o, const int32_t* row_of,
                            const float* weights, const int32_t* offsets, int64_t T, int k, int64_t R,
                            int H, int n, void* y, int accumulate, void* stream);

/* Its gradients: d_o[r, :] = weights[t, a] dy[t, :], rows of no pair left as they were; dweights[t, a] = sum over
 * the columns of o[r, :] dy[t, :], 0 for a pair without a row. dy [T,H] of `dtype`, o [R,H] of o_dtype, d_o [R,H] of
 * out_dtype, dweights [T,k] f32. d_o or dweights may be NULL: not wanted; o may be NULL without dweights. */
pcm_status pcm_combine_rows_grad(pcm_dtype dtype, pcm_dtype o_dtype, pcm_dtype out_dtype, const void* dy, const void* o,
                                 const int32_t* row_of, const float* weights, const int32_t* offsets,
                                 int64_t T, int k, int64_t R, int H, int n, void* d_o, float* dweights,
                                 void* stream);

/* SwiGLU between the experts' products: u[r, :] = SiLU(gate) * up. gate_up [R, 2F], a row's gate values before its up
 * values; u [R,F]. count: as for pcm_swiglu_quant_fp8, which quantises the same values. SiLU is formed first, in float32:
 * gates below about -87, where its exponential leaves the normal range, have |gate| 2^-149 |up| of error. */
pcm_status pcm_swiglu(pcm_dtype dtype, pcm_dtype out_dtype, const void* gate_up, const int32_t* count,
                      int64_t R, int F, void* u, void* stream);

/* Its gradient by gate_up, from it and du [R,F] (both of `dtype`): dgate_up [R, 2F] of out_dtype, in the same order,
 * dgate = du up s (1 + gate (1 - s)), dup = du gate s, s = 1 / (1 + exp(-gate)). du * up is formed first. */
pcm_status pcm_swiglu_grad(pcm_dtype dtype, pcm_dtype out_dtype, const void* gate_up, const void* du,
                           const int32_t* count, int64_t R, int F, void* dgate_up, void* stream);

/* The mix along each token's paths: z[tgt_row_of[t, b], :] = sum over a (ascending) of beta[t, a, b] u[src_row_of[t, a],
 * :] over the paths (a, b) of path_bits [T] (bit a*k+b). beta [T,k,k] f32; src_row_of and tgt_row_of [T,k] i32: row_of
 * of a pcm_paths for both, src_row_of and tgt_row_of of a pcm_scored_paths. u [R_src,F], z [R_tgt,F]. A number that is no
 * row ([0, R_src), [0, R_tgt)) has no part; no two pairs have the same row of a buffer. A target without paths has
 * zeros; rows of no pair are left as they were. beta where there is no path and its source's row are not used. */
pcm_status pcm_mix_rows(pcm_dtype dtype, pcm_dtype out_dtype, const void* u, const uint64_t* path_bits,
                        const float* beta, const int32_t* src_row_of, const int32_t* tgt_row_of, int64_t T,
                        int k, int64_t R_src, int64_t R_tgt, int F, void* z, void* stream);

/* Its gradients: du[src_row_of[t, a], :] = sum over b (ascending) of beta[t, a, b] dz[tgt_row_of[t, b], :] over the paths
 * (zeros for a source without paths, rows of no pair left as they were); dbeta[t, a, b] = sum over the columns of
 * dz[tgt_row_of[t, b], :] u[src_row_of[t, a], :], 0 where there is no path. dz [R_tgt,F] and u [R_src,F] of `dtype`, du
 * [R_src,F] of out_dtype, dbeta [T,k,k] f32. du or dbeta may be NULL: not wanted; u may be NULL without dbeta. */
pcm_status pcm_mix_rows_grad(pcm_dtype dtype, pcm_dtype out_dtype, const void* dz, const void* u,
                             const uint64_t* path_bits, const float* beta, const int32_t* src_row_of,
                             const int32_t* tgt_row_of, int64_t T, int k, int64_t R_src, int64_t R_tgt, int F,
                             void* du, float* dbeta, void* stream);

/* The router's gradient: dlogits [T,n] of out_dtype from the gradients of what pcm_route and pcm_build_paths (or
 * pcm_route_paths) made of the logits: dw [T,k] f32 by topk_w, dbeta [T,k,k] f32 by beta (only the elements of the
 * paths in path_bits are read), either or both (the others NULL). Logits that were not selected get 0. Computed in
 * 64 bits from the float32 inputs, rounded to float32, then to out_dtype. */
pcm_status pcm_route_grad(pcm_dtype out_dtype, const int32_t* topk_ids, const float* topk_w,
                          const uint64_t* path_bits, const float* dbeta, pcm_beta_mode beta_mode,
                          const float* dw, int64_t T, int n, int k, void* dlogits, void* stream);

/* A gradient among all of a model's: `count` neighbouring elements of PCM_F32 or PCM_BF16. data need only be aligned
 * to its elements (a view into a flat buffer); it may be NULL where count is 0. */
typedef struct pcm_tensor {
    void* data;
    int64_t count;      /* at most 2^36 */
    pcm_dtype dtype;
} pcm_tensor;

/* The norm over all gradients: norm [1] f32 (device) = sqrt(sum of squares of every element of grads[0, m)), squares and
 * sums in 64 bits, the norm rounded (over float32's largest: infinite). `grads` is host memory, read before the
 * call returns; m <= 4096.
 * ws: pcm_workspace_bytes(PCM_OP_GRAD_NORM, m, 0, 0, 1, 1, 0) bytes. Calls that overlap in time must not share it. norm
 * and ws lie on no tensor of a call and not on each other; the norm that pcm_clip_grads reads, on none that it writes. */
pcm_status pcm_grad_norm(const pcm_tensor* grads, int m, float* norm, void* ws, size_t ws_bytes, void* stream);

/* Clipping by a norm on the device (pcm_grad_norm's, or one made of several ranks'): with norm > max_norm, out[i] =
 * grads[i] * (max_norm / norm), the factor rounded to float32, otherwise out[i] = grads[i]; a norm that is not finite
 * leaves the values as they are. out: tensors of the same counts, of either type; NULL: in place. Each out[i] is
 * grads[i] itself or overlaps no other tensor of the call; gradients do not overlap each other. */
pcm_status pcm_clip_grads(const pcm_tensor* grads, const pcm_tensor* out, int m, const float* norm,
                          float max_norm, void* stream);

/* Both, with the same results, in fewer launches where the gradients are small: norm [1] f32 is written. Arguments as
 * above. */
pcm_status pcm_clip_grad_norm(const pcm_tensor* grads, const pcm_tensor* out, int m, float max_norm,
                              float* norm, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------- tests and measurement
 * A layer never needs these. The *_tuned calls are the calls above with a pcm_tuning that
 * forces kernel choices the library otherwise makes by shape (every choice computes the same
 * bits, but for the large tiles' projection, which adds two partial sums where its tiles would
 * fill less than the chip and K is long) and that records HIP events between the internal stages
 * of a call; tuning = NULL is the plain call. They let tests check each kernel on the same inputs
 * and let benchmarks time each stage on the stream it runs on. Values outside the documented sets
 * give PCM_ERR_ARG. */
typedef struct pcm_tuning {
    int tile;              /* 0: chosen by the shape (smaller tiles of 64 rows among the choices); 'S' the few-row
                              streaming kernel, 'M' the medium tiles, 'L' the large tiles on four waves,
                              'W' the large tiles on eight waves (two per SIMD; the default
                              for an expansion that takes the large tiles); for 'L' and 'W'
                              the medium tiles run instead where 32-bit buffer offsets would
                              not reach */
    int order_expand;      /* work order of the large tiles in expansion GEMMs: -1 by shape,
                              0 grouped, 1 longest first, 2 expert-major */
    int order_down;        /* the same for projection GEMMs */
    int em_window;         /* workgroups per expert-major window (0: 8) */
    int group_n;           /* N tiles per group of the grouped order (0: 4) */
    int stream_depth;      /* streaming kernel: -1 by shape; 0 the register-ring kernel;
                              2, 3, 4 or 6 LDS ring slots */
    void* stage_events[4]; /* hipEvent_t each, or NULL: the project-and-combine calls record
                              them on `stream` before the mix, before the projection GEMM,
                              before the combine and after it (the caller creates them) */
} pcm_tuning;

pcm_status pcm_expand_tuned(pcm_dtype dtype, const void* x, const void* w_gate, const void* w_up,
                            const pcm_paths* paths, int64_t T, int H, int F, int n, int k, void* u,
                            void* ws, size_t ws_bytes, void* stream, const pcm_tuning* tuning);
pcm_status pcm_project_combine_tuned(pcm_dtype dtype, const void* u, const void* w_down,
                                     const pcm_paths* paths, int64_t T, int H, int F, int n, int k,
                                     float* y, int accumulate, void* ws, size_t ws_bytes,
                                     void* stream, const pcm_tuning* tuning);
pcm_status pcm_dense_swiglu_tuned(pcm_dtype dtype, const void* x, const void* w_gate,
                                  const void* w_up, const void* w_down, int64_t T, int H, int Fs,
                                  float* y, int accumulate, void* ws, size_t ws_bytes, void* stream,
                                  const pcm_tuning* tuning);
pcm_status pcm_expand_scored_tuned(pcm_dtype dtype, const void* x, const void* w_gate,
                                   const void* w_up, const pcm_scored_paths* paths, int64_t T,
                                   int H, int F, int n, int K, void* u, void* ws, size_t ws_bytes,
                                   void* stream, const pcm_tuning* tuning);
pcm_status pcm_project_combine_scored_tuned(pcm_dtype dtype, const void* u, const void* w_down,
                                            const pcm_scored_paths* paths, int64_t T, int H, int F,
                                            int n, int K, float* y, int accumulate, void* ws,
                                            size_t ws_bytes, void* stream,
                                            const pcm_tuning* tuning);

/* Where pcm_project_combine(_tuned) keeps its intermediates inside its workspace, so that a
 * test can read them back after the call: the projection input z [T*k, F] (bf16 layers:
 * float16 rows, each multiplied by a power of two; f32 layers: float32) at byte *z_off; the
 * inverse of each z row's power of two [T*k] f32 at *zscale_off (bf16 layers; 0 otherwise);
 * the projected rows o [ksplit, T*k, H] f32 at *o_off, K slice s of row r at (s*T*k + r)*H
 * (the combine adds the slices in order). All outputs are host pointers. */
pcm_status pcm_project_workspace_layout(pcm_dtype dtype, int64_t T, int H, int F, int n, int k,
                                        const pcm_tuning* tuning, size_t* z_off,
                                        size_t* zscale_off, size_t* o_off, int* ksplit);

/* Device workspace bytes an operation needs (0 if none). Returns 0 for invalid sizes. */
size_t pcm_workspace_bytes(pcm_op op, int64_t T, int H, int F, int n, int k, pcm_dtype dtype);

/* Static description of a status code (never NULL). */
const char* pcm_status_string(pcm_status status);

/* ABI version of this header (major * 100 + minor). */
int pcm_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* PCOMOE_H */
