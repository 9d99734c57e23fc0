/*
 * moe.h -- C ABI of the MI355X (gfx950) library for one GPU's share of one
 * expert-parallel MoE layer, the layer whose routing statistics Director
 * (arXiv 2607.08782) turns into expert placements.
 *
 * The share runs five steps, one entry point each, all enqueued on the
 * caller's HIP stream:
 *   moe_route_topk        gate scores and top-k routing            (Sec. II-A)
 *   moe_expert_histogram  per-expert workload counts W, co-activation
 *                                                     (Sec. VI-A; Sec. I)
 *   moe_permute           packaging of tokens for the experts placed on this
 *                         GPU, with per-GPU send counts (Sec. II-B; Eq. 1, 3)
 *   moe_grouped_ffn       the experts' FFNs over ragged groups of rows
 *                                                              (Sec. II-A)
 *   moe_combine           gate-weighted sum of expert outputs  (Sec. II-A)
 *
 * Conventions for every entry point
 *   - Pointers named "device" point to caller-owned device memory; pointers
 *     named "host" point to host memory that is read during the call and not
 *     kept.  The library allocates nothing and never synchronises the
 *     stream; outputs are valid once the stream reaches the end of the call.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *   - Matrices are row-major and densely packed.  Element type codes:
 *     MOE_F32 (float) and MOE_BF16 (bfloat16, round-to-nearest-even stored).
 *     Gate scores, logits and gates are always float; indices int32.
 *   - Arguments are validated before anything is enqueued.  A non-zero
 *     status means nothing was enqueued, except MOE_ERR_DEVICE, which
 *     reports a HIP launch error (the stream state is then unspecified).
 *   - Entry points are stateless and reentrant; concurrent calls on
 *     different streams must use different output and workspace buffers.
 */
#ifndef MOE_H
#define MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define MOE_F32  0
#define MOE_BF16 1

/* status codes */
#define MOE_OK            0
#define MOE_ERR_ARG       1   /* null pointer, negative size, k out of range, bad dtype/flags */
#define MOE_ERR_PLACEMENT 2   /* an expert with no host GPU, dev >= G, or more than c_max local experts */
#define MOE_ERR_SHAPE     3   /* unsupported d or f, cap_rows or workspace too small */
#define MOE_ERR_DEVICE    4   /* a HIP launch failed */

/* products of moe_grouped_ffn_products */
#define MOE_FFN_GATE_UP 1   /* h = SiLU(W1 x) * (W3 x), kept in the workspace */
#define MOE_FFN_DOWN    2   /* y = W2 h, from the workspace */
#define MOE_FFN_SMALL_GROUPS 4   /* hint: no group has more than 256 rows; all are streamed */
#define MOE_FFN_LARGE_GROUPS 8   /* hint: every non-empty group has more than 256 rows; none is streamed */

/* flags of moe_route_topk */
#define MOE_RENORM    1   /* gates = softmax over the k selected logits (else: full softmax, restricted) */
#define MOE_LOGITS_IN 2   /* skip the gate GEMM: `logits` is an input holding T*E scores */

/* limits */
#define MOE_MAX_E      256   /* experts per layer */
#define MOE_MAX_K      16    /* experts per token */
#define MOE_MAX_G      64    /* GPUs in the placement map */
#define MOE_MAX_GROUPS 128   /* local expert groups per moe_grouped_ffn call */
#define MOE_PERMUTE_NOALLOC_MAX_WS (4 << 20)   /* scratch bytes of moe_permute_noalloc */

/* Human-readable name of a status code (static string). */
const char* moe_status_string(int status);

/*
 * moe_route_topk -- gate scores and top-k routing (Sec. II-A: the gating
 * network scores every expert for each token and the token goes to the k
 * best; the gate is replicated on every GPU, Sec. II-B).
 *
 *   logits[t][e] = sum_i x[t][i] * w_router[e][i] + bias[e]     (fp32 accumulate)
 *   topk_idx[t][r] = r-th best expert of token t: descending logit; equal
 *                    logits (-0.0 == +0.0) go to the lower expert index
 *   topk_gate[t][r] = exp(l_r - l_0) / sum_{r'<k} exp(l_r' - l_0)  with MOE_RENORM,
 *                     else exp(l_r - l_0) / sum_{e<E} exp(l_e - l_0)
 *
 * x         device [T][d] of `dtype`        (unused with MOE_LOGITS_IN; may be NULL then)
 * w_router  device [E][d] of `dtype`        (unused with MOE_LOGITS_IN)
 * bias      device [E] float, nullable (= 0)
 * logits    device [T][E] float: output, or input with MOE_LOGITS_IN; nullable
 *           otherwise (then the scores are not stored)
 * topk_idx  device [T][k] int32 output;  topk_gate  device [T][k] float output
 * ws        device workspace of moe_route_topk_ws_bytes(dtype, T, d, E, flags)
 *           bytes, 256-byte aligned; may be NULL when that size is 0.  (bf16 batches
 *           whose scores run in a launch of their own keep them here: the long ones
 *           when logits is NULL, the short ones always, past d = 2048 as fp32 partial
 *           scores per K chunk, which are summed in chunk order.)
 * Requires 1 <= E <= MOE_MAX_E, 1 <= k <= min(E, MOE_MAX_K), T >= 0,
 * d >= 1 and, for MOE_BF16, d % 8 == 0 and E * d * 2 < 2^31 (else
 * MOE_ERR_SHAPE).  Logits must be finite.
 * Scores are deterministic: the same inputs give bitwise the same outputs.
 */
int moe_route_topk(const void* x, int dtype, const void* w_router, const float* bias,
                   int64_t T, int d, int E, int k, int flags,
                   float* logits, int32_t* topk_idx, float* topk_gate,
                   void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes moe_route_topk needs (0 = none). */
size_t moe_route_topk_ws_bytes(int dtype, int64_t T, int d, int E, int flags);

/*
 * moe_expert_histogram -- per-expert workload counts (Sec. VI-A: W_{j,i}
 * counts tokens routed to expert i; this share routes all T tokens, so
 * counts[e] is the inner sum of Eq. 1) and co-activation counts (the signal
 * for co-locating experts activated together, Sec. I).
 *
 *   counts[e]   = #{(t, r) : topk_idx[t][r] == e}
 *   coact[a][b] = #{t : a and b both among topk_idx[t][0..k-1]}   (diag = counts)
 *
 * topk_idx  device [T][k] int32, values in [0, E), distinct within a row
 * counts    device [E] int32 output (overwritten)
 * coact     device [E][E] int32 output, nullable (not computed)
 * Results are exact integers and independent of scheduling.
 */
int moe_expert_histogram(const int32_t* topk_idx, int64_t T, int k, int E,
                         int32_t* counts, int32_t* coact, void* stream);

/* Workspace bytes moe_permute needs for T tokens, k and E. */
size_t moe_permute_ws_bytes(int64_t T, int k, int E);

/*
 * moe_permute -- package the tokens for the experts placed on GPU `dev`
 * (Sec. II-B: tokens are packaged and sent to the GPUs hosting their
 * experts; Sec. VI-A: placement x[e][j], every expert hosted at least once,
 * Eq. 6d, at most C_max experts per GPU, Eq. 6e).
 *
 * placement  HOST [E][G] uint8, x[e][j] = placement[e*G + j] != 0
 * Local slot s = the s-th expert, by ascending id, with x[e][dev] = 1;
 * n_local = number of local slots.  An expert with n_e hosts splits its
 * tokens (ascending token order, c_e = counts[e] of them) into contiguous
 * blocks: its q-th host by ascending GPU id serves ranks
 * [floor(q*c_e/n_e), floor((q+1)*c_e/n_e)).  (The paper allows replicas but
 * leaves the split open; this is the rule the library fixes.)
 *
 * Outputs (rows are grouped by slot, ascending token order inside a group):
 *   group_offsets device [n_local+1] int32: exclusive prefix sum of rows per slot;
 *                 N = group_offsets[n_local] rows are written
 *   x_perm        device [cap_rows][d] of `dtype`: x_perm[p] = x[row_token[p]]
 *   row_token     device [cap_rows] int32;  row_gate  device [cap_rows] float
 *   token_row     device [T][k] int32: row of assignment (t, r) here, or -1
 *   send_counts   device [G] int32, nullable: rows each GPU's hosts take,
 *                 i.e. Eq. 3's D_{dev,j} / d; equals Eq. 1's lambda_j when
 *                 no expert is replicated
 * counts  device [E] int32 from moe_expert_histogram on the same topk_idx.
 * c_max   0 = unchecked, else MOE_ERR_PLACEMENT if n_local > c_max.
 * ws      device workspace of at least moe_permute_ws_bytes(T, k, E) bytes,
 *         256-byte aligned.
 * Requires cap_rows >= T * min(k, n_local), G <= MOE_MAX_G, and for
 * MOE_BF16 d % 8 == 0.  Rows past N are left untouched.
 */
int moe_permute(const void* x, int dtype, const int32_t* topk_idx, const float* topk_gate,
                const int32_t* counts, int64_t T, int d, int k, int E,
                const uint8_t* placement, int G, int dev, int c_max,
                void* x_perm, int64_t cap_rows, int32_t* group_offsets,
                int32_t* row_token, float* row_gate, int32_t* token_row,
                int32_t* send_counts, void* ws, size_t ws_bytes, void* stream);

/*
 * moe_permute_noalloc -- moe_permute without a workspace argument, for callers
 * that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc).  It packages the tokens
 * exactly as moe_permute does (same outputs, bit for bit) and keeps the
 * per-block counts it needs in a scratch array of this library: one copy per
 * GPU, MOE_PERMUTE_NOALLOC_MAX_WS (4 MiB) bytes, held until the process ends.
 * The call allocates nothing; its first call on a GPU looks up that GPU's
 * copy of the array.
 *
 * Arguments, outputs and errors as for moe_permute, without ws / ws_bytes.
 * Returns MOE_ERR_SHAPE when moe_permute_ws_bytes(T, k, E) exceeds
 * MOE_PERMUTE_NOALLOC_MAX_WS (more than about 524 000 tokens at 128 local
 * slots), and MOE_ERR_DEVICE if the scratch cannot be located on the current
 * device.  The scratch keeps the last call's contents; every call on one GPU
 * shares it, so calls that overlap in time on one GPU (different streams, or
 * different threads) race and must be serialised by the caller.
 */
int moe_permute_noalloc(const void* x, int dtype, const int32_t* topk_idx,
                        const float* topk_gate, const int32_t* counts, int64_t T, int d, int k,
                        int E, const uint8_t* placement, int G, int dev, int c_max, void* x_perm,
                        int64_t cap_rows, int32_t* group_offsets, int32_t* row_token,
                        float* row_gate, int32_t* token_row, int32_t* send_counts, void* stream);

/*
 * moe_route_package -- moe_route_topk, moe_expert_histogram and moe_permute of
 * one batch in one call (Sec. II-A, II-B, VI-A): the same outputs, bit for bit,
 * in fewer launches where the batch is short (a decode step's routing is two).
 *
 * x, dtype, w_router, bias, T, d, E, k, flags, logits, topk_idx, topk_gate,
 *           ws_route, ws_route_bytes as for moe_route_topk
 * counts, coact (nullable) as for moe_expert_histogram
 * placement .. send_counts, ws_perm, ws_perm_bytes as for moe_permute; x_perm
 *           NULL writes the row maps only (moe_permute with d = 0)
 * Requirements and errors as for the three calls; with MOE_LOGITS_IN and no row
 * copy x and w_router are not read and may be NULL.
 */
int moe_route_package(const void* x, int dtype, const void* w_router, const float* bias,
                      int64_t T, int d, int E, int k, int flags, float* logits,
                      int32_t* topk_idx, float* topk_gate, void* ws_route,
                      size_t ws_route_bytes, int32_t* counts, int32_t* coact,
                      const uint8_t* placement, int G, int dev, int c_max, void* x_perm,
                      int64_t cap_rows, int32_t* group_offsets, int32_t* row_token,
                      float* row_gate, int32_t* token_row, int32_t* send_counts, void* ws_perm,
                      size_t ws_perm_bytes, void* stream);

/* Workspace bytes moe_grouped_ffn needs. */
size_t moe_grouped_ffn_ws_bytes(int dtype, int64_t cap_rows, int d, int f, int n_groups);

/*
 * moe_grouped_ffn -- every local expert's FFN on its group of rows
 * (Sec. II-A: experts are FFN sub-networks).  Experts are SwiGLU:
 *
 *   for each slot s and row p in [group_offsets[s], group_offsets[s+1]):
 *     a = W1_s x_perm[p],  b = W3_s x_perm[p]               (f values each)
 *     h = SiLU(a) * b,     SiLU(a) = a / (1 + exp(-a))
 *     y_perm[p] = W2_s h
 *
 * x_perm         device [cap_rows][d] of `dtype`
 * group_offsets  device [n_groups+1] int32, non-decreasing, offsets[0] = 0,
 *                offsets[n_groups] <= cap_rows (read on the device only)
 * w13            HOST array of n_groups device pointers; w13[s] is [2f][d]:
 *                rows 0..f-1 are W1_s (gate), rows f..2f-1 are W3_s (up)
 * w2             HOST array of n_groups device pointers; w2[s] is [d][f]
 * y_perm         device [cap_rows][d] of `dtype` output (rows past
 *                offsets[n_groups] untouched)
 * ws             device workspace, moe_grouped_ffn_ws_bytes(...) bytes,
 *                256-byte aligned
 * For MOE_BF16 the products accumulate in fp32 and h is rounded to bf16
 * before the second product.  Requires 1 <= n_groups <= MOE_MAX_GROUPS and
 * for MOE_BF16 d % 64 == 0, f % 64 == 0 and d, f < 2^22 (else MOE_ERR_SHAPE).
 * A shared (always-on) expert is the call with x_perm = x, one group and
 * group_offsets = {0, T}.
 */
int moe_grouped_ffn(const void* x_perm, int dtype, const int32_t* group_offsets, int n_groups,
                    const void* const* w13, const void* const* w2, int d, int f,
                    int64_t cap_rows, void* y_perm, void* ws, size_t ws_bytes, void* stream);

/*
 * moe_grouped_ffn_products -- moe_grouped_ffn run one product at a time
 * (Sec. II-A: the expert FFN is the two products of the SwiGLU block), for
 * callers that schedule or time the two separately.  products is a mask:
 *   MOE_FFN_GATE_UP  h = SiLU(W1_s x_perm[p]) * (W3_s x_perm[p]) for every row,
 *                    kept in ws (with the call's group plan)
 *   MOE_FFN_DOWN     y_perm[p] = W2_s h[p], reading h and the plan from ws
 * MOE_FFN_GATE_UP | MOE_FFN_DOWN is exactly moe_grouped_ffn.  A
 * MOE_FFN_DOWN call must follow a MOE_FFN_GATE_UP call on the same stream
 * with the same ws, group_offsets (unchanged contents), n_groups, d, f and
 * cap_rows; ws must not be used in between.  The two calls in sequence give
 * bitwise the outputs of moe_grouped_ffn.  x_perm and w13 are read only with
 * MOE_FFN_GATE_UP (may be NULL otherwise), y_perm and w2 only with
 * MOE_FFN_DOWN.  Other arguments, requirements and errors as for
 * moe_grouped_ffn; products outside {1, 2, 3} give MOE_ERR_ARG.
 * Adding MOE_FFN_SMALL_GROUPS to products states that no group holds more
 * than 256 rows (true of a batch of at most 256 tokens: a token reaches an
 * expert at most once).  Every group then takes the weight-streaming kernels
 * and the call skips the launches of the tiled kernels.  Without the flag a
 * call streams every group when none holds more than 256 rows and its groups
 * above 64 rows make few tiles (always so when no group holds more than 64
 * rows), and tiles every group otherwise, each product by itself (some calls
 * with K past 8192 tile only the groups above 256 rows); so a call
 * whose groups all hold at most 64 rows gives bitwise the outputs it gives
 * without the flag, and a group that the call without the flag would tile sums
 * its products in another order (same tolerance).  Rows of a group that breaks
 * the statement are left unwritten.  It must be passed the same way to the
 * MOE_FFN_GATE_UP and the MOE_FFN_DOWN call of one pair.
 * Adding MOE_FFN_LARGE_GROUPS instead states that every non-empty group holds
 * more than 256 rows (true of a shared expert's call over more than 256
 * tokens): every group then takes the tiled kernels and the call skips the
 * weight-streaming launches.  Such a call gives bitwise the outputs it gives
 * without the flag; a group that breaks the statement is still computed in
 * full, by the tiled kernels (its products summed in another order, same
 * tolerance).  It must be passed the same way to both calls of a pair; the
 * two hints together give MOE_ERR_ARG.
 */
int moe_grouped_ffn_products(const void* x_perm, int dtype, const int32_t* group_offsets,
                             int n_groups, const void* const* w13, const void* const* w2, int d,
                             int f, int64_t cap_rows, void* y_perm, void* ws, size_t ws_bytes,
                             int products, void* stream);

/*
 * moe_grouped_ffn_combine -- moe_grouped_ffn followed by moe_combine, for calls
 * in which no group holds more than 256 rows (a batch of at most 256 tokens;
 * the MOE_FFN_SMALL_GROUPS statement): the expert outputs are combined inside the
 * down product's fixed-order sum of its K chunks (the gate-weighted sum of
 * Sec. II-A, the return trip of Sec. II-B), so y_perm is neither written nor
 * read back and the combine needs no launch of its own:
 *
 *   y[t] = sum_{r ascending, token_row[t][r] >= 0} topk_gate[t][r] * y_perm[token_row[t][r]]
 *          + y_shared[t]
 *
 * with y_perm[p] the bf16 value moe_grouped_ffn with MOE_FFN_SMALL_GROUPS would
 * store, summed in fp32 in the order moe_combine uses: bitwise that call
 * followed by moe_combine.
 * x_perm, group_offsets, n_groups, w13, w2, d, f, cap_rows and ws as for
 * moe_grouped_ffn; token_row, topk_gate, y_shared (nullable), T, k and y as for
 * moe_combine.  MOE_BF16 only (MOE_ERR_ARG otherwise).  Rows of a group that
 * holds more than 256 rows are left out of y.  If y_shared comes from another
 * stream, that stream must be joined before this call.
 */
int moe_grouped_ffn_combine(const void* x_perm, int dtype, const int32_t* group_offsets,
                            int n_groups, const void* const* w13, const void* const* w2, int d,
                            int f, int64_t cap_rows, const int32_t* token_row,
                            const float* topk_gate, const void* y_shared, int64_t T, int k,
                            void* y, void* ws, size_t ws_bytes, void* stream);

/*
 * moe_grouped_ffn_rows -- moe_grouped_ffn whose first product reads row p of
 * its input straight from the token rows, x[row_token[p]], instead of from a
 * packaged copy: the row map of the packaging step (Sec. II-B) is kept and the
 * copy of the rows, x_perm, is never written or read.  This is the one-GPU
 * part of fusing the dispatch gather into the expert GEMM; with moe_permute
 * called with d = 0 (row maps only) the outputs are bitwise identical to
 * moe_permute + moe_grouped_ffn.
 *
 * x          device [T][d] of `dtype`: the token rows
 * row_token  device [cap_rows] int32 (moe_permute's row map): entries of rows
 *            below group_offsets[n_groups] must lie in [0, T)
 * other arguments, workspace (moe_grouped_ffn_ws_bytes) and outputs as for
 * moe_grouped_ffn.  bf16 requires T * d * 2 < 2^31 (32-bit row offsets),
 * else MOE_ERR_SHAPE, and 16-byte aligned x.
 */
int moe_grouped_ffn_rows(const void* x, int64_t T, const int32_t* row_token, int dtype,
                         const int32_t* group_offsets, int n_groups, const void* const* w13,
                         const void* const* w2, int d, int f, int64_t cap_rows, void* y_perm,
                         void* ws, size_t ws_bytes, void* stream);

/*
 * moe_grouped_ffn_rows_products -- moe_grouped_ffn_rows with the products mask of
 * moe_grouped_ffn_products (one product at a time, and the MOE_FFN_SMALL_GROUPS
 * or MOE_FFN_LARGE_GROUPS statement, with the same meaning and the same
 * outputs): x and row_token are read only with MOE_FFN_GATE_UP (may be NULL
 * otherwise), y_perm and w2 only with MOE_FFN_DOWN.  Other arguments,
 * requirements and errors as for moe_grouped_ffn_rows; MOE_FFN_GATE_UP |
 * MOE_FFN_DOWN is exactly moe_grouped_ffn_rows.
 */
int moe_grouped_ffn_rows_products(const void* x, int64_t T, const int32_t* row_token, int dtype,
                                  const int32_t* group_offsets, int n_groups,
                                  const void* const* w13, const void* const* w2, int d, int f,
                                  int64_t cap_rows, void* y_perm, void* ws, size_t ws_bytes,
                                  int products, void* stream);

/*
 * moe_grouped_ffn_rows_shared -- moe_grouped_ffn_rows_products with the
 * always-on shared experts (Sec. II-A: every token also passes through them)
 * computed in the same launches as the routed experts, as n_shared leading
 * groups of T rows each: one call instead of a second FFN call, so the tiles of
 * both fill the GPU together.  A shared expert of width m * f takes m groups
 * (its gate, up and down rows cut into m blocks of f: SwiGLU is elementwise in
 * h, and the down product sums over h, so the m outputs sum to the expert's).
 *
 *   group s < n_shared       rows [s T, (s+1) T), weights w13[s], w2[s]
 *   routed group g            rows n_shared T + [group_offsets[g], group_offsets[g+1]),
 *                             weights w13[n_shared + g], w2[n_shared + g]
 *
 * row_token  device [n_shared T + cap_rows] int32: the caller's entries for the
 *            shared rows (row s T + t is token t: 0, 1, ..., T-1 per group,
 *            written once and kept), then the routed rows' map (moe_permute's
 *            row_token written at row_token + n_shared T)
 * group_offsets  device [n_groups+1], the routed groups as moe_permute writes
 *            them (n_groups may be 0: only group_offsets[0] = 0 is then read)
 * w13, w2    HOST arrays of n_shared + n_groups device pointers, shared first
 * cap_rows   routed row capacity;  y_perm device [n_shared T + cap_rows][d]: group
 *            s's output in rows [s T, (s+1) T) (the n_shared slices that
 *            moe_combine_shared adds), routed rows from n_shared T
 * ws         moe_grouped_ffn_ws_bytes(dtype, n_shared T + cap_rows, d, f,
 *            n_shared + n_groups) bytes
 * products   as for moe_grouped_ffn_rows_products; the hints state the sizes of
 *            every group, shared ones included.
 * Requires 0 <= n_shared, 1 <= n_shared + n_groups <= MOE_MAX_GROUPS, T >= 1
 * when n_shared > 0 and n_shared T + cap_rows < 2^31; other requirements and
 * errors as for moe_grouped_ffn_rows.  With n_shared = 0 it is
 * moe_grouped_ffn_rows_products.
 */
int moe_grouped_ffn_rows_shared(const void* x, int64_t T, const int32_t* row_token, int dtype,
                                const int32_t* group_offsets, int n_groups, int n_shared,
                                const void* const* w13, const void* const* w2, int d, int f,
                                int64_t cap_rows, void* y_perm, void* ws, size_t ws_bytes,
                                int products, void* stream);

/*
 * moe_combine -- gate-weighted sum of the experts' outputs (Sec. II-A) back
 * in token order (the return trip of Sec. II-B), plus shared experts with
 * weight 1:
 *
 *   y[t] = sum_{r ascending, token_row[t][r] >= 0} topk_gate[t][r] * y_perm[token_row[t][r]]
 *          + y_shared[t]
 *
 * y_perm    device [rows][d] of `dtype`, required when T > 0 (it may hold
 *           no rows that any token uses);  token_row device [T][k] int32
 * topk_gate device [T][k] float;  y_shared device [T][d] of `dtype`, nullable
 * y         device [T][d] of `dtype` output (fp32 accumulation, then stored).
 * Tokens with no local assignment get y_shared[t] (or 0).
 */
int moe_combine(const void* y_perm, int dtype, const int32_t* token_row, const float* topk_gate,
                const void* y_shared, int64_t T, int d, int k, void* y, void* stream);

/*
 * moe_combine_shared -- moe_combine with the shared experts' output in
 * n_shared slices (as moe_grouped_ffn_rows_shared leaves it), added after the
 * routed sum in slice order:
 *
 *   y[t] = sum_{r ascending, token_row[t][r] >= 0} topk_gate[t][r] * y_perm[token_row[t][r]]
 *          + y_shared[0][t] + y_shared[1][t] + ... + y_shared[n_shared-1][t]
 *
 * y_shared  device [n_shared][T][d] of `dtype` (NULL or n_shared = 0: none).
 * Requires 0 <= n_shared <= MOE_MAX_GROUPS; other arguments as for
 * moe_combine.  n_shared = 1 is exactly moe_combine.
 */
int moe_combine_shared(const void* y_perm, int dtype, const int32_t* token_row,
                       const float* topk_gate, const void* y_shared, int n_shared, int64_t T,
                       int d, int k, void* y, void* stream);

/*
 * moe_quantize_e4m3 -- per-row FP8 quantization for the quantized routing
 * predictor (Sec. V-A: a low-bit replica with weights and activations both
 * quantized; gfx950 multiplies OCP FP8 E4M3 natively).  For every row r:
 *
 *   scales[r] = max_i |x[r][i]| / 448          (fp32 division; 1 if the row is 0)
 *   q[r][i]   = E4M3(x[r][i] / scales[r])      (fp32 division, round to nearest,
 *                                               ties to even; |.| > 448 saturates)
 *
 * E4M3: 1 sign, 4 exponent bits (bias 7), 3 mantissa bits, subnormals, max 448,
 * no infinities; a value that rounds to zero is stored as +0 (code 0x00).
 * x       device [rows][cols] of `dtype` (MOE_F32 or MOE_BF16), finite
 * q       device [rows][cols] uint8 output;  scales device [rows] float output
 * Requires rows >= 0, cols >= 1.  Results are exact (bitwise reproducible).
 */
int moe_quantize_e4m3(const void* x, int dtype, int64_t rows, int cols, uint8_t* q,
                      float* scales, void* stream);

/*
 * moe_route_topk_e4m3 -- gate scores of the quantized predictor (Sec. V-A)
 * and their top-k, whose agreement with moe_route_topk's choice is the
 * predictor's accuracy (top-k match rate, Sec. VIII):
 *
 *   logits[t][e] = x_scale[t] * w_scale[e] * sum_i E4M3(xq[t][i]) * E4M3(wq[e][i])
 *                  + bias[e]
 *
 * then top-k and gates exactly as moe_route_topk does for given scores.
 * xq       device [T][d] uint8 E4M3 codes, x_scale device [T] float (from
 *          moe_quantize_e4m3 of the activations)
 * wq       device [E][d] uint8 E4M3 codes, w_scale device [E] float (of the
 *          router weights [E][d])
 * bias     device [E] float, nullable
 * logits   device [T][E] float output (required: the top-k reads it back)
 * topk_idx device [T][k] int32 output;  topk_gate device [T][k] float output
 * flags    MOE_RENORM or 0
 * Requires d % 64 == 0, xq and wq 16-byte aligned, 1 <= E <= MOE_MAX_E,
 * 1 <= k <= min(E, MOE_MAX_K), T >= 0.  The code products are exact in fp32;
 * their sum is accumulated in fp32 in a fixed order (deterministic).
 */
int moe_route_topk_e4m3(const uint8_t* xq, const float* x_scale, const uint8_t* wq,
                        const float* w_scale, const float* bias, int64_t T, int d, int E, int k,
                        int flags, float* logits, int32_t* topk_idx, float* topk_gate,
                        void* stream);

/*
 * MXFP4 matrices (microscaled 4-bit floating point): rows of E2M1 elements in
 * blocks of 32, each block with one E8M0 scale.
 *
 *   E2M1: 1 sign, 2 exponent and 1 mantissa bits: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
 *         their negatives (codes 0..7, plus 8 for the sign); no infinities, no NaN
 *   E8M0: the byte b is the scale 2^(b - 127); 255 is NaN
 *
 * A matrix of `cols` columns is stored with its rows padded to
 * P = MOE_MXFP4_COLS(cols) columns, the next multiple of 128:
 *   codes   uint8 [rows][P / 2]: column 2 i in the lower, 2 i + 1 in the upper half
 *           of byte i
 *   scales  uint8 [rows][P / 32]: byte j scales columns 32 j .. 32 j + 31
 * Padding columns hold code 0; a block of padding alone has scale byte 0.
 */
#define MOE_MXFP4_COLS(cols) (((int64_t)(cols) + 127) / 128 * 128)

/*
 * moe_quantize_mxfp4 -- a matrix to MXFP4.  For every block of 32 columns (the last
 * one of a row padded with zeros):
 *
 *   b = max(E - 2, 0), E the biased exponent of the block's largest |x| (as a float;
 *       0 if that is zero or subnormal)
 *   code = E2M1(x * 2^(127 - b)), round to nearest, ties to the even code, magnitudes
 *       above 6 saturate; the sign of x is kept, also on a zero
 *
 * A block that holds an infinity or a NaN gets scale byte 255 and zero codes: all of
 * it reads as NaN, its neighbours are not touched.
 * x       device [rows][cols] of `dtype` (MOE_F32 or MOE_BF16)
 * codes, scales  device outputs as above
 * Requires rows >= 0, 1 <= cols < 2^28 (else MOE_ERR_SHAPE), codes 16-byte and scales
 * 4-byte aligned.  Results are exact (bitwise reproducible).
 */
int moe_quantize_mxfp4(const void* x, int dtype, int64_t rows, int cols, uint8_t* codes,
                       uint8_t* scales, void* stream);

/*
 * moe_dequantize_mxfp4 -- the values an MXFP4 matrix holds: y[r][c] = E2M1(code) *
 * 2^(b - 127), NaN where b = 255.  Exact in MOE_F32, and in MOE_BF16 for every value
 * above its subnormal range (rounded to nearest even there); values of 2^128 and more, which
 * only scale bytes 253 and 254 reach and no quantization gives, are infinities.
 * codes, scales  device, as above;  y  device [rows][cols] of `dtype` output
 * Requirements as for moe_quantize_mxfp4.
 */
int moe_dequantize_mxfp4(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                         int dtype, void* y, void* stream);

/*
 * moe_mxfp4_lay_out -- an MXFP4 matrix as moe_grouped_ffn_mxfp4 reads a weight's:
 * step-major, so that a product's step of 128 columns finds its rows side by side.
 *
 *   step_codes[g][r][0..63] = codes[r][64 g .. 64 g + 63]
 *   step_scales[g][r] = scale bytes 4 g .. 4 g + 3 of row r (byte i in bits 8 i)
 *
 * Made once for a weight matrix that is kept; the row-major one is then not needed.
 * codes, scales  device, as above;  step_codes  device uint8 [P / 128][rows][64] and
 * step_scales  device uint32 [P / 128][rows] outputs, P = MOE_MXFP4_COLS(cols).
 * Requires rows >= 0, 1 <= cols < 2^28 (else MOE_ERR_SHAPE), codes and step_codes 16-byte,
 * scales and step_scales 4-byte aligned.
 */
int moe_mxfp4_lay_out(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                      uint8_t* step_codes, uint32_t* step_scales, void* stream);

/* Workspace bytes moe_grouped_ffn_mxfp4 needs (T rows of x; all groups together n_groups,
 * rows of every group, shared ones included, at most cap_rows). */
size_t moe_grouped_ffn_mxfp4_ws_bytes(int64_t T, int64_t cap_rows, int d, int f, int n_groups);

/*
 * moe_grouped_ffn_mxfp4 -- moe_grouped_ffn of experts whose weights are MXFP4
 * matrices.  The rows of x are quantized to MXFP4, and the hidden rows between the
 * products, so both products multiply 4-bit operands (the matrix cores do so
 * natively, block scales included):
 *
 *   for each group s and row p of it, with Q(.) = the values moe_quantize_mxfp4 keeps:
 *     a = W1_s Q(x_p),  b = W3_s Q(x_p),  h = SiLU(a) * b          (fp32)
 *     y_perm[p] = W2_s Q(h)                                        (fp32, stored in bf16)
 *
 * x          device [T][d] bf16: row p reads x[row_token[p]]; row_token NULL: x is the
 *            packaged rows, row p reads x[p]
 * row_token  device [n_shared T + cap_rows] int32, nullable, as for
 *            moe_grouped_ffn_rows_shared (entries of rows that exist lie in [0, T))
 * group_offsets, n_groups, n_shared, cap_rows, y_perm  as for moe_grouped_ffn_rows_shared:
 *            n_shared leading groups of T rows each (0 without row_token)
 * w13, s13   HOST arrays of n_shared + n_groups device pointers: step-major codes and
 *            scales (moe_mxfp4_lay_out) of the MXFP4 matrix [2f][d], rows 0..f-1 W1
 *            (gate), f..2f-1 W3 (up)
 * w2, s2     the same of the MXFP4 matrix [d][f]
 * ws         moe_grouped_ffn_mxfp4_ws_bytes(T, n_shared T + cap_rows, d, f, n_shared +
 *            n_groups) bytes, 256-byte aligned
 * An infinity or NaN in x makes its own rows of y_perm NaN and no other.  Deterministic.
 * Requires d % 8 == 0, d and f below 2^21, T below 2^25 (else MOE_ERR_SHAPE),
 * 1 <= n_shared + n_groups <= MOE_MAX_GROUPS, x, y_perm and codes 16-byte, scales 4-byte
 * aligned.
 */
int moe_grouped_ffn_mxfp4(const void* x, int64_t T, const int32_t* row_token,
                          const int32_t* group_offsets, int n_groups, int n_shared,
                          const uint8_t* const* w13, const uint32_t* const* s13,
                          const uint8_t* const* w2, const uint32_t* const* s2, int d, int f,
                          int64_t cap_rows, void* y_perm, void* ws, size_t ws_bytes,
                          void* stream);

/*
 * moe_combine_backward -- gradient of moe_combine: of dy, the loss gradient of y,
 *
 *   dy_perm[p]  = topk_gate[t][r] * dy[t]           for p = token_row[t][r] >= 0
 *   dgate[t][r] = sum_i dy[t][i] * y_perm[p][i]     (fp32; 0 where token_row is -1)
 *
 * The gradient of y_shared is dy itself.
 * dy         device [T][d] of `dtype`;  y_perm  device [rows][d] of `dtype`, the rows
 *            that moe_combine read (not read, may be NULL, when dgate is NULL)
 * token_row  device [T][k] int32, every row at most once
 * topk_gate  device [T][k] float (not read, may be NULL, when dy_perm is NULL)
 * dy_perm    device [rows][d] of `dtype` output, nullable; rows that no token_row names
 *            are left untouched.  It must not overlap the inputs.
 * dgate      device [T][k] float output, nullable
 * Sums are fp32 in a fixed order (deterministic).  Requires T >= 0, d >= 1,
 * 1 <= k <= MOE_MAX_K; 16-byte aligned matrices where a row is a multiple of 16 bytes.
 */
int moe_combine_backward(const void* dy, const void* y_perm, int dtype, const int32_t* token_row,
                         const float* topk_gate, int64_t T, int d, int k, void* dy_perm,
                         float* dgate, void* stream);

/*
 * moe_permute_backward -- gradient of moe_permute's row copy: a token's gradient is the
 * sum of its rows' (every row's copy went to one expert), on top of what reached it by
 * another way:
 *
 *   dx[t] = sum_{r ascending, token_row[t][r] >= 0} dx_perm[token_row[t][r]] + dx_add[t]
 *
 * dx_perm    device [rows][d] of `dtype`, required when T > 0 (it may hold no rows)
 * token_row  device [T][k] int32;  dx_add  device [T][d] of `dtype`, nullable
 * dx         device [T][d] of `dtype` output (fp32 sum, then stored; may be dx_add)
 * Requirements as for moe_combine_backward.
 */
int moe_permute_backward(const void* dx_perm, int dtype, const int32_t* token_row,
                         const void* dx_add, int64_t T, int d, int k, void* dx, void* stream);

/* Workspace bytes moe_route_topk_backward needs. */
size_t moe_route_topk_backward_ws_bytes(int dtype, int64_t T, int d, int E, int k, int flags);

/*
 * moe_route_topk_backward -- gradient of moe_route_topk from dgate, the loss gradient of
 * topk_gate (the choice of experts itself has none):
 *
 *   m = sum_r topk_gate[t][r] * dgate[t][r]
 *   with MOE_RENORM: dlogits[t][topk_idx[t][r]] = topk_gate[t][r] * (dgate[t][r] - m),
 *                    0 for experts that were not chosen
 *   else:            dlogits[t][e] = p_e * ((dgate[t][r] if topk_idx[t][r] == e) - m),
 *                    p = softmax(logits[t])
 *   dx[t] = sum_e dlogits[t][e] * w_router[e];   dw[e] = sum_t dlogits[t][e] * x[t]
 *   dbias[e] = sum_t dlogits[t][e]
 *
 * dgate, topk_gate  device [T][k] float;  topk_idx  device [T][k] int32, distinct in a row
 * logits     device [T][E] float, as moe_route_topk left them (not read, may be NULL, with
 *            MOE_RENORM)
 * x          device [T][d] of `dtype` (not read, may be NULL, when dw is NULL)
 * w_router   device [E][d] of `dtype` (not read, may be NULL, when dx is NULL)
 * dlogits    device [T][E] float, dx  device [T][d] of `dtype`, dw  device [E][d] float,
 * dbias      device [E] float: outputs, each nullable (then not computed)
 * ws         moe_route_topk_backward_ws_bytes(...) bytes, 256-byte aligned
 * flags      MOE_RENORM or 0
 * Products and sums are fp32 in a fixed order (deterministic); with MOE_BF16, dlogits
 * enter dw with all 24 bits and dx, which keeps 8, with 16.  Infinite dlogits give infinite
 * sums; an infinity in x (w_router) gives infinities or, with MOE_BF16, NaN in the sums of dw
 * (dx) that it enters, and in no others.  Outputs must not overlap inputs or each other.
 * Requires T >= 0, 1 <= E <= MOE_MAX_E, 1 <= k <= min(E, MOE_MAX_K), 1 <= d < 2^22 and, for
 * MOE_BF16, d % 8 == 0 (else MOE_ERR_SHAPE); 16-byte aligned matrices where a row is a
 * multiple of 16 bytes.
 */
int moe_route_topk_backward(const float* dgate, const float* topk_gate, const int32_t* topk_idx,
                            const float* logits, const void* x, const void* w_router, int dtype,
                            int64_t T, int d, int E, int k, int flags, float* dlogits, void* dx,
                            float* dw, float* dbias, void* ws, size_t ws_bytes, void* stream);

/*
 * moe_route_topk_backward_aux -- moe_route_topk_backward with a gradient that reaches the gate
 * scores another way (moe_balance_loss_backward's): dlogits_add is added to dlogits before dx, dw
 * and dbias are taken of it.
 *
 * dlogits_add  device [T][E] float, nullable (then it is moe_route_topk_backward); may be dlogits
 * Other arguments, requirements and errors as for moe_route_topk_backward.
 */
int moe_route_topk_backward_aux(const float* dgate, const float* topk_gate, const int32_t* topk_idx,
                                const float* logits, const float* dlogits_add, const void* x,
                                const void* w_router, int dtype, int64_t T, int d, int E, int k,
                                int flags, float* dlogits, void* dx, float* dw, float* dbias, void* ws,
                                size_t ws_bytes, void* stream);

/*
 * Rows in 8-bit integers: a matrix of `cols` columns as
 *   q       int8 [rows][MOE_INT8_COLS(cols)]: codes -127 .. 127, the padding zero
 *   scales  float [rows]: value = q * scale
 * The scale belongs to a token where the rows are activations, to an output channel where they
 * are a weight matrix's.
 */
#define MOE_INT8_COLS(cols) (((int64_t)(cols) + 127) / 128 * 128)

/*
 * moe_quantize_int8 -- a matrix to 8-bit rows.  For every row r:
 *
 *   scales[r] = max(max_i |x[r][i]| / 127, 2^-126)      (fp32 division)
 *   q[r][i]   = x[r][i] / scales[r]                     (fp32 division, then rounded to a
 *                                                        whole number, ties to even)
 *
 * A row that holds an infinity or a NaN gets scale NaN and zero codes: all of it reads as
 * NaN, and no other row does.
 * x       device [rows][cols] of `dtype` (MOE_F32 or MOE_BF16)
 * q, scales  device outputs as above, q 16-byte and scales 4-byte aligned
 * Requires rows >= 0, 1 <= cols < 2^28 (else MOE_ERR_SHAPE).  Results are exact (bitwise
 * reproducible).
 */
int moe_quantize_int8(const void* x, int dtype, int64_t rows, int cols, int8_t* q, float* scales,
                      void* stream);

/*
 * moe_dequantize_int8 -- the values that 8-bit rows hold: y[r][c] = q[r][c] * scales[r] (the
 * fp32 product, rounded to `dtype`).
 * q, scales  device, as above;  y  device [rows][cols] of `dtype` output
 * Requirements as for moe_quantize_int8.
 */
int moe_dequantize_int8(const int8_t* q, const float* scales, int64_t rows, int cols, int dtype,
                        void* y, void* stream);

/* Workspace bytes moe_grouped_ffn_int8 needs (all groups together n_groups, rows of every group,
 * shared ones included, at most cap_rows). */
size_t moe_grouped_ffn_int8_ws_bytes(int64_t cap_rows, int d, int f, int n_groups);

/*
 * moe_grouped_ffn_int8 -- moe_grouped_ffn of experts whose weights are 8-bit rows, over token rows
 * in 8 bits: both products multiply 8-bit integers, a scale for each token and each output
 * channel, and the hidden rows are quantized between them:
 *
 *   for each group s and row p of it, with x the 8-bit row xq[row_token[p]] of scale sx:
 *     a = (W1_s x) sx s13_s[.],  b = (W3_s x) sx s13_s[f + .]     (whole sums, then fp32)
 *     h = SiLU(a) * b                                              (rounded to bf16)
 *     hq, sh = h as moe_quantize_int8 keeps it
 *     y_perm[p] = (W2_s hq) sh s2_s[.]                             (fp32, stored in bf16)
 *
 * xq, x_scale  device [T][MOE_INT8_COLS(d)] and [T]: token rows (moe_quantize_int8, moe_rmsnorm)
 * row_token  device [n_shared T + cap_rows] int32, as for moe_grouped_ffn_rows_shared (entries of
 *            rows that exist lie in [0, T)); NULL: row p reads xq[p]
 * group_offsets, n_groups, n_shared, cap_rows, y_perm  as for moe_grouped_ffn_rows_shared:
 *            n_shared leading groups of T rows each (0 without row_token); y_perm in bf16
 * w13, s13   HOST arrays of n_shared + n_groups device pointers: codes [2f][MOE_INT8_COLS(d)] and
 *            scales [2f], rows 0..f-1 W1 (gate), f..2f-1 W3 (up)
 * w2, s2     the same of [d][MOE_INT8_COLS(f)] and [d]
 * ws         moe_grouped_ffn_int8_ws_bytes(n_shared T + cap_rows, d, f, n_shared + n_groups)
 *            bytes, 256-byte aligned
 * The sums of products are exact.  A token whose scale is NaN makes its own rows of y_perm NaN and
 * no other; so does a row whose h overflows bf16.  Codes are -127 .. 127 (-128 in one operand of a
 * product keeps its sums exact too); padding columns are zero.  The same bits for a row in every
 * batch.
 * Requires d % 8 == 0, d and f at most 2^17, and T * MOE_INT8_COLS(d), 2 f * MOE_INT8_COLS(d)
 * and d * MOE_INT8_COLS(f) below 2^31 (else MOE_ERR_SHAPE), 1 <= n_shared + n_groups <=
 * MOE_MAX_GROUPS, codes and y_perm 16-byte, scales 4-byte aligned.
 */
int moe_grouped_ffn_int8(const int8_t* xq, const float* x_scale, int64_t T, const int32_t* row_token,
                         const int32_t* group_offsets, int n_groups, int n_shared,
                         const int8_t* const* w13, const float* const* s13, const int8_t* const* w2,
                         const float* const* s2, int d, int f, int64_t cap_rows, void* y_perm,
                         void* ws, size_t ws_bytes, void* stream);

/*
 * moe_rmsnorm -- the root-mean-square norm in front of a layer, with the residual's addition
 * before and the normed rows in 8 bits beside:
 *
 *   h[t] = x[t] + residual[t]              (fp32, rounded to `dtype`; x[t] without residual)
 *   rstd[t] = 1 / sqrt(mean_i h[t][i]^2 + eps)
 *   y[t][i] = h[t][i] * rstd[t] * weight[i]              (fp32, rounded to `dtype`)
 *   q[t], scales[t] = y[t], as rounded, as moe_quantize_int8 keeps it (bit for bit)
 *
 * x        device [T][d] of `dtype`;  residual  device [T][d] of `dtype`, nullable
 * weight   device [d] of `dtype`
 * h        device [T][d] of `dtype` output, required with a residual and not written without
 *          one; may be x or residual
 * y        device [T][d] of `dtype` output, nullable; may be x or residual, where h is not the same
 * rstd     device [T] float output, nullable (moe_rmsnorm_backward reads it)
 * q, scales  device [T][MOE_INT8_COLS(d)] and [T] outputs, nullable together
 * Apart from these, outputs must not overlap inputs or each other.
 * Squares are summed in 64 bits, in a fixed order (deterministic).  A row that holds a NaN gives
 * NaN; one that holds an infinity has rstd 0 (NaN at its infinities, zeros beside them, q's row
 * NaN); no other row is touched.  A row of zeros gives zeros (with eps > 0).
 * Requires T >= 0, 1 <= d < 2^22 (else MOE_ERR_SHAPE), eps >= 0 and finite, q 16-byte aligned.
 */
int moe_rmsnorm(const void* x, const void* residual, int dtype, const void* weight, float eps, int64_t T,
                int d, void* h, void* y, float* rstd, int8_t* q, float* scales, void* stream);

/* Workspace bytes moe_rmsnorm_backward needs for dw. */
size_t moe_rmsnorm_backward_ws_bytes(int dtype, int64_t T, int d);

/*
 * moe_rmsnorm_backward -- gradient of moe_rmsnorm's y: from dy, the loss gradient of y, to h (whose
 * gradient is x's and the residual's alike) and to the weight, with n = h rstd:
 *
 *   dh[t][i] = rstd[t] (dy[t][i] weight[i] - n[t][i] mean_j(dy[t][j] weight[j] n[t][j])) + dh_add[t][i]
 *   dw[i]    = sum_t dy[t][i] n[t][i]                     (fp32)
 *
 * dy, h    device [T][d] of `dtype`;  weight  device [d] of `dtype`;  rstd  device [T] float
 * dh_add   device [T][d] of `dtype`, nullable: what reaches h another way (the residual stream)
 * dh       device [T][d] of `dtype` output, nullable (fp32, then stored; may be dh_add)
 * dw       device [d] float output, nullable (zeros when T = 0)
 * ws       moe_rmsnorm_backward_ws_bytes(dtype, T, d) bytes, 256-byte aligned (may be NULL without dw)
 * Apart from dh over dh_add, outputs must not overlap inputs or each other.  Sums are fp32, dw's over
 * more than a range of ceil(T / 512) rows (4 at least) in 64 bits, in a fixed order (deterministic).
 * Requires T >= 0, 1 <= d < 2^22 (else MOE_ERR_SHAPE).
 */
int moe_rmsnorm_backward(const void* dy, const void* h, int dtype, const void* weight, const float* rstd,
                         const void* dh_add, int64_t T, int d, void* dh, float* dw, void* ws,
                         size_t ws_bytes, void* stream);

/* Workspace bytes moe_balance_loss needs. */
size_t moe_balance_loss_ws_bytes(int64_t T, int E);

/*
 * moe_balance_loss -- how far a batch's routing is from even (the popularity skew of Sec. III,
 * Finding 1, as the loss that training holds it down with), with the counts behind it: over the
 * n tokens that count, p[t] = softmax(logits[t]),
 *
 *   n_tokens = #{t : mask[t] != 0}
 *   counts[e] = #{(t, r) : mask[t] != 0, topk_idx[t][r] == e}
 *   prob_sum[e] = sum_{t : mask[t] != 0} p[t][e]
 *   loss = E sum_e (counts[e] / (k n_tokens)) (prob_sum[e] / n_tokens)      (1 when even)
 *
 * logits    device [T][E] float, as moe_route_topk leaves them
 * topk_idx  device [T][k] int32, values in [0, E)
 * mask      device [T] bytes, nullable (every token counts).  Where it is 0 (the padding of a
 *           batch) what logits and topk_idx hold, NaN and any index included, changes no output.
 * counts    device [E] int32, prob_sum  device [E] float, n_tokens  device [1] int32,
 * loss      device [1] float: outputs (all zero when no token counts).  counts, prob_sum and
 *           n_tokens may be summed over GPUs for the loss, and its gradient, of all their tokens.
 * ws        moe_balance_loss_ws_bytes(T, E) bytes, 256-byte aligned
 * A score of -infinity leaves its expert out (p = 0); a counted token needs one finite score.
 * Sums have a fixed order (deterministic).  Requires 0 <= T, T * k < 2^31, 1 <= E <= MOE_MAX_E,
 * 1 <= k <= min(E, MOE_MAX_K).
 */
int moe_balance_loss(const float* logits, const int32_t* topk_idx, const uint8_t* mask, int64_t T, int E,
                     int k, int32_t* counts, float* prob_sum, int32_t* n_tokens, float* loss, void* ws,
                     size_t ws_bytes, void* stream);

/*
 * moe_balance_loss_backward -- gradient of moe_balance_loss to the gate scores (the counts are
 * constants: the choice of experts has no gradient), times `scale`:
 *
 *   dlogits[t][e] = scale E / (k n_tokens^2) p[t][e] (counts[e] - sum_e' p[t][e'] counts[e'])
 *
 * and 0 where mask[t] is 0.
 * logits, mask, counts, n_tokens  device, as above (counts and n_tokens this batch's, or the sums
 *           over several GPUs' batches)
 * dlogits   device [T][E] float output; may be logits
 * Requirements as for moe_balance_loss.
 */
int moe_balance_loss_backward(const float* logits, const uint8_t* mask, const int32_t* counts,
                              const int32_t* n_tokens, int64_t T, int E, int k, float scale,
                              float* dlogits, void* stream);

/* Workspace bytes moe_grad_norm needs (sizes: HOST [n], elements of each gradient). */
size_t moe_grad_norm_ws_bytes(const int64_t* sizes, int n);

/*
 * moe_grad_norm -- the Euclidean norm over all elements of n tensors together:
 *
 *   norm = sqrt(sum_i sum_j grads[i][j]^2)
 *
 * grads     HOST array of n device pointers;  sizes  HOST [n], their elements (0 allowed)
 * dtypes    HOST [n], MOE_F32 or MOE_BF16
 * norm      device [1] float output (0 when there are no elements)
 * ws        moe_grad_norm_ws_bytes(sizes, n) bytes, 256-byte aligned
 * Squares and sums are in 64 bits, in a fixed order (deterministic).  An infinity gives an
 * infinite norm, a NaN a NaN.
 */
int moe_grad_norm(const void* const* grads, const int64_t* sizes, const int* dtypes, int n, float* norm,
                  void* ws, size_t ws_bytes, void* stream);

/*
 * moe_clip_grads -- the same tensors scaled down to a largest norm:
 *
 *   factor = 1 if norm <= max_norm else max_norm / norm   (fp32 division)
 *   out[i][j] = grads[i][j] * factor                      (fp32, rounded to the tensor's type)
 *
 * norm      device [1] float (moe_grad_norm's, or that over several GPUs' tensors)
 * out       HOST array of n device pointers; out[i] may be grads[i], and then nothing is read or
 *           written where the factor is 1.  No other overlap.
 * A NaN norm makes every element NaN, an infinite one makes finite elements zero.
 * Requires max_norm >= 0.
 */
int moe_clip_grads(const void* const* grads, const int64_t* sizes, const int* dtypes, int n,
                   const float* norm, float max_norm, void* const* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOE_H */
