/*
 * buddy.h -- C ABI of the MI355X (gfx950) budget-routed decode step of
 * BUDDY (Budget-Driven Dynamic depth routing, arXiv 2606.09514).
 *
 * One call of buddy_decode_step advances every sequence of a batch by one
 * token:
 *   1. the first block runs for every sequence and appends its K/V row;
 *   2. the KV-aware planner (Sec. 4.3) averages the first layer's K and V
 *      cache rows 0..pos (the new row included) and joins them with the new
 *      token's hidden state after the first block:
 *          z = [mean K | mean V | h]          (din = 2 n_kv hd + d)
 *   3. the Decision Module (Sec. 4.2.3, App. C.1) scores the L-2 routable
 *      blocks, s = W2 act(W1 z + b1) + b2, and fuses the prior,
 *      s' = s + omega p~ (Eq. 2);
 *   4. a deterministic top-k keeps the k_b best blocks of sequence b
 *      (Eq. 2; ties go to the lower block index, NaN ranks last);
 *   5. each routable block runs only on the sequences that selected it
 *      (grouping by mask, App. C.1); a skipped block leaves h unchanged
 *      (Eq. 1) and gets a zero-filled K/V row at pos (Sec. 6, limitations);
 *   6. the last block runs for every sequence.
 * Start layer (the Decision Module placement ablation of Sec. 4.3):
 * with buddy_config.start_layer = S > 1, step 1 runs blocks 0..S-1, the
 * planner reads block S-1's cache and the hidden state after block S-1, and
 * the routable blocks are S..L-2.  L_mid = L - 1 - S routable blocks (L-2
 * for the default S = 1) size every mask, score and budget below.
 * The decoder block is Llama-style (App. C.2): RMSNorm, Q/K/V projection,
 * rotary embedding (rotate-half pairing, angle pos * theta^(-2i/hd)), grouped
 * query attention over the cache including the new row (App. "Background",
 * KV-cache equation), output projection, residual, RMSNorm, SwiGLU MLP,
 * residual.  Projections are bias-free.
 *
 * Conventions shared by every entry point:
 *   - Memory: every pointer marked "device" is memory the caller allocated on
 *     the current HIP device; the caller owns it and keeps it alive until the
 *     enqueued work has finished.  The library never frees caller memory.
 *     A model handle owns only its workspace.
 *   - Precision: weights and the KV cache are stored in the configured dtype
 *     (fp32 or bf16); hidden states, scores and all accumulation are fp32.
 *     New K/V rows are rounded to the storage dtype (nearest, ties to even).
 *   - Layouts are row-major.  Weight matrices are [out][in]:
 *       wqkv     [(n_heads + 2 n_kv_heads) hd][d]    rows q | k | v
 *       wo       [d][n_heads hd]
 *       wgate_up [2 d_ffn][d]                        rows gate | up
 *       wdown    [d][d_ffn]
 *       attn_norm, mlp_norm [d]
 *       Decision Module: w1 [dm_hidden][din], b1 [dm_hidden],
 *                        w2 [L_mid][dm_hidden], b2 [L_mid]  (storage dtype),
 *                        prior [L_mid] fp32 (already normalised p~) or NULL.
 *     KV cache: K and V each [n_layers][max_batch][n_kv_heads][max_ctx][hd].
 *   - Positions: pos[b] (host array) is the number of cached rows of
 *     sequence b before the step; the step writes row pos[b] of every layer
 *     and attends rows 0..pos[b].  The caller advances pos.
 *   - Streams: `stream` is a hipStream_t (NULL = the null stream).  All work
 *     is enqueued on it; outputs are valid once the stream reaches the
 *     enqueued work.  The only host wait is the optional one of the
 *     host-routed launch policy (buddy_set_launch_policy).
 *   - Errors: arguments are validated on the host before anything is
 *     enqueued; on a validation failure nothing is written and a status is
 *     returned.  BUDDY_EDEVICE reports a HIP launch error; its text is
 *     available from buddy_last_error.  Handles are not thread-safe; calls
 *     on one handle must not overlap (they share its workspace).
 */
#ifndef BUDDY_H
#define BUDDY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BUDDY_OK = 0,
    BUDDY_EINVAL = 1,       /* null pointer, bad enum, k or pos out of range */
    BUDDY_ESHAPE = 2,       /* configuration shape the kernels do not support */
    BUDDY_ECAPACITY = 3,    /* batch above max_batch */
    BUDDY_ENOMEM = 4,       /* workspace allocation failed */
    BUDDY_EDEVICE = 5,      /* HIP error (see buddy_last_error) */
    BUDDY_EUNSUPPORTED = 6  /* valid request the library does not implement  */
} buddy_status;

typedef enum { BUDDY_F32 = 0, BUDDY_BF16 = 1 } buddy_dtype;

/* Decision Module activation: SiLU (App. C.1) or exact GELU (erf form). */
typedef enum { BUDDY_ACT_SILU = 0, BUDDY_ACT_GELU_ERF = 1 } buddy_dm_act;

/* Router context (Sec. 4.3 and the feature ablation of Sec. 5): pooled
 * first-layer cache features followed by the newest token's hidden state
 * after the first block.
 *   BUDDY_CTX_KV:   [mean K | mean V | h]  (2 n_kv hd + d values)
 *   BUDDY_CTX_K:    [mean K | h]           (n_kv hd + d)
 *   BUDDY_CTX_V:    [mean V | h]           (the paper's default feature)
 *   BUDDY_CTX_K_PLUS_V: [mean K + mean V | h]
 * Means run over positions 0..pos (the new row included); the Decision
 * Module's first layer has this many inputs (w1 is [dm_hidden][din]). */
typedef enum { BUDDY_CTX_KV = 0, BUDDY_CTX_K = 1, BUDDY_CTX_V = 2, BUDDY_CTX_K_PLUS_V = 3 } buddy_router_ctx;

/* KV treatment of a skipped block.
 *   BUDDY_SKIP_KV_ZERO: the slot at the step's position is zero-filled and
 *     later steps attend to it as an ordinary entry (logit 0, value 0): the
 *     treatment the paper uses (Conclusion, limitations).
 *   BUDDY_SKIP_KV_MASK: the slot is still zero-filled, and the step also
 *     records which blocks ran in the caller's execution map (buddy_kv.exec);
 *     attention leaves out the positions at which a block did not run (the
 *     masking alternative the paper names as future work). */
typedef enum { BUDDY_SKIP_KV_ZERO = 0, BUDDY_SKIP_KV_MASK = 1 } buddy_skip_kv;

typedef struct {
    int32_t n_layers;     /* L >= 2; blocks 0 and L-1 always run          */
    int32_t d_model;      /* multiple of 8; bf16: at most 8192, a multiple
                             of 512 above 4096; fp32: at most 2048        */
    int32_t n_heads;      /* query heads, multiple of n_kv_heads           */
    int32_t n_kv_heads;   /* n_heads / n_kv_heads <= 8                     */
    int32_t head_dim;     /* 64 or 128                                     */
    int32_t d_ffn;        /* multiple of 8; bf16: at most 32768, a multiple
                             of 512 above 4096; fp32: at most 2048        */
    int32_t dm_hidden;    /* Decision Module hidden width, multiple of 8   */
    int32_t dm_act;       /* buddy_dm_act                                  */
    int32_t dtype;        /* buddy_dtype of weights and KV cache           */
    int32_t max_batch;    /* 1..256: workspace and KV cache batch capacity */
    int32_t max_ctx;      /* rows per sequence in the KV cache             */
    float rms_eps;        /* RMSNorm epsilon                               */
    float rope_theta;     /* rotary base                                   */
    int32_t router_ctx;   /* buddy_router_ctx                              */
    int32_t start_layer;  /* S: blocks 0..S-1 always run, the router reads
                             block S-1; 1 <= S <= n_layers - 1, 0 reads as
                             1 (the paper's default)                       */
} buddy_config;

typedef struct {
    const void *attn_norm, *wqkv, *wo, *mlp_norm, *wgate_up, *wdown; /* device */
} buddy_layer_weights;

typedef struct {
    const void *w1, *b1, *w2, *b2;  /* device, storage dtype              */
    const float* prior;             /* device [L_mid] fp32, or NULL       */
    float omega;                    /* prior weight of Eq. 2 (paper: 0.1) */
} buddy_dm_weights;

typedef struct {
    void* k;        /* device [L][max_batch][n_kv][max_ctx][hd], storage dtype */
    void* v;        /* same layout as k                                         */
    uint8_t* exec;  /* device [L][max_batch][max_ctx] execution map, or NULL:
                       exec[l][b][j] != 0 when block l ran for sequence b's
                       token at position j.  Read and written only with
                       BUDDY_SKIP_KV_MASK (required then); the caller fills
                       the rows of cached positions (e.g. all ones after a
                       dense prefill), each step writes every block's entry
                       at its position.  Blocks 0 and L-1 run for every
                       token, so their maps are all ones.                  */
    /* Running-sum pool (optional; both NULL or both set).  The KV-aware
     * planner's context is the mean of the first block's K and V rows
     * 0..pos (Sec. 4.3).  With these arrays the planner keeps, per sequence
     * and KV head, the fp32 sums of rows 0..pool_rows-1 and adds only the
     * rows it has not seen, instead of summing all pos + 1 rows each call:
     *   pool_sum:  device fp32 [max_batch][n_kv][2][hd], K sums then V sums
     *   pool_rows: device int32 [max_batch][n_kv], rows held in pool_sum
     * A call at position p adds rows pool_rows..p-1 (rows older than the
     * step, which the step does not rewrite) and sets pool_rows = p; row p
     * enters that call's mean without entering the sums, so repeating a step
     * at the same position stays exact.  pool_rows > p starts the sums over;
     * where pool_rows is 0 the contents of pool_sum are not read.
     * The caller zeroes pool_rows before first use and again for a slot
     * whenever it rewrites that slot's cached rows below pool_rows;
     * buddy_prefill does so itself for the slots it fills.  Sums are in a
     * different order than a fresh scan: equal up to fp32 rounding.       */
    float* pool_sum;
    int32_t* pool_rows;
} buddy_kv;

typedef struct buddy_model buddy_model;

/* Creates a model handle on the current HIP device.  `layers` holds
 * n_layers entries; the weight pointers are copied, the weights are not.
 * Allocates the handle's workspace (sized by max_batch and max_ctx).
 * Returns BUDDY_OK and *out, or an error status with *out = NULL:
 * BUDDY_ESHAPE for a shape outside the limits of the fields above (the
 * query width n_heads * head_dim within those of d_ffn, the router input
 * of at most 20480 elements), BUDDY_ECAPACITY for max_batch or max_ctx. */
buddy_status buddy_model_create(const buddy_config* cfg, const buddy_layer_weights* layers,
                                const buddy_dm_weights* dm, buddy_model** out);

/* Waits for the device, then frees the handle's workspace.  NULL is a no-op. */
void buddy_model_destroy(buddy_model* m);

/* KV-aware planner plus Decision Module (Sec. 4.3, Sec. 4.2.3, Eq. 2 fusion)
 * without routing: for b < B, pools the first layer's K/V rows 0..pos[b] of
 * kv (the newest token's row already written) with h_new[b] (device
 * [B][d] fp32) and writes s' to scores_out (device [B][L_mid] fp32).
 * pos: host [B].  B = 0 is a no-op. */
buddy_status buddy_pool_route(buddy_model* m, const buddy_kv* kv, const int32_t* pos,
                              const float* h_new, int32_t B, float* scores_out,
                              void* stream);

/* buddy_pool_route for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * allocation): the same planner and Decision Module scores, bit for bit, with
 * no model handle and no allocation of any kind.  The configuration and the
 * Decision Module weights come as arguments (cfg as for buddy_model_create;
 * cfg->max_batch is the batch capacity of the KV cache layout); kv, pos,
 * h_new, B, scores_out and stream as for buddy_pool_route.  Every buffer
 * the kernels need beyond the inputs and outputs (positions, pool partial
 * sums, the Decision Module's hidden activations, scores) lives in a scratch
 * array that the library holds once per device for the life of the
 * process (12 MiB, 8 of them counted here; no part of it needs to start at
 * zero).  That limits a call to
 * pieces of 4 B bytes (three of them), 4, 4 B L_mid + 4, 4 B dm_hidden and
 * 8 B n_kv_heads head_dim splits bytes, each rounded up to 256, totalling at
 * most 8 MiB, where splits, the pool's position splits, is 1 with
 * kv->pool_sum and otherwise min(ceil(1024 / (B n_kv_heads)),
 * ceil((max pos + 1) / 64), ceil(max_ctx / 64), 64), at least 1 (e.g. a
 * Llama-3-8B shape fits any batch up to 256; a 40-KV-head, head_dim 128
 * shape fits batches up to about 190).  Beyond it the call returns
 * BUDDY_ECAPACITY and writes nothing.  Calls on one GPU
 * share its array: calls that overlap on a device (other streams or host
 * threads) race and must be ordered by the caller.  Errors as for
 * buddy_model_create and buddy_pool_route; BUDDY_EDEVICE when the scratch
 * address cannot be obtained on the current device. */
buddy_status buddy_pool_route_noalloc(const buddy_config* cfg, const buddy_dm_weights* dm,
                                      const buddy_kv* kv, const int32_t* pos, const float* h_new,
                                      int32_t B, float* scores_out, void* stream);

/* Deterministic per-row top-k (Eq. 2): mask_out[b][i] = 1 iff layer i is
 * among the k[b] largest of scores[b][0..n) under (score desc, index asc,
 * NaN last).  scores: device [B][n] fp32; k: host [B], 0 <= k[b] <= n;
 * mask_out: device [B][n] uint8; 1 <= n <= 255; B <= 65535.  Needs no
 * model handle. */
buddy_status buddy_select_topk(const float* scores, const int32_t* k, int32_t B, int32_t n,
                               uint8_t* mask_out, void* stream);

/* Batch-level path grouping (the Conclusion names grouping requests by
 * their path among its open questions): orders the B sequences of a batch
 * by route and marks the groups of identical routes, e.g. to serve each
 * group as one sub-batch with route_override.  mask: device [B][n] uint8,
 * nonzero = the block runs (as buddy_decode_step's mask_out); routes
 * compare lexicographically in block order with a skipped block before a
 * run one, and equal routes keep their batch order, so the result is
 * unique.  perm_out: device int32 [B], the sequence at each position;
 * starts_out: device int32 [B + 1], the first position of group g at
 * [g] and B after the last group; n_groups_out: device int32 [1].
 * 1 <= n <= 255, B <= 1024; B = 0 is a no-op.  Needs no model handle. */
buddy_status buddy_group_by_route(const uint8_t* mask, int32_t B, int32_t n, int32_t* perm_out,
                                  int32_t* starts_out, int32_t* n_groups_out, void* stream);

/* One budget-routed decode step for B sequences (steps 1-6 above).
 *   hidden: device [B][d] fp32; input H_0 of the new token, overwritten
 *           with the last block's output H_L (no final norm).
 *   pos:    host [B]; 0 <= pos[b] < max_ctx.
 *   k:      host [B]; 0 <= k[b] <= L_mid routable blocks to run.
 *   skip_kv: buddy_skip_kv; BUDDY_SKIP_KV_MASK needs kv->exec
 *           (BUDDY_EINVAL otherwise).
 *   route_override: device [B][L_mid] uint8 (nonzero = run) or NULL; when
 *           given, the planner and Decision Module are not run, k is
 *           ignored and scores_out is left untouched.
 *   mask_out: device [B][L_mid] uint8 or NULL: the mask that was executed.
 *   scores_out: device [B][L_mid] fp32 or NULL: s' of step 3.
 * B = 0 is a no-op; B > max_batch gives BUDDY_ECAPACITY. */
buddy_status buddy_decode_step(buddy_model* m, const buddy_kv* kv, float* hidden,
                               const int32_t* pos, const int32_t* k, int32_t B,
                               int32_t skip_kv, const uint8_t* route_override,
                               uint8_t* mask_out, float* scores_out, void* stream);

/* Budget Predictor head (Sec. 4.4): a categorical policy over k = 1..L_mid
 * from the same router context as the Decision Module, read as the Decision
 * Module's form (the paper does not give its layers): logits = w2 act(w1 z
 * + b1) + b2 with the Decision Module's activation. */
typedef struct {
    const void *w1, *b1, *w2, *b2;  /* device, storage dtype: w1 [hidden][din],
                                       b1 [hidden], w2 [L_mid][hidden], b2 [L_mid] */
    int32_t hidden;                 /* multiple of 8                          */
} buddy_predictor_weights;

/* Attaches a Budget Predictor head to the handle (the pointers are copied,
 * the weights are not; they must outlive the handle), or detaches it with
 * p == NULL.  Waits for the device, then allocates the head's workspace.
 * Errors: BUDDY_EINVAL (null pointers, hidden not a positive multiple of 8,
 * no routable block), BUDDY_ESHAPE (hidden too wide), BUDDY_ENOMEM. */
buddy_status buddy_set_budget_predictor(buddy_model* m, const buddy_predictor_weights* p);

/* Planner and Budget Predictor only (steps 3 and 4 with the predictor's
 * output layer): k_out device [B] int32 receives k_hat = 1 + argmax of the
 * logits (fp32; the smaller k on equal logits; the budget is b_hat =
 * (k_hat + 2) / L); logits_out device [B][L_mid] fp32 or NULL.  pos and h_new
 * as for buddy_pool_route.  BUDDY_EINVAL without an attached predictor. */
buddy_status buddy_predict_budget(buddy_model* m, const buddy_kv* kv, const int32_t* pos,
                                  const float* h_new, int32_t B, int32_t* k_out,
                                  float* logits_out, void* stream);

/* buddy_decode_step without budgets: each sequence's k is the Budget
 * Predictor's k_hat from the step's own router context, then the step runs
 * as buddy_decode_step with that k.  k_out: device [B] int32 or NULL.
 * BUDDY_EINVAL without an attached predictor. */
buddy_status buddy_decode_step_auto(buddy_model* m, const buddy_kv* kv, float* hidden,
                                    const int32_t* pos, int32_t B, int32_t skip_kv,
                                    int32_t* k_out, uint8_t* mask_out, float* scores_out,
                                    void* stream);

/* Routed prefill of B prompts into cache rows 0..len[b]-1 (one route per
 * prompt; the Reuse setting of Sec. 5 keeps decoding on the prefill's
 * decision, so the prefill itself is routed).  The first block (blocks
 * 0..S-1 with a start layer S) runs over
 * every prompt token; the planner and Decision Module decide the route once
 * per prompt at its last token (as a decode step at position len[b]-1
 * would), unless route_override gives it; each selected block then runs
 * causally over the prompt, and every skipped block's K/V rows 0..len[b]-1
 * are zero-filled (with BUDDY_SKIP_KV_MASK also marked in kv->exec).
 *   hidden: device [B][t_stride][d] fp32, the prompt tokens' inputs,
 *           overwritten with their last-block outputs (rows t >= len[b]
 *           untouched).
 *   len:    host [B], 1 <= len[b] <= min(t_stride, max_ctx).
 *   k:      host [B] budgets 0..L_mid (ignored with route_override).
 *   route_override, mask_out, scores_out: as buddy_decode_step.
 * Rows of all prompts together: B * t_stride <= 65535.  Grows the handle's
 * prefill workspace when needed: for each row of the largest call so far
 * 8 n_heads head_dim + 4 d_ffn bytes of activations, 8 times the widest of
 * d_model, d_ffn, n_heads head_dim and the router input in staged ones,
 * 12 n_layers of lists and, in bf16 from 64 rows on, 8 d_model bytes of partial
 * sums or, if that is more and the device has room, those of up to eight K
 * splits (at most 192 KiB a row and 128 MiB in all).  Returns after the device has finished
 * (the host waits for the route to build the per-block token lists). */
buddy_status buddy_prefill(buddy_model* m, const buddy_kv* kv, float* hidden, int32_t t_stride,
                           const int32_t* len, const int32_t* k, int32_t B, int32_t skip_kv,
                           const uint8_t* route_override, uint8_t* mask_out, float* scores_out,
                           void* stream);

/* How buddy_decode_step launches the routable blocks.
 *   BUDDY_LAUNCH_DEVICE_ROUTED: everything is enqueued without waiting; every
 *     routable block is launched and its kernels read the routed row count
 *     on the device, so a block nobody selected costs only empty launches.
 *     The call never blocks the host (suitable for stream capture).
 *   BUDDY_LAUNCH_HOST_ROUTED: after the router, the call waits for the
 *     per-block routed counts (written by the device to mapped pinned host
 *     memory owned by the handle) and launches only the blocks some sequence
 *     runs, with grids sized to the routed rows.  The host blocks until the
 *     first block and the router have run; a device error during that wait
 *     is reported (BUDDY_EDEVICE) within about 0.1 s, and no answer within a
 *     minute also ends it with BUDDY_EDEVICE.
 *   BUDDY_LAUNCH_AUTO (default): host-routed when B <= 16 and not every
 *     sequence runs every block, device-routed otherwise, and always
 *     device-routed while the stream is being captured into a graph.
 * Under stream capture (hipStreamBeginCapture) an explicit host-routed
 * policy makes buddy_decode_step and buddy_decode_step_auto return
 * BUDDY_EINVAL with nothing enqueued, and buddy_prefill, which waits for its
 * route on the host, always returns BUDDY_EINVAL.  A captured step replays
 * with the positions and budgets it was captured with (they are kernel
 * arguments). */
typedef enum {
    BUDDY_LAUNCH_AUTO = 0,
    BUDDY_LAUNCH_DEVICE_ROUTED = 1,
    BUDDY_LAUNCH_HOST_ROUTED = 2
} buddy_launch_policy;

/* Sets the launch policy of a handle; BUDDY_EINVAL for an unknown policy. */
buddy_status buddy_set_launch_policy(buddy_model* m, int32_t policy);

/* Output tile of the prefill's tiled projections (bf16 weights, many prompt
 * tokens).
 *   BUDDY_GEMM_TILE_AUTO (default): the tile (128 x 128, 128 x 256 or
 *     256 x 256, the last with a final, partly filled round on 128 x 256
 *     ones) and K split of least estimated time for the projection's weight
 *     rows and prompt tokens.  Up to 1536 tokens any projection may split K
 *     in up to eight parts; beyond, the residual-add projections (O, down)
 *     in two.  The parts' sums are added in a fixed order;
 *   BUDDY_GEMM_TILE_128, BUDDY_GEMM_TILE_256: always that tile (weight
 *     rows x token rows), K never split;
 *   BUDDY_GEMM_TILE_256_SPLIT: 256 x 256, K split in two for the
 *     residual-add projections (on 128 x 128 tiles where K is not a multiple
 *     of 128).
 * The tiles without a split give the same results bit for bit; a split adds
 * its two to eight partial sums, a different rounding order. */
typedef enum {
    BUDDY_GEMM_TILE_AUTO = 0,
    BUDDY_GEMM_TILE_128 = 1,
    BUDDY_GEMM_TILE_256 = 2,
    BUDDY_GEMM_TILE_256_SPLIT = 3
} buddy_gemm_tile;

/* Sets the tile choice of a handle; BUDDY_EINVAL for an unknown value. */
buddy_status buddy_set_gemm_tile(buddy_model* m, int32_t tile);

/* Kernels of a decoder block, for buddy_set_timing_events. */
typedef enum {
    BUDDY_KERNEL_QKV = 0,        /* RMSNorm + QKV projection + rotary + KV append */
    BUDDY_KERNEL_ATTENTION = 1,  /* split-K decode attention                      */
    BUDDY_KERNEL_O_PROJ = 2,     /* output projection + residual                  */
    BUDDY_KERNEL_GATE_UP = 3,    /* RMSNorm + gate/up projection + SwiGLU         */
    BUDDY_KERNEL_DOWN = 4,       /* down projection + residual                    */
    BUDDY_KERNEL_ATTN_MERGE = 5  /* merge of the attention's position-chunk partials
                                    (no launch when one chunk covers every row:
                                    the events then mark an empty interval)      */
} buddy_kernel;

/* Measurement hook.  For the next n calls of buddy_decode_step on this
 * handle, call i times `kernel` in block `layer`: start[i] and stop[i] are
 * recorded at the dispatch begin and end of that kernel's main launch (the
 * projection itself, not the activation staging of the batched path; the
 * attention score kernel, not the chunk merge), the interval a kernel trace
 * reports.  If the block does not run, both are recorded back to back on the
 * stream at that point of the step.  start and stop are
 * arrays of n hipEvent_t handles that the caller created and keeps alive
 * until the calls have run; the handle copies the arrays.  n = 0 turns the
 * hook off.  Errors: BUDDY_EINVAL for a bad kernel, layer or n < 0, or null
 * arrays with n > 0. */
buddy_status buddy_set_timing_events(buddy_model* m, int32_t kernel, int32_t layer,
                                     void* const* start, void* const* stop, int32_t n);

/* Kinds of raw per-layer importance indicator (App. B, direction
 * unification): the skip-induced perplexity increase PPL_skip - PPL_full,
 * a Taylor / Fisher / gradient-norm score, or the cosine similarity of a
 * block's input and output. */
typedef enum {
    BUDDY_PRIOR_DELTA_PPL = 0,
    BUDDY_PRIOR_TAYLOR = 1,
    BUDDY_PRIOR_COSINE = 2
} buddy_prior_kind;

/* Offline prior normalisation (App. B, then Eq. 2), host code.  raw: host
 * [n] indicator values of the n routable layers (finite); prior_out: host
 * [n] fp32, the prior p~ for buddy_dm_weights.prior (copy it to the device).
 * Steps over the n layers: larger-is-more-important (max(0, x) for the
 * perplexity and Taylor kinds, 1 - x for cosine), log(1 + x) for the
 * perplexity and Taylor kinds, robust z = (x - median) / (IQR + 1e-6) with
 * linearly interpolated quartiles, clipped to [-winsor, winsor] when winsor
 * > 0, rank normalisation u = (1 + rank) / (n + 1) with 0-based ranks and
 * ties at their mean rank, and p~ = (u - mean u) / (population std + 1e-6).
 * Errors: BUDDY_EINVAL for null pointers, n < 1, an unknown kind, a negative
 * or non-finite winsor, or a non-finite raw value (nothing written). */
buddy_status buddy_prior_normalize(const float* raw, int32_t n, int32_t kind, float winsor,
                                   float* prior_out);

/* Budget to routable-block count, k = round(b L) - 2 (Eq. 2), halves away
 * from zero, limited to [0, L-2]; -1 when b is outside (0, 1].  This is the
 * default start layer's count; with start layer S the blocks 0..S-1 and
 * L-1 always run and k = round(b L) - (S + 1), which callers compute. */
int32_t buddy_budget_to_k(float b, int32_t n_layers);

/* ------------------------------------------------------------------------
 * Serving from a paged cache of 4-bit keys and values.
 *
 * The calls below need no model handle and keep no state: a scheduler holds
 * the page tables, the pool and the workspaces in device memory and runs, for
 * each step, buddy_release_pages and buddy_plan_pages once, then for each
 * layer buddy_kv4_append_qkv on the QKV projection's output and
 * buddy_kv4_attention.  Nothing in a call waits for the device or allocates,
 * and lengths, positions, slots and tables are read on the device, so a
 * captured step replays with whatever they then hold.  Calls on different
 * streams or host threads are independent of each other as far as the memory
 * they are given is.  buddy_decode_step, buddy_prefill and buddy_pool_route
 * read the flat cache of buddy_kv and not this one.
 *
 * Cache format: elements are e2m1 (4 bits: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and
 * their negatives), 32 neighbours of a row share a scale of 8 bits, the power
 * of two 2^(code - 127) (code 255: the 32 are NaN): 4.25 bits an element
 * against the 16 of a bf16 cache.  A page holds page_rows rows of every KV
 * head; a row of the pool is named by its slot, page * page_rows + row.
 * Written groups take the least exponent e with amax <= 7 * 2^e (within
 * -125..125) and round to nearest, ties to even; an infinity or NaN makes its
 * group NaN.
 *
 * Page ids and slots are read on the device and checked there against the
 * pool: a slot outside it is not written or read (its output row is left as
 * it was), and attention leaves out the rows of a page outside it.  Arrays of
 * heads and codes must be 16-byte aligned, their row strides multiples of 16
 * bytes (BUDDY_EINVAL otherwise); other strides between rows are free.  A call
 * takes up to 2^24 rows of heads (BUDDY_ECAPACITY).
 */

typedef struct {
    uint8_t *k, *v;              /* device [n_pages][n_kv_heads][page_rows][head_dim / 2]
                                    codes, element 2 i in the low half of byte i       */
    uint8_t *k_scale, *v_scale;  /* device [n_pages][n_kv_heads][head_dim / 32][page_rows] */
    int32_t n_pages;             /* n_pages * page_rows <= 2^31 - 1                      */
    int32_t page_rows;           /* 16, 32, 64, 128 or 256                               */
    int32_t n_kv_heads;          /* 1..1024                                              */
    int32_t head_dim;            /* 64 or 128                                            */
} buddy_kv4;

/* Pages, positions and slots for the rows that B requests are about to add
 * (a scheduler's step; beside buddy_select_topk and buddy_group_by_route).
 *   len:    device [B], rows that each request has cached;
 *   n_new:  device [B], rows it adds (0: none);
 *   table:  device [B][max_pages], the request's pages in order; the entries
 *           of the pages it holds, ceil(len / page_rows), are read, those of
 *           new pages written, the others left as they were;
 *   ring:   device [n_pages], the free pages: ring_state[1] entries from
 *           entry ring_state[0] on (modulo n_pages); new pages are taken from
 *           the front, for the requests in order.
 * Written:
 *   ring_state_out: device [2], the ring after the call (may be ring_state);
 *   len_out:  device [B], len + n_new (may be len);
 *   cu_rows:  device [B + 1], rows of request b at cu_rows[b]..cu_rows[b + 1];
 *   pos, slots: device [n_rows], each row's position and slot; -1 behind the
 *           last request's rows;
 *   refused: device [B], 0 or why a request adds nothing this step (its rows
 *           count as 0 then): 1 lengths that are negative or pass max_pages
 *           pages, 2 too few free pages, 3 too few row entries.  2 and 3 are
 *           decided in order: a request is refused when all pages (for one
 *           that needs pages) or rows asked for up to it, those of refused
 *           requests of valid lengths included, pass what there is.
 * B <= 1024, page_rows as buddy_kv4, n_rows < 2^30; B = 0 is a no-op. */
buddy_status buddy_plan_pages(const int32_t* len, const int32_t* n_new, int32_t B, int32_t page_rows,
                              int32_t* table, int32_t max_pages, const int32_t* ring,
                              int32_t n_pages, const int32_t* ring_state, int32_t* ring_state_out,
                              int32_t* len_out, int32_t* cu_rows, int32_t* pos, int32_t* slots,
                              int32_t n_rows, uint8_t* refused, void* stream);

/* Gives the pages of ended requests back: for each b with done[b] != 0, in
 * order, its ceil(len[b] / page_rows) pages go to the end of the ring and
 * len_out[b] = 0; for the others len_out[b] = len[b].  len_out may be len,
 * ring_state_out ring_state.  A length that is negative or passes max_pages
 * pages gives nothing back.  Limits as buddy_plan_pages. */
buddy_status buddy_release_pages(const int32_t* len, const uint8_t* done, int32_t B,
                                 int32_t page_rows, const int32_t* table, int32_t max_pages,
                                 int32_t* ring, int32_t n_pages, const int32_t* ring_state,
                                 int32_t* ring_state_out, int32_t* len_out, void* stream);

/* How queries and keys are normed and rotated: y = x * rsqrt(mean(x^2) +
 * rms_eps) * w over each head where the side has weights, then the first
 * rope_dim elements rotated in pairs by pos * rope_theta^(-2 i / rope_dim).
 * All arithmetic in fp32, angles reduced in fp64, one rounding at the end. */
typedef struct {
    int32_t n_heads, n_kv_heads;      /* 1..1024 each                             */
    int32_t head_dim;                 /* 64 or 128                                */
    int32_t rope_dim;                 /* 0..head_dim, a multiple of 16; 0: none   */
    int32_t interleaved;              /* 0: pairs (i, i + rope_dim / 2);
                                         nonzero: pairs (2 i, 2 i + 1)            */
    int32_t dtype;                    /* buddy_dtype of all arrays and weights    */
    float rms_eps, rope_theta;
    const void *q_norm, *k_norm;      /* device [head_dim], or NULL: not normed   */
} buddy_qk_form;

/* Norms and rotates n_rows rows of queries and keys in one pass.  q, k and
 * the outputs: device rows [heads][head_dim], row strides in elements; an
 * output may be its input.  pos: device [n_rows]; rows with pos < 0 are left
 * as they were.  n_rows = 0 is a no-op. */
buddy_status buddy_qk_norm_rope(const buddy_qk_form* f, const void* q, int64_t q_stride,
                                const void* k, int64_t k_stride, const int32_t* pos, int32_t n_rows,
                                void* q_out, int64_t q_out_stride, void* k_out,
                                int64_t k_out_stride, void* stream);

/* Writes rows of finished keys and values into their slots of the cache.
 * k, v: device rows [n_kv_heads][head_dim] of dtype; slots: device [n_rows],
 * no slot twice (the slot's row would be a mixture).  n_rows = 0 is a no-op. */
buddy_status buddy_kv4_append(const buddy_kv4* cache, int32_t dtype, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, const int32_t* slots, int32_t n_rows,
                              void* stream);

/* buddy_qk_norm_rope and buddy_kv4_append in one pass over a projection's
 * output: queries normed and rotated to q_out (which may be q), keys normed,
 * rotated and written into the cache without a rounding between, values
 * written into the cache.  A row with pos < 0 is left out altogether. */
buddy_status buddy_kv4_append_qkv(const buddy_kv4* cache, const buddy_qk_form* f, const void* q,
                                  int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                  int64_t v_stride, const int32_t* pos, const int32_t* slots,
                                  int32_t n_rows, void* q_out, int64_t q_out_stride, void* stream);

/* Cache rows back as values, of either dtype (e.g. to move a sequence to the
 * flat cache of buddy_kv).  Every 4-bit value is a bf16 number: exact. */
buddy_status buddy_kv4_read(const buddy_kv4* cache, const int32_t* slots, int32_t n_rows, int32_t dtype,
                            void* k_out, int64_t k_stride, void* v_out, int64_t v_stride, void* stream);

/* Grouped-query attention of new rows over the paged cache, which holds them
 * already: row i of sequence b (of its n = cu_rows[b + 1] - cu_rows[b] rows)
 * stands at position p = len[b] - n + i and attends the cached rows j <= p
 * with mask[b][j] != 0; out = sum_j softmax_j(scale * q . k_j) v_j, zeros for
 * a row that attends nothing.  One row per sequence is a decode step, more
 * are a prompt or a piece of one.  Scores, statistics and sums are fp32; the
 * weights exp(s - max) enter the product with V as two bf16 parts (16 bits),
 * for fp32 calls as three (24), and in bf16 calls with more than 64 columns
 * (max_rows times the query heads of a KV head) may be rounded to bf16, as
 * the output is: buddy_kv4_attention_form tells.  All sequences of a call are
 * run alike: a step of prompts beside many single tokens is faster as two
 * calls, each over a range of the sequences (table, len and cu_rows from its
 * first on, q and out whole). */
typedef struct {
    const void* q;           /* device [n_rows] rows [n_heads][head_dim]          */
    void* out;               /* device, the same form; rows outside cu_rows[0]..
                                cu_rows[B] are left as they were                  */
    int64_t q_stride, out_stride; /* elements from row to row                     */
    int32_t dtype;           /* buddy_dtype of q and out                          */
    int32_t n_heads;         /* a multiple of n_kv_heads, at most 16 times it     */
    int32_t n_rows;          /* rows that q and out hold                          */
    int32_t max_rows;        /* at least the rows of any sequence, 1 or more      */
    int32_t max_len;         /* at least the length of any sequence (a smaller
                                bound costs speed, not rows)                      */
    int32_t max_pages;       /* table entries of a sequence                       */
    const int32_t* table;    /* device [B][max_pages]; lengths past max_pages
                                pages count as max_pages pages                    */
    const int32_t* len;      /* device [B], cached rows, the new ones included    */
    const int32_t* cu_rows;  /* device [B + 1]                                    */
    const uint8_t* mask;     /* device [B] rows of mask_stride >= max_len bytes, or
                                NULL: every row (as buddy_kv.exec: which tokens ran
                                the block); positions from mask_stride on count as 0 */
    int64_t mask_stride;
    float scale;             /* 1e-30 to 1e30 in magnitude                        */
    void* workspace;         /* device, 16-byte aligned; contents need no
                                preparation; one for each call that may run at
                                the same time (two captured graphs that may)      */
    size_t workspace_bytes;  /* at least buddy_kv4_attention_workspace            */
} buddy_kv4_attn;

/* Bytes of workspace that buddy_kv4_attention needs for B sequences with
 * a's n_heads, n_rows, max_rows and max_len (its pointers are not read);
 * 0 for arguments that the call refuses.  Those of a step are enough for every
 * step of the same n_heads, n_kv_heads and head_dim whose n_rows and max_len
 * are not larger, so one workspace serves a batch that shrinks.  At most
 * 2^17 * (head_dim + 2) * 4 bytes. */
size_t buddy_kv4_attention_workspace(const buddy_kv4* cache, const buddy_kv4_attn* a, int32_t B);

/* How buddy_kv4_attention runs a call for B sequences with a's dtype, n_heads,
 * n_rows, max_rows and max_len (its pointers are not read): the bf16 parts in
 * which weights enter the product with V (1, 2 or 3), for every sequence of
 * the call, and the chunks that the longest sequence's rows are split into.
 * Either pointer may be NULL; both are host memory. */
buddy_status buddy_kv4_attention_form(const buddy_kv4* cache, const buddy_kv4_attn* a, int32_t B,
                                      int32_t* weight_parts, int32_t* chunks);

/* B <= 1024; B = 0 and n_rows = 0 are no-ops. */
buddy_status buddy_kv4_attention(const buddy_kv4* cache, const buddy_kv4_attn* a, int32_t B, void* stream);

/* ------------------------------------------------------------------------
 * The rest of a served block, and the end of a step.
 *
 * Around buddy_kv4_append_qkv and buddy_kv4_attention a block adds to its
 * residual stream and norms it (buddy_add_rmsnorm), projects (buddy_mx8_linear)
 * and gates (buddy_mx8_quantize); requests may bring low-rank adapters for a
 * projection (buddy_lora_plan once a step, buddy_lora_add behind each adapted
 * projection); the step ends with a token for each sequence (buddy_sample).
 * The calls need no model handle and keep no state, wait for nothing and
 * allocate nothing; positions, adapter ids, plans and sampling parameters are
 * read on the device, so a captured step replays with whatever they then hold.
 * buddy_decode_step keeps its own norms and projections.
 *
 * 8-bit rows: elements are e4m3 (1 sign, 4 exponent, 3 mantissa bits, up to
 * 448, no infinities), 32 neighbours of a row share a scale of 8 bits, the
 * power of two 2^(code - 127) (code 255: the 32 are NaN); the last group of a
 * row may be short.  8.25 bits an element.  Written groups take the least
 * exponent e with amax <= 448 * 2^e (within -117..120) and round to nearest,
 * ties to even; an infinity or NaN makes its group NaN.
 *
 * Arrays of rows are 16-byte aligned, their row strides multiples of 16 bytes
 * (BUDDY_EINVAL otherwise); other strides between rows are free.  A call takes
 * up to 2^24 rows, of projections (rows of weights, too), adapters and their
 * plans 2^20 (BUDDY_ECAPACITY).  n_rows = 0 is a no-op.  What a call
 * writes overlaps nothing that it reads, but where that is said.
 */

typedef struct {
    uint8_t* codes;        /* device [n_rows] rows of width codes                  */
    uint8_t* scales;       /* device [n_rows] rows, byte g for elements 32 g .. + 31;
                              the other bytes of a row are neither read nor written
                              to any effect                                        */
    int64_t code_stride;   /* bytes from row to row, a multiple of 16, >= width     */
    int64_t scale_stride;  /* a multiple of 16, >= 16 ceil(width / 512)             */
    int32_t n_rows;
    int32_t width;         /* a multiple of 16, up to 2^20                          */
} buddy_mx8;

/* h' = h + delta, y = h' * rsqrt(mean(h'^2) + rms_eps) * weight, row by row:
 * the residual's addition and the norm before the next projection.  The sum is
 * taken in fp32, stored in h's type and normed as stored; statistics and
 * products are fp32, y is rounded once, to dtype or to 8-bit rows (or to each
 * of both). */
typedef struct {
    int32_t n_rows;
    int32_t width;           /* a multiple of 16, up to 32768                       */
    int32_t hidden_dtype;    /* buddy_dtype of h and h_out                          */
    int32_t dtype;           /* buddy_dtype of delta, weight and y                  */
    const void* h;           /* device rows                                         */
    const void* delta;       /* device rows, or NULL: h' = h                        */
    const void* weight;      /* device [width]                                      */
    void* h_out;             /* device rows, may be h with h's stride; NULL without
                                delta                                               */
    void* y;                 /* device rows, or NULL                                */
    const buddy_mx8* y_mx8;  /* n_rows rows of width, or NULL; y or y_mx8 is given  */
    int64_t h_stride, delta_stride, h_out_stride, y_stride;   /* elements           */
    const int32_t* pos;      /* device [n_rows]: rows with pos < 0 are left as they
                                were (padding); or NULL: all rows                   */
    float rms_eps;
} buddy_norm;
buddy_status buddy_add_rmsnorm(const buddy_norm* a, void* stream);

/* Rows of fp32 or bf16 values as 8-bit rows: x, or with gate SiLU(gate) * x
 * in fp32.  x, gate: device rows of out->width elements, strides in elements;
 * pos as buddy_norm (or NULL). */
buddy_status buddy_mx8_quantize(const buddy_mx8* out, int32_t dtype, const void* x, int64_t x_stride,
                                const void* gate, int64_t gate_stride, const int32_t* pos, void* stream);

/* 8-bit rows back as values.  An e4m3 value times its scale is a bf16 number:
 * exact, but that 2^128 (which magnitudes from 2^128 - 2^122 on round to) comes
 * back infinite, as does what scales that buddy_mx8_quantize does not write
 * take past the range; values below it are rounded. */
buddy_status buddy_mx8_read(const buddy_mx8* m, int32_t dtype, void* out, int64_t out_stride, void* stream);

/* out[r][n] = sum_k x[r][k] w[n][k]: a projection of 8-bit rows by 8-bit
 * weights [out features][in features] (buddy_mx8_quantize of the weight
 * matrix).  x->width = w->width; out: device rows of w->n_rows elements of
 * dtype, any alignment of the type, stride in elements.  bf16 outputs: fp32
 * sums of the matrix unit's 8-bit products, which within each 8 neighbours
 * keep at least 13 bits behind the largest product; fp32 outputs: all products
 * and sums in fp32, at less than half the rate, of the elements as
 * buddy_mx8_read gives them in bf16 (one of 2^128 is infinite; of scales that
 * buddy_mx8_quantize does not write, elements past bf16's range are infinite or
 * lose bits). */
buddy_status buddy_mx8_linear(const buddy_mx8* x, const buddy_mx8* w, int32_t dtype, void* out,
                              int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace that buddy_mx8_linear needs for x->n_rows rows or fewer
 * with weights of w's n_rows and width (pointers are not read), either dtype;
 * 0 for sizes that the call refuses.  16-byte aligned, contents need no
 * preparation; one for each call that may run at the same time. */
size_t buddy_mx8_linear_workspace(const buddy_mx8* x, const buddy_mx8* w);

/* How buddy_mx8_linear runs a call with these rows, weights and dtype (pointers
 * are not read, strides are). */
typedef struct {
    int32_t form;          /* 0: weights straight to registers, for few rows and for
                              rows 8 MB apart or more; 1: up to 128 rows of x for a
                              pass over the weights, both through LDS; 2: tiles of
                              256 x 256                                           */
    int32_t row_tiles;     /* of 16 rows of x, of a workgroup                      */
    int32_t weight_tiles;  /* of 16 rows of weights, of a workgroup                */
    int32_t parts;         /* of k, of a workgroup: each has wavefronts of its own */
    int32_t splits;        /* of k, over workgroups, joined by a further launch    */
} buddy_mx8_form;
buddy_status buddy_mx8_linear_form(const buddy_mx8* x, const buddy_mx8* w, int32_t dtype, buddy_mx8_form* form);

/* Low-rank adapters of one projection, all of one rank (a smaller one filled
 * up with zeros). */
typedef struct {
    const void* a;          /* device [n_adapters][rank][d_in]                     */
    const void* b;          /* device [n_adapters][d_out][rank]                    */
    const float* scale;     /* device [n_adapters]                                 */
    int32_t dtype;          /* buddy_dtype of a, b and the rows                    */
    int32_t n_adapters;     /* 1..4096                                             */
    int32_t rank;           /* a multiple of 8, 8..128                             */
    int32_t d_in, d_out;    /* multiples of 8, up to 2^20                          */
} buddy_lora;

/* Which rows use which adapter, once for all projections of a step.
 *   ids:  device [n_rows], in any order: 0..n_adapters-1, -1 for none, others
 *         for rows that buddy_lora_add leaves as they were (padding);
 *   plan: device, buddy_lora_plan_size(n_rows, n_adapters) int32, written. */
buddy_status buddy_lora_plan(const int32_t* ids, int32_t n_rows, int32_t n_adapters, int32_t* plan, void* stream);
int64_t buddy_lora_plan_size(int32_t n_rows, int32_t n_adapters);   /* 0: sizes that are refused */

/* out[r] = y[r] + scale[i] * b[i] (a[i] x[r]) for rows of adapter i, y[r] for
 * rows of none: the adapters beside a projection's output y.  x: device rows of
 * d_in, y and out (which may be y, with y's stride) of d_out, strides in
 * elements.  a x is kept in fp32 (for bf16 it enters the product with b as two
 * bf16 parts, 16 bits), the sum is rounded once.  plan: buddy_lora_plan's for the
 * same n_rows and n_adapters (another one's: rows may be left out). */
buddy_status buddy_lora_add(const buddy_lora* l, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                            void* out, int64_t out_stride, int32_t n_rows, const int32_t* plan, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Bytes of workspace for n_rows rows or fewer (l's pointers are not read); 0
 * for sizes that are refused.  As buddy_mx8_linear_workspace. */
size_t buddy_lora_workspace(const buddy_lora* l, int32_t n_rows);

/* A token for each row of logits, from a given random number.
 * A token's weight is exp((logit - max) / temperature), in 64 bits and then
 * rounded to a multiple of 2^-40, so that all sums of weights are exact and
 * the answer does not depend on an order of additions.  Of the tokens by
 * falling logit (of equal ones the lowest first):
 *   the first top_k (<= 0: all), of them those with weight >= min_p (clamped
 *   to 1; NaN: none is left out), of them the fewest whose weights reach
 *   ceil(top_p * their sum) (top_p >= 1 or NaN: all; the first in any case);
 * token = the first in the order of the vocabulary up to which the weights of
 * those kept pass floor(u * their sum) (this product and top_p's in 64-bit
 * floating point).
 * temperature not above 0 (or NaN): the largest logit's, the lowest token of
 * equal ones.  A NaN logit counts as -inf.  +inf is a largest logit like any
 * other.  A row of nothing but -inf: token -1. */
typedef struct {
    const void* logits;        /* device [B] rows of vocab, any alignment of the type */
    int64_t stride;            /* elements from row to row                            */
    int32_t dtype;             /* buddy_dtype                                         */
    int32_t B;                 /* up to 65535                                         */
    int32_t vocab;             /* 1..2^20                                             */
    const float* temperature;  /* device [B]                                          */
    const int32_t* top_k;      /* device [B], or NULL: all                            */
    const float* top_p;        /* device [B], or NULL: 1                              */
    const float* min_p;        /* device [B], or NULL: 0                              */
    const float* u;            /* device [B], in [0, 1) (others: the nearest token)   */
    int32_t* token;            /* device [B], written                                 */
    void* workspace;           /* as buddy_mx8_linear's                               */
    size_t workspace_bytes;
} buddy_sampling;
buddy_status buddy_sample(const buddy_sampling* s, void* stream);
size_t buddy_sample_workspace(int32_t B, int32_t vocab);   /* for B rows or fewer; 0: refused */

const char* buddy_status_string(buddy_status s);

/* Text of the last HIP error seen by this handle ("" if none). */
const char* buddy_last_error(const buddy_model* m);

#ifdef __cplusplus
}
#endif
#endif
