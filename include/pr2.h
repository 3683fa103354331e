/*
 * pr2.h -- C ABI of the MI355X (gfx950) Predictive Routing Replay MoE-layer hot path.
 *
 * One MoE layer of a Pr^2 model, in both phases of the method:
 *   rollout:  predictive route  I_hat = TopK(Softmax(h W + h W_p), k)   (Sec. 4.1,
 *             Eq. pr2_predict, Eq. pr2_route; Alg. 2 in Appendix D), recorded into a
 *             caller-owned route buffer;
 *   training: replay of the recorded ids with weights from the current router and the
 *             predictor bypassed, o = sum_{j in I_hat} rho_j E_j(h)  (Sec. 4.1, Eq. pr2_output;
 *             Alg. 3), experts being gated MLPs with gate, up and down projections
 *             (Appendix E.2).
 *
 * Conventions shared by every entry point
 *   - All tensor arguments are DEVICE pointers owned by the caller, row-major.  Alignment:
 *     activations (x, y, dy, dx) and expert weights and their gradients 16 bytes; fp32
 *     router, predictor, gate and logit tensors 4 bytes; id buffers their element size.
 *     The library never allocates, frees or keeps them; scratch memory comes from the
 *     caller's workspace `ws` of at least pr2_workspace_bytes(desc, op) bytes (any
 *     alignment; may be NULL when that size is 0).
 *   - Calls are asynchronous on `stream` (NULL = the null stream of the current device) and
 *     run on the current HIP device.  They return once the kernels are enqueued; every
 *     launch of a call goes on `stream` (the library owns no stream), so a call can be
 *     captured into a HIP graph.  Global state: the per-device gfx950 check and the
 *     workspace split records of pr2_route_predict_reuse, both host-side and guarded by
 *     mutexes, so calls may come from several threads (each with its own workspace).
 *   - Every argument is checked on the host before any HIP call.  On an error nothing is
 *     enqueued, outputs are untouched, the status says what was wrong and pr2_last_error()
 *     (thread-local) gives a sentence naming the argument.
 *   - T == 0 is a no-op returning PR2_OK (the backward then zeroes its weight gradients).
 *   - Expert ids are 0-based.  Results are deterministic: the same inputs on the same device
 *     give bitwise identical outputs (no floating-point atomics anywhere).
 *   - Route contents (0 <= id < N, distinct within a row) are a precondition.  Kernels never
 *     touch memory out of bounds for any id value: an out-of-range id is skipped and counted.
 *     With the environment variable PR2_VALIDATE=1 each call that reads a route also
 *     synchronises its stream and returns PR2_ERR_ROUTE if any id was out of range or
 *     repeated within its row (PR2_ERR_UNSUPPORTED, nothing enqueued, if the stream is
 *     being captured into a HIP graph).
 *   - Inputs must be finite; NaN or Inf give unspecified (but memory-safe) results, except
 *     where a call says what they give.
 */
#ifndef PR2_H
#define PR2_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Same type as hipStream_t. */
typedef struct ihipStream_t* pr2_stream_t;

typedef enum {
    PR2_OK = 0,
    PR2_ERR_NULL = 1,        /* a required pointer is NULL                                  */
    PR2_ERR_SHAPE = 2,       /* a size is out of range (k > N, k < 1, d < 1, ldi < k, ...)     */
    PR2_ERR_DTYPE = 3,       /* unknown act_dtype / idx_dtype code                             */
    PR2_ERR_ALIGN = 4,       /* a pointer is not aligned as its argument requires              */
    PR2_ERR_WORKSPACE = 5,   /* workspace smaller than pr2_workspace_bytes(desc, op)           */
    PR2_ERR_UNSUPPORTED = 6, /* valid but not implemented (e.g. N > 1024)                      */
    PR2_ERR_ROUTE = 7,       /* PR2_VALIDATE=1 found an out-of-range or repeated id             */
    PR2_ERR_DEVICE = 8,      /* no usable HIP device, or the device is not gfx950              */
    PR2_ERR_HIP = 9          /* a HIP runtime call or kernel launch failed                     */
} pr2_status;

/* act_dtype: storage type of activations (x, y, dy, dx) and expert weights.
 * The router W_r, its bias, the predictor factors A, B, gates and logits are always fp32. */
enum { PR2_F32 = 0, PR2_BF16 = 1 };
/* idx_dtype: storage type of recorded expert ids; token_dtype: of sampled token ids
 * (PR2_I32 or PR2_I64). */
enum { PR2_I32 = 0, PR2_I16 = 1, PR2_I64 = 2 };
/* op codes for pr2_workspace_bytes. */
enum {
    PR2_OP_ROUTE = 0,
    PR2_OP_REPLAY_FWD = 1,
    PR2_OP_REPLAY_BWD = 2,
    PR2_OP_ROLLOUT_FWD = 3,
    PR2_OP_ROUTE_DIAG = 4,
    PR2_OP_PREDICTOR_LOSS = 5,
    PR2_OP_DISPATCH_PLAN = 6
};

/*
 * Layer descriptor.
 *   T tokens (>= 0), d hidden size, N experts (1..1024), k experts per token (1..N),
 *   m expert intermediate size, r predictor rank (>= 0; 0 = no predictor),
 *   act_dtype PR2_F32 | PR2_BF16, idx_dtype PR2_I32 | PR2_I16 (PR2_I16 needs N <= 32767),
 *   renorm: 1 = the k weights are the softmax restricted to the k ids (they sum to one);
 *           0 = the weight of id j is rho_j of the softmax over all N experts, as Eq.
 *               pr2_old_output and Eq. pr2_output print it.
 */
typedef struct {
    int64_t T;
    int32_t d, N, k, m, r;
    int32_t act_dtype;
    int32_t idx_dtype;
    int32_t renorm;
} pr2_moe_desc;

/* Bytes of workspace an op needs for this descriptor (0 if none).  Never fails: an invalid
 * descriptor yields 0 and the call itself then reports the error.  The size does not
 * decrease with T: a workspace sized for a batch also serves any smaller batch of the
 * same layer shape. */
size_t pr2_workspace_bytes(const pr2_moe_desc* desc, int op);

/*
 * Route prediction during rollout (Sec. 4.1 "Route Prediction During Rollout";
 * Eq. pr2_predict, Eq. pr2_route; Alg. 2 in Appendix D, its logits, top-k and caching steps).
 *
 *   p = x W_r + b_r                      router logits (the feature-cache p_old)
 *   z = p + (x A) B                      predictive logits, W_p = A B of rank r
 *   idx = TopK(z, k)                     ties to the lower id, stored ASCENDING by id
 *   gate_j = softmax(z) restricted to idx (renorm = 1) or softmax over all N (renorm = 0)
 *
 *   x          [T, d] act_dtype
 *   W_r        [d, N] fp32;  b_r [N] fp32 or NULL (no router bias)
 *   A          [d, r] fp32;  B [r, N] fp32.  Both ignored when r == 0.  B may be NULL only
 *              when r == N, meaning the identity (a full-rank predictor W_p = A).
 *   idx_out    route record: token t's k ids go to idx_out + t*ldi (elements of idx_dtype),
 *              ldi >= k.  Rows of other tokens and elements beyond k in a row are never
 *              written, so a [seq, pos, k] buffer can be filled one decode step at a time
 *              (pass idx_out = buf + pos*k, ldi = n_pos*k).
 *   gate_out   [T, k] fp32, aligned with idx_out's order; may be NULL.
 *   logits_out [T, N] fp32 router logits p (without the predictor term); may be NULL.
 *   ws         scratch of at least pr2_workspace_bytes(desc, PR2_OP_ROUTE) bytes (the bf16
 *              three-way split of [W_r | A] that the MFMA router reads, and for batches of at
 *              most 2048 tokens the partial logits of its split-K form; 0 bytes when the
 *              shape takes the fp64 vector path).  Reused freely between calls on one stream.
 * Logits are accumulated from exact products (fp32 weights split into three bf16 parts times
 * bf16 x, or fp64 FMA for fp32 x) in fp32 chunks summed in fp64, then rounded once to fp32.
 */
pr2_status pr2_route_predict(const pr2_moe_desc* desc, const void* x, const float* W_r,
                             const float* b_r, const float* A, const float* B, void* idx_out,
                             int64_t ldi, float* gate_out, float* logits_out, void* ws,
                             size_t ws_bytes, pr2_stream_t stream);

/*
 * Route prediction for the later steps of a rollout (Sec. 4.1 "Route Prediction During
 * Rollout": the policy's router and predictor stay fixed while a batch is generated, so one
 * decode step follows another with the same W_r, A, B).  Same arguments, checks and results
 * as pr2_route_predict, except that the bf16 three-way split of the weights is not formed
 * again: the call reads the split that the previous pr2_route_predict (or _reuse) call on
 * this workspace left there.  The library keeps a host-side record per workspace address of
 * the split it holds (device, W_r, A, B pointers, d, N, r and the layout, which depends on the
 * NULL-ness of logits_out); any other call that takes the workspace drops the records inside
 * it.  The call returns PR2_ERR_WORKSPACE, with nothing enqueued, when ws holds no record or
 * one that differs from this call in any of those.  The caller still guarantees that the
 * VALUES of W_r, A and B did not change since the split was formed (only pointers are
 * compared).  Shapes that take the fp64 vector path keep no split and behave exactly as
 * pr2_route_predict.
 */
pr2_status pr2_route_predict_reuse(const pr2_moe_desc* desc, const void* x, const float* W_r,
                                   const float* b_r, const float* A, const float* B,
                                   void* idx_out, int64_t ldi, float* gate_out, float* logits_out,
                                   void* ws, size_t ws_bytes, pr2_stream_t stream);

/*
 * Route prediction that allocates nothing, for callers that cannot allocate device memory:
 * code being captured into a HIP graph, tight serving loops, harnesses that forbid it.
 * Same arguments (minus the workspace), checks and results as pr2_route_predict: the same
 * kernels, always the fused (non-split-K) form, whose logits are bitwise those of the split-K
 * form.  The bf16 split of the weights goes to a file-scope device array of 6 MiB that the
 * library holds on each GPU it runs on until the process ends; a shape whose split needs more
 * (3 x 2 bytes x d x the columns N, or N + r when logits_out is given, rounded up to 64)
 * returns PR2_ERR_UNSUPPORTED with nothing enqueued.  The call allocates and frees nothing;
 * its first call on a device looks up that device's copy of the array (make it outside a
 * capture).  Every call on a GPU shares that GPU's array: calls that overlap on one GPU (two
 * streams, two threads) race and give unspecified routes; order them on one stream.
 */
pr2_status pr2_route_predict_noalloc(const pr2_moe_desc* desc, const void* x, const float* W_r,
                                     const float* b_r, const float* A, const float* B,
                                     void* idx_out, int64_t ldi, float* gate_out,
                                     float* logits_out, pr2_stream_t stream);

/*
 * Replay forward during training (Sec. 4.1 "Replay During Training"; Eq. pr2_output;
 * Alg. 3 in Appendix D, its first two steps).  No fresh top-k: the recorded ids are used as
 * given, in any order; the weights come from the current router with the predictor bypassed:
 *
 *   p = x W_r + b_r,  g_{t,s} = softmax over the k recorded ids (renorm = 1) or rho of the
 *   softmax over all N (renorm = 0),
 *   y_t = sum_s g_{t,s} E_{idx[t,s]}(x_t),  E_j(h) = W_down_j (silu(W_gate_j h) * (W_up_j h)).
 *
 *   x        [T, d] act_dtype;  idx: token t's ids at idx + t*ldi (idx_dtype), ldi >= k
 *   W_r      [d, N] fp32;  b_r [N] fp32 or NULL
 *   W_gate   [N, m, d], W_up [N, m, d], W_down [N, d, m]   act_dtype
 *   y        [T, d] act_dtype (overwritten)
 *   gate_out [T, k] fp32 replay weights in idx's slot order; may be NULL.
 *   ws       >= pr2_workspace_bytes(desc, PR2_OP_REPLAY_FWD)
 * bf16 expert GEMMs use MFMA with fp32 accumulation; the SwiGLU activation is rounded to
 * act_dtype before the down projection and the weighted expert outputs are rounded to
 * act_dtype before the combine, which sums each token's k terms in slot order in fp32.
 */
pr2_status pr2_moe_replay_forward(const pr2_moe_desc* desc, const void* x, const void* idx,
                                  int64_t ldi, const float* W_r, const float* b_r,
                                  const void* W_gate, const void* W_up, const void* W_down,
                                  void* y, float* gate_out, void* ws, size_t ws_bytes,
                                  pr2_stream_t stream);

/*
 * Replay forward that also saves the experts' pre-activations for the backward (Sec. 4.1
 * "Replay During Training", Alg. 3: the training pass runs the replay forward and then its
 * backward under the same recorded routes).  Everything pr2_moe_replay_forward does, plus
 *
 *   au_out  [T*k, 2m] act_dtype, 16-byte aligned: row q holds a = x W_gate_e^T (first m) and
 *           u = x W_up_e^T (last m), rounded to act_dtype, for the q-th route in the
 *           library's expert-sorted order (a stable sort of the routes by expert id, which the
 *           backward forms again from the same ids).  Opaque to the caller: pass it unchanged
 *           to pr2_moe_replay_backward_saved with the same desc, x, idx, W_gate and W_up.
 *
 * y and gate_out are bitwise those of pr2_moe_replay_forward.  The saved rows are bitwise
 * what the backward would otherwise recompute, so the saved backward's gradients are bitwise
 * those of pr2_moe_replay_backward.  Same workspace and checks as pr2_moe_replay_forward, and
 * au_out NULL with T > 0 returns PR2_ERR_NULL, a misaligned au_out PR2_ERR_ALIGN (nothing
 * enqueued).
 */
pr2_status pr2_moe_replay_forward_save(const pr2_moe_desc* desc, const void* x, const void* idx,
                                       int64_t ldi, const float* W_r, const float* b_r,
                                       const void* W_gate, const void* W_up, const void* W_down,
                                       void* y, float* gate_out, void* au_out, void* ws,
                                       size_t ws_bytes, pr2_stream_t stream);

/*
 * Replay forward with the route-tracking diagnostics of Sec. 5.4 (top-k agreement, routing
 * deviation, route KL) formed in the same pass: the replay-weight epilogue already holds all N
 * current router logits of each token, so it also selects their top-k and compares it with the
 * recorded ids.  Everything pr2_moe_replay_forward does, plus (each output may be NULL):
 *
 *   p = x W_r + b_r (the replay router, predictor bypassed),  I = TopK(p, k) (ties to the lower
 *   id, decided on the fp32 logits)
 *   cur_idx_out [T, k] idx_dtype   I, ascending
 *   overlap_out [T] int32          |idx_t ∩ I_t|   (agreement = overlap / k, deviation = k - overlap)
 *   kl_out      [T] fp32           KL(softmax(p_t) || softmax(z_ref_t)), evaluated in fp64
 *   hist_out    [k + 1] uint64     tokens per deviation value, overwritten (8-byte aligned)
 *   z_ref       [T, N] fp32 reference logits (e.g. the rollout's predictive logits); needed only
 *               with kl_out
 * Same workspace, streams and checks as pr2_moe_replay_forward; y and gate_out are bitwise
 * those of pr2_moe_replay_forward, and the diagnostics bitwise those of pr2_route_diagnostics
 * on the same inputs.  T = 0 only zeroes hist_out.
 */
pr2_status pr2_moe_replay_forward_diag(const pr2_moe_desc* desc, const void* x, const void* idx,
                                       int64_t ldi, const float* W_r, const float* b_r,
                                       const void* W_gate, const void* W_up, const void* W_down,
                                       void* y, float* gate_out, const float* z_ref,
                                       void* cur_idx_out, int32_t* overlap_out, float* kl_out,
                                       uint64_t* hist_out, void* ws, size_t ws_bytes,
                                       pr2_stream_t stream);

/*
 * Rollout-phase layer forward (Sec. 4.1 "Route Prediction During Rollout"; Eq. pr2_old_output;
 * Alg. 2 in Appendix D): route prediction exactly as pr2_route_predict, then the layer output
 * under the predictive weights,
 *
 *   o_old,t = sum_s rho_hat_{t,s} E_{idx[t,s]}(x_t)
 *
 * with rho_hat renormalised over the k predicted ids (renorm = 1) or the softmax of the
 * predictive logits over all N (renorm = 0, the printed equation).  Arguments as for
 * pr2_route_predict and pr2_moe_replay_forward; idx_out and gate_out receive the recorded
 * route and its predictive weights (gate_out may be NULL).
 *   ws       >= pr2_workspace_bytes(desc, PR2_OP_ROLLOUT_FWD)
 */
pr2_status pr2_moe_rollout_forward(const pr2_moe_desc* desc, const void* x, const float* W_r,
                                   const float* b_r, const float* A, const float* B,
                                   const void* W_gate, const void* W_up, const void* W_down,
                                   void* idx_out, int64_t ldi, float* gate_out, float* logits_out,
                                   void* y, void* ws, size_t ws_bytes, pr2_stream_t stream);

/*
 * Replay backward (Sec. 4.1 "Replay During Training": the current experts and router are
 * trained through the replayed routes; Alg. 3 in Appendix D, its backward step).  Gradients
 * of L = sum_t <dy_t, y_t> for the replay forward above, with the recorded ids held fixed:
 *
 *   dg_ts = <dy_t, E_j(x_t)>                                        (j = idx[t, s])
 *   renorm = 1 (g = softmax over the k recorded logits):
 *     dp_t,j = g_ts (dg_ts - sum_s' g_ts' dg_ts') at the recorded ids, 0 at the others
 *   renorm = 0 (g_ts = rho_j of the softmax over all N logits, Eq. pr2_output as printed):
 *     dp_t,i = rho_ti ([i recorded] dg_ti - sum_s g_ts dg_ts) for every i < N (k <= 64)
 *   dW_r = sum_t x_t^T dp_t,  db_r = sum_t dp_t
 *   dW_gate_j, dW_up_j, dW_down_j = sums over the routes through expert j of the SwiGLU
 *   expert's weight gradients, each route's output scaled by g_ts
 *   dx_t = sum_s g_ts dE_j/dx(x_t)^T dy_t + dp_t W_r^T
 *
 * The predictor (A, B) is bypassed in replay and gets no gradient.  Arguments as for
 * pr2_moe_replay_forward, plus:
 *   dy       [T, d] act_dtype, gradient of the output y
 *   dx       [T, d] act_dtype (out)
 *   dW_r     [d, N] fp32 (out);  db_r [N] fp32 (out) or NULL when not wanted
 *   dW_gate  [N, m, d], dW_up [N, m, d], dW_down [N, d, m] fp32 (out), 16-byte aligned
 *   ws       >= pr2_workspace_bytes(desc, PR2_OP_REPLAY_BWD)
 * Every gradient is overwritten (not accumulated); an expert no route uses gets zeros, and
 * T = 0 writes zeros to all weight gradients (x, idx, dy, dx, ws may then be NULL).  Results
 * are bitwise deterministic.  With renorm = 0 the router gradients are dense over N (fp32
 * FMA passes over x and the [T, N] logit gradient) and k > 64 returns PR2_ERR_UNSUPPORTED.
 * The pre-activations
 * are recomputed (nothing is saved from the forward call); on the bf16 MFMA path
 * (d % 256 == 0, m % 128 == 0) a, u, their gradients, g H and the per-route input gradients
 * are held in bf16, with fp32 accumulation everywhere.
 */
pr2_status pr2_moe_replay_backward(const pr2_moe_desc* desc, const void* x, const void* idx,
                                   int64_t ldi, const float* W_r, const float* b_r,
                                   const void* W_gate, const void* W_up, const void* W_down,
                                   const void* dy, void* dx, float* dW_r, float* db_r,
                                   float* dW_gate, float* dW_up, float* dW_down, void* ws,
                                   size_t ws_bytes, pr2_stream_t stream);

/*
 * Replay backward from saved pre-activations: pr2_moe_replay_backward with the gate/up
 * pre-activations read from au_saved (written by pr2_moe_replay_forward_save with the same
 * desc, x, idx, W_gate and W_up) instead of recomputed by a grouped GEMM.  au_saved is only
 * read.  Same arguments otherwise, same workspace, bitwise the same gradients; au_saved NULL
 * with T > 0 returns PR2_ERR_NULL, a misaligned one PR2_ERR_ALIGN (nothing enqueued).  A
 * buffer not written by pr2_moe_replay_forward_save for these inputs gives wrong gradients
 * (nothing detects it).
 */
pr2_status pr2_moe_replay_backward_saved(const pr2_moe_desc* desc, const void* x, const void* idx,
                                         int64_t ldi, const float* W_r, const float* b_r,
                                         const void* W_gate, const void* W_up,
                                         const void* W_down, const void* au_saved,
                                         const void* dy, void* dx, float* dW_r, float* db_r,
                                         float* dW_gate, float* dW_up, float* dW_down, void* ws,
                                         size_t ws_bytes, pr2_stream_t stream);

/*
 * Route-tracking diagnostics (Sec. 5.4: top-k agreement, routing deviation and route KL) of a
 * recorded route against the current router, the predictor bypassed as in replay:
 *
 *   p = x W_r + b_r,  I = TopK(p, k)   (ties to the lower id, decided on the fp32 logits)
 *   overlap_t = |idx_t ∩ I_t|           (agreement = overlap / k, deviation = k - overlap)
 *   kl_t = KL(softmax(p_t) || softmax(z_ref_t))
 *   hist[v] = number of tokens whose deviation is v, v = 0..k
 *
 *   x, idx, ldi, W_r, b_r   as for pr2_moe_replay_forward (desc.m, desc.r, desc.renorm unused)
 *   z_ref        [T, N] fp32 reference logits, e.g. the rollout-time predictive logits; may be
 *                NULL when kl_out is NULL
 *   cur_idx_out  [T, k] idx_dtype, the current top-k ascending, or NULL
 *   overlap_out  [T] int32 or NULL;  kl_out [T] fp32 or NULL
 *   hist_out     [k + 1] uint64 (8-byte aligned), overwritten with exact counts, or NULL
 *   ws           >= pr2_workspace_bytes(desc, PR2_OP_ROUTE_DIAG)
 * The logits are the replay router's (exact bf16 x times fp32 W_r, one rounding to fp32); the
 * route KL is evaluated in fp64 from them.  T = 0 only zeroes hist_out.
 */
pr2_status pr2_route_diagnostics(const pr2_moe_desc* desc, const void* x, const void* idx,
                                 int64_t ldi, const float* W_r, const float* b_r,
                                 const float* z_ref, void* cur_idx_out, int32_t* overlap_out,
                                 float* kl_out, uint64_t* hist_out, void* ws, size_t ws_bytes,
                                 pr2_stream_t stream);

/*
 * Feature-cache positions (Appendix E.2, feature-cache paragraph: a fixed number Tc of token
 * positions per response keep their route-recording features, drawn by uniform
 * sub-sampling along the rollout).  HOST function, no device work: fills pos_out[0..n) with
 * n = min(T, Tc) increasing positions in [0, T): Tc >= T keeps every position; otherwise
 * position i is drawn uniformly inside the stratum [floor(i T / Tc), floor((i+1) T / Tc))
 * with the i-th output of SplitMix64 (Steele, Lea and Flood, 2014) for `seed`, so the cache
 * covers the whole rollout evenly.  Returns n, or -1 on a bad argument (pr2_last_error).
 */
int64_t pr2_feature_cache_positions(int64_t T, int64_t Tc, uint64_t seed, int64_t* pos_out);

/*
 * Route prediction with the feature-cache write fused in (Alg. 2 in Appendix D, its caching
 * step: the predicted ids go to the index cache and the retained tokens' route-recording
 * features (h_old, p_old) to the feature cache).  Same as pr2_route_predict with
 * logits_out = NULL, plus: token t with 0 <= cache_row[t] < cache_rows copies its input row
 * x_t to h_cache[cache_row[t]] ([cache_rows, d] act_dtype, 16-byte aligned) and writes its
 * router logits p_t (no predictor term) to p_cache[cache_row[t]] ([cache_rows, N] fp32);
 * tokens with any other cache_row value are not cached.  cache_row is a device int32 [T];
 * rows must be distinct.  ws >= pr2_workspace_bytes(desc, PR2_OP_ROUTE).
 */
pr2_status pr2_route_predict_cached(const pr2_moe_desc* desc, const void* x, const float* W_r,
                                    const float* b_r, const float* A, const float* B,
                                    void* idx_out, int64_t ldi, float* gate_out,
                                    const int32_t* cache_row, void* h_cache, float* p_cache,
                                    int64_t cache_rows, void* ws, size_t ws_bytes,
                                    pr2_stream_t stream);

/*
 * Evolution-predictor loss and gradients on the feature cache (Sec. 4.2, Eq. pr2_loss; Alg. 3
 * in Appendix D, its predictive-loss steps).  desc.T = number of cached tokens; desc.d, N, r
 * as for the layer (r >= 1); desc.k must be valid; m, idx_dtype and renorm are unused.
 *
 *   p_t = h_t W_r + b_r               the current router on the same tokens (teacher)
 *   zhat_t = p_old,t + h_old,t A B    rebuilt predictive logits
 *   loss_kind 0:  kl_t = KL(softmax(p_t) || softmax(zhat_t))                  (Eq. pr2_loss)
 *   loss_kind 1:  kl_t = KL(softmax(p_t - p_old,t) || softmax(h_old,t A B))   (delta matching,
 *                 the objective ablation of Appendix G)
 *   loss = mean_t kl_t;  dA, dB = gradients of loss (the router gets none: stop-gradient)
 *
 *   h, h_old   [T, d] act_dtype (16-byte aligned);  W_r [d, N], b_r [N] or NULL, p_old [T, N],
 *              A [d, r], B [r, N] fp32 (B NULL means the identity, needs r == N; dB unused)
 *   mini_step  1-based index of the update within the batch: mini_step == 1 is the
 *              on-policy first step, where the loss is skipped (zeros written, h, h_old, W_r,
 *              p_old and ws may be NULL)
 *   kl_out [T] fp32 or NULL;  loss_out [1] fp32;  dA [d, r], dB [r, N] fp32 (overwritten)
 *   ws         >= pr2_workspace_bytes(desc, PR2_OP_PREDICTOR_LOSS)
 * p is computed as by the replay router (exact products, one rounding to fp32); everything
 * after it, including the gradient sums over tokens, in fp64 with a fixed summation order.
 */
pr2_status pr2_predictor_loss(const pr2_moe_desc* desc, const void* h, const float* W_r,
                              const float* b_r, const void* h_old, const float* p_old,
                              const float* A, const float* B, int loss_kind, int mini_step,
                              float* kl_out, float* loss_out, float* dA, float* dB, void* ws,
                              size_t ws_bytes, pr2_stream_t stream);

/* ------------------------------------------------------------------------------------------
 * The policy's loss on the sampled tokens (Sec. 2, the clipped objective with a KL regulariser
 * that the method is trained with; Appendix E.1: clip bounds 0.2 below and 0.28 above).
 *
 * Row t of the logits belongs to sampled token y_t.  With z = logits[t, 0..V) and
 * s = inv_temp (1 / sampling temperature):
 *   logp_t    = s z_y - log sum_v exp(s z_v),   p_v = exp(s z_v) / sum exp(s z),
 *   entropy_t = -sum_v p_v log p_v,
 *   ratio r_t = exp(logp_t - logp_old_t),
 *   surr_t    = min(r_t A_t, clamp(r_t, 1 - clip_low, 1 + clip_high) A_t),
 *   kl_t      = exp(d_t) - d_t - 1 with d_t = logp_ref_t - logp_t   (0 without logp_ref),
 *   loss      = sum_t w_t (-surr_t + kl_coef kl_t),
 *   coef_t    = d loss / d logp_t
 *             = w_t (-A_t r_t [not clipped] + kl_coef (1 - exp(d_t))),   clipped meaning
 *               A_t > 0 and r_t > 1 + clip_high, or A_t < 0 and r_t < 1 - clip_low,
 *   dlogits[t, v] = coef_t s ([v = y_t] - p_v).
 * A_t = 0 has surr_t = 0 and no gradient through it, whatever r_t is.
 *
 * A row counts only if w_t != 0, 0 <= y_t < V and some logit of it is above -infinity.  Any
 * other row has loss, logp, entropy and coef 0 and a gradient of zeros, whatever stands in its
 * other inputs (NaN included); its lse is -infinity.  A logit of -infinity (an id that may not
 * be sampled) has probability 0.  NaN or +infinity in the logits of a row that counts make its
 * logp, lse and entropy NaN and with them whatever is formed from them: with A_t = 0 and no KL
 * term (logp_ref NULL or kl_coef 0) loss, coef and gradient are not, and stay 0.
 *
 * T rows (>= 0, below 2^25), V vocabulary size (>= 1), ldl and ldd (>= V, at most 2^35) the row
 * strides in elements of logits and dlogits (ldd is read only by calls that write dlogits),
 * act_dtype of both, token_dtype PR2_I32 or PR2_I64 of the ids, inv_temp > 0, clip_low,
 * clip_high and kl_coef >= 0, all finite.  Logits and gradients need only their element's
 * alignment, rows may start anywhere.
 * Per-token tensors are [T] fp32, contiguous.
 */
typedef struct {
    int64_t T, ldl, ldd;
    int32_t V;
    int32_t act_dtype;
    int32_t token_dtype;
    float inv_temp;
    float clip_low, clip_high;
    float kl_coef;
} pr2_policy_desc;

/* Bytes of workspace that pr2_token_logprob and pr2_policy_loss need for this descriptor
 * (0 for an invalid one, which the call then reports).  Does not decrease with T. */
size_t pr2_policy_workspace_bytes(const pr2_policy_desc* desc);

/*
 * Log-probability of the sampled tokens, for the rollout's record and for the passes that
 * form logp_old and logp_ref.  clip_low, clip_high, kl_coef and ldd are not read.
 *   logits [T, V] act_dtype;  token [T]
 *   logp_out [T];  lse_out [T] log sum_v exp(s z_v) or NULL;  entropy_out [T] or NULL
 *   ws >= pr2_policy_workspace_bytes(desc)
 */
pr2_status pr2_token_logprob(const pr2_policy_desc* desc, const void* logits, const void* token,
                             float* logp_out, float* lse_out, float* entropy_out, void* ws,
                             size_t ws_bytes, pr2_stream_t stream);

/*
 * The loss, and in the same pass (dlogits not NULL) its gradient.
 *   logp_old, adv [T];  logp_ref [T] or NULL (no KL term);  weight [T] or NULL (all 1)
 *   sums_out [4]: sum_t w_t times the loss, kl_t, [clipped] and entropy_t
 *   logp_out, lse_out, entropy_out, coef_out [T], each may be NULL (lse and coef are what
 *              pr2_policy_loss_backward reads)
 *   dlogits    [T, V] act_dtype at row stride ldd, or NULL; may be logits itself (same
 *              stride), otherwise the two must not overlap (rows of the same stride may lie
 *              between each other, as halves of one buffer's columns do)
 *   No other output may overlap an input or another output.
 * Statistics are held in fp32 (differences to the row's maximum), and the gradient is formed from
 * them, so that neither depends on how far from zero the logits lie; the sums over tokens are
 * held in fp64.  The same call gives the same bits.  (Calls of other batch sizes may split a row
 * differently and differ in its last bits.)  T = 0 writes zeros to sums_out.
 */
pr2_status pr2_policy_loss(const pr2_policy_desc* desc, const void* logits, const void* token,
                           const float* logp_old, const float* logp_ref, const float* adv,
                           const float* weight, float* sums_out, float* logp_out, float* lse_out,
                           float* entropy_out, float* coef_out, void* dlogits, void* ws,
                           size_t ws_bytes, pr2_stream_t stream);

/*
 * The gradient alone, from what the forward call kept: dlogits = grad coef_t s ([v = y_t] - p_v)
 * with p_v = exp(s z_v - lse_t).  grad_loss: one fp32 on the device (the gradient of the first
 * of the sums) or NULL for 1.  Rows with coef_t = 0 get zeros and are not read.  dlogits as
 * above (it may be logits itself).  clip_low, clip_high and kl_coef are not read.  No workspace.
 * lse_t is one fp32 number, and log p_v = s z_v - lse_t has its rounding, up to |lse_t| 2^-23: p_v is
 * off by that relatively and 1 - p_y by that times p_y.  (At a level of the logits of 30 that is
 * 4e-6, at 1e4 1e-3.)  pr2_policy_loss with dlogits has no such error at any level.
 */
pr2_status pr2_policy_loss_backward(const pr2_policy_desc* desc, const void* logits,
                                    const void* token, const float* lse, const float* coef,
                                    const float* grad_loss, void* dlogits, pr2_stream_t stream);

/* ------------------------------------------------------------------------------------------
 * Experts of the caller's own behind the recorded routes: tokens sorted by expert, the
 * experts' outputs summed back under the route weights, and both gradients (Eq. pr2_output
 * with any E_j).  desc.T, d, N, k, act_dtype and, for the plan, idx_dtype are read.
 *
 * A route is a (token t, slot s) pair, numbered t k + s.  Rows are the routes sorted by expert,
 * stably in route order; expert e's rows are offsets[e] .. offsets[e + 1).  A route whose id
 * is outside [0, N) (-1 for one that was dropped) has no row.  Rows from offsets[N] on belong
 * to no route.
 */

/*
 *   idx           token t's ids at idx + t * ldi, ldi >= k
 *   offsets       [N + 1] int32 (out)
 *   row_of_route  [T, k] int32 (out), -1 for a route without a row
 *   route_of_row  [T * k] int32 (out), -1 for a row without a route
 *   ws            >= pr2_workspace_bytes(desc, PR2_OP_DISPATCH_PLAN)
 * A dropped or repeated id is no fault here: PR2_VALIDATE does not apply.  T = 0 writes zeros
 * to offsets.
 */
pr2_status pr2_dispatch_plan(const pr2_moe_desc* desc, const void* idx, int64_t ldi,
                             int32_t* offsets, int32_t* row_of_route, int32_t* route_of_row,
                             void* ws, size_t ws_bytes, pr2_stream_t stream);

/* xs[row_of_route[t, s], :] = x[t, :], zeros in the rows from offsets[N] on.
 *   x [T, d], xs [T * k, d] act_dtype (16-byte aligned, not overlapping).  Here and in the
 *   three calls below a row index outside [0, T k) counts as none. */
pr2_status pr2_dispatch(const pr2_moe_desc* desc, const void* x, const int32_t* offsets,
                        const int32_t* row_of_route, void* xs, pr2_stream_t stream);

/* dx[t, :] = sum over slots of dxs[row_of_route[t, s], :], in slot order in fp32, zeros for a
 * token without rows. */
pr2_status pr2_dispatch_backward(const pr2_moe_desc* desc, const void* dxs,
                                 const int32_t* row_of_route, void* dx, pr2_stream_t stream);

/* y[t, :] = sum over slots of gate[t, s] o[row_of_route[t, s], :], in slot order in fp32.
 *   o [T * k, d], y [T, d] act_dtype;  gate [T, k] fp32 */
pr2_status pr2_combine(const pr2_moe_desc* desc, const void* o, const int32_t* row_of_route,
                       const float* gate, void* y, pr2_stream_t stream);

/* d_o[row_of_route[t, s], :] = gate[t, s] dy[t, :], zeros in the rows from offsets[N] on;
 * dgate[t, s] = <dy[t, :], o[row_of_route[t, s], :]> in fp32, 0 for a route without a row.
 * d_o may be o itself. */
pr2_status pr2_combine_backward(const pr2_moe_desc* desc, const void* dy, const void* o,
                                const int32_t* offsets, const int32_t* row_of_route,
                                const float* gate, void* d_o, float* dgate,
                                pr2_stream_t stream);

/* ------------------------------------------------------------------------------------------
 * Activations kept in 8 bits between the forward and the backward pass.
 *
 * The packed form of x [R, C]: q [R, C] int8 and scale [R, ceil(C / 32)] uint8, one scale for
 * each group of 32 consecutive columns of a row (the last group may be shorter).  With E the
 * exponent field (fp32) of the group's largest magnitude, scale = max(E - 6, 1) and
 *   q = clamp(round_to_even(x 2^(127 - scale)), -127, 127),   value = q 2^(scale - 127):
 * a power of two, so that value is exact in bf16 and fp32 and packing gives the same bits on
 * any machine.  A step, 2^(scale - 127), is 1/128 to 1/64 of the group's largest magnitude (2^-126
 * where that is below 2^-120).  x is held to half a step, its largest magnitude too: q has 7 bits, a
 * bf16 magnitude 8.  An fp32 magnitude above 127.5 steps is cut to 127, up to a whole step.  A group
 * that holds an infinity or a NaN has scale 255 and q = 0, and all its values are NaN.
 * R >= 0 rows of C >= 1 columns, contiguous; q and scale 16-byte aligned.
 */
pr2_status pr2_act_pack(int64_t R, int32_t C, int act_dtype, const void* x, int8_t* q,
                        uint8_t* scale, pr2_stream_t stream);
/* x [R, C] act_dtype (out): the values that (q, scale) stand for. */
pr2_status pr2_act_unpack(int64_t R, int32_t C, int act_dtype, const int8_t* q,
                          const uint8_t* scale, void* x, pr2_stream_t stream);

/* SwiGLU that keeps its input in 8 bits: au [R, 2m] holds a (first m columns) and u;
 *   h [R, m] = silu(a) u (from au itself), (q, scale) = the packed form of au as [R, 2m]. */
pr2_status pr2_swiglu_pack(int64_t R, int32_t m, int act_dtype, const void* au, void* h,
                           int8_t* q, uint8_t* scale, pr2_stream_t stream);
/* Its backward from the packed form, with a, u the values that it stands for:
 *   d_au [R, 2m]: da = dh u sig(a) (1 + a (1 - sig(a))) and du = dh silu(a);
 *   h_out [R, m] = silu(a) u (what a down projection's weight gradient reads), or NULL. */
pr2_status pr2_swiglu_backward_packed(int64_t R, int32_t m, int act_dtype, const int8_t* q,
                                      const uint8_t* scale, const void* dh, void* d_au,
                                      void* h_out, pr2_stream_t stream);

/*
 * Weight gradients of linear layers (out = x W^T, W [n_out, n_in]) whose input x was packed:
 *   dW[e] = sum over the rows r of expert e of dy[r, :]^T value(x)[src(r), :]
 * with expert e's rows offsets[e] .. offsets[e + 1) and src(r) = route_of_row[r] / k (the token
 * of the route), or src(r) = r when route_of_row is NULL.  A row whose route_of_row is
 * outside [0, k Rx) adds nothing.  offsets NULL (then N = 1): one weight over all R rows.
 *   R rows of dy [R, n_out];  q [Rx, n_in], scale [Rx, ceil(n_in / 32)] as packed;
 *   dW [N, n_out, n_in] fp32, overwritten (zeros for an expert without rows).
 *   Without route_of_row, R <= Rx.  N <= 1024; R and Rx below 2^31.
 *   ws >= pr2_weight_grad_workspace_bytes(desc)
 * act_dtype is dy's.  bf16: MFMA with fp32 accumulation of exact products (the packed values
 * are bf16 values); fp32: fp32 products and sums.  Sums run in a fixed order.
 */
typedef struct {
    int64_t R, Rx;
    int32_t n_out, n_in, N, k;
    int32_t act_dtype;
} pr2_wgrad_desc;
/* Bytes of workspace that pr2_weight_grad_packed needs (0 where R, N, n_out or n_in is out of its
 * range, which the call then reports).  Does not decrease with R. */
size_t pr2_weight_grad_workspace_bytes(const pr2_wgrad_desc* desc);
pr2_status pr2_weight_grad_packed(const pr2_wgrad_desc* desc, const void* dy, const int8_t* q,
                                  const uint8_t* scale, const int32_t* offsets,
                                  const int32_t* route_of_row, float* dW, void* ws,
                                  size_t ws_bytes, pr2_stream_t stream);

/*
 * The same from x itself: x [Rx, n_in] of dy's type, 16-byte aligned, in the place of (q, scale);
 * dW apart from dy and x.
 * bf16: MFMA with fp32 accumulation; fp32: fp32 products and sums.  Same workspace.
 */
pr2_status pr2_weight_grad(const pr2_wgrad_desc* desc, const void* dy, const void* x,
                           const int32_t* offsets, const int32_t* route_of_row, float* dW, void* ws,
                           size_t ws_bytes, pr2_stream_t stream);

/* ------------------------------------------------------------------------------------------
 * Products of rows sorted by expert with their experts' weights (desc as for the weight gradients;
 * act_dtype of x, W and out), for experts of the caller's own behind the recorded routes.
 *   out[r, :] = x[src(r), :] W[e]^T        for the rows r of expert e, offsets[e] .. offsets[e + 1)
 *   x [Rx, n_in], W [N, n_out, n_in], out [R, n_out], 16-byte aligned, out apart from x and W
 * with src(r) as above: the token of row r's route (x is then read through the plan and need not be
 * dispatched), or r itself where route_of_row is NULL (then R <= Rx).  offsets NULL (then N = 1): one
 * weight for all rows.  A row whose route_of_row is outside [0, k Rx) and the rows from offsets[N] on
 * are written as zeros.  offsets[0] is 0 and offsets rise to at most R (others give unspecified rows,
 * no access out of bounds).  R = 0 is a no-op.  NaN and infinities reach the rows and columns that
 * they are terms of, no others.
 * Sums in fp32, one rounding to act_dtype at the end; bf16 products are exact.  N <= 1024, R and Rx
 * below 2^31 - 1024, n_out and n_in at most 2^20, N n_out n_in at most 2^36.  No workspace.  The same
 * call gives the same bits.  (Speed: rows of a multiple of 16 bytes, and tokens below 4 GiB where they are
 * read through the plan, take the fast tiles; larger ones are better sorted first by pr2_dispatch.)
 */
pr2_status pr2_grouped_mm(const pr2_wgrad_desc* desc, const void* x, const void* W,
                          const int32_t* offsets, const int32_t* route_of_row, void* out,
                          pr2_stream_t stream);
/* The gradient of the rows: dx[r, :] = dy[r, :] W[e], dy [R, n_out], dx [R, n_in]; zeros from
 * offsets[N] on.  (Where the product read x through the plan, pr2_dispatch_backward sums a token's
 * rows of dx.  The weights' gradient is pr2_weight_grad.)  desc.Rx and k are not read. */
pr2_status pr2_grouped_mm_backward(const pr2_wgrad_desc* desc, const void* dy, const void* W,
                                   const int32_t* offsets, void* dx, pr2_stream_t stream);

/*
 * The product in 8 bits, for a rollout whose weights stay fixed:
 *   out[r, o] = ((float)(sum_c q[src(r), c] Wq[e, o, c]) row_scale[src(r)]) w_scale[e, o]
 *   q [Rx, n_in] int8, row_scale [Rx] fp32;  Wq [N, n_out, n_in] int8, w_scale [N, n_out] fp32
 *   out [R, n_out] of act_dtype
 * The sum is exact (int32; n_in below 2^17), then rounded to fp32, as is each product with a scale.
 * Otherwise as pr2_grouped_mm.
 */
pr2_status pr2_grouped_mm_quant(const pr2_wgrad_desc* desc, const int8_t* q, const float* row_scale,
                                const int8_t* Wq, const float* w_scale, const int32_t* offsets,
                                const int32_t* route_of_row, void* out, pr2_stream_t stream);

/*
 * Rows in 8 bits with one scale each (the row form), of x [R, C] act_dtype: with m the row's largest
 * magnitude
 *   row_scale = fp32(max(m, 2^-100) fp32(1 / 127)),  q = rint(x / row_scale)  in [-127, 127],
 * the quotient as in exact arithmetic, ties to even, so that q row_scale is x to half of row_scale.  A row that
 * holds an infinity or a NaN has row_scale NaN and q = 0.  Weights [N, n_out, n_in] brought to
 * this form as N n_out rows are what pr2_grouped_mm_quant reads as Wq and w_scale.
 *   q [R, C] int8, x 16-byte aligned;  row_scale [R] fp32
 */
pr2_status pr2_act_quant(int64_t R, int32_t C, int act_dtype, const void* x, int8_t* q,
                         float* row_scale, pr2_stream_t stream);
/* The row form of a / (1 + exp(-a)) u (fp32 operations, to a few last places), au [R, 2m] as for pr2_swiglu_pack;
 * q [R, m]. */
pr2_status pr2_swiglu_quant(int64_t R, int32_t m, int act_dtype, const void* au, int8_t* q,
                            float* row_scale, pr2_stream_t stream);

/* ------------------------------------------------------------------------------------------
 * Root-mean-square norm in front of the layer, the residual's addition in the same pass.
 *   h = round(x + residual)  (the sum in fp32; x itself without residual),  r = (mean_i h_i^2 + eps)^(-1/2),
 *   y_i = round(h_i r w_i)                                  round: to act_dtype, of y through fp32
 *   x, residual [T, d] act_dtype; weight [d] fp32; residual may be NULL
 *   h_out [T, d], y [T, d] act_dtype; rstd_out [T] fp32 (what the backward call reads)
 *   q [T, d] int8 with scale [T, ceil(d / 32)] uint8: the packed form of y, the bits of pr2_act_pack
 *   q [T, d] int8 with row_scale [T] fp32: the row form of h r w (not rounded to act_dtype), q that of
 *     fp32(h w) under pr2_act_quant and row_scale = r times its scale
 * Each output may be NULL, q goes with one of scale and row_scale.  h_out and y may lie on x or
 * residual (not both on the same); other overlaps are not allowed.  d <= 32768, T < 2^31, 16-byte
 * alignment of all but the fp32 tensors.  The sum of squares, r and h r w are formed
 * in fp64: y and rstd_out are the roundings of the exact values, also where the squares or r w pass
 * fp32's range.  A row's results have the same bits in any batch, and a NaN or an infinity in a row
 * reaches that row alone.  T = 0 is a no-op.
 */
pr2_status pr2_rms_norm(int64_t T, int32_t d, int act_dtype, float eps, const void* x,
                        const void* residual, const float* weight, void* h_out, void* y,
                        float* rstd_out, int8_t* q, uint8_t* scale, float* row_scale,
                        pr2_stream_t stream);

/* Bytes of workspace for the gradient of the weight (0 where T or d is out of its range).  Does not
 * decrease with T. */
size_t pr2_rms_norm_workspace_bytes(int64_t T, int32_t d);
/*
 * Its gradients, from h (x where there was no residual) and rstd:
 *   g = dy w,  dx = round(dh + r (g - h r^2 mean_i(g_i h_i))),  dweight = sum_t dy_t h_t r_t
 *   dy, h, dx [T, d] act_dtype; dh [T, d] or NULL: the gradient that reaches h beside the norm (its
 *   use as the residual stream).  dx is the gradient of x and of residual alike; it may be dy, dh or h.
 *   dweight [d] fp32, overwritten, or NULL when not wanted (then no workspace is needed)
 *   ws >= pr2_rms_norm_workspace_bytes(T, d)
 * A row of dx has the same bits in any batch.  Sums over rows in fp32 in a fixed order.  T = 0 writes
 * zeros to dweight.
 */
pr2_status pr2_rms_norm_backward(int64_t T, int32_t d, int act_dtype, const void* dy, const void* dh,
                                 const void* h, const float* rstd, const float* weight, void* dx,
                                 float* dweight, void* ws, size_t ws_bytes, pr2_stream_t stream);

/* Status name ("PR2_OK", ...); never NULL. */
const char* pr2_status_string(pr2_status s);
/* Detail of the last error on this thread ("" if none); valid until the next call. */
const char* pr2_last_error(void);
/* Library version string. */
const char* pr2_version(void);

/*
 * Measurement hooks (not part of the method).  While enabled, every kernel the library
 * enqueues is bracketed by a pair of HIP events recorded on the same stream.
 * pr2_profile_collect waits for the recorded events, adds each kernel's elapsed time to a
 * per-kernel-name total and fills up to `cap` entries of names / total_ms / launches,
 * returning the number of distinct kernel names seen since the last reset (or -1 on a HIP
 * error).  Names are static strings.  Not thread-safe; for single-threaded benchmarking.
 */
void pr2_profile_enable(int on);
void pr2_profile_reset(void);
int pr2_profile_collect(const char** names, double* total_ms, int64_t* launches, int cap);

#ifdef __cplusplus
}
#endif
#endif /* PR2_H */
