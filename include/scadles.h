/*
 * scadles.h -- C ABI of the ScaDLES data-parallel hot path on MI355X (gfx950).
 *
 * The hot path of one training step of ScaDLES (Tyagi & Swany, "ScaDLES:
 * Scalable Deep Learning over Streaming data at the Edge", arXiv 2301.08897):
 * K simulated edge devices each hold a flat fp32 gradient of n elements in the
 * HBM of one GPU. For every device the library
 *   1. keeps the Top-k entries by magnitude (Top-k sparsification, §III-C and
 *      §IV "High communication cost"), ties broken towards the lower index,
 *      with k = clamp(floor(ratio * n), 1, n) (compression ratio CR, §V-G);
 *   2. measures the energies ||g||^2 and ||Top-k(g)||^2 that drive the
 *      adaptive compression rule of §IV (send Top-k(g) when the relative
 *      energy loss is at most delta, else send g);
 * then
 *   3. aggregates all devices' (sparse or dense) gradients weighted by each
 *      device's streaming rate, g~ = sum_j r_j g_j (Eqn 4b, weights of Eqn 4a);
 *   4. applies the SGD update w <- w - eta_scaled * g~ (Eqn 4c).
 *
 * Conventions for every entry point:
 *   - Pointers marked (dev) are device pointers owned by the caller; the
 *     library never frees or retains them. Pointers marked (host) are host
 *     memory read during the call only.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Every device-side effect is asynchronous on that stream; outputs are
 *     valid once the stream has been synchronised.
 *   - No entry point allocates device memory. Scratch space is the
 *     caller-provided workspace `ws` of `ws_bytes` bytes (dev, 256-byte
 *     aligned), sized by the matching *_workspace_bytes() query. A workspace
 *     must not be shared by calls that may run concurrently.
 *   - All arguments are validated on the host before anything is launched; an
 *     invalid call returns a non-zero scadles_status, launches nothing, and
 *     scadles_last_error() describes the problem.
 *   - Gradients must be finite (NaN/Inf give unspecified results, never a
 *     memory fault). Magnitude ranking uses the 31-bit key bits(g) & 0x7FFFFFFF,
 *     so -0 and +0 rank equal and denormals are ranked exactly (no flushing).
 *   - Results are deterministic: re-running a call on the same inputs gives
 *     bit-identical outputs.
 */
#ifndef SCADLES_H
#define SCADLES_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SCADLES_OK = 0,
  SCADLES_EINVAL = 1,      /* invalid argument (NULL pointer, size, ratio, weight ...) */
  SCADLES_EWORKSPACE = 2,  /* workspace NULL, misaligned or smaller than required     */
  SCADLES_EHIP = 3,        /* the HIP runtime reported an error while launching        */
  SCADLES_EUNSORTED = 4,   /* validation mode only: a sparse set's idx is not strictly
                              ascending or holds an entry >= n                          */
  SCADLES_EINTERNAL = 5    /* validation mode only: an internal consistency check of a
                              selection failed (a radix pass missed, the threshold was
                              not found, or the kept count is not k)                   */
} scadles_status;

/* Largest number of devices one call accepts. */
#define SCADLES_MAX_DEVICES 64

/* One device's contribution to the weighted aggregation (Eqn 4b).
 * Sparse: idx (dev, k entries, strictly ascending, each < n) and val (dev, k
 * entries) hold the kept gradient entries; every other position is zero.
 * Dense: idx == NULL and k == n; val (dev, n entries) is the full gradient.
 * Empty: k == 0 (idx and val are ignored and may be NULL); contributes nothing.
 * idx and val must be 4-byte aligned.                                        */
typedef struct {
  const uint32_t* idx;
  const float* val;
  uint64_t k;
} scadles_sparse;

/* Number of entries Top-k keeps for a vector of n elements at compression
 * ratio `ratio` (§V-G: CR 0.1 keeps a tenth of the entries):
 * k = clamp(floor(ratio * n), 1, n), computed in IEEE double.
 * Returns 0 when n == 0, n > 2^32 - 1 or ratio is not in (0, 1].            */
uint64_t scadles_topk_k(uint64_t n, double ratio);

/* Workspace bytes needed by scadles_step_fused for K devices of n elements at
 * the given per-device compression ratios (host[K]); scadles_topk_select uses
 * K = 1. Returns 0 for arguments the calls would reject.                    */
size_t scadles_workspace_bytes(uint32_t K, uint64_t n, const double* ratios);

/* Workspace bytes needed by scadles_weighted_aggregate for K sets over n
 * positions. Returns 0 for arguments the call would reject.                 */
size_t scadles_aggregate_workspace_bytes(uint32_t K, uint64_t n);

/* Top-k sparsification of one gradient (§IV "High communication cost";
 * Top-k as in §III-C), with the energies of the adaptive rule.
 *   grad      (dev, n floats, 4-byte aligned) the gradient; not modified.
 *   n         1 <= n <= 2^32 - 1.
 *   ratio     compression ratio in (0, 1]; k = scadles_topk_k(n, ratio).
 *   idx, val  (dev, k entries each) receive the kept positions in strictly
 *             ascending order and their signed values (bit copies of grad).
 *             The kept set holds the k largest |grad|; among equal magnitudes
 *             the lower index is kept.
 *   energies  (dev, 2 doubles) or NULL: receives sum grad^2 and the sum over
 *             the kept entries, both accumulated in double.
 * Returns SCADLES_EINVAL for a NULL or misaligned pointer, n out of range or
 * a ratio outside (0, 1]; SCADLES_EWORKSPACE for an undersized workspace.   */
scadles_status scadles_topk_select(const float* grad, uint64_t n, double ratio,
                                   uint32_t* idx, float* val, double* energies,
                                   void* ws, size_t ws_bytes, void* stream);

/* scadles_topk_select without a workspace argument and without allocating,
 * for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation). The
 * workspace is a static array of SCADLES_NOALLOC_SCRATCH_BYTES bytes that the
 * library holds on every GPU it runs on until the process ends; its address is
 * looked up once per GPU, on the first call there. The call allocates nothing
 * and launches the same kernels as scadles_topk_select, with the same
 * results, and clears the parts of the scratch that must start at zero.
 * Every call on one GPU shares that GPU's scratch: calls that may overlap on
 * one GPU (several host threads, or streams that do not order them) race and
 * give unspecified results; order them on one stream. Arguments and errors as
 * for scadles_topk_select; in addition SCADLES_EWORKSPACE when the selection
 * needs more scratch than the maximum (scadles_workspace_bytes(1, n, &ratio) >
 * SCADLES_NOALLOC_SCRATCH_BYTES; e.g. a gradient of 143,667,240 elements fits
 * at ratio 0.01 but not at 0.1). The first call on a GPU may return
 * SCADLES_EHIP if the scratch address cannot be looked up.               */
#define SCADLES_NOALLOC_SCRATCH_BYTES ((size_t)128 << 20)
scadles_status scadles_topk_select_noalloc(const float* grad, uint64_t n, double ratio,
                                           uint32_t* idx, float* val, double* energies,
                                           void* stream);

/* Per-layer Top-k: the per-layer reading of the Top-k sparsification of §IV
 * (each layer of the model keeps its own top fraction) for K devices whose
 * flat gradients share one layer layout. Layer l is positions
 * [seg_off[l], seg_off[l+1]) of every gradient and keeps k_l =
 * scadles_topk_k(seg_off[l+1] - seg_off[l], ratio_j) entries of device j,
 * chosen as scadles_topk_select chooses them within the layer. Device j's
 * kept set is the union over its layers, written in ascending index order
 * (layer after layer, indices relative to the whole gradient) to idx[j] /
 * val[j]: scadles_layers_k(seg_off, L, ratio_j) entries.
 *   grads     (host[K] of dev pointers, seg_off[L] floats each, 4-byte aligned).
 *   seg_off   (host[L+1]) 0 = seg_off[0] < seg_off[1] < ... < seg_off[L] <= 2^32 - 1;
 *             1 <= L <= 2^24.
 *   ratios    (host[K]) in (0, 1].
 *   idx, val  (host[K] of dev pointers, 4-byte aligned).
 *   energies  (dev, 2K doubles) or NULL: E_all and E_kept of each whole gradient.
 *   ws        scadles_layers_workspace_bytes(K, seg_off, L, ratios) bytes.
 * Layers of at most "row_max" elements (scadles_set_option) are selected as
 * (device, layer) rows, all at once: one workgroup per row, or, for rows of
 * more than "row_split" elements, one workgroup per 16384-element part of the
 * row in each of its passes. Longer layers are selected by the selection of
 * scadles_topk_select, one layer after the other, overlapped with each other
 * on a second and third stream the library creates per GPU (default
 * priority; those streams start after the caller's earlier work on `stream`,
 * and the caller's stream waits for them before the call's work ends on it).
 * Results do not depend on these splits. Feed the sets to
 * scadles_weighted_aggregate for Eqn 4b, or use scadles_step_fused_layers.
 * Same error convention as above.                                           */
uint64_t scadles_layers_k(const uint64_t* seg_off, uint32_t L, double ratio);
size_t scadles_layers_workspace_bytes(uint32_t K, const uint64_t* seg_off, uint32_t L, const double* ratios);
scadles_status scadles_topk_select_layers(const float* const* grads, uint32_t K, const uint64_t* seg_off,
                                          uint32_t L, const double* ratios, uint32_t* const* idx,
                                          float* const* val, double* energies, void* ws, size_t ws_bytes,
                                          void* stream);

/* Weighted aggregation of K devices' contributions (Eqn 4b):
 *   dense[i] = sum over j = 0..K-1, in that order, of w_j * v_j(i)
 * where v_j(i) is device j's value at i (zero when i is not in a sparse set).
 * The sum is accumulated in double with one fused multiply-add per term and
 * rounded to float once, so the result does not depend on the launch shape.
 *   sets     (host[K]) the contributions, see scadles_sparse.
 *   weights  (host[K]) r_j of Eqn 4a: finite, >= 0, summing to 1 within
 *            K * 2^-23.
 *   dense    (dev, n floats, 16-byte aligned) overwritten; +0 where no device
 *            contributes.
 * Returns SCADLES_EINVAL for bad arguments; with the "validate" option set it
 * also synchronises `stream` and returns SCADLES_EUNSORTED if a set's idx is
 * not strictly ascending or reaches n. Without it such input gives
 * unspecified values (never an out-of-bounds access).                       */
scadles_status scadles_weighted_aggregate(const scadles_sparse* sets, const float* weights,
                                          uint32_t K, uint64_t n, float* dense,
                                          void* ws, size_t ws_bytes, void* stream);

/* SGD update (Eqn 4c): params[i] <- params[i] - lr * grad[i], evaluated as
 * one fused multiply-add in double and rounded to float once.
 *   params (dev, n floats) updated in place; grad (dev, n floats), may not
 *   alias params. Both 16-byte aligned. lr finite.                          */
scadles_status scadles_apply_sgd(float* params, const float* grad, uint64_t n, float lr,
                                 void* stream);

/* Momentum SGD with weight decay: the optimizer of the paper's evaluation
 * (§V training setup: momentum 0.9, weight decay 1e-4 for ResNet152 and
 * 5e-4 for VGG19), applied in place of the plain step of Eqn 4c. Per
 * element, without dampening or Nesterov:
 *   d         = grad[i] + weight_decay * params[i]
 *   buf[i]    = momentum * buf[i] + d
 *   params[i] = params[i] - lr * buf[i]     (with the buf[i] just stored)
 * Each line is evaluated in double as one fused multiply-add (every product
 * of two floats is exact in double) and rounded to float once. A zero-filled
 * buf gives buf = d on the first step; momentum = weight_decay = 0 is Eqn 4c.
 *   params, momentum_buf (dev, n floats) updated in place; grad (dev, n
 *   floats). All 16-byte aligned, no two overlapping. lr, momentum and
 *   weight_decay finite.                                                    */
scadles_status scadles_apply_momentum_sgd(float* params, float* momentum_buf, const float* grad, uint64_t n,
                                          float lr, float momentum, float weight_decay, void* stream);

/* One whole hot-path step for K devices in one call (the training step of
 * §IV): Top-k + energies for every device, the adaptive decision, weighted
 * aggregation and, optionally, the SGD update.
 *   grads      (host[K] of dev pointers, n floats each, 4-byte aligned).
 *   ratios     (host[K]) per-device compression ratio in (0, 1].
 *   delta      compression threshold of §IV: device j sends Top-k(g_j) when
 *              |E_all - E_kept| / E_all <= delta (E_all == 0 counts as 0) and
 *              its dense gradient otherwise. +INFINITY always compresses.
 *   weights    (host[K]) as for scadles_weighted_aggregate.
 *   idx, val   (host[K] of dev pointers) per-device outputs of k_j entries,
 *              exactly as scadles_topk_select writes them (always written,
 *              whatever the decision).
 *   dense      (dev, n floats, 16-byte aligned) receives g~ of Eqn 4b.
 *   energies   (dev, 2K doubles) or NULL: E_all and E_kept per device.
 *   compressed (dev, K bytes) or NULL: 1 if the device sent Top-k, else 0.
 *   params     (dev, n floats, 16-byte aligned) or NULL: when non-NULL the
 *              SGD update of Eqn 4c with learning rate lr is applied to it
 *              using the float g~ written to dense.
 * K <= SCADLES_MAX_DEVICES. Same error convention as above.                 */
scadles_status scadles_step_fused(const float* const* grads, uint32_t K, uint64_t n,
                                  const double* ratios, double delta, const float* weights,
                                  uint32_t* const* idx, float* const* val, float* dense,
                                  double* energies, uint8_t* compressed,
                                  float* params, float lr,
                                  void* ws, size_t ws_bytes, void* stream);

/* Options of scadles_step_fused_ex; an all-zero struct gives exactly
 * scadles_step_fused.
 *   momentum_buf  (dev, n floats, 16-byte aligned, not overlapping params or
 *                 dense) or NULL. When set, the update after the aggregation
 *                 is the momentum SGD of scadles_apply_momentum_sgd with
 *                 `momentum` and `weight_decay` (finite) in place of Eqn 4c,
 *                 computed from the float g~ written to dense; params is
 *                 then required.
 *   ewma          (dev, 2K doubles, 8-byte aligned) or NULL. When set, the
 *                 adaptive rule of §IV is applied to moving averages of each
 *                 device's energies kept here (the paper tracks them as an
 *                 exponentially weighted moving average but prints no
 *                 factor): ewma[2j], ewma[2j+1] <- ewma_beta * ewma + (1 -
 *                 ewma_beta) * (E_all, E_kept), in double; a device whose
 *                 pair is (0, 0) has no history and takes its energies as they
 *                 are. Zero-fill before the first step. ewma_beta in [0, 1);
 *                 0 is the instantaneous rule.
 *   counters      (dev, 3K uint64, 8-byte aligned) or NULL. When set, each
 *                 call adds per device j: counters[3j] += 1 if it sent Top-k,
 *                 counters[3j+1] += 1, counters[3j+2] += k_j if it sent
 *                 Top-k else n (floats sent; values only, as §V-G counts
 *                 them). The CNC ratio of §V-G is counters[3j] /
 *                 counters[3j+1].                                           */
typedef struct scadles_step_options {
  float* momentum_buf;
  float momentum;
  float weight_decay;
  double* ewma;
  double ewma_beta;
  uint64_t* counters;
} scadles_step_options;

/* scadles_step_fused with the options above (momentum SGD, moving-average
 * adaptive rule, CNC and floats-sent accounting). options must not be NULL.
 * Other arguments and errors as for scadles_step_fused.                    */
scadles_status scadles_step_fused_ex(const float* const* grads, uint32_t K, uint64_t n,
                                     const double* ratios, double delta, const float* weights,
                                     uint32_t* const* idx, float* const* val, float* dense,
                                     double* energies, uint8_t* compressed, float* params, float lr,
                                     const scadles_step_options* options, void* ws, size_t ws_bytes,
                                     void* stream);

/* The fused step with the per-layer Top-k: scadles_topk_select_layers for
 * every device, the adaptive rule of §IV on each device's whole-gradient
 * energies (with the moving average and accounting of `options`, which may
 * be NULL), then Eqn 4b over the layered sets (or the dense gradients of
 * devices that send g) and the update (Eqn 4c, or momentum SGD when
 * options->momentum_buf is set), as scadles_step_fused_ex does for the
 * whole-vector Top-k. idx[j] / val[j] hold scadles_layers_k(seg_off, L,
 * ratios[j]) entries; dense, params and the options as for
 * scadles_step_fused_ex; ws is scadles_step_layers_workspace_bytes(...) bytes.
 * Same error convention as above.                                           */
size_t scadles_step_layers_workspace_bytes(uint32_t K, const uint64_t* seg_off, uint32_t L, const double* ratios);
scadles_status scadles_step_fused_layers(const float* const* grads, uint32_t K, const uint64_t* seg_off, uint32_t L,
                                         const double* ratios, double delta, const float* weights,
                                         uint32_t* const* idx, float* const* val, float* dense, double* energies,
                                         uint8_t* compressed, float* params, float lr,
                                         const scadles_step_options* options, void* ws, size_t ws_bytes,
                                         void* stream);

/* Aggregation weights and learning-rate scale from streaming rates
 * (§IV "Heterogeneous streams", Eqn 4a and the linear scaling rule):
 *   b_j = clamp(S_j, b_min, b_max)   (batch bounded to [b_min, b_max]),
 *   r_j = b_j / sum_i b_i            (computed in double, stored as float),
 *   gamma = sum_i b_i / base_batch   (eta_scaled = gamma * eta).
 *   rates   (host[K]) S_j, finite and >= 0, not all zero after clamping.
 *   b_min <= b_max; pass 0 and +INFINITY for no bounds.
 *   weights (host[K]) receives r_j. gamma (host) may be NULL; if not,
 *   base_batch must be > 0.
 * Host-only; touches no GPU state.                                          */
scadles_status scadles_stream_weights(const double* rates, uint32_t K, double b_min,
                                      double b_max, double base_batch, float* weights,
                                      double* gamma);

/* ---- streaming buffers, batch sizes, weights and learning-rate scale --------
 * The step before the aggregation (§II-C, Eqns 2 and 3; §IV "Heterogeneous
 * streams" and "Limited memory and storage"): device j receives a continuous
 * stream of S_j samples per second into its buffer and trains one iteration
 * of t_j seconds on a batch of b_j = clamp(S_j, b_min, b_max) samples, or on
 * all it holds when that is fewer. After an iteration the samples that
 * arrived meanwhile join the buffer. Stream persistence keeps every sample;
 * stream truncation discards the residual the iteration left and keeps at
 * most S_j of the new arrivals (the newest), so its buffer stays O(S_j)
 * while persistence grows as (t_j S_j - b_j) T + S_j after T iterations
 * (Eqn 2). A continuous stream has delivered floor(S_j * us / 10^6) samples
 * after `us` microseconds; a buffer starts with one second of it (S_j).
 * Host-only: none of these calls touches GPU state.                         */
#define SCADLES_PERSISTENCE 0
#define SCADLES_TRUNCATION 1

/* One device's stream buffer. */
typedef struct scadles_stream {
  uint64_t rate;        /* S_j, samples per second, < 2^32                      */
  uint64_t elapsed_us;  /* stream time covered by the iterations so far         */
  uint64_t queued;      /* samples in the buffer                                */
  uint64_t trained;     /* samples trained on so far                            */
  uint64_t dropped;     /* samples discarded by truncation so far               */
} scadles_stream;

/* Sets st[j] to a fresh buffer of stream rate rate[j] (queued = rate[j]).
 *   rate (host[K]) < 2^32; st (host[K]).                                    */
scadles_status scadles_stream_init(uint32_t K, const uint64_t* rate, scadles_stream* st);

/* One training iteration of K devices: every device takes its batch from its
 * buffer (batch[j] = min(clamp(S_j, b_min, b_max), queued)), the weights and
 * learning-rate scale of that iteration follow from the batches as in
 * scadles_stream_weights (r_j = batch_j / sum batch, Eqn 4a; gamma = sum
 * batch / base_batch), then the arrivals of iter_us[j] microseconds join the
 * buffer under `policy`.
 *   st       (host[K], in/out) from scadles_stream_init.
 *   iter_us  (host[K]) this iteration's duration per device, < 2^32.
 *   b_min <= b_max (UINT64_MAX: no upper bound). policy: SCADLES_PERSISTENCE
 *   or SCADLES_TRUNCATION. base_batch > 0 when gamma is not NULL.
 *   batch (host[K]) or NULL; weights (host[K]) or NULL; gamma or NULL.
 * When no device holds a sample, weights are all 0 and gamma is 0 (there is
 * nothing to aggregate). Errors leave st unchanged.                        */
scadles_status scadles_stream_iteration(uint32_t K, scadles_stream* st, const uint64_t* iter_us, uint64_t b_min,
                                        uint64_t b_max, int policy, double base_batch, uint64_t* batch,
                                        float* weights, double* gamma);

/* T iterations of constant duration iter_us[j] from fresh buffers.
 *   queued (host[(T+1) x K]) or NULL: row t = buffer before iteration t, row T
 *   after the last; batch (host[T x K]) or NULL; dropped (host[K]) or NULL.   */
scadles_status scadles_stream_simulate(uint32_t K, const uint64_t* rate, const uint64_t* iter_us, uint64_t b_min,
                                       uint64_t b_max, int policy, uint64_t T, uint64_t* queued, uint64_t* batch,
                                       uint64_t* dropped);

/* ---- AdamW over many tensors at once ----------------------------------------------------
 * The optimizer that language models are trained with, in place of Eqn 4c:
 * the gradients are any tensors, or the parts of the aggregate of Eqn 4b. A
 * plan lists the tensors once; a step is one launch over all of them. Per
 * element, with t the step's number from 1 and every operation rounded once to
 * float in this order:
 *   g = grad * factor                  (with a clip; see scadles_grad_norm)
 *   m = beta1 * m + (1 - beta1) * g
 *   v = beta2 * v + (1 - beta2) * (g * g)
 *   d = sqrt(v) * (1 / sqrt(1 - beta2^t)) + eps
 *   param = param * (1 - lr * weight_decay) - (m / d) * (lr / (1 - beta1^t))
 * (the factors in parentheses are computed in double and rounded to float).
 *
 * 8-bit moments. Blocks of SCADLES_MOMENT_BLOCK consecutive elements of a
 * tensor share one word of `tops`: the largest step of m in its lower half, of
 * v in its upper half. The step of a value x is (bits(x) + u) >> 20 of the
 * bits of |x| (the exponent and three bits of the mantissa), at most 2039, u in
 * [0, 2^20) the dither ((i * A + t * B) mod 2^32) >> 12 of element i of its
 * tensor at step t: A, B = 0x9E3779B9, 0xBB67AE85 for m and 0x6A09E667,
 * 0x9E3779B9 for v. With base = max(top, span) - span, a code is step - base,
 * clamped to [0, span]: span 127 for m, whose sign is the code's bit 7 (0 for
 * code 0), 255 for v, where values > 0 have at least code 1. A code c > 0
 * stands for the float of bits (c + base) << 20. The update itself uses the
 * moments before this rounding. If a value of the block is not finite, all of
 * the block's codes stand for NaN. All-zero bytes are zero moments.
 *
 *   param  (dev, n floats, 4-byte aligned) updated in place.
 *   grad   (dev, n of the plan's type, aligned to it); not modified.
 *   m, v   (dev, 4-byte aligned) n floats each, or n bytes each with 8-bit
 *          moments.
 *   tops   (dev, ceil(n / SCADLES_MOMENT_BLOCK) words) with 8-bit moments,
 *          NULL else.
 *   copy   (dev, n bfloat16) or NULL: receives param rounded to nearest even.
 *   n      0 <= n <= 2^32 - 1; an empty tensor's pointers are ignored.
 *   weight_decay  finite; 0 for tensors without decay (biases, norms).
 * No two arrays of a tensor may overlap, nor those of different tensors (the
 * latter is not checked).                                                   */
#define SCADLES_F32 0
#define SCADLES_BF16 1
#define SCADLES_MOMENT_BLOCK 256
typedef struct scadles_adamw_tensor {
  float* param;
  const void* grad;
  void* m;
  void* v;
  uint32_t* tops;
  uint16_t* copy;
  uint64_t n;
  float weight_decay;
} scadles_adamw_tensor;

/* A plan: a small host struct filled by scadles_adamw_plan_build (its fields
 * are the library's), and a table in device memory of the caller that must
 * stay in place, unmodified, as long as the plan is used.                   */
typedef struct scadles_adamw_plan {
  void* table;
  uint64_t chunks_at, chunks, n;
  uint32_t moment_bits, grad_type, magic, reserved;
} scadles_adamw_plan;

/* Bytes of the table of a plan for these tensors (only their sizes are read);
 * 0 for arguments the build would reject: count outside [1, 2^20], a tensor
 * of more than 2^32 - 1 elements, or more than about 2^34 elements in all.  */
size_t scadles_adamw_plan_bytes(const scadles_adamw_tensor* tensors, uint32_t count);

/* Lists the tensors (host[count], read during the call) in a plan.
 *   moment_bits 32 or 8; grad_type SCADLES_F32 or SCADLES_BF16 (of all tensors).
 *   table  (dev, scadles_adamw_plan_bytes(...) bytes, 256-byte aligned).
 *   plan   (host) receives the handle.
 * The table is written by launches on `stream`; later calls on other streams
 * must be ordered after them. Calls with the same plan must not overlap.
 * Build again when a pointer, a size or a weight decay changes: a step goes on
 * with the addresses that it was built with.                                 */
scadles_status scadles_adamw_plan_build(const scadles_adamw_tensor* tensors, uint32_t count, int moment_bits,
                                        int grad_type, void* table, size_t table_bytes, scadles_adamw_plan* plan,
                                        void* stream);

/* Global norm of the plan's gradients and the clip factor that follows, in one
 * launch: norm = sqrt(sum of all grad^2), squares and sums in double in a fixed
 * order; factor = max_norm / norm where norm > max_norm, else 1.
 *   max_norm  > 0; +INFINITY never clips.
 *   clip      (dev, 2 floats, 4-byte aligned) receives norm and factor. If the
 *             norm is not finite (some gradient is not), the factor is NaN,
 *             and a step given this clip changes nothing.                    */
scadles_status scadles_grad_norm(const scadles_adamw_plan* plan, double max_norm, float* clip, void* stream);

/* One AdamW step of every tensor of the plan, in one launch.
 *   options (host) lr finite; beta1, beta2 in [0, 1); eps > 0 as a float;
 *           step the step's number, from 1 (a step that its clip turned off
 *           counts as one if the caller counts it).
 *   clip    (dev, 2 floats) from scadles_grad_norm, or NULL: gradients as
 *           they are.
 * Infinities and NaN in gradients without a clip go into the moments and
 * parameters they belong to (with 8-bit moments: their block's moments).     */
typedef struct scadles_adamw_options {
  double lr, beta1, beta2, eps;
  uint64_t step;
} scadles_adamw_options;
scadles_status scadles_adamw_step(const scadles_adamw_plan* plan, const scadles_adamw_options* options,
                                  const float* clip, void* stream);

/* The moments' values as floats, packed in the tensors' order (dev, as many
 * floats as all tensors have elements, 4-byte aligned, m and v not
 * overlapping): out of the plan's moments, or into them. 8-bit moments are
 * rounded with the dither of `step`; values that came from
 * scadles_adamw_get_moments are kept exactly.                                */
scadles_status scadles_adamw_get_moments(const scadles_adamw_plan* plan, float* m, float* v, void* stream);
scadles_status scadles_adamw_set_moments(const scadles_adamw_plan* plan, const float* m, const float* v,
                                         uint64_t step, void* stream);

/* ---- the router of a mixture of experts ----------------------------------------------------
 * The tokens of K devices (of streams of different rates, so of batches of
 * different sizes) are routed to E experts, k per token, and the losses that
 * keep the experts evenly used are taken over all devices with the Eqn 4a
 * weights, not device by device: a slow stream's few tokens say little about
 * the load. For row t of device d, x its logits and n_d the device's counted
 * rows:
 *   p = softmax(x), lse = log sum exp(x)
 *   idx  = the k experts of the largest x, in descending order, ties to the
 *          lower index (as scadles_topk_select breaks them)
 *   gate = p of those, divided by their sum if renormalise is set
 *   counts[d][e] = choices of e by d's rows
 *   load_e = sum_d weights[d] * counts[d][e] / (k * n_d)
 *   prob_e = sum_d weights[d] / n_d * sum_t p_e
 *   loss[0] = E * sum_e load_e * prob_e           (balance; 1 when even)
 *   loss[1] = sum_d weights[d] / n_d * sum_t lse^2    (z)
 * Softmax statistics are kept in float. Sums over rows are taken in a fixed
 * order: of lse^2 in double; of probabilities in float over the rows of a
 * workgroup and then of up to 16 workgroups, fewer than 300 additions of values
 * that are not negative (relative error below 300 * 2^-24), and from there in
 * double. All of this holds for finite logits of any size; loss[1] is infinite
 * where it passes the largest float. An expert at -infinity is never chosen:
 * missing choices have index -1 and gate 0. A row with `valid` 0, or with every
 * logit at -infinity, routes nowhere: indices -1, gates, lse and gradient 0, not
 * counted. A device without counted rows adds nothing. A NaN or +infinity makes its row's gates, lse and
 * gradient and the losses NaN; indices stay within [-1, E).                  */
#define SCADLES_ROUTER_MAX_EXPERTS 1024
#define SCADLES_ROUTER_MAX_K 16

/* Shape of a call.
 *   tokens       rows of logits, 0 <= tokens <= 2^31 - 1.
 *   experts, k   1 <= experts <= SCADLES_ROUTER_MAX_EXPERTS; 1 <= k <=
 *                min(experts, SCADLES_ROUTER_MAX_K).
 *   devices      1 <= devices <= SCADLES_MAX_DEVICES.
 *   tok_off      (host[devices + 1]) rows [tok_off[d], tok_off[d + 1]) are
 *                device d's; from 0 to tokens, not decreasing.
 *   weights      (host[devices]) finite and >= 0.
 *   ld           elements between the starts of two rows, >= experts.
 *   logits_type  SCADLES_F32 or SCADLES_BF16.                                */
typedef struct scadles_router {
  uint64_t tokens;
  uint64_t ld;
  const uint64_t* tok_off;
  const float* weights;
  uint32_t experts, k, devices;
  int32_t logits_type;
  int32_t renormalise;
} scadles_router;

/* What the forward pass writes and the backward pass reads (dev, 4-byte
 * aligned, not overlapping): idx and gate tokens x k, lse tokens, counts
 * devices x experts, load experts, share devices (1 / n_d, 0 without rows),
 * loss 2.                                                                    */
typedef struct scadles_router_out {
  int32_t* idx;
  float* gate;
  float* lse;
  int32_t* counts;
  float* load;
  float* share;
  float* loss;
} scadles_router_out;

/* Workspace bytes of scadles_router_forward for up to `tokens` rows, however
 * they are spread over the devices; 0 for arguments the call would reject.  */
size_t scadles_router_workspace_bytes(uint64_t tokens, uint32_t experts, uint32_t devices);

/* Forward pass.
 *   logits  (dev, tokens rows of experts elements, aligned to its type).
 *   valid   (dev, tokens bytes) or NULL: 0 marks rows that are padding.
 *   router->weights must sum to 1 within devices * 2^-23.                    */
scadles_status scadles_router_forward(const scadles_router* router, const void* logits, const uint8_t* valid,
                                      const scadles_router_out* out, void* ws, size_t ws_bytes, void* stream);

/* Gradient of the logits, with load held constant:
 *   dlogits = weights[d] / n_d * p * (dloss[0] * E * (load - sum_j load_j p_j)
 *             + 2 * dloss[1] * lse) + the gradient of the gates under dgate.
 *   router   as in the forward pass, except for the weights, which need not
 *            sum to 1: the forward's give the gradient of its losses; ones
 *            give each device's own share, for scadles_weighted_aggregate
 *            to weight.
 *   out      the forward pass's; counts and loss are not read. An index outside
 *            [0, experts) is a missing choice.
 *   dgate    (dev, tokens x k floats) or NULL (zero).
 *   dloss    (dev, 2 floats) or NULL (zero).
 *   dlogits  (dev, tokens rows of experts elements of the logits' type, ld_out
 *            elements between rows) overwritten; may not overlap an input.    */
scadles_status scadles_router_backward(const scadles_router* router, const void* logits, const scadles_router_out* out,
                                       const float* dgate, const float* dloss, void* dlogits, uint64_t ld_out,
                                       void* stream);

/* Message for the last non-OK status returned on the calling thread.        */
const char* scadles_last_error(void);

/* Process-wide options, for testing and diagnosis:
 *   "validate"       1: scadles_weighted_aggregate checks its sets, and
 *                       scadles_topk_select(_noalloc), scadles_step_fused and
 *                       scadles_step_fused_ex read every device's selection
 *                       state back after the call and return
 *                       SCADLES_EINTERNAL if its internal checks failed;
 *                       scadles_topk_select_layers and
 *                       scadles_step_fused_layers do the same for their
 *                       layers that are not rows, see "row_max" (all of these
 *                       then synchronise `stream`).
 *   "inject_count_error" 1 (testing): the multi-launch selection (of the
 *                       whole vector, and of a per-layer selection's long
 *                       layers) reports a failed count check for device 0
 *                       (its outputs are unaffected), to exercise the
 *                       validation above.
 *   "force_exact"    1: Top-k skips the sampled single-read path and always
 *                       runs the exact multi-pass radix select.
 *   "force_fallback" 1: the sampled path runs but its result is discarded as
 *                       if the bracket had missed, exercising the fallback.
 *   "parts"          1..4 (default 1): device groups whose selections are
 *                       pipelined in scadles_step_fused (group i's main pass
 *                       overlaps the end of group i-1's selection, which runs
 *                       on a second stream the library creates per GPU, at the
 *                       default priority). Results do not depend on it.
 *   "row_max"        -1..2^32-1 (default -1): in the per-layer selection,
 *                       layers of at most this many elements are selected as
 *                       (device, layer) rows; longer ones by the multi-launch
 *                       selection, consecutive ones pipelined on the library's
 *                       second stream and the rows on a third. -1: layers of
 *                       up to 2^21 elements, and of up to 2^22 where their
 *                       rows can be split (see row_split) and few enough
 *                       entries are kept. The kept sets do not depend on it
 *                       (the energies are summed in another order).
 *   "row_split"      0..2^32-1 (default 65536, the least that takes effect):
 *                       rows of more than this many elements (and at most
 *                       2^24) are read by one workgroup per 16384-element part
 *                       (their candidates staged, so each row is read once)
 *                       instead of one workgroup per row, unless their ratio
 *                       is so high that a part's candidates could exceed half
 *                       its elements. Results do not depend on it.
 *   "layer_order"    0..2 (default 1): the order in which the per-layer
 *                       selection runs its layers of more than "row_max"
 *                       elements: 0 index order, 1 ascending length (the
 *                       longest last, so the end of every earlier layer's
 *                       selection overlaps a long main pass), 2 descending
 *                       length. Every layer writes its own part of the
 *                       outputs and of the energy sums, so results do not
 *                       depend on it.
 * Returns SCADLES_EINVAL for an unknown name or a value out of range.       */
scadles_status scadles_set_option(const char* name, int64_t value);

/* Stage timing. While enabled, every scadles_topk_select / scadles_step_fused
 * call records HIP events on its stream at the boundaries of its stages.
 * scadles_profile_read synchronises those events, writes the summed
 * milliseconds of each stage to stage_ms (host[SCADLES_PROFILE_STAGES]) and
 * the number of calls recorded to *calls, and clears the record.
 * Stages: 0 bracket (sampling), 1 main select pass (one read of every
 * gradient; the sum over the device groups), 2 the rest of the selection
 * after the last main pass (exact threshold, ordered compaction, energies;
 * earlier groups' share overlaps the main passes), 3 weighted aggregation
 * (+SGD; empty for scadles_topk_select), 4 the whole call.                  */
#define SCADLES_PROFILE_STAGES 5
scadles_status scadles_profile_enable(int on);
scadles_status scadles_profile_read(double* stage_ms, uint32_t* calls);

#ifdef __cplusplus
}
#endif

#endif /* SCADLES_H */
