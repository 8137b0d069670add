/*
 * map_gb300.h -- C ABI of the GB300 (sm_103a) implementation of MAP's inference-time
 * visual-token pruning path (arxiv 2608.06411, "Learning to Predict Middle-layer
 * Attention in MLLMs for Visual Token Pruning").
 *
 * The path:  (T, V) --map_score--> p_hat --map_select--> keep set --map_gather--> tokens
 *
 * Conventions for every call
 *   - Tensors are plain pointers to row-major, densely packed arrays; bf16 tensors are
 *     passed as void* to 16-bit storage.  Unless a call says otherwise, pointers are
 *     DEVICE pointers owned by the caller and must stay valid until the stream work
 *     completes; map_prune alone also accepts host pointers.
 *   - `stream` is a cudaStream_t passed as void* (NULL = legacy default stream).  Work
 *     is enqueued asynchronously on it; the call returns once enqueued.
 *   - Return value: MAP_OK (0) or a negative MAP_E* code.  Arguments are validated on
 *     the host before anything is enqueued; on an argument error nothing is enqueued.
 *     Device-side failures (a bounded wait that ran out) are recorded in the context
 *     and reported by map_status.
 *   - A context is not thread-safe: one host thread (and one stream at a time) per
 *     context.  Workspace is owned by the context, allocated on first use and grown on
 *     demand (growth synchronises the device).
 */
#ifndef MAP_GB300_H
#define MAP_GB300_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MAP_OK            0
#define MAP_EINVAL       -1   /* bad argument (null pointer, size, alignment) */
#define MAP_ENOMEM       -2   /* device or host allocation failed */
#define MAP_ECUDA        -3   /* a CUDA runtime / driver call failed */
#define MAP_ETIMEOUT     -4   /* a bounded device-side wait ran out (kernel aborted) */
#define MAP_EUNSUPPORTED -5   /* shape outside what the kernels support (see each call) */
#define MAP_EINTERNAL    -6   /* device-side consistency check failed */

typedef struct map_ctx map_ctx;   /* opaque, owned by the library */

/*
 * Predictor and selection settings.
 *   D, Dh, dp  feature width, predictor MLP width, query/key width d of Eq. 3.
 *              The paper calls the predictor lightweight without giving widths; the
 *              defaults are Dh = 1024, dp = 128 (D = 4096 for LLaVA-NeXT-7B).
 *              Supported: D % 64 == 0, Dh % 256 == 0, dp in {64, 128}.
 *   rope_theta RoPE base (10000); rope_on = 1 applies RoPE to q and k as the paper's
 *              predictor does (section "Cross-Modal Attention Distillation"); 0 turns it
 *              off (used by tests of permutation equivariance).
 *   k0_frac, k0_abs  |R0| (section "Inference-Time Token Pruning"): k0_abs if >= 0,
 *              else floor(k0_frac * K); clamped to [0, K].  The paper does not state
 *              K0; the default is K/2.
 *   lambda     diversity weight: value_i = p_hat_i * rho_i^lambda.  lambda = 1 is Eq. 4;
 *              lambda = 0 reduces the selection to the top-K of p_hat.
 *   tau        a residual with rho_i^2 <= tau * ||v_i||^2 counts as zero (the token is
 *              already in the span); picking such a token keeps it without extending
 *              the basis.  Default 1e-5.
 */
typedef struct {
    int   D, Dh, dp;
    float rope_theta;
    int   rope_on;
    float k0_frac;
    int   k0_abs;
    float lambda;
    float tau;
} map_config;

/* Predictor weights, bf16, PyTorch Linear layout [out, in]; host OR device pointers
 * (map_init copies them).  f_T: wT1 [Dh, D], bT1 [Dh], wT2 [Dh, Dh], bT2 [Dh];
 * W_Q: wQ [dp, Dh]; f_V: wV1, bV1, wV2, bV2 likewise; W_K: wK [dp, Dh]. */
typedef struct {
    const void *wT1, *bT1, *wT2, *bT2, *wQ;
    const void *wV1, *bV1, *wV2, *bV2, *wK;
} map_weights;

/* Fills *cfg with the defaults above (D = 4096, Dh = 1024, dp = 128, theta = 1e4,
 * rope on, K0 = K/2, lambda = 1, tau = 1e-5).  Returns MAP_EINVAL for NULL. */
int map_config_default(map_config *cfg);

/* Creates a context on the current CUDA device, copying the weights (synchronous).
 * Returns MAP_EINVAL for a bad config or NULL pointers, MAP_ENOMEM / MAP_ECUDA on
 * failure (then *out is NULL). */
int map_init(const map_config *cfg, const map_weights *w, map_ctx **out);

/*
 * Predicted attention, Eq. 3 (section "Cross-Modal Attention Distillation"):
 *   p_hat[b, n] = (1/M_b) sum_m softmax_n( <RoPE(W_Q f_T(t_m)), RoPE(W_K f_V(v_n))> / sqrt(dp) )
 * with visual token n at position n and question token m at position N + m.
 *   text_feats  bf16 [sum(lens), D]: the question tokens of all images, packed in
 *               image order (device).
 *   vis_feats   bf16 [B, N, D] (device), 16-byte aligned.
 *   lens        int32 [B] HOST array: question tokens per image, each >= 1.
 *   scores      float32 [B, N] output (device).
 * B >= 1, N >= 1.  Inputs and weights are bf16; every product is accumulated in fp32,
 * and the hidden MLP activations are kept to about 16 significant bits (a bf16 pair)
 * rather than rounded to bf16; q, k, logits and p_hat are fp32.
 */
int map_score(map_ctx *ctx, const void *text_feats, const void *vis_feats,
              const int32_t *lens, int B, int N, float *scores, void *stream);

/*
 * Diversity-aware selection, Eq. 4 (section "Inference-Time Token Pruning"):
 * R0 = top-K0 by p_hat (ties to the lower index), then greedily
 *   i_t = argmax_{i in C} p_hat_i * ||v_i - B B^T v_i||^lambda
 * until k tokens are kept (ties to the lower index).
 *   scores      float32 [B, N] (device), p_hat from map_score (or any non-negative
 *               importance).
 *   vis_feats   bf16 [B, N, D] (device): the embeddings v_i of the diversity term.
 *   keep_idx    int32 [B, k] output (device): kept token indices restored to ascending
 *               original order; they are also the kept tokens' position ids.
 *   pick_order  int32 [B, k] output (device) or NULL: the same tokens in the order they
 *               were retained (R0 in p_hat order first).
 * k == N keeps every token (keep_idx = pick_order = 0..N-1); k == 0 is a no-op;
 * k > N is MAP_EINVAL.  Supported: N <= 16384; k <= 4096 for plain top-k (lambda = 0 or
 * K0 = k), k <= 768 with the diversity term (MAP_EUNSUPPORTED beyond).
 * Asynchronous like the other calls: after its first rounds the selection runs as a
 * device-side loop (a CUDA graph whose WHILE node repeats a round while an image still
 * selects; built on the first call of a shape and workspace, then cached in the context), so
 * the host never waits for it.  A device-side failure (a bounded wait that ran out, or the
 * loop's iteration cap, set at the most rounds the selection can take:
 * k * (ceil(N / 256) + 1) + ceil(k / 88) + 64) is reported by map_status.
 */
int map_select(map_ctx *ctx, const float *scores, const void *vis_feats, int B, int N,
               int k, int32_t *keep_idx, int32_t *pick_order, void *stream);

/*
 * Compaction (last step of section "Inference-Time Token Pruning"):
 *   out[b, j, :] = vis_feats[b, keep_idx[b, j], :]   (a bit copy of bf16 rows)
 * vis_feats [B, N, D], out [B, k, D], keep_idx [B, k] (device).  vis_feats and out
 * must be 16-byte aligned (MAP_EINVAL otherwise).  Indices outside [0, N) are not
 * copied; they set MAP_EINTERNAL for map_status.
 */
int map_gather(map_ctx *ctx, const void *vis_feats, const int32_t *keep_idx, int B, int N,
               int k, void *out, void *stream);

/*
 * Hand-off to the language model (last paragraph of section "Inference-Time Token
 * Pruning"): the kept tokens, restored to their original order, keep their positional
 * indices and are combined with the question tokens.  For image b, whose sequence starts
 * at row o_b = b k + sum_{b' < b} lens[b'] of `seq`:
 *   seq[o_b + j]     = vis_feats[b, keep_idx[b, j]],  pos_ids[o_b + j]     = keep_idx[b, j] + pos_offset
 *   seq[o_b + k + m] = text_feats[t_b + m],           pos_ids[o_b + k + m] = N + m + pos_offset
 * for j < k and m < lens[b], with t_b = sum_{b' < b} lens[b'] (the question follows the
 * whole image, as in map_score).  pos_offset shifts every position (e.g. by the length of
 * a system prompt placed before the image).
 *   vis_feats  bf16 [B, N, D]; keep_idx int32 [B, k] (map_select's output);
 *   text_feats bf16 [sum(lens), D]; lens int32 [B] HOST array, each >= 0;
 *   seq        bf16 [sum_b (k + lens[b]), D] output; pos_ids int32 [same rows] output.
 * Device pointers, caller-owned; vis_feats, text_feats and seq 16-byte aligned (MAP_EINVAL
 * otherwise); 0 <= k <= N.  An index outside [0, N) is not copied: its pos_ids entry is
 * -1 and map_status reports MAP_EINTERNAL.
 */
int map_assemble(map_ctx *ctx, const void *vis_feats, const int32_t *keep_idx,
                 const void *text_feats, const int32_t *lens, int B, int N, int k,
                 int pos_offset, void *seq, int32_t *pos_ids, void *stream);

/*
 * The hand-off for a language model whose rotary positions have three axes (time, height,
 * width), as image and video models use them: map_assemble_ragged's rows, with position ids
 * on each axis.  Image b is a grid of T x H x W visual tokens, its rows 0 .. T H W - 1 of
 * vis_feats in time-major order (H W per frame, W per row of a frame).
 *   kept token n:     (n / (H W)) * t_step,  (n / W) % H,  n % W
 *   question token m: max((T - 1) * t_step + 1, H, W) + m  on every axis
 * each plus pos_offset: a pruned image's question sits where the whole image's would.
 *   grids    int32 [B, 3] HOST array: T, H, W >= 1 of each image, T H W <= N, k <= T H W.
 *   t_step   int32 [B] HOST array: positions from one frame to the next, >= 0; NULL: 1.
 *   pos_ids  int32 [3, sum_b (k + lens[b])] output (device): time, height, width.
 * Everything else as for map_assemble.  An index outside [0, T H W) is not copied: its ids are
 * -1 and map_status reports MAP_EINTERNAL.  Positions must stay below 2^31 (MAP_EUNSUPPORTED).
 */
int map_assemble_axes(map_ctx *ctx, const void *vis_feats, const int32_t *keep_idx,
                      const void *text_feats, const int32_t *lens, const int32_t *grids,
                      const int32_t *t_step, int B, int N, int k, int pos_offset, void *seq,
                      int32_t *pos_ids, void *stream);

/*
 * map_select without allocating memory in the call (the paper has no counterpart; this
 * is a deployment variant of map_select).  Same arguments and limits as map_select, and
 * the same exact greedy picks (a near-tie below fp32 resolution may go either way, as
 * between any two fp32 evaluations), but every scratch buffer is carved from one static
 * device array of MAP_NOALLOC_SCRATCH_BYTES, held by each GPU that loads the library
 * until the process exits.  It is for callers that cannot allocate device memory while
 * they prune: code that runs inside another framework's caching pool or under a fixed
 * device-memory budget, where a cudaMalloc would take memory the budget does not have or
 * fail, and serving paths that must not stall on the allocator (cudaMalloc and cudaFree
 * may synchronise the device).  The call makes no cudaMalloc / cudaFree and allocates
 * through no library.
 * Workspace needed, in bytes (each array rounded up to 256): 17 B*N + 16 B*k + 4 B*256
 * + 8 B + small per-image counters, plus, when the diversity term is on (lambda > 0 and
 * K0 < k), 4 B*N*ceil4(k) + 2 B*R*D + 4 B*256*R with R = ceil16(256 + k).  A request
 * that does not fit returns MAP_EUNSUPPORTED and does nothing.  One LLaVA-NeXT image
 * (N = 2880, k = 160, D = 4096) counts as about 6 MB.  (2 B*R*D of it is reserved and no longer
 * written: the same requests fit as before.)
 * Unlike map_select, whose later rounds run as a device-side loop, it waits on the host
 * for bursts of selection rounds (it synchronises `stream`); a device-side error is
 * returned and also recorded for map_status.  It skips map_select's tensor-core
 * projection pass (every candidate starts from its bound p_hat * ||v||^lambda), so it
 * runs more selection rounds for the same picks.
 * The first call on a device looks the array's address up (device must be current);
 * make that call before any stream capture.  All calls share the array and it keeps the
 * last call's contents; calls whose GPU work overlaps (other streams, other threads)
 * race on it and must be serialised by the caller.
 */
#define MAP_NOALLOC_SCRATCH_BYTES (16u * 1024u * 1024u)
int map_select_noalloc(map_ctx *ctx, const float *scores, const void *vis_feats, int B, int N,
                       int k, int32_t *keep_idx, int32_t *pick_order, void *stream);

/*
 * The whole path in one call: score, select, gather.  Pointers may be HOST or DEVICE
 * memory (detected per pointer); host inputs are copied in and host outputs copied out
 * on `stream`, and the call synchronises `stream` before returning when any pointer is
 * host memory.  text_feats, vis_feats, lens as for map_score (lens is always host);
 * out bf16 [B, k, D]; keep_idx int32 [B, k]; scores float32 [B, N] or NULL.
 */
int map_prune(map_ctx *ctx, const void *text_feats, const void *vis_feats,
              const int32_t *lens, int B, int N, int k, void *out, int32_t *keep_idx,
              float *scores, void *stream);

/*
 * Question Contrastive Teacher Selection (section "Question Contrastive Teacher
 * Selection", Eq. 1 and Eq. 2): the teacher layer whose attention supervises the
 * predictor during training.  For every sample b and language-model layer l:
 *   a^l_n     = 1/(H M_b) sum_h sum_m A^l[h, m, n]                        (Eq. 1)
 *   p^l       = a^l / sum_n a^l_n          (l1 normalisation over visual tokens)
 *   p_ref^l   = the same for the reference question's attention (M_ref tokens)
 *   js[b, l]  = D_JS(p^l, p_ref^l) in nats (natural logarithm)
 *   teacher[b] = l* = argmax_l js[b, l], ties to the lower layer               (Eq. 2)
 * A layer whose aggregate sums to zero (M_b = 0, or attention that is all zero) gets the
 * uniform distribution 1/N.  Context-free: it needs no map_init and no workspace.
 *   attn       bf16, the samples' text-to-vision attention, packed in sample order: sample
 *              b is a dense [L, H, lens[b], N] block (row (h, m) of layer l holds the
 *              attention of question token m to the N visual tokens at head h).  Values
 *              must be finite and non-negative (attention probabilities).
 *   lens       int32 [B] HOST array: question tokens M_b per sample, each >= 0.
 *   attn_ref   bf16 [B, L, H, M_ref, N]: the reference question's attention.
 *   p, p_ref   float32 [B, L, N] outputs: the distributions p^l and p_ref^l.
 *   js         float32 [B, L] output; teacher int32 [B] output (while the call runs it
 *              also counts the finished layers of each sample).
 *   teacher_p  float32 [B, N] output (p^{l*} of each sample) or NULL.
 * All device pointers, caller-owned; attn and attn_ref 2-byte aligned (16-byte alignment
 * with N % 8 == 0 takes the fastest path).  B, L, H, N, M_ref >= 1 (MAP_EINVAL
 * otherwise); L <= 65535.  Asynchronous on `stream`; no device-side error conditions.
 */
int map_qcts(const void *attn, const int32_t *lens, const void *attn_ref, int M_ref, int B,
             int L, int H, int N, float *p, float *p_ref, float *js, int32_t *teacher,
             float *teacher_p, void *stream);

/*
 * Ragged batches (variable-resolution images, e.g. Qwen2.5-VL's dynamic token counts): the
 * same three steps on a padded layout.  vis_feats is [B, N, D] with N the largest token
 * count; image b's visual tokens are rows 0 .. n_valid[b]-1 and the rows after them are
 * padding whose contents are never used.  n_valid int32 [B] is a HOST array with
 * 1 <= n_valid[b] <= N (MAP_EINVAL otherwise).  Per image, the results equal those of the
 * unpadded call on its n_valid[b] tokens: Eq. 3's softmax runs over n < n_valid[b] only and
 * the question follows the image (positions n_valid[b] + m); scores[b, n] = 0 for padding;
 * the selection never retains padding, so k <= min_b n_valid[b] (MAP_EINVAL otherwise).
 * Other arguments, limits and buffer rules as for map_score / map_select / map_prune
 * (map_prune_ragged also accepts host buffers).  The padding rows still pass through the
 * predictor's GEMMs, so the cost is that of the padded batch.
 */
int map_score_ragged(map_ctx *ctx, const void *text_feats, const void *vis_feats,
                     const int32_t *lens, const int32_t *n_valid, int B, int N, float *scores,
                     void *stream);
int map_select_ragged(map_ctx *ctx, const float *scores, const void *vis_feats,
                      const int32_t *n_valid, int B, int N, int k, int32_t *keep_idx,
                      int32_t *pick_order, void *stream);
int map_prune_ragged(map_ctx *ctx, const void *text_feats, const void *vis_feats,
                     const int32_t *lens, const int32_t *n_valid, int B, int N, int k, void *out,
                     int32_t *keep_idx, float *scores, void *stream);
/* map_assemble for a ragged batch: question token m of image b sits at position
 * n_valid[b] + m (+ pos_offset), and kept indices must lie in [0, n_valid[b]). */
int map_assemble_ragged(map_ctx *ctx, const void *vis_feats, const int32_t *keep_idx,
                        const void *text_feats, const int32_t *lens, const int32_t *n_valid,
                        int B, int N, int k, int pos_offset, void *seq, int32_t *pos_ids,
                        void *stream);

/*
 * Predictor distillation step (section "Cross-Modal Attention Distillation"): the predictor
 * is trained offline by minimising D_KL(p^{l*} || p_hat) (the teacher distribution chosen by
 * QCTS, e.g. map_qcts's teacher_p, against Eq. 3's prediction).  This call computes the batch
 * loss  L = (1/B) sum_b sum_n p*_b[n] log(p*_b[n] / p_hat_b[n])  (0 log 0 = 0) with the
 * context's weights and the gradient dL/dW of every predictor weight, through Eq. 3's
 * softmax-mean, RoPE, W_Q / W_K and both MLPs (the second MLP layer and the projection are
 * kept separate here, unlike the inference path).  The optimiser update is the caller's.
 *   text_feats, vis_feats, lens  as for map_score (lens HOST, each >= 1).
 *   teacher    float32 [B, N] (device): each row a distribution over the N visual tokens.
 *   loss       float32 [1] output (device).
 *   grads      float32 device outputs, each with its weight's shape (wT1 [Dh, D], bT1 [Dh],
 *              wT2 [Dh, Dh], bT2 [Dh], wQ [dp, Dh], and the same for V / K); overwritten.
 * fp32 arithmetic throughout (bf16 inputs decoded exactly); deterministic.  Workspace (about
 * (B N + sum(lens)) (32 Dh + 20 dp) + 10 P N bytes, P the question tokens with each image's rounded up
 * to 64, plus the K slices of contractions with few output tiles and a copy of features that are
 * not 16-byte aligned) is owned by the context.
 * B N <= 2097120 and sum(lens) <= 2097120 (MAP_EUNSUPPORTED beyond).
 */
typedef struct {
    float *wT1, *bT1, *wT2, *bT2, *wQ;
    float *wV1, *bV1, *wV2, *bV2, *wK;
} map_grads;

int map_distill_grad(map_ctx *ctx, const void *text_feats, const void *vis_feats,
                     const int32_t *lens, const float *teacher, int B, int N, float *loss,
                     const map_grads *grads, void *stream);

/* ---------------------------------------------------------------- queries and keys
 * What a language model does with the hand-off sequence before its attention: the norm of
 * each query and key head and the rotation by position, forward and backward.  Context-free
 * like map_qcts: no map_init, no device workspace of the library's own.
 */

/* Element types of the calls below. */
#define MAP_BF16 0
#define MAP_F16  1
#define MAP_F32  2

/* Heads of `heads` vectors a row: element (r, h, i) at p[r * row + h * head + i] (strides in
 * elements, >= 0).  A view of one projection's output, or [heads, rows, dh] arrays, need no copy. */
typedef struct {
    void *p;
    long long row, head;
    int heads;
} map_heads;

/*
 * A rotation plan: host memory only, immutable, usable from any thread, stream and device.
 *   dh        head width, 1 .. 256.
 *   rot       columns that are rotated, the first of each head: even, 0 .. dh.
 *   adjacent  0: pair i is columns (i, i + rot / 2); 1: columns (2 i, 2 i + 1).
 *   n_axes    position axes, 1 .. 4.
 *   inv_freq  double [rot / 2] HOST: radians per position of each pair, finite.
 *   axis      int32 [rot / 2] HOST: the axis whose position turns the pair, 0 .. n_axes - 1
 *             (time, height and width in runs, by turns, or any other way); NULL: axis 0.
 *   eps       added to the mean square of a head before its root, >= 0.
 * The angle pos * inv_freq is taken modulo 2 pi in 64-bit fixed point: within 2^-29 radians for
 * any int32 position and frequencies up to 2^40.  Returns MAP_EINVAL for arguments outside these ranges.
 */
typedef struct map_rope map_rope;
int map_rope_init(int dh, int rot, int adjacent, int n_axes, const double *inv_freq, const int32_t *axis,
                  double eps, map_rope **out);
void map_rope_destroy(map_rope *rope);

/*
 * Per head x of q and k:  z = x * (mean_i x_i^2 + eps)^(-1/2) * w   (z = x where w is NULL),
 * then pair (a, b) of the rotated columns:  (z_a cos t - z_b sin t, z_b cos t + z_a sin t),
 * t = pos[axis, row] * inv_freq.  Computed in fp32, rounded once to the output's type.
 *   type      MAP_BF16, MAP_F16 or MAP_F32: of q, k, wq, wk and the outputs.
 *   pos       int32 [n_axes, rows] (device); NULL only if rot = 0.
 *   q, k      inputs; either may be absent (NULL or heads = 0).
 *   wq, wk    [dh] norm weights (device) or NULL: no norm of that side.
 *   q_out, k_out  outputs with the inputs' heads; they may be the inputs themselves (same p,
 *             row and head), else must not overlap them.  Vectors of one output must not
 *             overlap each other (MAP_EINVAL).
 * rows >= 0 (0: no-op), rows * heads < 2^31 per side.  16-byte aligned bases, strides that are
 * multiples of 8 elements and dh and rot / 2 that are multiples of 8 take the widest accesses.
 */
int map_qk_rotate(const map_rope *rope, int type, long long rows, const int32_t *pos, const map_heads *q,
                  const map_heads *k, const void *wq, const void *wk, const map_heads *q_out,
                  const map_heads *k_out, void *stream);

/*
 * Gradient of map_qk_rotate.  dq_out, dk_out: gradients of its outputs; q, k: its inputs (only
 * read where wq / wk is given; else may be NULL); dq, dk: outputs, of `type` (may be dq_out,
 * dk_out themselves); dwq, dwk: float [dh] outputs, overwritten, for the sides with a norm:
 * sums over all rows and heads in fp32, in a fixed order.  ws: device scratch of
 * map_qk_rotate_grad_workspace(rope) bytes, 16-byte aligned, the caller's until the call's work
 * completes (may be NULL without norms).  Other arguments as for map_qk_rotate.  rows = 0 zeroes
 * dwq and dwk, a dq_out or dk_out of 0 heads that of its side (NULL leaves it alone).
 */
size_t map_qk_rotate_grad_workspace(const map_rope *rope);
int map_qk_rotate_grad(const map_rope *rope, int type, long long rows, const int32_t *pos,
                       const map_heads *dq_out, const map_heads *dk_out, const map_heads *q, const map_heads *k,
                       const void *wq, const void *wk, const map_heads *dq, const map_heads *dk, float *dwq,
                       float *dwk, void *ws, void *stream);

/* ---------------------------------------------------------------- pages of a cache
 * Keys and values of the sequences that a language model is answering, in pages of a pool that
 * all layers share one page table for.  Sequences of one image share its pages: a question
 * takes the parent's rows with its own kept visual tokens (map_cache_fork) and frees them when
 * answered.  Everything below is device memory of the caller, initially zero but for the pool;
 * the calls keep no other state, never synchronise and may be captured.  Calls on one cache
 * are ordered by the caller (one stream, or events).
 *   pool    [layers][2: K, V][pages][heads][page][dh] of `type`, 16-byte aligned.
 *   table   int32 [seqs, max_pages]: the pages of each sequence; only the first
 *           ceil(len / page) entries of a row mean anything.
 *   len     int32 [seqs]: rows of each sequence.
 *   refs    int32 [pages]: sequences that hold the page; 0: free.
 *   status  int32 [MAP_CACHE_STATUS_WORDS]: error bits for map_cache_status; the calls' own counters.
 * type MAP_BF16 or MAP_F16; dh a multiple of 8 up to 256; page 1 .. 1024; pages <= 1048576;
 * seqs <= 262144; max_pages * page < 2^31; heads <= 65535, layers * heads <= 2^23
 * (MAP_EUNSUPPORTED beyond these).  New pages are the free ones with the lowest numbers, in the
 * order of the call's entries: results do not depend on timing.
 * A call that names a bad sequence, names one twice where that is not allowed, or needs more
 * pages than are free or than a table row holds, changes no length and no page (map_cache_free
 * apart): map_cache_status then reports it.  Table entries outside the pool and lengths that no
 * row holds are reported too and never followed: such rows read as zeros or as page 0, get slot
 * -1, are not freed.
 */
#define MAP_CACHE_STATUS_WORDS 1024
typedef struct {
    void *pool;
    int32_t *table, *len, *refs, *status;
    int type, layers, pages, heads, page, dh, seqs, max_pages;
} map_cache;

/*
 * Appends rows: entry i adds counts[i] rows to sequence seqs[i], taking pages where they are
 * needed, and gives them their slots (page * cache->page + row in the page), packed in the
 * entries' order: slots [rows], those past the last entry's rows are -1.
 *   seqs, counts  int32 [n] (device).  seqs[i] = -1: the entry is padding, without rows.  A
 *                 sequence may appear once.  counts >= 0, sum <= rows (else the call is refused
 *                 as above and every slot is -1).  counts = NULL, for a decoding step: one row
 *                 each, entry i's is row i, a padding entry's slot is -1; rows >= n.
 *   n <= 4096, rows <= 1048576 (MAP_EUNSUPPORTED).
 */
int map_cache_extend(const map_cache *cache, const int32_t *seqs, const int32_t *counts, int n, long long rows,
                     int32_t *slots, void *stream);

/*
 * map_qk_rotate whose keys go to the cache: row r's rotated k and its v (copied) are written to
 * slot slots[r] of `layer`, its rotated q to q_out.  k and v have cache->heads heads of
 * cache->dh = the plan's dh columns, and the cache's type.  A row with slot -1 is padding:
 * nothing of it is written.  A slot outside the pool is skipped like padding and reported by
 * map_cache_status.  No slot may appear twice.
 */
int map_qk_rotate_append(const map_rope *rope, const map_cache *cache, int layer, long long rows,
                         const int32_t *pos, const int32_t *slots, const map_heads *q, const map_heads *k,
                         const map_heads *v, const void *wq, const void *wk, const map_heads *q_out, void *stream);

/*
 * Forks sequences: the empty sequence children[i] gets the rows of parents[i] in all layers.
 *   keep, base and span NULL, k = 0: all rows.
 *   keep int32 [n, k] (device), base, span int32 [n] (device): rows base .. base + span - 1 of
 *        the parent (its visual tokens) are replaced by its rows base + keep[i, 0 .. k); the rows
 *        before and after stay.  keep is map_select's keep_idx: a question's own pruned view of
 *        an image that stays cached whole.  base, span >= 0, base + span <= the parent's
 *        length.  An index outside [0, span) gives a row of zeros and is reported.  With k = 0
 *        (keep may be NULL) the rows of the span are left out.
 * Pages that are full and end before the first replaced row are shared (not copied); the other
 * rows are copied to new pages.  parents may repeat, children may not, and no child may be a
 * parent.  Compaction in place is a fork of the kept rows followed by map_cache_free of the
 * parent.  n <= 4096, 0 <= k <= 2^24 (MAP_EUNSUPPORTED beyond).
 */
int map_cache_fork(const map_cache *cache, const int32_t *parents, const int32_t *children, int n,
                   const int32_t *keep, int k, const int32_t *base, const int32_t *span, void *stream);

/* Frees sequences: each page loses one holder, the length becomes 0.  seqs int32 [n] (device);
 * -1 is padding, a sequence that is empty or appears again is left alone.  n <= 1048576
 * (MAP_EUNSUPPORTED beyond).  Alone of these calls it goes entry by entry: a bad sequence, or one
 * whose length no row can hold, is reported and left as it is, the others are freed. */
int map_cache_free(const map_cache *cache, const int32_t *seqs, int n, void *stream);

/*
 * Attention of single tokens over the cache: for query row i of sequence s = seqs[i] and head h,
 *   out[i, h] = sum_t softmax_t(scale <q[i, h], K[t, h / G]>) V[t, h / G],  t < len[s],
 * G = q heads / cache->heads (a whole number).  Scores, softmax statistics and sums in fp32.
 *   q, out    heads of cache->dh columns in the cache's type, [n] rows; 16-byte aligned, strides
 *             that are multiples of 8; out must not overlap q.
 *   seqs      int32 [n] (device); -1: padding, that row of out is left as it was.  A sequence
 *             without rows gives zeros.  A sequence may appear in several rows.
 *   ws        device scratch of map_cache_attend_workspace(cache) bytes, 16-byte aligned, the
 *             caller's until the call's work completes.
 * dh 64, 80, 96, 128, 192 or 256 (MAP_EUNSUPPORTED otherwise); n <= 65535.
 */
size_t map_cache_attend_workspace(const map_cache *cache);
int map_cache_attend(const map_cache *cache, int layer, const map_heads *q, const int32_t *seqs, int n, float scale,
                     const map_heads *out, void *ws, void *stream);

/*
 * map_cache_attend for groups of sequences that begin with the same pages (questions and samples on one cached image): the rows
 * that all of a group's sequences share are read once for the group.  The same result as map_cache_attend's, but for the order
 * of its sums; what is shared is found in the page table, so that any groups are right.
 *   starts    int32 [groups + 1] (device): entries starts[g] .. starts[g + 1] - 1 of seqs form group g; ascending from 0 to n
 *             (else it is reported, and nothing is shared).  Shared are the whole pages that the sequences of a group (those with
 *             rows) have in common in front; a group whose sequences have none is attended as by map_cache_attend.
 *   ws        device scratch of map_cache_attend_shared_workspace(cache, q heads, n, groups) bytes, 16-byte aligned, the
 *             caller's until the call's work completes.
 * groups 1 .. 65535, n * q heads < 2^31 (MAP_EUNSUPPORTED beyond); everything else as for map_cache_attend.
 */
size_t map_cache_attend_shared_workspace(const map_cache *cache, int heads, int n, int groups);
int map_cache_attend_shared(const map_cache *cache, int layer, const map_heads *q, const int32_t *seqs, int n,
                            const int32_t *starts, int groups, float scale, const map_heads *out, void *ws, void *stream);

/*
 * map_cache_attend that also keeps count of who is looked at: for each query row i of sequence s = seqs[i], key head h and t < len[s]
 *   weights[layer, s, h, t] += sum over the G query heads of h of softmax_t(scale <q, K[t, h]>).
 *   weights   float32 [layers, seqs, heads, max_pages * page] (device).  The caller zeroes a sequence's when it begins, is forked
 *             or freed; a row that is appended must find its weight as the caller wants it to begin.  What lies at or behind a
 *             sequence's length is not read or written.
 *   ws        device scratch of map_cache_attend_weigh_workspace(cache, q heads, n) bytes, 16-byte aligned, the caller's until
 *             the call's work completes; 4 bytes for each row that a sequence can have (not those that it has) and query head.
 * A sequence that appears in several rows gets the weights of all, added up in their order.  Everything else as for
 * map_cache_attend.
 */
size_t map_cache_attend_weigh_workspace(const map_cache *cache, int heads, int n);
int map_cache_attend_weigh(const map_cache *cache, int layer, const map_heads *q, const int32_t *seqs, int n, float scale,
                           const map_heads *out, float *weights, void *ws, void *stream);

/*
 * Takes the rows of least weight out of sequences, for each layer and key head by itself: of sequence seqs[i]'s rows first[i] ..
 * len - last[i] - 1 the k of greatest weights[layer, seqs[i], h, .] stay (of equal ones those in front; NaN is the greatest), in
 * their order; the rows before and after stay.  Rows behind one that leaves move up, their weights with them, and len shrinks by
 * as many rows as leave, which is the same in all layers and heads.  A sequence with k candidates or fewer is left as it is.
 *   seqs         int32 [n] (device); -1: padding.  A sequence may appear once.
 *   first, last  int32 [n] (device), >= 0; NULL: 0.
 *   weights      as map_cache_attend_weigh's; those behind the new length, up to the old one, become 0.
 *   ws           device scratch of map_cache_evict_workspace(cache, n, k) bytes, 16-byte aligned, the caller's until the call's work
 *                completes.
 * Pages that other sequences hold as well keep their rows: of a sequence that loses rows, those from row first[i]'s page up to the
 * new length are replaced by new ones, taken before any is given up (row first[i]'s also where only rows before it are left of it:
 * what is appended next goes there).  Pages behind the new length lose a holder.
 * Keys stay rotated by the positions that they were appended with: the next token's position follows from the tokens so far,
 * not from len, which an eviction has made smaller.
 * n <= 4096, n * max_pages < 2^31, n * layers * heads <= 2^24 (MAP_EUNSUPPORTED beyond).
 */
size_t map_cache_evict_workspace(const map_cache *cache, int n, int k);
int map_cache_evict(const map_cache *cache, float *weights, const int32_t *seqs, int n, const int32_t *first,
                    const int32_t *last, int k, void *ws, void *stream);

/* Synchronises `stream` and returns the error recorded by calls on this cache since the last
 * call (MAP_ENOMEM: no free page or a full table row; MAP_EINTERNAL: a bad sequence, slot, count or index),
 * clearing it; else a CUDA error as MAP_ECUDA; else MAP_OK. */
int map_cache_status(const map_cache *cache, void *stream);

/* Synchronises `stream` and returns the first deferred device-side error recorded by
 * this context since the last call (MAP_ETIMEOUT, MAP_EINTERNAL), clearing it; else a
 * CUDA error as MAP_ECUDA; else MAP_OK. */
int map_status(map_ctx *ctx, void *stream);

/* Frees the context and its workspace (synchronises the device first).  NULL is a no-op. */
void map_destroy(map_ctx *ctx);

/* Static description of a MAP_E* code. */
const char *map_strerror(int code);

/* ---------------------------------------------------------------- instrumentation
 * Counters and per-kernel CUDA-event timing used by the benchmark; not part of the
 * paper's method. */
typedef struct {
    long long launches;       /* kernels this context has launched */
    long long select_rounds;  /* selection rounds run (one round = choose, Gram, greedy) */
    long long gram_rows;      /* Gram-block rows evaluated by the selection */
} map_counters;

/* The launches of the selection's device-side loop are counted on the device: this call reads
 * that count (a synchronous copy), so it includes the loop iterations that have completed. */
int map_get_counters(map_ctx *ctx, map_counters *out);

/* Kernel ids for timing. */
#define MAP_K_GEMM_FV1    0   /* f_V layer 1: V [B*N, D] x wV1^T, GELU */
#define MAP_K_GEMM_FV2    1   /* no launches: f_V layer 2 is folded into W_K (W_K wV2) */
#define MAP_K_GEMM_WK     2   /* folded W_K wV2 projection with RoPE */
#define MAP_K_GEMM_TEXT   3   /* f_T layer 1 and the folded W_Q wT2 projection together */
#define MAP_K_SCORES      4   /* softmax statistics + mean */
#define MAP_K_SELECT      5   /* everything in map_select */
#define MAP_K_GATHER      6
#define MAP_K_NUM         7

/* enable != 0 records a CUDA event pair around every launch of the kernels above.  Where a call
 * otherwise runs two of them in one launch (the two modalities' layers, the kept indices' order and
 * the compaction), it launches them separately while timing is on; the results are the same. */
int map_set_timing(map_ctx *ctx, int enable);
/* Synchronises the device; returns the summed event time (ms) and count of kernel `id`
 * since timing was enabled, and resets them. */
int map_read_timing(map_ctx *ctx, int id, double *total_ms, long long *count);

/* ---------------------------------------------------------------- diagnostics
 * Entry points that expose internal stages for tests.  Not on the pruning path. */

/* y[M, Nout] = epi(x[M, K] @ w[Nout, K]^T + b) with the library's tcgen05 GEMM.
 * epi: 0 = GELU then bf16, 1 = bf16, 3 = fp32 (bias ignored for 3; b may be NULL).
 * Device pointers; x, w bf16; K % 64 == 0, Nout % 64 == 0. */
int map_linear(map_ctx *ctx, const void *x, const void *w, const void *b, int M, int K,
               int Nout, int epi, void *y, void *stream);

/* Limit, in ns, of every wait inside the tensor-core GEMM kernels that this context launches
 * (ns <= 0 restores the default of 2 s).  A wait that runs out makes the kernel stop issuing
 * work, let the copies and MMAs already in flight land, release its tensor memory and exit;
 * map_status then reports MAP_ETIMEOUT.  For tests of that path; MAP_EINVAL for NULL. */
int map_set_wait_limit(map_ctx *ctx, long long ns);

/* map_score that also writes q [sum(lens), dp] and k [B*N, dp] (fp32, after RoPE). */
int map_score_debug(map_ctx *ctx, const void *text_feats, const void *vis_feats,
                    const int32_t *lens, int B, int N, float *scores, float *q_out,
                    float *k_out, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* MAP_GB300_H */
