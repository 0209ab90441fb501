/*
 * zo_layers.h - C ABI of the layers of a recurrent language model that is
 * trained by exact gradients: linear attention with a decay for each head
 * (forward, backward and the step for single tokens), layer norm (forward and
 * backward) and the AdamW step over many tensors. Part of the same library as
 * zo.h (MI355X, gfx950).
 *
 * Conventions are zo.h's: buffers are device pointers owned by the caller;
 * every call only enqueues work on `stream` (a hipStream_t) and returns; arguments are
 * validated on the host before anything is enqueued; calls return a zo_status
 * and zo_last_error() describes the last failure. Nothing is allocated,
 * retained or cleared beforehand, and calls may be captured into a HIP graph.
 * Calls on distinct streams with distinct workspaces may run concurrently.
 *
 * Types. Activations are fp32 or bf16 (ZO_WFP32, ZO_WBF16); sums, statistics,
 * states and moments are fp32 (or codes of 8 bits), and every output is rounded once, to nearest even.
 */
#ifndef ZO_LAYERS_H
#define ZO_LAYERS_H

#include "zo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- linear attention with a decay for each head ----
 *
 * Every sequence b and key/value head h keeps a state S [key_dim][value_dim]
 * with gamma_h = exp(log_decay[h]); query heads g = h * (q_heads / kv_heads) ..
 * read it:
 *   S_t = gamma S_{t-1} + k_t v_t^T,    o_t = scale S_t^T q_t,    0 <= t < length_b
 * S_{-1} is the initial state (zero if NULL), the final state is the state after
 * the sequence's last position. Outputs from length_b on are zero, and inputs
 * there are never used, whatever they hold. log_decay is expected <= 0 (-inf:
 * gamma = 0); larger values are used as they are. The decay is a constant of
 * the head: it has no gradient.
 *
 * A position reaches the outputs from itself on only: a value that is not finite
 * leaves every earlier output of its sequence as it would be without it.
 *
 * Precision: products and sums as fp32; with bf16 activations the operands
 * formed inside (the masked scores, and the states that queries read) are held in
 * two bf16 parts, 2^-16 of them left out at most, states and their gradients in fp32. */

/* Head sizes up to ZO_LINATTN_MAX_DIM (ZO_ESHAPE beyond). */
#define ZO_LINATTN_MAX_DIM 256
/* Distance of neighbouring positions in memory, in elements (ZO_ESHAPE beyond). */
#define ZO_LINATTN_MAX_STRIDE ((int64_t)1 << 24)

typedef struct {
    int32_t batch;      /* sequences, >= 0 */
    int32_t length;     /* positions, 0 .. 2^30 (the step takes one, whatever this says within the range) */
    int32_t q_heads;    /* a multiple of kv_heads */
    int32_t kv_heads;   /* > 0 */
    int32_t key_dim;    /* 1 .. ZO_LINATTN_MAX_DIM */
    int32_t value_dim;  /* 1 .. ZO_LINATTN_MAX_DIM */
    int32_t dtype;      /* of q, k, v, o and their gradients: ZO_WFP32 or ZO_WBF16 */
    float scale;        /* finite */
} zo_linattn;

/* A tensor [batch][length][heads][dim]: element (b, t, h, d) at
 * data[b * batch_stride + t * position_stride + h * head_stride + d], strides
 * in elements, any sign (position_stride within
 * ZO_LINATTN_MAX_STRIDE; not used where there is one position or none). Any alignment of data that its type needs. Inputs may
 * overlap (slices of one projection); an output may share no value with them or
 * another output (ZO_EINVAL where that is certain: the same first value, both without gaps,
 * or the same strides). */
typedef struct {
    void* data;
    int64_t batch_stride, position_stride, head_stride;
} zo_heads;

/* Bytes of device workspace that zo_linear_attention (backward = 0) or
 * zo_linear_attention_backward (1) uses; possibly 0. Host only. */
size_t zo_linear_attention_workspace_bytes(const zo_linattn* shape, int32_t backward);

/* Whole sequences. q [B][T][q_heads][key_dim], k [B][T][kv_heads][key_dim],
 * v [B][T][kv_heads][value_dim] -> o [B][T][q_heads][value_dim].
 *   log_decay      device fp32 [kv_heads]
 *   lengths        device int32 [B], or NULL (all T); values outside [0, T]
 *                  count as the nearer end
 *   initial_state  device fp32 [B][kv_heads][key_dim][value_dim], or NULL (zeros)
 *   final_state    the same shape, or NULL (not wanted); nothing of initial_state
 *                  (ZO_EINVAL): workgroups read the one while others write the other
 *   workspace, ws_bytes  at least zo_linear_attention_workspace_bytes(); NULL if that is 0 */
int zo_linear_attention(const zo_linattn* shape, const zo_heads* q, const zo_heads* k, const zo_heads* v,
                        const zo_heads* o, const float* log_decay, const int32_t* lengths,
                        const float* initial_state, float* final_state, void* workspace, size_t ws_bytes,
                        void* stream);

/* The gradients of zo_linear_attention, recomputed from its inputs. With
 * dS_t = scale sum_g q_t do_t^T + gamma dS_{t+1} (sum over the query heads of a
 * state; the last position's dS also takes dfinal_state):
 *   dq_t = scale S_t do_t,  dk_t = dS_t v_t,  dv_t = dS_t^T k_t,  dinitial = gamma dS_0
 * (length 0: dinitial = dfinal).
 *   dout           gradient of o
 *   dfinal_state   device fp32, the final state's gradient, or NULL (zeros)
 *   dinitial_state device fp32, or NULL (not wanted); nothing of dfinal_state (ZO_EINVAL)
 * Gradients from length_b on are zero. */
int zo_linear_attention_backward(const zo_linattn* shape, const zo_heads* dout, const zo_heads* q,
                                 const zo_heads* k, const zo_heads* v, const zo_heads* dq, const zo_heads* dk,
                                 const zo_heads* dv, const float* log_decay, const int32_t* lengths,
                                 const float* initial_state, const float* dfinal_state, float* dinitial_state,
                                 void* workspace, size_t ws_bytes, void* stream);

/* One token for each of B sequences, their states updated in place.
 * shape->length and the tensors' position strides are not used. state is a pool
 * of n_slots states [n_slots][kv_heads][key_dim][value_dim]; sequence b's is
 * slots[b] (device int32; no two alike), or b itself where slots is NULL
 * (n_slots >= B then). A slot of -1 is a sequence without a state: its output is
 * zero. Any other slot outside [0, n_slots) is never used to address memory and
 * makes its sequence's output NaN. */
int zo_linear_attention_step(const zo_linattn* shape, const zo_heads* q, const zo_heads* k, const zo_heads* v,
                             const zo_heads* o, const float* log_decay, float* state, int32_t n_slots,
                             const int32_t* slots, void* stream);

/* ---- layer norm ----
 * Over each of `rows` rows of D values, x at x + r * x_stride (elements), y at
 * y + r * y_stride:
 *   mean, var over the row;  rstd = 1 / sqrt(var + eps);
 *   y = (x - mean) rstd w + b
 * xdtype is the type of x and y (and dy, dx), wdtype that of weight and bias;
 * weight and bias may be NULL (1 and 0). mean and rstd: device fp32 [rows],
 * kept for the backward pass, or both NULL. y may be x with its stride (ZO_EINVAL if they
 * share memory in another way). */
int zo_layer_norm(int32_t xdtype, int32_t wdtype, int64_t rows, int64_t D, const void* x, int64_t x_stride,
                  const void* weight, const void* bias, float eps, void* y, int64_t y_stride, float* mean,
                  float* rstd, void* stream);

/* Bytes of device workspace of zo_layer_norm_backward. Host only. */
size_t zo_layer_norm_workspace_bytes(int64_t rows, int64_t D);

/* xhat = (x - mean) rstd, g = dy w:
 *   dx = rstd (g - avg(g) - xhat avg(g xhat));  dweight = sum_rows dy xhat;  dbias = sum_rows dy
 * dweight, dbias: device fp32 [D], each may be NULL (not wanted). Their sums run
 * in a fixed order: the same call gives the same bits. dx may be dy or x, with its stride. */
int zo_layer_norm_backward(int32_t xdtype, int32_t wdtype, int64_t rows, int64_t D, const void* dy,
                           int64_t dy_stride, const void* x, int64_t x_stride, const void* weight,
                           const float* mean, const float* rstd, void* dx, int64_t dx_stride, float* dweight,
                           float* dbias, void* workspace, size_t ws_bytes, void* stream);

/* ---- AdamW over many tensors ----
 * For every value of every tensor, in fp32, with g' = g * grad_scale:
 *   m = beta1 m + (1 - beta1) g';  v = beta2 v + (1 - beta2) g'^2
 *   p = p (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * The moments of all tensors lie in flat arrays; a tensor's begin at its
 * state_offset, a multiple of ZO_ADAMW_BLOCK, and take whole blocks. All tensors are updated
 * at once: the parameters of two, or their moments, may not overlap (ZO_EINVAL; a tied
 * tensor is given once, with the sum of its gradients). A gradient may be shared by tensors, but lies in
 * no parameter.
 *   32 bits  m and v fp32
 *   8 bits   m int8 and v uint8 codes, and m_scale and v_scale fp32, the largest |m| and v of each
 *            block: a code c stands for m_scale sign(c) (c / 127)^2, or v_scale (c / 255)^4.
 *            Codes are the nearest in the root's scale, and at least 1 for a positive v (a
 *            denominator that would be rounded to zero under a first moment that is not).
 *            The step itself uses the moments before they are coded. A moment
 *            that is not finite leaves its whole block NaN. */
#define ZO_ADAMW_BLOCK 256

typedef struct {
    void* param;          /* n values of type pdtype, updated in place */
    const void* grad;     /* n values of type gdtype */
    int64_t n;            /* >= 0 */
    int64_t state_offset; /* first value of its moments */
    double weight_decay;
    int32_t pdtype, gdtype;
} zo_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps;
    int64_t step;         /* of this update, >= 1 */
    int32_t state_bits;   /* 32 or 8 */
} zo_adamw_config;

/* One step over n_tensors tensors (a host array, read before the call returns).
 *   m, v             device moments; m_scale, v_scale: 8 bits only (NULL otherwise)
 *   grad_scale       device fp32 [1] or NULL (1): a clipping or unscaling factor. If it
 *                    is not finite the step is skipped on the device: parameters and
 *                    moments stay bit for bit as they are. Bias corrections go by cfg->step alone:
 *                    a caller that counts a skipped step corrects for an update that no moment holds
 *                    (a first step skipped makes the next one's change 0.74 of what it would be, at
 *                    betas of 0.9 and 0.999), one that does not, by skipped_out, has the formula's
 *   skipped_out      device int32 [1] or NULL: 1 if it was skipped, else 0
 * Parameters of 32-bit and 16-bit types may be mixed, and aligned as their type needs.
 * A parameter is rounded once, to nearest: in bf16 a change under 2^-9 of the value is lost, step after
 * step (a weight decay of 0.1 at an lr of 1e-3 alone changes nothing). Where small changes count, keep fp32
 * parameters and cast them. cfg is read by the call: a captured launch replays with its step's lr and bias corrections. */
int zo_adamw(const zo_adamw_config* cfg, const zo_adamw_tensor* tensors, int32_t n_tensors, void* m, void* v,
             float* m_scale, float* v_scale, const float* grad_scale, int32_t* skipped_out, void* stream);

/* The values that n (a multiple of ZO_ADAMW_BLOCK) 8-bit moments stand for, into fp32 m_out and v_out. */
int zo_adamw_moments(int64_t n, const void* m, const void* v, const float* m_scale, const float* v_scale,
                     float* m_out, float* v_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ZO_LAYERS_H */
