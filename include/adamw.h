/*
 * adamw.h - C ABI of the AdamW update of many tensors at once: the weights that
 * stage_param gives with the gradients that stage_grad gives, or any others.
 *
 * With t the number of steps, this one among them, lr the step's rate times the
 * tensor's lr_scale, wd the tensor's decay, and c = min(1, max_norm / norm) where
 * gradients are clipped by their global norm (norm^2 = the sum of all squares), else 1:
 *     g = c grad                       m = beta1 m + (1 - beta1) g
 *     v = beta2 v + (1 - beta2) g^2
 *     w = w - lr wd w - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
 *
 * Types
 *   - param: fp32, or bf16.  A bf16 parameter with a master copy (fp32) takes w from
 *     it and becomes its value rounded to nearest; one without takes w from itself and
 *     becomes one of w's two neighbours at random in proportion (nearest would lose every
 *     update below 2^-9 of the weight), or NaN if w is.
 *   - grad: fp32 or bf16.
 *   - m, v: fp32 (state_bits 32), or 8 bits in blocks of 256 elements with an fp32 scale
 *     each (state_bits 8): m = scale * e4m3, scale = max |m| / 448, and v = scale * e5m2,
 *     scale = max v / 57344.  Codes are rounded to one of the two neighbours at random in
 *     proportion: one step changes v by 0.1% of itself, a code by up to 25%, and rounded to
 *     nearest most changes would be lost for good.  A positive v never becomes 0.  A block
 *     whose largest value is below 2^-110 is held as 0.
 *   - The random bits of element i at step t are the 32-bit numbers
 *         x = i 0x9E3779B1 + t 0x6A09E667;        x = (x ^ x >> 15) 0xBB67AE85;
 *         x = (x ^ x >> 13) 0x3C6EF373;           x = x ^ x >> 16
 *     (mod 2^32): its low 16 bits for m, its high 16 for v and for a bf16 weight.  A
 *     value is rounded up if its part beyond the last bit, in steps, and those bits / 2^16
 *     come to 1 or more.  So the same steps give the same bits every time.
 *   - m, v and the norm are formed in 32 bits or more (the norm in 64).
 *
 * Conventions
 *   - Parameters, gradients and states are the caller's, contiguous, aligned to an element
 *     (16-byte aligned ones are fastest), updated in place; no memory may be given twice.
 *     The library holds their addresses, on the device, from adamw_init on.
 *   - The number of steps is an int64 of the caller's on the device, raised by each step, so
 *     that a captured step counts on.
 *   - Steps of one handle run one after the other: the caller orders those on several
 *     streams.  Different handles are independent.
 *   - adamw_step neither allocates nor synchronises, and can be captured into a HIP graph.
 *   - Results do not depend on the run: every sum has a fixed order.
 *   - A gradient that is not finite: with clipping the norm is not finite either, and the
 *     step changes nothing, not the number of steps either.  Without, it reaches its own
 *     weight and states (8 bits: its block's).  So does one whose square passes fp32's range
 *     after clipping, above 1.8e19: its v is infinite (8 bits: its block's m or v NaN).
 *   - Every call returns a stage_status and never aborts or throws; adamw_last_error gives a
 *     message for this thread's last failure.
 */
#ifndef SKY_ADAMW_H
#define SKY_ADAMW_H

#include "stage.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ADAMW_BLOCK 256 /* elements that share a scale of 8-bit states */

typedef struct adamw adamw_t; /* opaque, library-owned */

typedef struct {
  void* param;
  const void* grad;
  void* m;         /* fp32, or e4m3 codes */
  void* v;         /* fp32, or e5m2 codes */
  float* m_scale;  /* [ceil(numel / 256)] with state_bits 8, else NULL */
  float* v_scale;
  float* master;   /* fp32 copy of a bf16 parameter, or NULL */
  int64_t numel;
  stage_dtype dtype, grad_dtype;
  int state_bits;      /* 32 or 8 */
  float weight_decay;  /* wd */
  float lr_scale;
} adamw_tensor;

/*
 * A handle for n tensors of the current device.  Allocates device memory for their addresses
 * and copies them there; returns when that is done (so not during a capture).  steps: int64 on
 * the device, the number of steps done so far, 0 or more.  EINVAL for n < 0, a negative numel (0 is valid), null or misaligned
 * pointers, unknown types, scales or a master copy that do not fit the types, values that are
 * not finite, or 2^40 elements or more in all.
 */
stage_status adamw_init(const adamw_tensor* tensors, int n, int64_t* steps, adamw_t** out);

typedef struct {
  float lr;             /* used if lr_ptr is NULL */
  const float* lr_ptr;  /* one fp32 value on the device, read by the step */
  double beta1, beta2;  /* 0 <= beta < 1 */
  float eps;            /* 1e-30 or more, finite */
  float max_norm;       /* > 0: clip; 0: do not */
  float* norm;          /* receives the norm before clipping (fp32), or NULL; needs max_norm > 0 */
} adamw_args;

/* One step of all tensors, on hip_stream (NULL = default stream) of the handle's device, which
 * must be the current one.  EINVAL for what the comments rule out. */
stage_status adamw_step(adamw_t* h, const adamw_args* a, void* hip_stream);

/* Frees what the handle owns (waits for the device; graphs that captured a step of it may not be
 * replayed any more).  NULL is a no-op. */
void adamw_destroy(adamw_t* h);

/* Message of this thread's last failed adamw_ call ("" if none). */
const char* adamw_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SKY_ADAMW_H */
