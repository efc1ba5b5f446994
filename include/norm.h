/*
 * norm.h - C ABI of layer norm as an operator of its own: forward, with a residual
 * addition in front of it where there is one, and backward, with the sums of the
 * weights' gradients.  It stands beside the residual + LayerNorm inside a stage
 * (stage.h), for what enters a stage, follows it or is normalised elsewhere.
 *
 * For each row x of width w (residual r, or 0):
 *     z = x + r, rounded to the operands' type        mu = mean(z)
 *     rstd = 1 / sqrt(mean((z - mu)^2) + eps)         xh = (z - mu) rstd
 *     out = gamma xh + beta
 * The backward pass of <out, dy> + <z, dtotal>, from z, mu and rstd, d = gamma dy:
 *     dx = rstd (d - mean(d) - xh mean(d xh)) + dtotal        (the residual's too)
 *     dgamma = sum over rows of dy xh                 dbeta = sum over rows of dy
 *
 * Conventions
 *   - x, residual, total (z), out, dy, dtotal, dx are [batch, seq, width] in dtype
 *     (fp32 or bf16): element strides of batch and position are given, the values of
 *     a row lie side by side.  Pointers are aligned to an element, strides are any;
 *     16-byte aligned rows are fastest.  Inputs may be broadcast (stride 0: the
 *     gradient is then of the expanded tensor).  Outputs may not overlap themselves
 *     or each other; out or total may be x or residual itself, and dx dy, dtotal or
 *     total itself, with its strides; apart from that no output may overlap an input.
 *   - gamma and beta [width], mean and rstd [batch, seq], dgamma and dbeta are fp32,
 *     contiguous.  gamma NULL: 1.  beta NULL: 0.
 *   - Sums and statistics are fp32; what is stored is rounded once.  A row whose sum or
 *     whose mean times rstd is beyond fp32's range may become NaN.
 *   - width is 1 .. 16384; a call has at most 2^32 / 1024 (width 8193 on) to 2^32 / 8 (width
 *     64 or less) rows, by the threads that a row takes.
 *   - All device work is enqueued on hip_stream (NULL = default stream) of the
 *     current device, which must be the operands'; calls neither allocate nor
 *     synchronise, and can be captured into a HIP graph.  The workspace is the
 *     caller's: its contents are scratch during the call, so calls that may
 *     overlap, and graphs that may, need one each.
 *   - Results do not depend on the run: every sum has a fixed order.
 *   - Every call returns a stage_status and never aborts or throws;
 *     layer_norm_last_error gives a message for this thread's last failure.
 */
#ifndef SKY_NORM_H
#define SKY_NORM_H

#include "stage.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LAYER_NORM_MAX_WIDTH 16384

/* Strides in elements: batch, position. */
typedef struct {
  stage_dtype dtype;
  int batch, seq, width;
  float eps; /* >= 0, finite */
  int64_t x[2], residual[2], total[2], out[2];
  int64_t dy[2], dtotal[2], dx[2];
} layer_norm_shape;

/*
 * out, mean and rstd of the formulas above.  residual may be NULL; with it, total
 * receives z (NULL: it is not kept).  Without it total has to be NULL: z is x.  mean
 * and rstd may be NULL.  Lengths of 0 are valid (nothing is launched).  EINVAL, with
 * nothing launched, for what the conventions rule out.
 */
stage_status layer_norm_forward(const layer_norm_shape* s, const void* x, const void* residual,
                                const float* gamma, const float* beta, void* total, void* out,
                                float* mean, float* rstd, void* hip_stream);

/* Workspace bytes that layer_norm_backward needs for this shape where it makes dgamma or
 * dbeta (0 is possible).  Host arithmetic only; the strides are not looked at. */
stage_status layer_norm_workspace(const layer_norm_shape* s, size_t* bytes);

/*
 * dx, dgamma and dbeta of the formulas above, overwritten.  total is z (x, where there was
 * no residual), mean and rstd are the forward call's.  dtotal, dx, dgamma and dbeta may be
 * NULL (an output that is NULL is not made).  No rows: dgamma and dbeta become 0.  Errors as
 * layer_norm_forward; EINVAL for a workspace that is too small (16-byte aligned; NULL if
 * none is needed).
 */
stage_status layer_norm_backward(const layer_norm_shape* s, const void* dy, const void* total,
                                 const float* gamma, const float* mean, const float* rstd,
                                 const void* dtotal, void* dx, float* dgamma, float* dbeta,
                                 void* workspace, size_t workspace_bytes, void* hip_stream);

/* Message of this thread's last failed layer_norm_ call ("" if none). */
const char* layer_norm_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SKY_NORM_H */
