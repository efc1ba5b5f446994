/*
 * rotary.h - C ABI of rotary positions: queries and keys turned by angles that
 * grow with their positions, so that their products depend on the distance
 * alone.  They stand beside the relative position bias of attn.h and go in front
 * of attn_forward; the backward pass turns the gradients of q and k back.
 *
 * For a token at position p, pair i of the n = rot_dim / 2 pairs of a head:
 *     y0 = A (x0 cos a_i - x1 sin a_i),   y1 = A (x0 sin a_i + x1 cos a_i),
 *     a_i = p f_i,
 * where (x0, x1) are values i and n + i of the head (halves) or 2 i and 2 i + 1
 * (interleaved).  Values from rot_dim on go through as they are.  The backward
 * pass takes -a_i in a_i's place (A as it is).
 *
 * Conventions
 *   - Heads are 64 wide, as in attn.h.  q is [batch, seq, heads, 64], k [batch,
 *     seq, kv_heads, 64] (kv_heads 0: there is no k) in any memory order:
 *     element strides of batch, position and head are given, the 64 values of a
 *     head lie side by side.  Pointers are 16-byte aligned, strides multiples of
 *     16 bytes.  Inputs may be broadcast (stride 0).  q_out may be q itself, with
 *     its strides, and k_out k; otherwise outputs may not overlap themselves,
 *     each other or an input.
 *   - dtype: fp32 or bf16, of all four.  Angles are formed in 64 bits (in turns,
 *     of which only the fraction goes on), the rest in fp32, rounded once.
 *   - Positions: int32 [batch], the position of token 0 of each sequence, or
 *     (pos_each) [batch, seq], that of each token, with element strides; NULL =
 *     0, 1, ...  Any value is valid, negative ones too.  Read on the device, so
 *     that a captured call follows them.
 *   - All device work is enqueued on hip_stream (NULL = default stream) of the
 *     current device, which must be the operands'; calls neither allocate nor
 *     synchronise, and can be captured into a HIP graph.
 *   - Every call returns a stage_status and never aborts or throws;
 *     rotary_last_error gives a message for this thread's last failure.
 */
#ifndef SKY_ROTARY_H
#define SKY_ROTARY_H

#include "stage.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ROTARY_MAX_PAIRS 32

/* Frequencies of the pairs; plain host data, free to copy.  Filled by rotary_init
 * or rotary_init_freqs. */
typedef struct rotary_freqs {
  int rot_dim;                    /* values of a head that are turned: 2 i pairs */
  int interleaved;                /* 0: pairs (i, n + i); 1: pairs (2 i, 2 i + 1) */
  float amplitude;                /* A */
  double turns[ROTARY_MAX_PAIRS]; /* f_i / 2 pi */
} rotary_freqs;

/* How the frequencies f_i = base^(-i / n) change for contexts `factor` = s times
 * those of original_len positions that a model was trained on:
 *   NONE    not at all
 *   LINEAR  f_i / s: positions are squeezed
 *   BASE    base s^(n / (n - 1)) in base's place: the first pair as it was, the last
 *           one s times slower (one pair: as it was)
 *   PARTS   by the turns t_i = original_len f_i / 2 pi that a pair makes:
 *           f_i (w + (1 - w) / s), w = (t_i - low) / (high - low) within 0 .. 1, so
 *           that pairs of many turns stay and those of few are squeezed
 */
typedef enum SKY_ENUM_INT {
  ROTARY_NONE = 0,
  ROTARY_LINEAR = 1,
  ROTARY_BASE = 2,
  ROTARY_PARTS = 3
} rotary_scaling;

/*
 * EINVAL unless rot_dim is even from 2 to 64, interleaved is 0 or 1, base > 0, amplitude
 * is finite and, except for NONE, factor > 0; for PARTS also original_len >= 1 and
 * high > low; or if a frequency is not finite.  What a scaling does not use is not
 * looked at.  Host arithmetic only.
 */
stage_status rotary_init(int rot_dim, int interleaved, double base, rotary_scaling scaling,
                         double factor, int original_len, double low, double high,
                         double amplitude, rotary_freqs* out);
/* The same with rot_dim / 2 frequencies of the caller's, in radians a position. */
stage_status rotary_init_freqs(int rot_dim, int interleaved, const double* freqs, double amplitude,
                               rotary_freqs* out);

/* Strides in elements: batch, position, head (pos: batch, position). */
typedef struct {
  stage_dtype dtype;
  int batch, seq;
  int heads, kv_heads;
  int pos_each; /* 0 or 1 */
  int64_t q[3], k[3], q_out[3], k_out[3], pos[2];
} rotary_shape;

/*
 * q_out and k_out of the formulas above.  Lengths of 0 are valid (nothing is launched).
 * EINVAL, with nothing launched, for what the conventions rule out, sequences of 2^29
 * positions or more, 65536 heads or more, or more work-groups than a launch has.
 */
stage_status rotary_forward(const rotary_shape* s, const rotary_freqs* f, const void* q, const void* k,
                            const int32_t* pos, void* q_out, void* k_out, void* hip_stream);
/* The gradients of rotary_forward's q and k (into q_out, k_out) from those of its q_out
 * and k_out (q, k). */
stage_status rotary_backward(const rotary_shape* s, const rotary_freqs* f, const void* q,
                             const void* k, const int32_t* pos, void* q_out, void* k_out,
                             void* hip_stream);

/* Message of this thread's last failed rotary_ call ("" if none). */
const char* rotary_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SKY_ROTARY_H */
