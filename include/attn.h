/*
 * attn.h - C ABI of the attention operators: queries over the keys and values
 * of another sequence (cross attention), and a relative position bias learned
 * by buckets.  They stand beside the stage's own attention (stage.h), whose
 * queries, keys and values come from one projection of one sequence.
 *
 * For batch entry b, query i of head h and key j (g = h / (heads / kv_heads) is
 * the key head that query head h shares; p_b = q_pos[b], or 0):
 *     s_ij = scale * q_i . k_j + table[bucket(j - (i + p_b))][h]
 *     P_ij = exp(s_ij - lse_i) over the keys that i sees, else 0
 *     out_i = sum_j P_ij v_j,      lse_i = log sum_j exp(s_ij)
 * i sees j if key_mask[b][j] != 0 and, with `causal`, j <= i + p_b.  The bias
 * term is there only with a table.  A query that sees no key gets out = 0 and
 * lse = -inf, and adds nothing to any gradient, whatever its q and dout hold.
 *
 * The backward pass of <out, dout>, with D_i = sum_j P_ij (dout_i . v_j) and
 * dS_ij = P_ij (dout_i . v_j - D_i):
 *     dq_i = scale * sum_j dS_ij k_j       dk_j = scale * sum_{h of g} sum_i dS_ij q_i
 *     dv_j = sum_{h of g} sum_i P_ij dout_i
 *     dtable[c][h] = sum of dS_ij over all b, i, j with bucket(j - (i + p_b)) = c
 *
 * Conventions
 *   - Heads are 64 wide.  q and out are [batch, seq_q, heads, 64], k and v
 *     [batch, seq_k, kv_heads, 64] in any memory order: element strides of
 *     batch, position and head are given, the 64 values of a head lie side by
 *     side.  So the parts of a packed projection, and both orders of positions
 *     and heads, are read and written in place.  Inputs may be broadcast
 *     (stride 0); outputs may not overlap themselves, each other or an input.
 *     Pointers are 16-byte aligned, strides multiples of 16 bytes, and a
 *     position's stride is below 16 MiB.
 *   - dtype (fp32 or bf16) is the type of q, k, v, out, dout, dq, dk, dv.
 *     lse [batch, heads, seq_q], table and dtable [num_buckets, heads] are
 *     fp32, contiguous.  Scores, softmax statistics and sums are fp32; on bf16
 *     the probabilities and dS are rounded to bf16 where a matrix product takes
 *     them (dtable sums dS unrounded).  A bias below -2.35e38 (fp32's lowest
 *     value, -inf) hides its keys; a query all of whose keys are hidden so gets
 *     what one that sees none gets.  Other biases are finite, below 2.35e38.
 *   - key_mask: uint8 [batch, seq_k], contiguous, nonzero = may be attended;
 *     NULL = every key.  What the k and v rows of a key hold that the mask
 *     hides, or that no query may see, reaches no result, whatever it is (NaN
 *     included); its dk and dv are 0.  A row that some query of the call sees
 *     has to be finite.
 *   - q_pos: int32 [batch], the position of query 0 on the key axis, for
 *     `causal` and the bias; NULL = 0.  Read on the device, so that a captured
 *     call follows it.
 *   - All device work is enqueued on hip_stream (NULL = default stream) of the
 *     current device, which must be the operands'; calls neither allocate nor
 *     synchronise, and can be captured into a HIP graph.  The workspace is the
 *     caller's: its contents are scratch during the call, so calls that may
 *     overlap, and graphs that may, need one each.
 *   - Results do not depend on the run: every sum has a fixed order.
 *   - Every call returns a stage_status and never aborts or throws;
 *     attn_last_error gives a message for this thread's last failure.
 */
#ifndef SKY_ATTN_H
#define SKY_ATTN_H

#include "stage.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The buckets of a relative position bias.  With n buckets to a direction
 * (all of num_buckets, or half of them each for keys before and keys after the
 * query), the distances 0 .. n/2 - 1 have a bucket each, and the others grow
 * with the logarithm of the distance up to max_distance, the last one taking
 * all that is further: distance d >= o = n/2 has bucket
 *     min(n - 1, o + floor(log(d / o) / log(max_distance / o) * (n - o))),
 * in exact arithmetic (a border that is a whole number belongs to the bucket it
 * opens).  One direction: keys after the query have bucket 0.  Both: keys at or
 * before it have buckets 0 .. n - 1, keys after it n .. 2 n - 1.
 * Filled by attn_relpos_init; plain host data, free to copy.
 */
#define ATTN_MAX_BUCKETS 256
#define ATTN_MAX_DISTANCE 2048
typedef struct {
  int num_buckets;
  int max_distance;
  int bidirectional;
  int reach;     /* least distance of a direction's last bucket */
  int n_borders; /* border[i]: least distance of bucket o + 1 + i */
  int border[ATTN_MAX_BUCKETS / 2];
} attn_relpos;

/*
 * EINVAL unless bidirectional is 0 or 1, num_buckets is 2 .. 256 (both
 * directions: an even number from 4 on), and max_distance is above half a
 * direction's buckets and at most 2048.  Host arithmetic only.
 */
stage_status attn_relpos_init(int num_buckets, int max_distance, int bidirectional,
                              attn_relpos* out);
/* Bucket of key position - query position; -1 for a null or invalid rp. */
int attn_relpos_bucket(const attn_relpos* rp, int64_t distance);

/* Strides in elements: batch, position, head.  Those of dout, dq, dk and dv
 * are for attn_backward. */
typedef struct {
  stage_dtype dtype;
  int batch, seq_q, seq_k;
  int heads, kv_heads; /* heads a multiple of kv_heads */
  int causal;          /* 0 or 1 */
  float scale;         /* > 0, below 2.35e38 (fp32's largest over log2(e)) */
  int64_t q[3], k[3], v[3], out[3];
  int64_t dout[3], dq[3], dk[3], dv[3];
} attn_shape;

/*
 * Workspace bytes that attn_forward (backward = 0) or attn_backward (1) needs
 * for this shape (0 is possible); rp as in those calls.  Host arithmetic only;
 * the strides are not looked at.
 */
stage_status attn_workspace(const attn_shape* s, const attn_relpos* rp, int backward,
                            size_t* bytes);

/*
 * out and lse of the formulas above.  rp and table are both given or both NULL;
 * lse may be NULL.  Lengths of 0 are valid (nothing is launched for no
 * queries).  EINVAL, with nothing launched, for what the conventions rule out,
 * sequences of 2^29 positions or more, more work-groups than a launch has, or a
 * workspace that is too small (16-byte aligned; NULL if none is needed).
 */
stage_status attn_forward(const attn_shape* s, const attn_relpos* rp, const float* table,
                          const void* q, const void* k, const void* v, const uint8_t* key_mask,
                          const int32_t* q_pos, void* out, float* lse, void* workspace,
                          size_t workspace_bytes, void* hip_stream);

/*
 * dq, dk, dv and, with a table, dtable of the formulas above, from the inputs,
 * out and lse of a forward call; all are overwritten.  dtable may be NULL.
 * Errors as attn_forward.
 */
stage_status attn_backward(const attn_shape* s, const attn_relpos* rp, const float* table,
                           const void* q, const void* k, const void* v, const uint8_t* key_mask,
                           const int32_t* q_pos, const void* out, const float* lse,
                           const void* dout, void* dq, void* dk, void* dv, float* dtable,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

/* Message of this thread's last failed attn_ call ("" if none). */
const char* attn_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SKY_ATTN_H */
