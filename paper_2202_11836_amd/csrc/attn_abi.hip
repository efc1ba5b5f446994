// C ABI of the attention operators (include/attn.h): argument checks, the borders
// of the relative position buckets, the workspace's layout.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "xattn.h"

namespace {

thread_local char g_err[256];

stage_status bad(stage_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

// A natural number of up to 4096 bits, for exact powers.
struct Big {
  uint32_t w[128] = {1};
  int n = 1;  // words in use
  void mul(uint32_t f, int times) {
    while (times-- > 0) {
      uint64_t c = 0;
      for (int i = 0; i < n; ++i) {
        c += (uint64_t)w[i] * f;
        w[i] = (uint32_t)c;
        c >>= 32;
      }
      if (c) w[n++] = (uint32_t)c;
    }
  }
  bool operator>=(const Big& o) const {
    if (n != o.n) return n > o.n;
    for (int i = n - 1; i >= 0; --i)
      if (w[i] != o.w[i]) return w[i] > o.w[i];
    return true;
  }
};

// (n / one)^m >= (max / one)^j: distance n belongs to bucket one + j or a later one.
// (At most 128 + 127 factors below 2^11: 2805 bits.)
bool reaches(int n, int one, int m, int max, int j) {
  Big a, b;
  a.mul(n, m);
  a.mul(one, j);
  b.mul(one, m);
  b.mul(max, j);
  return a >= b;
}

struct Buckets {
  int n, one, m;  // to a direction; with one distance each; the others
};
bool buckets_of(int num_buckets, int max_distance, int both, Buckets* out) {
  if ((both != 0 && both != 1) || num_buckets < 2 || num_buckets > ATTN_MAX_BUCKETS) return false;
  if (both && (num_buckets < 4 || (num_buckets & 1))) return false;
  const int n = both ? num_buckets / 2 : num_buckets;
  *out = {n, n / 2, n - n / 2};
  return max_distance > out->one && max_distance <= ATTN_MAX_DISTANCE;
}

// Whether rp is what attn_relpos_init makes, as far as the kernels rely on it.
bool relpos_ok(const attn_relpos* rp) {
  Buckets k;
  if (!buckets_of(rp->num_buckets, rp->max_distance, rp->bidirectional, &k)) return false;
  if (rp->n_borders != k.m - 1) return false;
  int last = k.one;
  for (int i = 0; i < rp->n_borders; ++i) {
    if (rp->border[i] < last || rp->border[i] > rp->max_distance) return false;
    last = rp->border[i];
  }
  return rp->reach == last;
}

int64_t row_blocks(int n) { return ((int64_t)n + 127) / 128; }

struct Workspace {
  int64_t dsum, tpart, part, total;  // bytes
  XKvPlan kv;
  XFewPlan few;
  XDqPlan dq;
};
Workspace workspace_of(const attn_shape* s, const attn_relpos* rp, bool backward) {
  Workspace w{};
  const int rep = s->heads / s->kv_heads;
  if (!backward) {
    w.few = xattn_few_plan(s->batch, s->kv_heads, rep, s->seq_q, s->seq_k, rp ? rp->num_buckets : 0,
                           rp ? rp->reach : 0, s->dtype);
    if (w.few.splits > 1)
      w.part = (int64_t)w.few.splits * s->batch * s->kv_heads * xattn_few_tiles(rep, s->seq_q) * 32 *
               XFEW_ROW * 4;
    w.total = w.part;
    return w;
  }
  w.dsum = ((int64_t)s->batch * s->heads * s->seq_q * 4 + 15) / 16 * 16;
  w.dq = xattn_dq_plan(s->batch, s->heads, s->seq_q, s->seq_k, s->causal, rp != nullptr, s->dtype);
  const int64_t qb = 128 / w.dq.ks;  // queries of a work-group
  if (rp)
    w.tpart = ((int64_t)s->batch * s->heads * ((s->seq_q + qb - 1) / qb) * rp->num_buckets * 4 + 15) /
              16 * 16;
  w.kv = xattn_kv_plan(s->batch, s->kv_heads, rep, s->seq_q, s->seq_k, s->causal, rp != nullptr,
                       w.dq, s->dtype);
  if (w.kv.splits > 1)
    w.part = (int64_t)w.kv.splits * s->batch * s->kv_heads * s->seq_k * 2 * XHD * 4;
  if (w.dq.splits > 1)  // (its partial results are summed before those of dK, dV are made)
    w.part = std::max(w.part, (int64_t)w.dq.splits * s->batch * s->heads * s->seq_q *
                                  xattn_dq_row(s->dtype) * 4);
  w.total = w.dsum + w.tpart + w.part;
  return w;
}

stage_status check_shape(const attn_shape* s, const attn_relpos* rp) {
  if (!s) return bad(STAGE_EINVAL, "null shape");
  if (s->dtype != STAGE_F32 && s->dtype != STAGE_BF16) return bad(STAGE_EINVAL, "unknown dtype");
  if (s->batch < 0 || s->seq_q < 0 || s->seq_k < 0)
    return bad(STAGE_EINVAL, "negative batch or length");
  if (s->seq_q >= 1 << 29 || s->seq_k >= 1 << 29)
    return bad(STAGE_EINVAL, "sequences of 2^29 positions or more");
  if (s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads)
    return bad(STAGE_EINVAL, "heads must be a multiple of kv_heads, both >= 1");
  if (s->causal != 0 && s->causal != 1) return bad(STAGE_EINVAL, "causal must be 0 or 1");
  // (the kernels take it times log2(e))
  if (!(s->scale > 0.0f) || !std::isfinite(s->scale * XLOG2E))
    return bad(STAGE_EINVAL, "scale must be positive and below 2.35e38");
  if (rp && !relpos_ok(rp)) return bad(STAGE_EINVAL, "rp is not one that attn_relpos_init filled");
  // A launch holds fewer than 2^32 threads, 256 to a work-group.
  // (the dQ kernel may take two for 128 queries)
  const double most = 16777215.0;
  if (2.0 * s->batch * s->heads * (double)row_blocks(s->seq_q) > most ||
      (double)s->batch * s->kv_heads * (double)row_blocks(s->seq_k) +
              (rp ? (double)rp->num_buckets * s->heads : 0.0) > most)
    return bad(STAGE_EINVAL, "batch * heads * length too large");
  return STAGE_OK;
}

// Pointer and strides of one operand of [batch, n, heads, 64]; strides of
// dimensions of one or no element are not looked at (0 in *st).
stage_status check_operand(const char* name, const void* p, const int64_t* given, int batch, int n,
                           int heads, stage_dtype dt, bool output, int64_t* st) {
  const int64_t size[3] = {batch, n, heads};
  for (int i = 0; i < 3; ++i) st[i] = size[i] > 1 ? given[i] : 0;
  if (batch == 0 || n == 0) return STAGE_OK;
  const int esz = dt == STAGE_BF16 ? 2 : 4;
  if (!p) return bad(STAGE_EINVAL, "null %s", name);
  if ((uintptr_t)p % 16) return bad(STAGE_EINVAL, "%s is not 16-byte aligned", name);
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0) return bad(STAGE_EINVAL, "%s has a negative stride", name);
    if (st[i] > (int64_t)1 << 53 || st[i] * esz % 16)
      return bad(STAGE_EINVAL, "a stride of %s is not a multiple of 16 bytes", name);
    if (size[i] > 1 && st[i] > ((int64_t)1 << 53) / (size[i] - 1))
      return bad(STAGE_EINVAL, "%s spans more than 2^53 elements", name);
  }
  if (st[1] * esz >= 1 << 24) return bad(STAGE_EINVAL, "positions of %s lie 16 MiB or more apart", name);
  if (output) {
    // From the innermost dimension out, each must step over all that is inside.
    int64_t span = XHD;
    bool used[3] = {};
    for (int d = 0; d < 3; ++d) {
      int at = -1;
      for (int i = 0; i < 3; ++i)
        if (!used[i] && size[i] > 1 && (at < 0 || st[i] < st[at])) at = i;
      if (at < 0) break;
      used[at] = true;
      if (st[at] < span) return bad(STAGE_EINVAL, "%s overlaps itself", name);
      span += st[at] * (size[at] - 1);
    }
  }
  return STAGE_OK;
}

void fill_common(XAttnArgs* a, const attn_shape* s, const attn_relpos* rp, const float* table) {
  a->B = s->batch;
  a->Sq = s->seq_q;
  a->Sk = s->seq_k;
  a->H = s->heads;
  a->G = s->kv_heads;
  a->rep = s->heads / s->kv_heads;
  a->causal = s->causal;
  a->scale = s->scale;
  a->c = s->scale * XLOG2E;
  a->table = table;
  if (rp) {
    a->nb = rp->num_buckets;
    a->both = rp->bidirectional;
    a->nbd = rp->bidirectional ? rp->num_buckets / 2 : rp->num_buckets;
    a->one = a->nbd / 2;
    a->reach = rp->reach;
    a->n_borders = rp->n_borders;
    for (int i = 0; i < ATTN_MAX_BUCKETS / 2; ++i)
      a->border[i] = i < rp->n_borders ? rp->border[i] : INT_MAX;
  }
}

stage_status check_table(const attn_relpos* rp, const float* table) {
  if ((rp != nullptr) != (table != nullptr))
    return bad(STAGE_EINVAL, "rp and table go together");
  if ((uintptr_t)table % 4) return bad(STAGE_EINVAL, "table is not aligned");
  return STAGE_OK;
}

stage_status check_workspace(int64_t need, const void* ws, size_t bytes) {
  if (need == 0) return STAGE_OK;
  if (!ws || bytes < (size_t)need)
    return bad(STAGE_EINVAL, "the workspace holds %zu bytes of the %lld needed", ws ? bytes : 0,
               (long long)need);
  if ((uintptr_t)ws % 16) return bad(STAGE_EINVAL, "the workspace is not 16-byte aligned");
  return STAGE_OK;
}

#define CK(expr)                 \
  do {                           \
    stage_status st_ = (expr);   \
    if (st_) return st_;         \
  } while (0)

}  // namespace

extern "C" {

const char* attn_last_error(void) { return g_err; }

stage_status attn_relpos_init(int num_buckets, int max_distance, int bidirectional,
                              attn_relpos* out) {
  Buckets k;
  if (!out) return bad(STAGE_EINVAL, "null out");
  if (!buckets_of(num_buckets, max_distance, bidirectional, &k))
    return bad(STAGE_EINVAL,
               "need 2 .. 256 buckets (both directions: even, 4 or more) and a max_distance "
               "above half a direction's buckets and at most 2048");
  attn_relpos r{};
  r.num_buckets = num_buckets;
  r.max_distance = max_distance;
  r.bidirectional = bidirectional;
  r.n_borders = k.m - 1;
  r.reach = k.one;
  for (int j = 1; j < k.m; ++j) {
    // The border as a real number (at most 2048, in 53 bits) tells its least whole
    // number, except next to one, which is looked at exactly.
    const double x = k.one * std::pow((double)max_distance / k.one, (double)j / k.m);
    int n = (int)std::lround(x);
    if (std::fabs(x - n) > 1e-6 ? n < x : !reaches(n, k.one, k.m, max_distance, j)) ++n;
    r.border[j - 1] = r.reach = n;
  }
  *out = r;
  return STAGE_OK;
}

int attn_relpos_bucket(const attn_relpos* rp, int64_t distance) {
  if (!rp || !relpos_ok(rp)) return -1;
  const int n = rp->bidirectional ? rp->num_buckets / 2 : rp->num_buckets;
  const int base = rp->bidirectional && distance > 0 ? n : 0;
  uint64_t d = distance <= 0 ? 0 - (uint64_t)distance
                             : (rp->bidirectional ? (uint64_t)distance : 0);
  if (d < (uint64_t)(n / 2)) return base + (int)d;
  int b = n / 2;
  for (int i = 0; i < rp->n_borders; ++i) b += d >= (uint64_t)rp->border[i];
  return base + b;
}

stage_status attn_workspace(const attn_shape* s, const attn_relpos* rp, int backward,
                            size_t* bytes) {
  if (!bytes) return bad(STAGE_EINVAL, "null bytes");
  if (backward != 0 && backward != 1) return bad(STAGE_EINVAL, "backward must be 0 or 1");
  CK(check_shape(s, rp));
  *bytes = (size_t)workspace_of(s, rp, backward).total;
  return STAGE_OK;
}

stage_status attn_forward(const attn_shape* s, const attn_relpos* rp, const float* table,
                          const void* q, const void* k, const void* v, const uint8_t* key_mask,
                          const int32_t* q_pos, void* out, float* lse, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  CK(check_shape(s, rp));
  CK(check_table(rp, table));
  XAttnArgs a{};
  const int B = s->batch, H = s->heads, G = s->kv_heads;
  CK(check_operand("q", q, s->q, B, s->seq_q, H, s->dtype, false, a.sq));
  CK(check_operand("k", k, s->k, B, s->seq_k, G, s->dtype, false, a.sk));
  CK(check_operand("v", v, s->v, B, s->seq_k, G, s->dtype, false, a.sv));
  CK(check_operand("out", out, s->out, B, s->seq_q, H, s->dtype, true, a.so));
  if ((uintptr_t)lse % 4 || (uintptr_t)q_pos % 4)
    return bad(STAGE_EINVAL, "lse or q_pos is not aligned");
  if (B > 0 && s->seq_q > 0 && (out == q || (s->seq_k > 0 && (out == k || out == v))))
    return bad(STAGE_EINVAL, "out may not be an input");
  const Workspace w = workspace_of(s, rp, false);
  CK(check_workspace(w.total, workspace, workspace_bytes));
  if (B == 0 || s->seq_q == 0) return STAGE_OK;
  fill_common(&a, s, rp, table);
  a.q = q;
  a.k = k;
  a.v = v;
  a.mask = key_mask;
  a.q_pos = q_pos;
  a.out = out;
  a.lse = lse;
  a.part = (float*)workspace;
  a.few_waves = w.few.waves;
  a.few_splits = w.few.splits;
  a.few_stream = w.few.stream;
  xattn_fwd_time(s->batch, s->heads, s->seq_q, s->seq_k, s->causal, s->dtype, &a.fwd_ks);
  const hipError_t e = xattn_forward(a, s->dtype, (hipStream_t)hip_stream);
  if (e != hipSuccess) return bad(STAGE_EHIP, "attn_forward: %s", hipGetErrorString(e));
  return STAGE_OK;
}

stage_status attn_backward(const attn_shape* s, const attn_relpos* rp, const float* table,
                           const void* q, const void* k, const void* v, const uint8_t* key_mask,
                           const int32_t* q_pos, const void* out, const float* lse,
                           const void* dout, void* dq, void* dk, void* dv, float* dtable,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  CK(check_shape(s, rp));
  CK(check_table(rp, table));
  if (dtable && !table) return bad(STAGE_EINVAL, "dtable without a table");
  if (dtable && dtable == table)
    return bad(STAGE_EINVAL, "a gradient may not be written over an input");
  XAttnArgs a{};
  const int B = s->batch, H = s->heads, G = s->kv_heads, Sq = s->seq_q, Sk = s->seq_k;
  CK(check_operand("q", q, s->q, B, Sq, H, s->dtype, false, a.sq));
  CK(check_operand("k", k, s->k, B, Sk, G, s->dtype, false, a.sk));
  CK(check_operand("v", v, s->v, B, Sk, G, s->dtype, false, a.sv));
  CK(check_operand("out", out, s->out, B, Sq, H, s->dtype, false, a.so));
  CK(check_operand("dout", dout, s->dout, B, Sq, H, s->dtype, false, a.sdo));
  CK(check_operand("dq", dq, s->dq, B, Sq, H, s->dtype, true, a.sdq));
  CK(check_operand("dk", dk, s->dk, B, Sk, G, s->dtype, true, a.sdk));
  CK(check_operand("dv", dv, s->dv, B, Sk, G, s->dtype, true, a.sdv));
  if ((uintptr_t)lse % 4 || (uintptr_t)q_pos % 4 || (uintptr_t)dtable % 4)
    return bad(STAGE_EINVAL, "lse, q_pos or dtable is not aligned");
  if (B > 0 && Sq > 0 && !lse) return bad(STAGE_EINVAL, "null lse");
  const void* const outs[3] = {dq, dk, dv};
  const void* const ins[5] = {q, k, v, out, dout};
  const bool here[5] = {Sq > 0, Sk > 0, Sk > 0, Sq > 0, Sq > 0};
  const bool made[3] = {Sq > 0, Sk > 0, Sk > 0};
  for (int i = 0; i < 3 && B > 0; ++i) {
    for (int j = 0; j < 5; ++j)
      if (made[i] && here[j] && outs[i] == ins[j])
        return bad(STAGE_EINVAL, "a gradient may not be written over an input");
    for (int j = 0; j < i; ++j)
      if (made[i] && made[j] && outs[i] == outs[j])
        return bad(STAGE_EINVAL, "two gradients have the same memory");
  }
  const Workspace w = workspace_of(s, rp, true);
  CK(check_workspace(w.total, workspace, workspace_bytes));
  fill_common(&a, s, rp, table);
  a.q = q;
  a.k = k;
  a.v = v;
  a.mask = key_mask;
  a.q_pos = q_pos;
  a.o = out;
  a.lse = (float*)lse;
  a.dout = dout;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dtable = dtable;
  a.dsum = (float*)workspace;
  a.tpart = (float*)((char*)workspace + w.dsum);
  a.part = (float*)((char*)workspace + w.dsum + w.tpart);
  a.dq_ks = w.dq.ks;
  a.dq_splits = w.dq.splits;
  a.kv_chunk = w.kv.chunk;
  a.kv_qs = w.kv.qs;
  a.kv_splits = w.kv.splits;
  a.one_launch = xattn_one_launch(B, H, G, Sq, Sk, w.dq, w.kv, s->dtype);
  const hipError_t e = xattn_backward(a, s->dtype, (hipStream_t)hip_stream);
  if (e != hipSuccess) return bad(STAGE_EHIP, "attn_backward: %s", hipGetErrorString(e));
  return STAGE_OK;
}

}  // extern "C"
