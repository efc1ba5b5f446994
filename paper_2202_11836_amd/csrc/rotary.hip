// Rotary positions of queries and keys (include/rotary.h): the kernel, its plan, the
// argument checks of the C ABI.
//
// y0 = A (x0 cos a - x1 sin a), y1 = A (x0 sin a + x1 cos a): three operations a value
// read and written once, so HBM bounds it.  A work-group takes the tokens s0 .. s0 + P - 1
// of one sequence, all heads of q and of k: it forms the cosines and sines of its P * n
// angles once, in LDS, and turns every head by them, 16-byte accesses.  bf16, 32 x 512 tokens of
// 16 + 16 heads, part of a packed projection: 29.2 us (4.6 TB/s); 2 x 32768 of 16 + 4: 69-71 us
// (4.7-4.8).  Stores that bypass the caches are 3-10% faster alone, and slower with the attention
// that reads them next (86 -> 88 us).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/rotary.h"
#include "common.h"

namespace {

constexpr int HEAD = 64;
constexpr int MOST_THREADS = 512;
constexpr int MAX_P = 32;  // tokens of a work-group

struct Operand {
  const void* in;
  void* out;
  int64_t si[3], so[3];  // strides of batch, position, head
};
struct Args {
  Operand x[2];  // q, k
  int S, H, HG;  // positions; heads of q, of both
  int P, nblk;   // tokens of a work-group; work-groups of a sequence
  uint32_t inv_hg, inv_items;  // 2^32 / HG, 2^32 / items of a head, rounded up
  int items;
  int n;  // pairs
  int skip;  // bit i: x[i] is turned in place
  const int32_t* pos;
  int64_t sp[2];
  int pos_each;
  int no_step;  // without pos all tokens are at 0
  float amp, sign;
  double turns[ROTARY_MAX_PAIRS];
};

// a / b for a * b < 2^32, inv = floor(2^32 / b) + 1 (b = 1: 0, which stands for 2^32).
__device__ __forceinline__ uint32_t quotient(uint32_t a, uint32_t inv) {
  return inv ? __umulhi(a, inv) : a;
}

// (cos, sin) of `turns` whole turns.  The fraction of a turn is taken in 64 bits (a
// position of 2^31 times a frequency keeps 2^-23 of a turn), a quarter turn around its
// nearest multiple is left, |x| <= pi / 4, where the Taylor series to x^9 and x^10 are off
// by less than 2^-28.
__device__ __forceinline__ float2 cos_sin(double turns) {
  const double f = (turns - rint(turns)) * 4.0;
  const double q = rint(f);
  const float x = (float)((f - q) * 1.5707963267948966);
  const float z = x * x;
  const float s =
      x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), 1.0f);
  const float c = fmaf(
      z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f),
      1.0f);
  const int k = (int)q & 3;
  const float a = k & 1 ? s : c, b = k & 1 ? c : s;
  return {k == 1 || k == 2 ? -a : a, k >= 2 ? -b : b};
}

// 16 bytes of values, at any multiple of a value's size.
template <typename T> struct Vec;
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  typedef u32x4_t __attribute__((aligned(2))) any_t;
  u32x4_t r;
  __device__ __forceinline__ void load(const bf16_t* p) { r = *(const any_t*)p; }
  __device__ __forceinline__ void store(bf16_t* p) const { *(any_t*)p = r; }
  __device__ __forceinline__ float get(int i) const {
    return __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
  }
  __device__ __forceinline__ void set2(int i, float a, float b) { r[i >> 1] = pack_bf16x2(a, b); }
  __device__ __forceinline__ void store1(bf16_t* p, int i) const { p[i] = (bf16_t)(r[i >> 1] >> (16 * (i & 1))); }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  typedef f32x4_t __attribute__((aligned(4))) any_t;
  f32x4_t r;
  __device__ __forceinline__ void load(const float* p) { r = *(const any_t*)p; }
  __device__ __forceinline__ void store(float* p) const { *(any_t*)p = r; }
  __device__ __forceinline__ float get(int i) const { return r[i]; }
  __device__ __forceinline__ void set2(int i, float a, float b) { r[i] = a, r[i + 1] = b; }
  __device__ __forceinline__ void store1(float* p, int i) const { p[i] = r[i]; }
};

enum Pairs {
  HALVES,       // (i, n + i), n a multiple of Vec::N: both halves are whole vectors
  HALVES_ODD,   // other n: the second half and what follows it lie at any place
  INTERLEAVED,  // (2 i, 2 i + 1)
};

// An item: two vectors of a head.  HALVES: Vec::N pairs, or 2 Vec::N values behind them;
// HALVES_ODD: the same with a last one of fewer; INTERLEAVED: Vec::N values of each half of the
// head.  So the items of a head access 64 bytes or more in a row.
struct Item {
  int p, which;     // token, 0: q, 1: k
  int64_t in, out;  // offsets of the head
  int a, b;         // first value of each vector
  int pair;         // first pair, -1: values that go through
};

template <typename T, Pairs L>
__device__ __forceinline__ Item item_of(const Args& g, uint32_t idx, int b, int s0) {
  constexpr int N = Vec<T>::N;
  Item it;
  uint32_t t, j;
  if constexpr (L == HALVES_ODD) {
    t = quotient(idx, g.inv_items);
    j = idx - t * g.items;
  } else {
    constexpr int ITEMS = HEAD / (2 * N);
    t = idx / ITEMS;
    j = idx % ITEMS;
  }
  it.p = (int)quotient(t, g.inv_hg);
  int h = (int)(t - it.p * g.HG);
  it.which = h >= g.H;
  if (it.which) h -= g.H;
  const Operand& x = g.x[it.which];
  const int64_t s = s0 + it.p;
  it.in = b * x.si[0] + s * x.si[1] + h * x.si[2];
  it.out = b * x.so[0] + s * x.so[1] + h * x.so[2];
  if constexpr (L == INTERLEAVED) {
    it.a = N * j;
    it.b = HEAD / 2 + it.a;
    it.pair = it.a / 2;
  } else {
    const int np = L == HALVES ? g.n / N : (g.n + N - 1) / N;
    if ((int)j < np) {
      it.pair = N * j;
      // The last pairs, fewer than a vector holds: with some of those before them, unless these
      // may be turned by now.
      if (L == HALVES_ODD && it.pair + N > g.n && g.n >= N && !(g.skip >> it.which & 1)) it.pair = g.n - N;
      it.a = it.pair;
      it.b = g.n + it.pair;
    } else {
      it.pair = -1;
      it.a = 2 * g.n + 2 * N * ((int)j - np);
      it.b = it.a + N;
    }
  }
  return it;
}

template <typename T, Pairs L>
__device__ __forceinline__ void load_item(const Args& g, const Item& it, Vec<T>& u, Vec<T>& v) {
  constexpr int N = Vec<T>::N;
  const T* p = (const T*)g.x[it.which].in + it.in;
  if (L == HALVES_ODD && it.pair < 0) {  // (none beyond the head)
    u.load(p + min(it.a, HEAD - N));
    v.load(p + min(it.b, HEAD - N));
  } else {
    u.load(p + it.a);
    v.load(p + it.b);
  }
}

template <typename T, Pairs L>
__device__ __forceinline__ void turn_item(const Args& g, const Item& it, Vec<T> u, Vec<T> v,
                                          const float2* cs) {
  constexpr int N = Vec<T>::N;
  T* p = (T*)g.x[it.which].out + it.out;
  if (L != INTERLEAVED && it.pair < 0) {
    if (g.skip >> it.which & 1) return;
    if constexpr (L == HALVES) {
      u.store(p + it.a);
      v.store(p + it.b);
    } else {
      // u and v were read from HEAD - N on where the head ends before theirs do, and are stored so
      // where that is behind the pairs.
      const int ua = min(it.a, HEAD - N), vb = min(it.b, HEAD - N);
      if (ua >= 2 * g.n) {
        u.store(p + ua);
        v.store(p + vb);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (ua + i >= it.a) u.store1(p + ua, i);
      }
    }
    return;
  }
  const float2* c = cs + it.p * ROTARY_MAX_PAIRS + it.pair;
  if constexpr (L == INTERLEAVED) {
    constexpr int FAR = HEAD / 4;  // pairs from the first vector's to the second's
#pragma unroll
    for (int i = 0; i < N; i += 2) {  // pairs beyond the n go through
      const float a = u.get(i), b = u.get(i + 1), d = v.get(i), e = v.get(i + 1);
      const float2 r = c[i / 2], w = c[FAR + i / 2];
      const bool go = it.pair + i / 2 < g.n, go2 = it.pair + FAR + i / 2 < g.n;
      u.set2(i, go ? fmaf(a, r.x, -(b * r.y)) : a, go ? fmaf(a, r.y, b * r.x) : b);
      v.set2(i, go2 ? fmaf(d, w.x, -(e * w.y)) : d, go2 ? fmaf(d, w.y, e * w.x) : e);
    }
    const bool skip = g.skip >> it.which & 1;
    if (!skip || it.pair < g.n) u.store(p + it.a);
    if (!skip || it.pair + FAR < g.n) v.store(p + it.b);
  } else {
    Vec<T> y, z;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 r = c[i], w = c[i + 1];
      const float a = u.get(i), b = v.get(i), d = u.get(i + 1), e = v.get(i + 1);
      y.set2(i, fmaf(a, r.x, -(b * r.y)), fmaf(d, w.x, -(e * w.y)));
      z.set2(i, fmaf(a, r.y, b * r.x), fmaf(d, w.y, e * w.x));
    }
    if (L == HALVES || it.pair + N <= g.n) {
      y.store(p + it.a);
      z.store(p + it.b);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (it.pair + i < g.n) {
          y.store1(p + it.a, i);
          z.store1(p + it.b, i);
        }
    }
  }
}

template <typename T, Pairs L>
__global__ __launch_bounds__(MOST_THREADS) void rotary_kernel(const Args g) {
  __shared__ float2 cs[MAX_P * ROTARY_MAX_PAIRS];
  const int b = blockIdx.x / g.nblk;
  const int s0 = (blockIdx.x - b * g.nblk) * g.P;
  const int np = min(g.P, g.S - s0);
  const uint32_t total = (uint32_t)np * g.HG * (L == HALVES_ODD ? g.items : HEAD / (2 * Vec<T>::N));
  // The first items' loads are on their way while the angles are formed.
  uint32_t idx = threadIdx.x;
  Item it;
  Vec<T> u, v;
  if (idx < total) {
    it = item_of<T, L>(g, idx, b, s0);
    load_item<T, L>(g, it, u, v);
  }
  for (int i = threadIdx.x; i < np * ROTARY_MAX_PAIRS; i += blockDim.x) {
    const int p = i / ROTARY_MAX_PAIRS, pair = i % ROTARY_MAX_PAIRS;
    float2 r = {1.0f, 0.0f};
    if (pair < g.n) {
      int64_t at = g.no_step ? 0 : s0 + p;
      if (g.pos) {
        const int32_t given = g.pos[b * g.sp[0] + (g.pos_each ? (s0 + p) * g.sp[1] : 0)];
        at = g.pos_each ? given : at + given;
      }
      r = cos_sin((double)at * g.turns[pair]);
      r.x *= g.amp;
      r.y *= g.amp * g.sign;
    }
    cs[i] = r;
  }
  __syncthreads();
  while (idx < total) {
    const uint32_t next = idx + blockDim.x;
    Item it2;
    Vec<T> u2, v2;
    if (next < total) {
      it2 = item_of<T, L>(g, next, b, s0);
      load_item<T, L>(g, it2, u2, v2);
    }
    turn_item<T, L>(g, it, u, v, cs);
    it = it2;
    u = u2;
    v = v2;
    idx = next;
  }
}

thread_local char g_err[256];

stage_status bad(stage_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}
#define CK(expr)               \
  do {                         \
    stage_status st_ = (expr); \
    if (st_) return st_;       \
  } while (0)

stage_status check_freqs(const rotary_freqs* f) {
  if (!f) return bad(STAGE_EINVAL, "null frequencies");
  if (f->rot_dim < 2 || f->rot_dim > HEAD || f->rot_dim % 2)
    return bad(STAGE_EINVAL, "rot_dim must be even, from 2 to 64");
  if (f->interleaved != 0 && f->interleaved != 1)
    return bad(STAGE_EINVAL, "interleaved must be 0 or 1");
  if (!std::isfinite(f->amplitude)) return bad(STAGE_EINVAL, "the amplitude is not finite");
  for (int i = 0; i < f->rot_dim / 2; ++i)
    if (!std::isfinite(f->turns[i])) return bad(STAGE_EINVAL, "a frequency is not finite");
  return STAGE_OK;
}

// Pointers and strides of one operand and what it becomes; strides of dimensions of one or no
// element are not looked at.
stage_status check_operand(const char* name, const rotary_shape* s, int heads, const void* in,
                           const int64_t* si, void* out, const int64_t* so, Operand* o) {
  const int64_t size[3] = {s->batch, s->seq, heads};
  const int esz = s->dtype == STAGE_BF16 ? 2 : 4;
  o->in = in;
  o->out = out;
  for (int i = 0; i < 3; ++i) {
    o->si[i] = size[i] > 1 ? si[i] : 0;
    o->so[i] = size[i] > 1 ? so[i] : 0;
  }
  if (size[0] == 0 || size[1] == 0 || heads == 0) return STAGE_OK;
  if (!in || !out) return bad(STAGE_EINVAL, "null %s or %s_out", name, name);
  if ((uintptr_t)in % 16 || (uintptr_t)out % 16)
    return bad(STAGE_EINVAL, "%s or %s_out is not 16-byte aligned", name, name);
  for (int i = 0; i < 3; ++i)
    for (const int64_t st : {o->si[i], o->so[i]}) {
      if (st < 0) return bad(STAGE_EINVAL, "%s or %s_out has a negative stride", name, name);
      if (st > (int64_t)1 << 53 || st * esz % 16)
        return bad(STAGE_EINVAL, "a stride of %s or %s_out is not a multiple of 16 bytes", name, name);
      if (size[i] > 1 && st > ((int64_t)1 << 53) / (size[i] - 1))
        return bad(STAGE_EINVAL, "%s or %s_out spans more than 2^53 elements", name, name);
    }
  // From the innermost dimension out, each must step over all that is inside.
  int64_t span = HEAD;
  bool used[3] = {};
  for (int d = 0; d < 3; ++d) {
    int at = -1;
    for (int i = 0; i < 3; ++i)
      if (!used[i] && size[i] > 1 && (at < 0 || o->so[i] < o->so[at])) at = i;
    if (at < 0) break;
    used[at] = true;
    if (o->so[at] < span) return bad(STAGE_EINVAL, "%s_out overlaps itself", name);
    span += o->so[at] * (size[at] - 1);
  }
  if (in == out)
    for (int i = 0; i < 3; ++i)
      if (o->si[i] != o->so[i])
        return bad(STAGE_EINVAL, "%s_out over %s needs the same strides", name, name);
  return STAGE_OK;
}

template <typename T>
void launch(const Args& g, Pairs pairs, dim3 grid, dim3 block, hipStream_t st) {
  if (pairs == INTERLEAVED) hipLaunchKernelGGL((rotary_kernel<T, INTERLEAVED>), grid, block, 0, st, g);
  else if (pairs == HALVES) hipLaunchKernelGGL((rotary_kernel<T, HALVES>), grid, block, 0, st, g);
  else hipLaunchKernelGGL((rotary_kernel<T, HALVES_ODD>), grid, block, 0, st, g);
}

// Tokens of a work-group and its threads: whole wavefronts, one item a thread, about 256 of them
// (512 at most: more heads go in turns), as few idle as may be, but fewer tokens while there are too
// few work-groups to fill the device.  us by items a thread, 32 x 512 tokens of 32 heads in bf16:
// 1 30.4, 2 31.6, 4 32.7, 8 33.0; of 20 heads (65536 tokens), 160 of 256 threads at work 82, 240 72.7.
struct Group {
  int tokens, threads;
};
Group group_of(int batch, int S, int64_t per_token) {
  Group best = {1, (int)std::min<int64_t>(MOST_THREADS, (per_token + 63) / 64 * 64)};
  double most = 0.0;
  for (int p = 1; p <= MAX_P && p <= S; ++p) {
    const int64_t items = p * per_token, threads = (items + 63) / 64 * 64;
    if (p > 1 && (threads > 320 || batch * (((int64_t)S + p - 1) / p) < 1024)) break;
    // (a few more idle threads rather than work-groups of one or two wavefronts)
    const double used = (double)items / threads * std::min(1.0, 0.7 + threads / 640.0);
    if (threads <= MOST_THREADS && used > most) {
      most = used;
      best = {p, (int)threads};
    }
  }
  return best;
}

uint32_t inverse(uint32_t b) { return b == 1 ? 0 : (uint32_t)(((uint64_t)1 << 32) / b + 1); }

stage_status apply(const rotary_shape* s, const rotary_freqs* f, bool backward, const void* q,
                   const void* k, const int32_t* pos, void* q_out, void* k_out, void* hip_stream) {
  if (!s) return bad(STAGE_EINVAL, "null shape");
  if (s->dtype != STAGE_F32 && s->dtype != STAGE_BF16) return bad(STAGE_EINVAL, "unknown dtype");
  if (s->batch < 0 || s->seq < 0) return bad(STAGE_EINVAL, "negative batch or length");
  if (s->seq >= 1 << 29) return bad(STAGE_EINVAL, "sequences of 2^29 positions or more");
  if (s->heads < 1 || s->kv_heads < 0 || (int64_t)s->heads + s->kv_heads > 65535)
    return bad(STAGE_EINVAL, "heads must be >= 1, kv_heads >= 0, both together at most 65535");
  if (s->pos_each != 0 && s->pos_each != 1) return bad(STAGE_EINVAL, "pos_each must be 0 or 1");
  CK(check_freqs(f));
  Args g{};
  CK(check_operand("q", s, s->heads, q, s->q, q_out, s->q_out, &g.x[0]));
  CK(check_operand("k", s, s->kv_heads, k, s->k, k_out, s->k_out, &g.x[1]));
  if ((uintptr_t)pos % 4) return bad(STAGE_EINVAL, "pos is not aligned");
  for (int i = 0; i < 2; ++i) {
    const int64_t size = i ? s->seq : s->batch;
    g.sp[i] = size > 1 && (i == 0 || s->pos_each) ? s->pos[i] : 0;
    if (pos && (g.sp[i] < 0 || g.sp[i] > (int64_t)1 << 53 ||
                (size > 1 && g.sp[i] > ((int64_t)1 << 53) / (size - 1))))
      return bad(STAGE_EINVAL, "a stride of pos is out of range");
  }
  if (s->batch == 0 || s->seq == 0) return STAGE_OK;
  if (s->kv_heads > 0 && (q_out == k || k_out == q || q_out == k_out))
    return bad(STAGE_EINVAL, "an output may be its own input, not another operand");
  if (pos && ((const void*)pos == q_out || (s->kv_heads > 0 && (const void*)pos == k_out)))
    return bad(STAGE_EINVAL, "an output may not be written over pos");
  g.S = s->seq;
  g.H = s->heads;
  g.HG = s->heads + s->kv_heads;
  g.n = f->rot_dim / 2;
  g.pos = pos;
  g.pos_each = s->pos_each;
  g.amp = f->amplitude;
  g.sign = backward ? -1.0f : 1.0f;
  for (int i = 0; i < g.n; ++i) g.turns[i] = f->turns[i];
  g.skip = (q == q_out) | (k == k_out) << 1;
  const int N = s->dtype == STAGE_BF16 ? 8 : 4;
  const Pairs pairs = f->interleaved ? INTERLEAVED : g.n % N == 0 ? HALVES : HALVES_ODD;
  g.items = pairs != HALVES_ODD ? HEAD / (2 * N) : (g.n + N - 1) / N + (HEAD - 2 * g.n + 2 * N - 1) / (2 * N);
  int batch = s->batch;
  if (g.S == 1 && batch > 1) {
    // Sequences of one token each are tokens of one sequence whose positions are given, or all 0.
    g.S = batch;
    batch = 1;
    for (Operand& x : g.x) {
      x.si[1] = x.si[0];
      x.so[1] = x.so[0];
    }
    g.pos_each = 1;
    g.sp[1] = g.sp[0];
    g.no_step = !pos;
  }
  const Group group = group_of(batch, g.S, (int64_t)g.HG * g.items);
  g.P = group.tokens;
  g.nblk = (int)(((int64_t)g.S + g.P - 1) / g.P);
  g.inv_hg = inverse(g.HG);
  g.inv_items = inverse(g.items);
  const int64_t grid = (int64_t)batch * g.nblk;
  if (grid * group.threads >= (int64_t)1 << 32) return bad(STAGE_EINVAL, "batch * length too large");
  if (s->dtype == STAGE_BF16) launch<bf16_t>(g, pairs, dim3((unsigned)grid), dim3(group.threads), (hipStream_t)hip_stream);
  else launch<float>(g, pairs, dim3((unsigned)grid), dim3(group.threads), (hipStream_t)hip_stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess)
    return bad(STAGE_EHIP, "rotary_%s: %s", backward ? "backward" : "forward", hipGetErrorString(e));
  return STAGE_OK;
}

}  // namespace

extern "C" {

const char* rotary_last_error(void) { return g_err; }

stage_status rotary_init_freqs(int rot_dim, int interleaved, const double* freqs, double amplitude,
                               rotary_freqs* out) {
  if (!out || !freqs) return bad(STAGE_EINVAL, "null out or freqs");
  rotary_freqs r{};
  r.rot_dim = rot_dim;
  r.interleaved = interleaved;
  r.amplitude = (float)amplitude;
  if (rot_dim < 2 || rot_dim > HEAD) return bad(STAGE_EINVAL, "rot_dim must be even, from 2 to 64");
  for (int i = 0; i < rot_dim / 2; ++i) r.turns[i] = freqs[i] / 6.283185307179586476925;
  CK(check_freqs(&r));
  *out = r;
  return STAGE_OK;
}

stage_status rotary_init(int rot_dim, int interleaved, double base, rotary_scaling scaling,
                         double factor, int original_len, double low, double high,
                         double amplitude, rotary_freqs* out) {
  if (rot_dim < 2 || rot_dim > HEAD) return bad(STAGE_EINVAL, "rot_dim must be even, from 2 to 64");
  if (!(base > 0.0)) return bad(STAGE_EINVAL, "base must be positive");
  if (scaling < ROTARY_NONE || scaling > ROTARY_PARTS) return bad(STAGE_EINVAL, "unknown scaling");
  if (scaling != ROTARY_NONE && !(factor > 0.0 && std::isfinite(factor)))
    return bad(STAGE_EINVAL, "factor must be positive");
  if (scaling == ROTARY_PARTS && !(original_len >= 1 && std::isfinite(low) && std::isfinite(high) && high > low))
    return bad(STAGE_EINVAL, "need original_len >= 1 and high > low");
  const int n = rot_dim / 2;
  double f[ROTARY_MAX_PAIRS];
  if (scaling == ROTARY_BASE && n > 1) base *= std::pow(factor, (double)n / (n - 1));
  for (int i = 0; i < n; ++i) {
    f[i] = std::pow(base, -(double)i / n);
    if (scaling == ROTARY_LINEAR) f[i] /= factor;
    if (scaling == ROTARY_PARTS) {
      const double t = original_len * f[i] / 6.283185307179586476925;
      const double w = std::min(1.0, std::max(0.0, (t - low) / (high - low)));
      f[i] *= w + (1.0 - w) / factor;
    }
  }
  return rotary_init_freqs(rot_dim, interleaved, f, amplitude, out);
}

stage_status rotary_forward(const rotary_shape* s, const rotary_freqs* f, const void* q, const void* k,
                            const int32_t* pos, void* q_out, void* k_out, void* hip_stream) {
  return apply(s, f, false, q, k, pos, q_out, k_out, hip_stream);
}

stage_status rotary_backward(const rotary_shape* s, const rotary_freqs* f, const void* q,
                             const void* k, const int32_t* pos, void* q_out, void* k_out,
                             void* hip_stream) {
  return apply(s, f, true, q, k, pos, q_out, k_out, hip_stream);
}

}  // extern "C"
