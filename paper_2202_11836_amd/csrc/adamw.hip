// AdamW of many tensors at once (include/adamw.h): the kernels, and the handle of the C ABI.
//
// An element is read once and written once with its states, 28 bytes with fp32 states, 18 with
// 8-bit ones (and a master copy): HBM bounds it.  All tensors are one launch: they are cut
// into chunks of 2048 elements, whose table lies on the device, and work-groups take every
// gridDim-th one.  50M bf16 weights with master copies, 8-bit states and bf16 gradients: 150 us,
// 5.4 TB/s (counted traffic equals the bytes it cannot do without); 504M with fp32 states and
// gradients 2975 us, 5.1 TB/s, and 346 us for the gradients' norm, 5.8 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <vector>

#include "../../include/adamw.h"
#include "common.h"

namespace {

constexpr int THREADS = 256;
constexpr int CHUNK = THREADS * 8;  // elements: eight a thread, a block of 8-bit states 32 threads
constexpr int GROUPS = 512, GROUPS_LIGHT = 1024;  // most work-groups, 2 or 4 to a CU
constexpr int LIGHT = 14;           // bytes to and from memory for an element, of which it is 4
constexpr int MOST_PARTS = 1024;    // work-groups of the norm
// The tickets: one counter, and behind it in memory those that many work-groups take first, a
// COUNTERS'th of them each, in cache lines of their own.
constexpr int COUNTERS = 32, TICKET_STEP = 32;

enum Kind : int { P_F32, P_BF16_MASTER, P_BF16 };

struct Tensor {
  void* p;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale, *master;
  int64_t n;
  float decay, lr_scale;
  int kind, grad_bf16, bits;
  int pad;
};
struct Chunk {
  int tensor, index;  // elements [index * CHUNK, ...) of the tensor
};
// (the tables never change, and all threads of a work-group read the same entry: scalar loads)
typedef const __attribute__((address_space(4))) Tensor* TensorTable;
typedef const __attribute__((address_space(4))) Chunk* ChunkTable;
struct StepArgs {
  TensorTable tensors;
  ChunkTable chunks;
  int n_chunks;
  int64_t* steps;
  unsigned* ticket;     // (and the other counters) 0 between launches
  const double* parts;  // sums of squares, or NULL: no clipping
  int n_parts;
  float max_norm;
  float* norm;
  float lr;
  const float* lr_ptr;
  double beta1, beta2;
  float eps;
};

// The tensors' addresses come from memory: accesses through them are told to be global.
template <typename V, typename T>
__device__ __forceinline__ V get(const T* p) {
  return *(const __attribute__((address_space(1))) V*)(uintptr_t)p;
}
template <typename V, typename T>
__device__ __forceinline__ void put(T* p, V v) {
  *(__attribute__((address_space(1))) V*)(uintptr_t)p = v;
}

// What a tensor has of a thread's eight elements: all (WHOLE); or the first n, behind which the tensor
// ends (n <= 0: none), and which come as the last of the tensor's last eight (PART: no branch keeps a
// load from starting before another is done; one tensor of 2047 in fp32 4.4 -> 4.1 us, in bf16 with
// 8-bit states 6.7 -> 4.9); or, of a tensor of fewer than eight, one at a time (FEW).
enum Reach { WHOLE, PART, FEW };

// Eight elements from p on, element-aligned accesses of 8 and 16 bytes; FEW: the first n.
template <Reach R>
__device__ __forceinline__ void load8(const float* p, int n, float v[8]) {
  typedef f32x4_t __attribute__((aligned(4))) any_t;
  if constexpr (R != FEW) {
    const f32x4_t a = get<any_t>(p), b = get<any_t>(p + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? get<float>(p + k) : 0.0f;
  }
}
template <Reach R>
__device__ __forceinline__ void load8(const bf16_t* p, int n, float v[8]) {
  typedef u32x4_t __attribute__((aligned(2))) any_t;
  if constexpr (R != FEW) {
    const u32x4_t a = get<any_t>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(a[k] << 16);
      v[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? bf2f(get<bf16_t>(p + k)) : 0.0f;
  }
}
template <Reach R>
__device__ __forceinline__ u32x2_t load8(const uint8_t* p, int n) {
  typedef u32x2_t __attribute__((aligned(1))) any_t;
  if constexpr (R != FEW) return get<any_t>(p);
  u32x2_t r = {0, 0};
#pragma unroll
  for (int k = 0; k < 8; ++k) r[k >> 2] |= (k < n ? (uint32_t)get<uint8_t>(p + k) : 0) << (8 * (k & 3));
  return r;
}
// PART: the first `gone` of eight go, zeros come in at the end (8 or more: all).
template <Reach R>
__device__ __forceinline__ void drop(float v[8], int gone) {
  if constexpr (R == PART) {
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = gone & o ? (k + o < 8 ? v[k + o < 8 ? k + o : 7] : 0.0f) : v[k];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = gone < 8 ? v[k] : 0.0f;
  }
}
template <Reach R>
__device__ __forceinline__ void drop(u32x2_t& c, int gone) {
  if constexpr (R == PART) {
    const uint64_t r = gone < 8 ? ((uint64_t)c[1] << 32 | c[0]) >> (8 * (gone & 7)) : 0;
    c = u32x2_t{(uint32_t)r, (uint32_t)(r >> 32)};
  }
}
template <Reach R>
__device__ __forceinline__ void store8(float* p, int n, const float v[8]) {
  typedef f32x4_t __attribute__((aligned(4))) any_t;
  if (R == WHOLE || n >= 8) {
    put<any_t>(p, f32x4_t{v[0], v[1], v[2], v[3]});
    put<any_t>(p + 4, f32x4_t{v[4], v[5], v[6], v[7]});
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) put<float>(p + k, v[k]);
  }
}
template <Reach R>
__device__ __forceinline__ void store8(bf16_t* p, int n, u32x4_t r) {
  typedef u32x4_t __attribute__((aligned(2))) any_t;
  if (R == WHOLE || n >= 8) {
    put<any_t>(p, r);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) put<bf16_t>(p + k, (bf16_t)(r[k >> 1] >> (16 * (k & 1))));
  }
}
template <Reach R>
__device__ __forceinline__ void store8(uint8_t* p, int n, const uint32_t c[8]) {
  typedef u32x2_t __attribute__((aligned(1))) any_t;
  if (R == WHOLE || n >= 8) {
    put<any_t>(p, u32x2_t{c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24,
                          c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24});
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) put<uint8_t>(p + k, (uint8_t)c[k]);
  }
}

// The values of eight codes times their scale: the device's own conversions, exact.
__device__ __forceinline__ void from_e4m3(u32x2_t c, float scale, float v[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], false);
    const f32x2_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], true);
    v[4 * k] = a[0] * scale, v[4 * k + 1] = a[1] * scale;
    v[4 * k + 2] = b[0] * scale, v[4 * k + 3] = b[1] * scale;
  }
}
__device__ __forceinline__ void from_e5m2(u32x2_t c, float scale, float v[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_bf8((int)c[k], false);
    const f32x2_t b = __builtin_amdgcn_cvt_pk_f32_bf8((int)c[k], true);
    v[4 * k] = a[0] * scale, v[4 * k + 1] = a[1] * scale;
    v[4 * k + 2] = b[0] * scale, v[4 * k + 3] = b[1] * scale;
  }
}
// Codes of eight x with |x| <= 448 (values times their block's inverse scale): up where the
// part beyond the last bit and r / 2^16 come to a step.  A normal code is a float's exponent
// and leading mantissa bits, so the sum may carry into either; a subnormal one counts 2^-9,
// and few meet one (below 2^-15 of a block's largest), so a wavefront branches for it.
__device__ __forceinline__ void to_e4m3(const float x[8], const uint32_t r[8], uint32_t c[8]) {
  float least = fabsf(x[0]);
#pragma unroll
  for (int k = 1; k < 8; ++k) least = fminf(least, fabsf(x[k]));
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t b = __float_as_uint(x[k]);
    c[k] = min(((b & 0x7fffffffu) + ((r[k] & 0xffffu) << 4)) >> 20, 0x7eu + 960u) - 960u | (b >> 24 & 0x80u);
  }
  if (__builtin_amdgcn_ballot_w64(least < 0x1p-6f)) {
    asm volatile("");  // (not to be made part of the way without)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t b = __float_as_uint(x[k]), n = ((uint32_t)(fabsf(x[k]) * 0x1p25f) + (r[k] & 0xffffu)) >> 16;
      if (fabsf(x[k]) < 0x1p-6f) c[k] = n | (b >> 24 & 0x80u);
    }
  }
}
// The same for 0 <= x <= 57344 and the high halves of r; x > 0 has a code above 0.
__device__ __forceinline__ void to_e5m2(const float x[8], const uint32_t r[8], uint32_t c[8]) {
  float least = x[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) least = fminf(least, x[k]);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    c[k] = min((__float_as_uint(x[k]) + (r[k] >> 16 << 5)) >> 21, 0x7bu + 448u) - 448u;
  if (__builtin_amdgcn_ballot_w64(least < 0x1p-14f)) {
    asm volatile("");
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t n = ((uint32_t)(x[k] * 0x1p32f) + (r[k] >> 16)) >> 16;
      if (x[k] < 0x1p-14f) c[k] = max(n, x[k] > 0.0f ? 1u : 0u);
    }
  }
}
// A block's scale and its inverse from the bits of its largest |value| (NaN above all), both
// rounded as a division is: 0 for values too small for the inverse, NaN where one is not
// finite.  The scale's quotient by `most`, 7 times a power of 2, is a product with its rounded
// reciprocal and one correction, which is exact there (P. Markstein, 1990).
__device__ __forceinline__ float2 scale_of(uint32_t top, float most, float reciprocal) {
  const float f = __uint_as_float(top);
  if (top >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.0f};
  if (f < 0x1p-110f) return {0.0f, 0.0f};
  const float q = f * reciprocal;
  return {fmaf(fmaf(-most, q, f), reciprocal, q), most / f};
}
// The largest over 32 lanes, to all of them.
__device__ __forceinline__ uint32_t max32(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));   // lane ^ 1
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true));   // lane ^ 2
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));  // lane ^ 7
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));  // lane ^ 15
  return max(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x401F));           // lane ^ 16
}
// Random bits of element i at step t (adamw.h).
__device__ __forceinline__ uint32_t random_bits(uint32_t i, uint32_t t) {
  uint32_t x = i * 0x9E3779B1u + t * 0x6A09E667u;
  x = (x ^ x >> 15) * 0xBB67AE85u;
  x = (x ^ x >> 13) * 0x3C6EF373u;
  return x ^ x >> 16;
}

struct Step {  // what all elements of a step share
  float clip, b1, c1, b2, c2;  // c1 = 1 - beta1, c2 = 1 - beta2, each rounded once
  float lr, lr_bias;           // lr, lr / (1 - beta1^t)
  float inv_root;              // 1 / sqrt(1 - beta2^t)
  float eps;
  // The device's square root of a subnormal is 0.  Roots of those are below 2^-63, and where eps is
  // 2^24 times what inv_root makes of that they do not count.  us with / without, 50M weights with 8-bit
  // states: 102.2 / 96.8 (bf16 alone), 150.3 / 149.0 (a master copy).
  bool small_roots;
  uint32_t t;
};

// New states of eight elements, from gradients g: each operation rounded by itself, as they
// are defined.
__device__ __forceinline__ void new_states(const float g[8], const Step& s, float m[8], float v[8]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float d = g[k] * s.clip;
    m[k] = m[k] * s.b1 + d * s.c1;
    v[k] = v[k] * s.b2 + d * d * s.c2;
  }
}

// Eight elements from i of a tensor, or what it has of them.
template <int KIND, bool GRAD_BF16, int BITS, Reach R>
__device__ __forceinline__ void update8(const Tensor& x, int64_t i, const Step& s) {
  const int64_t block = i / ADAMW_BLOCK;
  if (R != WHOLE && block * ADAMW_BLOCK >= x.n) return;  // (with the other lanes of the block)
  const int n = R == WHOLE ? 8 : (int)max((int64_t)0, min((int64_t)8, x.n - i));
  const int64_t at = R == PART ? min(i, x.n - 8) : i;
  const int gone = (int)(i - at);
  float w[8], g[8], m[8], v[8];
  if constexpr (KIND == P_F32) load8<R>((const float*)x.p + at, n, w);
  else if constexpr (KIND == P_BF16_MASTER) load8<R>(x.master + at, n, w);
  else load8<R>((const bf16_t*)x.p + at, n, w);
  if constexpr (GRAD_BF16) load8<R>((const bf16_t*)x.g + at, n, g);
  else load8<R>((const float*)x.g + at, n, g);
  if constexpr (BITS == 8) {
    u32x2_t cm = load8<R>((const uint8_t*)x.m + at, n), cv = load8<R>((const uint8_t*)x.v + at, n);
    const float sm = get<float>(x.m_scale + block), sv = get<float>(x.v_scale + block);
    drop<R>(cm, gone);
    drop<R>(cv, gone);
    from_e4m3(cm, sm, m);
    from_e5m2(cv, sv, v);
  } else {
    load8<R>((const float*)x.m + at, n, m);
    load8<R>((const float*)x.v + at, n, v);
    drop<R>(m, gone);
    drop<R>(v, gone);
  }
  drop<R>(w, gone);
  drop<R>(g, gone);
  new_states(g, s, m, v);
  const float keep = 1.0f - s.lr * x.lr_scale * x.decay, rate = s.lr_bias * x.lr_scale;
  float root[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) root[k] = __builtin_amdgcn_sqrtf(v[k]);
  if (s.small_roots) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (v[k] < 0x1p-126f) root[k] = __builtin_amdgcn_sqrtf(v[k] * 0x1p64f) * 0x1p-32f;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    // (square root and reciprocal of 1 ulp: a change of w, not w, is off by that)
    const float den = fmaf(root[k], s.inv_root, s.eps);
    w[k] = fmaf(w[k], keep, -(rate * m[k] * __builtin_amdgcn_rcpf(den)));
  }
  uint32_t r[8];
  if constexpr (BITS == 8 || KIND == P_BF16)
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = random_bits((uint32_t)i + k, s.t);
  if constexpr (KIND == P_F32) {
    store8<R>((float*)x.p + i, n, w);
  } else {
    u32x4_t b;
    if constexpr (KIND == P_BF16) {
      // The sum with a draw may carry out of a NaN, into the sign and beyond: a quiet one, as w is, is the
      // same without its low bits.  Few meet one, so a wavefront branches for it (50M weights in one
      // tensor, 8-bit states, us: no look 97.3, this 98.4, a choice for each weight 100.6).
      bool nan = false;
#pragma unroll
      for (int k = 0; k < 8; k += 2) nan |= __builtin_isunordered(w[k], w[k + 1]);
      if (__builtin_amdgcn_ballot_w64(nan)) {
        asm volatile("");
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (w[k] != w[k]) w[k] = __uint_as_float(__float_as_uint(w[k]) & 0xffff0000u);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      b[k] = KIND == P_BF16 ? (__float_as_uint(w[2 * k]) + (r[2 * k] >> 16)) >> 16 |
                                  ((__float_as_uint(w[2 * k + 1]) + (r[2 * k + 1] >> 16)) & 0xffff0000u)
                            : pack_bf16x2(w[2 * k], w[2 * k + 1]);
    store8<R>((bf16_t*)x.p + i, n, b);
    if constexpr (KIND == P_BF16_MASTER) store8<R>(x.master + i, n, w);
  }
  if constexpr (BITS == 8) {
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      top_m = max(top_m, __float_as_uint(m[k]) & 0x7fffffffu);
      top_v = max(top_v, __float_as_uint(v[k]));  // (a NaN is above all with either sign)
    }
    const float2 sm = scale_of(max32(top_m), 448.0f, 1.0f / 448.0f);
    const float2 sv = scale_of(max32(top_v), 57344.0f, 1.0f / 57344.0f);
    uint32_t cm[8], cv[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] *= sm.y, v[k] *= sv.y;
    to_e4m3(m, r, cm);
    to_e5m2(v, r, cv);
    if (sm.y == 0.0f || sv.y == 0.0f)  // (a block of zeros, or one that is not finite)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (sm.y == 0.0f) cm[k] = 0;
        if (sv.y == 0.0f) cv[k] = 0;
      }
    store8<R>((uint8_t*)x.m + i, n, cm);
    store8<R>((uint8_t*)x.v + i, n, cv);
    if ((threadIdx.x & 31) == 0 && n > 0) {
      put<float>(x.m_scale + block, sm.x);
      put<float>(x.v_scale + block, sv.x);
    }
  } else {
    store8<R>((float*)x.m + i, n, m);
    store8<R>((float*)x.v + i, n, v);
  }
}

template <int KIND, bool GRAD_BF16, int BITS>
__device__ __forceinline__ void update_chunk(const Tensor& x, int64_t i, Reach r, const Step& s) {
  if (r == WHOLE) update8<KIND, GRAD_BF16, BITS, WHOLE>(x, i, s);
  else if (r == PART) update8<KIND, GRAD_BF16, BITS, PART>(x, i, s);
  else update8<KIND, GRAD_BF16, BITS, FEW>(x, i, s);
}
template <int KIND, bool GRAD_BF16>
__device__ __forceinline__ void update_bits(const Tensor& x, int64_t i, Reach r, const Step& s) {
  if (x.bits == 8) update_chunk<KIND, GRAD_BF16, 8>(x, i, r, s);
  else update_chunk<KIND, GRAD_BF16, 32>(x, i, r, s);
}
template <int KIND>
__device__ __forceinline__ void update_grad(const Tensor& x, int64_t i, Reach r, const Step& s) {
  if (x.grad_bf16) update_bits<KIND, true>(x, i, r, s);
  else update_bits<KIND, false>(x, i, r, s);
}

// beta^t by squaring, in 64 bits.
__device__ __forceinline__ double power(double b, int64_t t) {
  double p = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) p *= b;
  return p;
}

// The sum over a work-group, in a fixed order, to all of it.
__device__ __forceinline__ double group_sum(double v, double* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int j = 1; j < THREADS / 64; ++j) v += lds[j];
  __syncthreads();
  return v;
}

__device__ __forceinline__ Tensor tensor_at(const StepArgs& a, int j) {
  TensorTable t = a.tensors + j;
  return {t->p, t->g, t->m, t->v, t->m_scale, t->v_scale, t->master, t->n, t->decay, t->lr_scale,
          t->kind, t->grad_bf16, t->bits, 0};
}
__device__ __forceinline__ Chunk chunk_at(const StepArgs& a, int c) {
  return {a.chunks[c].tensor, a.chunks[c].index};
}

// Two work-groups to a CU that take chunk after chunk: 128 bytes a thread in flight are enough, and
// what each has to set up (the powers, the norm's parts) is done 512 times.  us by work-groups a CU,
// 1 / 2 / 3 / 4: 50M weights with 8-bit states (0.8 GB) 240 / 150 / 165 / 166, 504M in bf16 (15 GB,
// clipped) 3365 / 3363 / 3385 / 3383, 5M in fp32 (139 MB, clipped) 31.6 / 32.2 / 31.9 / 33.5; numbers
// between leave CUs with unequal shares (1.25: 205, 4322, 33.8).  Four where an element is LIGHT: bf16
// without master copies and 8-bit states, 50M weights 133 / 119 with 2 / 4, with gradients in fp32
// 138 / 128, 19M weights 63 / 52.
__global__ __launch_bounds__(THREADS) void step_kernel(const StepArgs a) {
  __shared__ double lds[THREADS / 64];
  const int64_t t = *a.steps + 1;
  Chunk ch = chunk_at(a, blockIdx.x);  // (the table has an entry to read where there are no chunks)
  Step s;
  s.clip = 1.0f;
  bool go = true;
  if (a.parts) {
    double sum = 0.0;
    for (int j = threadIdx.x; j < a.n_parts; j += THREADS) sum += a.parts[j];
    const double norm = sqrt(group_sum(sum, lds));
    go = norm < INFINITY;
    s.clip = norm > a.max_norm ? (float)(a.max_norm / norm) : 1.0f;
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  }
  const float lr = a.lr_ptr ? *a.lr_ptr : a.lr;
  s.b1 = (float)a.beta1;
  s.c1 = (float)(1.0 - a.beta1);
  s.b2 = (float)a.beta2;
  s.c2 = (float)(1.0 - a.beta2);
  s.lr = lr;
  s.lr_bias = (float)(lr / (1.0 - power(a.beta1, t)));
  s.inv_root = (float)(1.0 / sqrt(1.0 - power(a.beta2, t)));
  s.eps = a.eps;
  s.small_roots = __builtin_amdgcn_readfirstlane(s.inv_root > a.eps * 0x1p39f);
  s.t = (uint32_t)t;
  for (int c = blockIdx.x; go && c < a.n_chunks; c += gridDim.x) {
    const Chunk next = chunk_at(a, min(c + (int)gridDim.x, a.n_chunks - 1));
    const Tensor x = tensor_at(a, ch.tensor);
    const int64_t first = (int64_t)ch.index * CHUNK, i = first + 8 * threadIdx.x;
    const Reach r = first + CHUNK <= x.n ? WHOLE : x.n >= 8 ? PART : FEW;
    if (x.kind == P_F32) update_grad<P_F32>(x, i, r, s);
    else if (x.kind == P_BF16_MASTER) update_grad<P_BF16_MASTER>(x, i, r, s);
    else update_grad<P_BF16>(x, i, r, s);
    ch = next;
  }
  // All of a work-group have read the number of steps before it takes a ticket, so the one with
  // the last ticket may raise it.  A counter serves a work-group in 9 ns, and many end together: 24
  // fp32 tensors of 208 chunks 6.8 us with the last counter alone, 5.4 so, 900 of a chunk each 10.8 and
  // 7.2 (and on the way in, tickets keep work-groups from their work: 139 MB 34.6 -> 48 us).
  __syncthreads();
  if (threadIdx.x != 0) return;
  unsigned last = gridDim.x;
  if (gridDim.x > COUNTERS) {
    last = COUNTERS;
    const unsigned mine = blockIdx.x % COUNTERS;
    unsigned* const first = a.ticket + TICKET_STEP * (1 + mine);
    if (atomicAdd(first, 1u) + 1 < (gridDim.x - mine + COUNTERS - 1) / COUNTERS) return;
    *first = 0;
  }
  if (atomicAdd(a.ticket, 1u) + 1 < last) return;
  *a.ticket = 0;
  if (go) *a.steps = t;
}

template <Reach R>
__device__ __forceinline__ void gradients(const Tensor& x, int64_t i, float g[8]) {
  const int n = R == WHOLE ? 8 : (int)max((int64_t)0, min((int64_t)8, x.n - i));
  const int64_t at = R == PART ? min(i, x.n - 8) : i;
  if (x.grad_bf16) load8<R>((const bf16_t*)x.g + at, n, g);
  else load8<R>((const float*)x.g + at, n, g);
  drop<R>(g, (int)(i - at));
}

// Sums of squares of the gradients, a work-group's chunks together, in 64 bits (squares of
// fp32 values neither overflow there nor vanish).
__global__ __launch_bounds__(THREADS) void norm_kernel(const StepArgs a, double* parts) {
  __shared__ double lds[THREADS / 64];
  double sum = 0.0;
  for (int c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
    const Chunk ch = chunk_at(a, c);
    const Tensor x = tensor_at(a, ch.tensor);
    const int64_t first = (int64_t)ch.index * CHUNK;
    float g[8];
    if (first + CHUNK <= x.n) gradients<WHOLE>(x, first + 8 * threadIdx.x, g);
    else if (x.n >= 8) gradients<PART>(x, first + 8 * threadIdx.x, g);
    else gradients<FEW>(x, first + 8 * threadIdx.x, g);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = fma((double)g[k], (double)g[k], sum);
  }
  sum = group_sum(sum, lds);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

thread_local char g_err[256];

stage_status bad(stage_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

}  // namespace

struct adamw {
  int device = 0;
  int n_chunks = 0;
  int groups = 0;          // most work-groups
  void* memory = nullptr;  // parts, ticket, tensors, chunks
  double* parts = nullptr;
  unsigned* ticket = nullptr;
  Tensor* tensors = nullptr;
  Chunk* chunks = nullptr;
  int64_t* steps = nullptr;
};

extern "C" {

const char* adamw_last_error(void) { return g_err; }

stage_status adamw_init(const adamw_tensor* tensors, int n, int64_t* steps, adamw_t** out) try {
  if (!out) return bad(STAGE_EINVAL, "null out");
  *out = nullptr;
  if (n < 0 || (n > 0 && !tensors)) return bad(STAGE_EINVAL, "null tensors or a negative number of them");
  if (!steps || (uintptr_t)steps % 8) return bad(STAGE_EINVAL, "steps is null or not aligned");
  std::vector<Tensor> host(n);
  std::vector<Chunk> chunks;
  int64_t all = 0;
  for (int j = 0; j < n; ++j) {
    const adamw_tensor& x = tensors[j];
    Tensor& t = host[j];
    t = Tensor{};
    if ((x.dtype != STAGE_F32 && x.dtype != STAGE_BF16) || (x.grad_dtype != STAGE_F32 && x.grad_dtype != STAGE_BF16))
      return bad(STAGE_EINVAL, "tensor %d: unknown type", j);
    if (x.state_bits != 32 && x.state_bits != 8)
      return bad(STAGE_EINVAL, "tensor %d: state_bits must be 32 or 8", j);
    if (x.numel < 0) return bad(STAGE_EINVAL, "tensor %d: a negative number of elements", j);
    all += std::min(x.numel, (int64_t)1 << 40);
    if (all >= (int64_t)1 << 40) return bad(STAGE_EINVAL, "2^40 elements or more");
    if (!std::isfinite(x.weight_decay) || !std::isfinite(x.lr_scale))
      return bad(STAGE_EINVAL, "tensor %d: weight_decay or lr_scale is not finite", j);
    const bool eight = x.state_bits == 8, bf = x.dtype == STAGE_BF16;
    if (x.numel == 0) continue;
    if (!x.param || !x.grad || !x.m || !x.v || (eight && (!x.m_scale || !x.v_scale)))
      return bad(STAGE_EINVAL, "tensor %d: a null pointer", j);
    if (!eight && (x.m_scale || x.v_scale)) return bad(STAGE_EINVAL, "tensor %d: scales of 32-bit states", j);
    if (x.master && !bf) return bad(STAGE_EINVAL, "tensor %d: a master copy of an fp32 parameter", j);
    if ((uintptr_t)x.param % (bf ? 2 : 4) || (uintptr_t)x.grad % (x.grad_dtype == STAGE_BF16 ? 2 : 4) ||
        (!eight && ((uintptr_t)x.m % 4 || (uintptr_t)x.v % 4)) || (uintptr_t)x.m_scale % 4 ||
        (uintptr_t)x.v_scale % 4 || (uintptr_t)x.master % 4)
      return bad(STAGE_EINVAL, "tensor %d: a pointer is not aligned", j);
    t = {x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.master, x.numel, x.weight_decay, x.lr_scale,
         !bf ? P_F32 : x.master ? P_BF16_MASTER : P_BF16, x.grad_dtype == STAGE_BF16, x.state_bits, 0};
  }
  // What a step writes, and the gradients that it reads, are apart.
  std::vector<std::pair<uintptr_t, uintptr_t>> spans;
  for (const Tensor& t : host) {
    const int64_t blocks = (t.n + ADAMW_BLOCK - 1) / ADAMW_BLOCK, se = t.bits == 8 ? 1 : 4;
    const std::pair<const void*, int64_t> mem[6] = {{t.p, t.n * (t.kind == P_F32 ? 4 : 2)}, {t.m, t.n * se},
                                                    {t.v, t.n * se}, {t.m_scale, blocks * 4},
                                                    {t.v_scale, blocks * 4}, {t.master, t.n * 4}};
    for (const auto& s : mem)
      if (s.first && s.second) spans.push_back({(uintptr_t)s.first, (uintptr_t)s.first + s.second});
  }
  spans.push_back({(uintptr_t)steps, (uintptr_t)steps + 8});
  std::sort(spans.begin(), spans.end());
  for (size_t j = 1; j < spans.size(); ++j)
    if (spans[j].first < spans[j - 1].second)
      return bad(STAGE_EINVAL, "two of the parameters and states share memory");
  for (int j = 0; j < n; ++j) {
    const Tensor& t = host[j];
    if (!t.n) continue;
    const uintptr_t a = (uintptr_t)t.g, b = a + t.n * (t.grad_bf16 ? 2 : 4);
    const auto next = std::upper_bound(spans.begin(), spans.end(), std::make_pair(b - 1, ~(uintptr_t)0));
    if (next != spans.begin() && std::prev(next)->second > a)
      return bad(STAGE_EINVAL, "tensor %d: the gradient shares memory with a parameter or state", j);
  }
  for (int j = 0; j < n; ++j)
    for (int64_t i = 0; i * CHUNK < host[j].n; ++i) {
      if (chunks.size() >= (size_t)1 << 30) return bad(STAGE_EINVAL, "too many elements");
      chunks.push_back({j, (int)i});
    }
  const int n_chunks = (int)chunks.size();
  // (an entry each to read where there is nothing to do)
  if (chunks.empty()) chunks.push_back({0, 0});
  if (host.empty()) host.push_back(Tensor{});
  adamw_t* h = new adamw_t;
  h->steps = steps;
  h->n_chunks = n_chunks;
  int64_t elements = 0, traffic = 0;
  for (const Tensor& t : host) {
    elements += t.n;
    traffic += t.n * ((t.kind == P_F32 ? 8 : t.kind == P_BF16_MASTER ? 10 : 4) + (t.grad_bf16 ? 2 : 4) +
                      (t.bits == 8 ? 4 : 16));
  }
  h->groups = traffic < LIGHT * elements ? GROUPS_LIGHT : GROUPS;
  const size_t at_ticket = MOST_PARTS * sizeof(double), at_tensors = at_ticket + (1 + COUNTERS) * TICKET_STEP * 4;
  const size_t at_chunks = at_tensors + host.size() * sizeof(Tensor);
  const size_t bytes = at_chunks + chunks.size() * sizeof(Chunk);
  hipError_t e = hipGetDevice(&h->device);
  if (e == hipSuccess) e = hipMalloc(&h->memory, bytes);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete h;
    return bad(e == hipErrorOutOfMemory ? STAGE_ENOMEM : STAGE_EHIP, "adamw_init: %s", hipGetErrorString(e));
  }
  char* base = (char*)h->memory;
  h->parts = (double*)base;
  h->ticket = (unsigned*)(base + at_ticket);
  h->tensors = (Tensor*)(base + at_tensors);
  h->chunks = (Chunk*)(base + at_chunks);
  e = hipMemset(base, 0, at_tensors);
  if (e == hipSuccess)
    e = hipMemcpy(h->tensors, host.data(), host.size() * sizeof(Tensor), hipMemcpyHostToDevice);
  if (e == hipSuccess)
    e = hipMemcpy(h->chunks, chunks.data(), chunks.size() * sizeof(Chunk), hipMemcpyHostToDevice);
  if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    (void)hipFree(h->memory);
    delete h;
    return bad(STAGE_EHIP, "adamw_init: %s", hipGetErrorString(e));
  }
  *out = h;
  return STAGE_OK;
} catch (const std::bad_alloc&) {
  return bad(STAGE_ENOMEM, "adamw_init: out of host memory");
}

stage_status adamw_step(adamw_t* h, const adamw_args* a, void* hip_stream) {
  if (!h || !a) return bad(STAGE_EINVAL, "null handle or arguments");
  if (!(a->beta1 >= 0.0 && a->beta1 < 1.0 && a->beta2 >= 0.0 && a->beta2 < 1.0))
    return bad(STAGE_EINVAL, "betas must be at least 0 and below 1");
  if (!(a->eps >= 1e-30f && std::isfinite(a->eps))) return bad(STAGE_EINVAL, "eps must be finite, 1e-30 or more");
  if (!(a->max_norm >= 0.0f && std::isfinite(a->max_norm)))
    return bad(STAGE_EINVAL, "max_norm must be finite and not negative");
  if (!a->lr_ptr && !std::isfinite(a->lr)) return bad(STAGE_EINVAL, "lr must be finite");
  if (a->norm && a->max_norm == 0.0f) return bad(STAGE_EINVAL, "norm without max_norm");
  if ((uintptr_t)a->norm % 4 || (uintptr_t)a->lr_ptr % 4) return bad(STAGE_EINVAL, "norm or lr_ptr is not aligned");
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess || device != h->device)
    return bad(STAGE_EINVAL, "the handle is of device %d, the current one is %d", h->device, device);
  const hipStream_t st = (hipStream_t)hip_stream;
  StepArgs k{};
  k.tensors = (TensorTable)h->tensors;
  k.chunks = (ChunkTable)h->chunks;
  k.n_chunks = h->n_chunks;
  k.steps = h->steps;
  k.ticket = h->ticket;
  k.max_norm = a->max_norm;
  k.norm = a->norm;
  k.lr = a->lr;
  k.lr_ptr = a->lr_ptr;
  k.beta1 = a->beta1;
  k.beta2 = a->beta2;
  k.eps = a->eps;
  if (a->max_norm > 0.0f) {
    k.parts = h->parts;
    k.n_parts = std::max(1, std::min(MOST_PARTS, h->n_chunks));
    hipLaunchKernelGGL(norm_kernel, dim3(k.n_parts), dim3(THREADS), 0, st, k, h->parts);
  }
  hipLaunchKernelGGL(step_kernel, dim3(std::max(1, std::min(h->groups, h->n_chunks))), dim3(THREADS), 0, st, k);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return bad(STAGE_EHIP, "adamw_step: %s", hipGetErrorString(e));
  return STAGE_OK;
}

void adamw_destroy(adamw_t* h) {
  if (!h) return;
  (void)hipFree(h->memory);
  delete h;
}

}  // extern "C"
