// AdamW of many tensors at once (include/adamw.h): the kernels, and the handle of the C ABI.
//
// An element is read once and written once with its states, 28 bytes with fp32 states, 18 with
// 8-bit ones (and a master copy): HBM bounds it.  All tensors are one launch: they are cut
// into chunks of 2048 elements, whose table lies on the device, and work-groups take every
// gridDim-th one.
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
constexpr int MOST_GROUPS = 2048;   // work-groups: 8 to a CU
constexpr int MOST_PARTS = 1024;    // work-groups of the norm

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
struct StepArgs {
  const Tensor* tensors;
  const Chunk* chunks;
  int n_chunks;
  int64_t* steps;
  unsigned* ticket;     // 0 between launches
  const double* parts;  // sums of squares, or NULL: no clipping
  int n_parts;
  float max_norm;
  float* norm;
  float lr;
  const float* lr_ptr;
  double beta1, beta2;
  float eps;
};

// Eight elements, element-aligned 16-byte accesses; n >= 8 of them, or the first n.
__device__ __forceinline__ void load8(const float* p, int64_t n, float v[8]) {
  typedef f32x4_t __attribute__((aligned(4))) any_t;
  if (n >= 8) {
    const f32x4_t a = *(const any_t*)p, b = *(const any_t*)(p + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? p[k] : 0.0f;
  }
}
__device__ __forceinline__ void load8(const bf16_t* p, int64_t n, float v[8]) {
  typedef u32x4_t __attribute__((aligned(2))) any_t;
  if (n >= 8) {
    const u32x4_t a = *(const any_t*)p;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(a[k] << 16);
      v[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? bf2f(p[k]) : 0.0f;
  }
}
__device__ __forceinline__ void store8(float* p, int64_t n, const float v[8]) {
  typedef f32x4_t __attribute__((aligned(4))) any_t;
  if (n >= 8) {
    *(any_t*)p = f32x4_t{v[0], v[1], v[2], v[3]};
    *(any_t*)(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = v[k];
  }
}
__device__ __forceinline__ void store8(bf16_t* p, int64_t n, const bf16_t v[8]) {
  typedef u32x4_t __attribute__((aligned(2))) any_t;
  if (n >= 8) {
    u32x4_t r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = v[2 * k] | (uint32_t)v[2 * k + 1] << 16;
    *(any_t*)p = r;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = v[k];
  }
}
__device__ __forceinline__ void load8(const uint8_t* p, int64_t n, uint8_t v[8]) {
  typedef u32x2_t __attribute__((aligned(1))) any_t;
  if (n >= 8) {
    const u32x2_t a = *(const any_t*)p;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (uint8_t)(a[k >> 2] >> (8 * (k & 3)));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? p[k] : 0;
  }
}
__device__ __forceinline__ void store8(uint8_t* p, int64_t n, const uint32_t v[8]) {
  typedef u32x2_t __attribute__((aligned(1))) any_t;
  if (n >= 8) {
    u32x2_t r;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      r[k] = v[4 * k] | v[4 * k + 1] << 8 | v[4 * k + 2] << 16 | v[4 * k + 3] << 24;
    *(any_t*)p = r;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = (uint8_t)v[k];
  }
}

// e4m3 and e5m2 codes (no infinities or NaNs among them: codes stay below) by their bits: a
// normal one is a float's exponent and leading mantissa bits, a subnormal one counts
// 2^-9 or 2^-16.
__device__ __forceinline__ float from_e4m3(uint32_t c) {
  const uint32_t a = c & 0x7f;
  const float f = a < 8 ? (float)a * 0x1p-9f : __uint_as_float((a + (120 << 3)) << 20);
  return c & 0x80 ? -f : f;
}
__device__ __forceinline__ float from_e5m2(uint32_t c) {
  return c < 4 ? (float)c * 0x1p-16f : __uint_as_float((c + (112 << 2)) << 21);
}
// The code of |x| <= 448 (x times a block's scale): up where its part beyond the last bit and
// r / 2^16 come to a step.
__device__ __forceinline__ uint32_t to_e4m3(float x, uint32_t r) {
  const float a = fabsf(x);
  const uint32_t c = a < 0x1p-6f ? ((uint32_t)(a * 0x1p25f) + r) >> 16
                                 : ((__float_as_uint(a) + (r << 4)) >> 20) - (120 << 3);
  return min(c, 0x7eu) | (__float_as_uint(x) >> 31 << 7);
}
// The same for 0 <= x <= 57344; x > 0 has a code above 0.
__device__ __forceinline__ uint32_t to_e5m2(float x, uint32_t r) {
  const uint32_t c = x < 0x1p-14f ? ((uint32_t)(x * 0x1p32f) + r) >> 16
                                  : ((__float_as_uint(x) + (r << 5)) >> 21) - (112 << 2);
  return min(max(c, x > 0.0f ? 1u : 0u), 0x7bu);
}
// A block's scale and its inverse from the bits of its largest |value| (NaN above all): 0 for
// values too small for the inverse, NaN where one is not finite.
__device__ __forceinline__ float2 scale_of(uint32_t top, float most) {
  const float f = __uint_as_float(top);
  if (top >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.0f};
  if (f < 0x1p-110f) return {0.0f, 0.0f};
  return {f / most, most / f};
}
__device__ __forceinline__ uint32_t max32(uint32_t v) {  // over 32 lanes
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
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
  uint32_t t;
};

// Eight elements from i of a tensor.
template <int KIND, bool GRAD_BF16, int BITS>
__device__ __forceinline__ void update8(const Tensor& x, int64_t i, const Step& s) {
  // (the states' operations are rounded one by one, as they are defined)
#pragma clang fp contract(off)
  const int64_t n = x.n - i;
  float w[8], g[8], m[8], v[8];
  if constexpr (KIND == P_F32) load8((const float*)x.p + i, n, w);
  else if constexpr (KIND == P_BF16_MASTER) load8(x.master + i, n, w);
  else load8((const bf16_t*)x.p + i, n, w);
  if constexpr (GRAD_BF16) load8((const bf16_t*)x.g + i, n, g);
  else load8((const float*)x.g + i, n, g);
  const int64_t block = i / ADAMW_BLOCK;
  if constexpr (BITS == 8) {
    uint8_t cm[8], cv[8];
    load8((const uint8_t*)x.m + i, n, cm);
    load8((const uint8_t*)x.v + i, n, cv);
    const float sm = n > 0 ? x.m_scale[block] : 0.0f, sv = n > 0 ? x.v_scale[block] : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = from_e4m3(cm[k]) * sm, v[k] = from_e5m2(cv[k]) * sv;
  } else {
    load8((const float*)x.m + i, n, m);
    load8((const float*)x.v + i, n, v);
  }
  const float keep = 1.0f - s.lr * x.lr_scale * x.decay, rate = s.lr_bias * x.lr_scale;
  uint32_t top_m = 0, top_v = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float d = g[k] * s.clip;
    m[k] = m[k] * s.b1 + d * s.c1;
    v[k] = v[k] * s.b2 + d * d * s.c2;
    // (square root and reciprocal of 1 ulp: a change of w, not w, is off by that)
    const float den = __builtin_amdgcn_sqrtf(v[k]) * s.inv_root + s.eps;
    w[k] = w[k] * keep - rate * m[k] * __builtin_amdgcn_rcpf(den);
    top_m = max(top_m, __float_as_uint(m[k]) & 0x7fffffffu);
    top_v = max(top_v, __float_as_uint(v[k]) & 0x7fffffffu);
  }
  uint32_t r[8];
  if constexpr (BITS == 8 || KIND == P_BF16)
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = random_bits((uint32_t)i + k, s.t);
  if constexpr (KIND == P_F32) {
    store8((float*)x.p + i, n, w);
  } else {
    bf16_t b[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      b[k] = KIND == P_BF16 ? (bf16_t)((__float_as_uint(w[k]) + (r[k] >> 16)) >> 16) : f2bf(w[k]);
    store8((bf16_t*)x.p + i, n, b);
    if constexpr (KIND == P_BF16_MASTER) store8(x.master + i, n, w);
  }
  if constexpr (BITS == 8) {
    const float2 sm = scale_of(max32(top_m), 448.0f), sv = scale_of(max32(top_v), 57344.0f);
    uint32_t cm[8], cv[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      cm[k] = sm.y == 0.0f ? 0 : to_e4m3(m[k] * sm.y, r[k] & 0xffff);
      cv[k] = sv.y == 0.0f ? 0 : to_e5m2(v[k] * sv.y, r[k] >> 16);
    }
    store8((uint8_t*)x.m + i, n, cm);
    store8((uint8_t*)x.v + i, n, cv);
    if ((threadIdx.x & 31) == 0 && n > 0) {
      x.m_scale[block] = sm.x;
      x.v_scale[block] = sv.x;
    }
  } else {
    store8((float*)x.m + i, n, m);
    store8((float*)x.v + i, n, v);
  }
}

template <int KIND, bool GRAD_BF16>
__device__ __forceinline__ void update_bits(const Tensor& x, int64_t i, const Step& s) {
  if (x.bits == 8) update8<KIND, GRAD_BF16, 8>(x, i, s);
  else update8<KIND, GRAD_BF16, 32>(x, i, s);
}
template <int KIND>
__device__ __forceinline__ void update_grad(const Tensor& x, int64_t i, const Step& s) {
  if (x.grad_bf16) update_bits<KIND, true>(x, i, s);
  else update_bits<KIND, false>(x, i, s);
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

__global__ __launch_bounds__(THREADS) void step_kernel(const StepArgs a) {
  __shared__ double lds[THREADS / 64];
  __shared__ int64_t steps;
  if (threadIdx.x == 0) steps = *a.steps;
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
  } else {
    __syncthreads();
  }
  // Every work-group reads the number of steps before it takes a ticket, so the one with the
  // last ticket may raise it.
  const int64_t t = steps + 1;
  if (threadIdx.x == 0 && atomicAdd(a.ticket, 1u) == gridDim.x - 1) {
    if (go) *a.steps = t;
    *a.ticket = 0;
  }
  if (!go) return;
  const float lr = a.lr_ptr ? *a.lr_ptr : a.lr;
  s.b1 = (float)a.beta1;
  s.c1 = (float)(1.0 - a.beta1);
  s.b2 = (float)a.beta2;
  s.c2 = (float)(1.0 - a.beta2);
  s.lr = lr;
  s.lr_bias = (float)(lr / (1.0 - power(a.beta1, t)));
  s.inv_root = (float)(1.0 / sqrt(1.0 - power(a.beta2, t)));
  s.eps = a.eps;
  s.t = (uint32_t)t;
  for (int c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
    const Chunk ch = a.chunks[c];
    const Tensor& x = a.tensors[ch.tensor];
    const int64_t i = (int64_t)ch.index * CHUNK + 8 * threadIdx.x;
    if (x.kind == P_F32) update_grad<P_F32>(x, i, s);
    else if (x.kind == P_BF16_MASTER) update_grad<P_BF16_MASTER>(x, i, s);
    else update_grad<P_BF16>(x, i, s);
  }
}

// Sums of squares of the gradients, a work-group's chunks together, in 64 bits (squares of
// fp32 values neither overflow there nor vanish).
__global__ __launch_bounds__(THREADS) void norm_kernel(const StepArgs a, double* parts) {
  __shared__ double lds[THREADS / 64];
  double sum = 0.0;
  for (int c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
    const Chunk ch = a.chunks[c];
    const Tensor& x = a.tensors[ch.tensor];
    const int64_t i = (int64_t)ch.index * CHUNK + 8 * threadIdx.x;
    float g[8];
    if (x.grad_bf16) load8((const bf16_t*)x.g + i, x.n - i, g);
    else load8((const float*)x.g + i, x.n - i, g);
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
  adamw_t* h = new adamw_t;
  h->steps = steps;
  h->n_chunks = (int)chunks.size();
  const size_t at_ticket = MOST_PARTS * sizeof(double), at_tensors = at_ticket + 64;
  const size_t at_chunks = at_tensors + (size_t)n * sizeof(Tensor);
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
  if (e == hipSuccess && n > 0) e = hipMemcpy(h->tensors, host.data(), n * sizeof(Tensor), hipMemcpyHostToDevice);
  if (e == hipSuccess && !chunks.empty())
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
  k.tensors = h->tensors;
  k.chunks = h->chunks;
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
  hipLaunchKernelGGL(step_kernel, dim3(std::max(1, std::min(MOST_GROUPS, h->n_chunks))), dim3(THREADS), 0, st, k);
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
