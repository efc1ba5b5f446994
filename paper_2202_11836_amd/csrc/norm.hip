// Layer norm as an operator of its own (include/norm.h): forward with an optional residual
// addition, backward with the sums of the weights' gradients; plan and argument checks of
// the C ABI.
//
// A few operations a value, so HBM bounds it.  A row stays in the registers of its TPR
// threads (8 to 1024 of them by its width) from its one read to its one write: forward reads
// x (and the residual) and writes out (and the sum), backward reads dy, z and dtotal and
// writes dx, while every thread adds up dy xh and dy of its columns over the rows of its
// work-group, which leaves one partial row a work-group to a second launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/norm.h"
#include "common.h"

namespace {

struct Rows {  // an operand: its memory, strides of batch and position
  void* p;
  int64_t sb, ss;
};
struct FwdArgs {
  Rows x, res, total, out;
  const float *gamma, *beta;
  float *mean, *rstd;
  int rows, seq, batch, w;  // (batch 1: rows = seq)
  float eps;
};
struct BwdArgs {
  Rows dy, z, dtotal, dx;
  const float *gamma, *mean, *rstd;
  float *part, *dgamma, *dbeta;  // part [work-groups][2][w]
  int rows, seq, batch, w, rpb;  // rpb: rows of a work-group
};

// Eight values of a row in their storage type; element-aligned 16-byte accesses (rows of
// any width lie at any element).
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
  typedef u32x4_t __attribute__((aligned(2))) any_t;
  u32x4_t r;
  __device__ __forceinline__ void zero() { r = u32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const bf16_t* p) { r = *(const any_t*)p; }
  __device__ __forceinline__ void load_part(const bf16_t* p, int n) {
    uint32_t v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? p[k] : 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = v[2 * k] | v[2 * k + 1] << 16;
  }
  __device__ __forceinline__ float get(int k) const {
    return __uint_as_float(k & 1 ? r[k >> 1] & 0xffff0000u : r[k >> 1] << 16);
  }
  __device__ __forceinline__ void set(const float v[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
  }
  __device__ __forceinline__ void store(bf16_t* p) const { *(any_t*)p = r; }
  __device__ __forceinline__ void store_part(bf16_t* p, int n) const {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = (bf16_t)(r[k >> 1] >> (16 * (k & 1)));
  }
};
template <> struct Chunk<float> {
  typedef f32x4_t __attribute__((aligned(4))) any_t;
  f32x4_t a, b;
  __device__ __forceinline__ void zero() { a = b = f32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const float* p) {
    a = *(const any_t*)p;
    b = *(const any_t*)(p + 4);
  }
  __device__ __forceinline__ void load_part(const float* p, int n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      a[k] = k < n ? p[k] : 0.0f;
      b[k] = 4 + k < n ? p[4 + k] : 0.0f;
    }
  }
  __device__ __forceinline__ float get(int k) const { return k < 4 ? a[k & 3] : b[k & 3]; }
  __device__ __forceinline__ void set(const float v[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = v[k], b[k] = v[4 + k];
  }
  __device__ __forceinline__ void store(float* p) const {
    *(any_t*)p = a;
    *(any_t*)(p + 4) = b;
  }
  __device__ __forceinline__ void store_part(float* p, int n) const {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = get(k);
  }
};
// n of the eight (<= 0: none).
template <typename T>
__device__ __forceinline__ void load_n(Chunk<T>& c, const T* p, int n) {
  if (n >= 8) c.load(p);
  else if (n > 0) c.load_part(p, n);
  else c.zero();
}
template <typename T>
__device__ __forceinline__ void store_n(const Chunk<T>& c, T* p, int n) {
  if (n >= 8) c.store(p);
  else if (n > 0) c.store_part(p, n);
}
// eight weights (absent: all `none`)
__device__ __forceinline__ void weights(const float* w, int at, int n, float none, float v[8]) {
  Chunk<float> c;
  if (!w) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = none;
    return;
  }
  load_n(c, w + at, n);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = c.get(k);
}

template <typename T>
__device__ __forceinline__ T* row_at(const Rows& r, int batch, int seq, int row) {
  if (batch == 1) return (T*)r.p + (int64_t)row * r.ss;
  const int b = row / seq;
  return (T*)r.p + b * r.sb + (int64_t)(row - b * seq) * r.ss;
}

// Sums over the TPR threads of a row, N of them together.  Up to 64 threads: lanes of a
// wavefront.  More: its wavefronts meet in LDS, twice buffered by `turn` (one barrier a sum).
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float v[N], float* lds, int turn) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = (TPR < 64 ? TPR : 64) / 2; o > 0; o >>= 1) v[i] += __shfl_xor(v[i], o, 64);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float* at = lds + turn * N * W;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) at[i * W + (threadIdx.x >> 6)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = at[i * W];
#pragma unroll
      for (int j = 1; j < W; ++j) t += at[i * W + j];
      v[i] = t;
    }
  }
}

// A row a TPR threads, NC chunks of eight values each: thread j owns chunks j + TPR i.
template <typename T, int TPR, int NC, bool RES>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void fwd_kernel(const FwdArgs g) {
  __shared__ float lds[TPR > 64 ? 2 * (TPR / 64) : 1];
  constexpr int RPB = TPR > 256 ? 1 : 256 / TPR;
  const int lane = threadIdx.x % TPR;
  const int row = blockIdx.x * RPB + threadIdx.x / TPR;
  if (TPR <= 64 && row >= g.rows) return;  // (work-groups of whole rows have no other)
  const T* x = row_at<T>(g.x, g.batch, g.seq, row);
  Chunk<T> c[NC], r[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) load_n(c[i], x + 8 * (lane + TPR * i), g.w - 8 * (lane + TPR * i));
  if constexpr (RES) {
    const T* res = row_at<T>(g.res, g.batch, g.seq, row);
#pragma unroll
    for (int i = 0; i < NC; ++i) load_n(r[i], res + 8 * (lane + TPR * i), g.w - 8 * (lane + TPR * i));
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = c[i].get(k) + r[i].get(k);
      c[i].set(v);  // (what follows sees the sum as it is stored)
    }
    if (g.total.p) {
      T* t = row_at<T>(g.total, g.batch, g.seq, row);
#pragma unroll
      for (int i = 0; i < NC; ++i) store_n(c[i], t + 8 * (lane + TPR * i), g.w - 8 * (lane + TPR * i));
    }
  }
  float s[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) s[0] += c[i].get(k);
  row_sums<TPR, 1>(s, lds, 0);
  const float mean = s[0] / (float)g.w;
  s[0] = 0.0f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int n = g.w - 8 * (lane + TPR * i);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float d = k < n ? c[i].get(k) - mean : 0.0f;
      s[0] += d * d;
    }
  }
  row_sums<TPR, 1>(s, lds, 1);
  const float rstd = 1.0f / sqrtf(s[0] / (float)g.w + g.eps);
  T* out = row_at<T>(g.out, g.batch, g.seq, row);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int at = 8 * (lane + TPR * i), n = g.w - at;
    float ga[8], be[8], v[8];
    weights(g.gamma, at, n, 1.0f, ga);
    weights(g.beta, at, n, 0.0f, be);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = fmaf((c[i].get(k) - mean) * rstd, ga[k], be[k]);
    c[i].set(v);
    store_n(c[i], out + at, n);
  }
  if (lane == 0) {
    if (g.mean) g.mean[row] = mean;
    if (g.rstd) g.rstd[row] = rstd;
  }
}

// U rows of a TPR threads at a time, so that the loads of all are on their way together.
template <typename T, int TPR, int NC, int U, bool GRADS>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void bwd_kernel(const BwdArgs g) {
  constexpr int THREADS = TPR > 256 ? TPR : 256;
  constexpr int SLOTS = THREADS / TPR;  // rows side by side
  constexpr int WAVES = THREADS / 64;
  __shared__ float lds[TPR > 64 ? 4 * U * (TPR / 64) : 1];
  const int lane = threadIdx.x % TPR, slot = threadIdx.x / TPR;
  const int r0 = blockIdx.x * g.rpb, r1 = min(g.rows, r0 + g.rpb);
  const float inv_w = 1.0f / (float)g.w;
  // (rows of 1024 threads have 128 registers a thread: gamma is read again for each row)
  constexpr bool KEEP = TPR <= 256;
  float gm[NC][8], pg[GRADS ? NC : 1][8], pb[GRADS ? NC : 1][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int at = 8 * (lane + TPR * i);
    if constexpr (KEEP) weights(g.gamma, at, g.w - at, 1.0f, gm[i]);
    if constexpr (GRADS)
#pragma unroll
      for (int k = 0; k < 8; ++k) pg[i][k] = pb[i][k] = 0.0f;
  }
  int turn = 0;
  // (the same number of passes for all wavefronts of a row)
  for (int first = r0; first < r1; first += SLOTS * U) {
    Chunk<T> dy[U][NC], z[U][NC], dt[U][NC];
    float mean[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = first + slot + SLOTS * u;
      const bool live = row < r1;
      const T* pd = live ? row_at<T>(g.dy, g.batch, g.seq, row) : nullptr;
      const T* pz = live ? row_at<T>(g.z, g.batch, g.seq, row) : nullptr;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = 8 * (lane + TPR * i), n = live ? g.w - at : 0;
        load_n(dy[u][i], pd + at, n);
        load_n(z[u][i], pz + at, n);
      }
      if (g.dtotal.p) {
        const T* pt = live ? row_at<T>(g.dtotal, g.batch, g.seq, row) : nullptr;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int at = 8 * (lane + TPR * i);
          load_n(dt[u][i], pt + at, live ? g.w - at : 0);
        }
      }
      mean[u] = live ? g.mean[row] : 0.0f;
      rstd[u] = live ? g.rstd[row] : 0.0f;
    }
    float s[2 * U];
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) s[u] = 0.0f;
    // (behind a row's end dy is 0, and so is all that comes of it)
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = 8 * (lane + TPR * i);
        if constexpr (!KEEP) weights(g.gamma, at, g.w - at, 1.0f, gm[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float d = dy[u][i].get(k), xh = (z[u][i].get(k) - mean[u]) * rstd[u];
          const float dg = d * gm[i][k];
          s[2 * u] += dg;
          s[2 * u + 1] += dg * xh;
          if constexpr (GRADS) {
            pg[i][k] += d * xh;
            pb[i][k] += d;
          }
        }
      }
    if (g.dx.p) {
      row_sums<TPR, 2 * U>(s, lds, turn);
      turn ^= 1;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = first + slot + SLOTS * u;
        if (row >= r1) continue;
        T* px = row_at<T>(g.dx, g.batch, g.seq, row);
        const float a = s[2 * u] * inv_w, b = s[2 * u + 1] * inv_w;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int at = 8 * (lane + TPR * i);
          float v[8];
          if constexpr (!KEEP) weights(g.gamma, at, g.w - at, 1.0f, gm[i]);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float xh = (z[u][i].get(k) - mean[u]) * rstd[u];
            v[k] = rstd[u] * (dy[u][i].get(k) * gm[i][k] - a - xh * b);
            if (g.dtotal.p) v[k] += dt[u][i].get(k);
          }
          dy[u][i].set(v);
          store_n(dy[u][i], px + at, g.w - at);
        }
      }
    }
  }
  if constexpr (GRADS) {
    // The work-group's rows side by side: lanes of a wavefront first, then wavefronts in order.
    extern __shared__ float red[];  // TPR <= 64: [wavefront][2][w]
    float* to = gridDim.x == 1 && g.dgamma ? nullptr : g.part + (int64_t)blockIdx.x * 2 * g.w;
    if constexpr (TPR < 64) {
#pragma unroll
      for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int o = TPR; o < 64; o <<= 1) {
            pg[i][k] += __shfl_xor(pg[i][k], o, 64);
            pb[i][k] += __shfl_xor(pb[i][k], o, 64);
          }
    }
    if constexpr (TPR <= 64) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) < TPR) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int at = 8 * (lane + TPR * i) + k;
            if (at < g.w) {
              red[wave * 2 * g.w + at] = pg[i][k];
              red[wave * 2 * g.w + g.w + at] = pb[i][k];
            }
          }
      }
      __syncthreads();
      for (int e = threadIdx.x; e < 2 * g.w; e += THREADS) {
        float t = red[e];
#pragma unroll
        for (int j = 1; j < WAVES; ++j) t += red[j * 2 * g.w + e];
        if (to) to[e] = t;
        else if (e < g.w) g.dgamma[e] = t;
        else if (g.dbeta) g.dbeta[e - g.w] = t;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = 8 * (lane + TPR * i), n = g.w - at;
        Chunk<float> c;
        float* dg = to ? to : g.dgamma;
        float* db = to ? to + g.w : g.dbeta;
        c.set(pg[i]);
        store_n(c, dg + at, n);
        c.set(pb[i]);
        if (db) store_n(c, db + at, n);
      }
    }
  }
}

// dgamma and dbeta: the sums over the work-groups' partial rows, `parts` of them, in order within
// each of a work-group's 16 stripes, then over the stripes.
constexpr int RED_COLS = 64;
__global__ __launch_bounds__(1024) void reduce_kernel(const float* __restrict__ part, int parts, int w,
                                                      float* dgamma, float* dbeta) {
  __shared__ float lds[16][RED_COLS];
  const int col = blockIdx.x * RED_COLS + (threadIdx.x & 63), stripe = threadIdx.x >> 6;
  float t = 0.0f;
  if (col < 2 * w) {
    const float* p = part + col;
    const int64_t step = (int64_t)2 * w;
    int b = stripe;
    for (; b + 16 * 7 < parts; b += 16 * 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = p[(b + 16 * j) * step];
#pragma unroll
      for (int j = 0; j < 8; ++j) t += v[j];
    }
    for (; b < parts; b += 16) t += p[b * step];
  }
  lds[stripe][threadIdx.x & 63] = t;
  __syncthreads();
  if (stripe == 0 && col < 2 * w) {
    for (int j = 1; j < 16; ++j) t += lds[j][threadIdx.x];
    if (col < w) {
      if (dgamma) dgamma[col] = t;
    } else if (dbeta) {
      dbeta[col - w] = t;
    }
  }
}

__global__ void zero_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  if (a) a[i] = 0.0f;
  if (b) b[i] = 0.0f;
}

// ---------------------------------------------------------------------------
// Plan
// ---------------------------------------------------------------------------
// Threads of a row: a wavefront or less while its rows fit (no barriers), then 256 and 1024,
// with at most four chunks of eight values a thread; backward, which holds dy, z, gamma and
// both sums, two.
int fwd_threads(int w) {
  return w <= 64 ? 8 : w <= 128 ? 16 : w <= 256 ? 32 : w <= 2048 ? 64 : w <= 8192 ? 256 : 1024;
}
int bwd_threads(int w) {
  return w <= 64 ? 8 : w <= 128 ? 16 : w <= 256 ? 32 : w <= 1024 ? 64 : w <= 4096 ? 256 : 1024;
}
// Rows of a work-group at a time (rows side by side times U of bwd_kernel).
int bwd_rows(int w) {
  const int t = bwd_threads(w);
  return t > 256 ? 1 : 2 * (256 / t);
}
struct BwdPlan {
  int blocks, rpb;
};
BwdPlan bwd_plan(int rows, int w) {
  const int step = bwd_rows(w);
  const int most = w <= 4096 ? 512 : 256;
  int blocks = std::min(most, (rows + step - 1) / step);
  const int rpb = ((rows + blocks - 1) / blocks + step - 1) / step * step;
  return {(rows + rpb - 1) / rpb, rpb};
}

template <typename T, int TPR, int NC>
void launch_fwd(const FwdArgs& g, hipStream_t st) {
  constexpr int RPB = TPR > 256 ? 1 : 256 / TPR;
  const dim3 grid((unsigned)((g.rows + RPB - 1) / RPB)), block(TPR > 256 ? TPR : 256);
  if (g.res.p) hipLaunchKernelGGL((fwd_kernel<T, TPR, NC, true>), grid, block, 0, st, g);
  else hipLaunchKernelGGL((fwd_kernel<T, TPR, NC, false>), grid, block, 0, st, g);
}
template <typename T>
void forward(const FwdArgs& g, hipStream_t st) {
  const int w = g.w;
  if (w <= 64) launch_fwd<T, 8, 1>(g, st);
  else if (w <= 128) launch_fwd<T, 16, 1>(g, st);
  else if (w <= 256) launch_fwd<T, 32, 1>(g, st);
  else if (w <= 512) launch_fwd<T, 64, 1>(g, st);
  else if (w <= 1024) launch_fwd<T, 64, 2>(g, st);
  else if (w <= 2048) launch_fwd<T, 64, 4>(g, st);
  else if (w <= 4096) launch_fwd<T, 256, 2>(g, st);
  else if (w <= 8192) launch_fwd<T, 256, 4>(g, st);
  else launch_fwd<T, 1024, 2>(g, st);
}

template <typename T, int TPR, int NC>
void launch_bwd(const BwdArgs& g, int blocks, hipStream_t st) {
  constexpr int U = TPR > 256 ? 1 : 2;
  const dim3 grid((unsigned)blocks), block(TPR > 256 ? TPR : 256);
  const size_t lds = TPR <= 64 ? (size_t)4 * 2 * g.w * 4 : 0;
  if (g.dgamma || g.dbeta) hipLaunchKernelGGL((bwd_kernel<T, TPR, NC, U, true>), grid, block, lds, st, g);
  else hipLaunchKernelGGL((bwd_kernel<T, TPR, NC, U, false>), grid, block, 0, st, g);
}
template <typename T>
void backward(const BwdArgs& g, int blocks, hipStream_t st) {
  const int w = g.w;
  if (w <= 64) launch_bwd<T, 8, 1>(g, blocks, st);
  else if (w <= 128) launch_bwd<T, 16, 1>(g, blocks, st);
  else if (w <= 256) launch_bwd<T, 32, 1>(g, blocks, st);
  else if (w <= 512) launch_bwd<T, 64, 1>(g, blocks, st);
  else if (w <= 1024) launch_bwd<T, 64, 2>(g, blocks, st);
  else if (w <= 2048) launch_bwd<T, 256, 1>(g, blocks, st);
  else if (w <= 4096) launch_bwd<T, 256, 2>(g, blocks, st);
  else if (w <= 8192) launch_bwd<T, 1024, 1>(g, blocks, st);
  else launch_bwd<T, 1024, 2>(g, blocks, st);
}

// ---------------------------------------------------------------------------
// Argument checks
// ---------------------------------------------------------------------------
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

stage_status check_shape(const layer_norm_shape* s) {
  if (!s) return bad(STAGE_EINVAL, "null shape");
  if (s->dtype != STAGE_F32 && s->dtype != STAGE_BF16) return bad(STAGE_EINVAL, "unknown dtype");
  if (s->batch < 0 || s->seq < 0) return bad(STAGE_EINVAL, "negative batch or length");
  if (s->width < 1 || s->width > LAYER_NORM_MAX_WIDTH)
    return bad(STAGE_EINVAL, "width must be 1 .. %d", LAYER_NORM_MAX_WIDTH);
  // A launch holds fewer than 2^32 threads.
  if ((int64_t)s->batch * s->seq > 4294967040LL / fwd_threads(s->width))
    return bad(STAGE_EINVAL, "batch * seq too large");
  return STAGE_OK;
}

// One operand; strides of dimensions of one or no element are not looked at.
stage_status check_rows(const char* name, const layer_norm_shape* s, const void* p, const int64_t* given,
                        bool output, Rows* r) {
  const int64_t size[2] = {s->batch, s->seq};
  int64_t st[2];
  r->p = const_cast<void*>(p);
  for (int i = 0; i < 2; ++i) st[i] = size[i] > 1 ? given[i] : 0;
  r->sb = st[0];
  r->ss = st[1];
  if (size[0] == 0 || size[1] == 0) return STAGE_OK;
  if (!p) return bad(STAGE_EINVAL, "null %s", name);
  if ((uintptr_t)p % (s->dtype == STAGE_BF16 ? 2 : 4)) return bad(STAGE_EINVAL, "%s is not aligned", name);
  for (int i = 0; i < 2; ++i) {
    if (st[i] < 0) return bad(STAGE_EINVAL, "%s has a negative stride", name);
    if (size[i] > 1 && st[i] > ((int64_t)1 << 53) / size[i])
      return bad(STAGE_EINVAL, "%s spans more than 2^53 elements", name);
  }
  if (output) {
    const int in = size[0] > 1 && size[1] > 1 && st[0] < st[1] ? 0 : size[1] > 1 ? 1 : 0;
    const int64_t span = s->width + (size[in] > 1 ? st[in] * (size[in] - 1) : 0);
    if ((size[in] > 1 && st[in] < s->width) || (size[1 - in] > 1 && st[1 - in] < span))
      return bad(STAGE_EINVAL, "%s overlaps itself", name);
  }
  return STAGE_OK;
}

// An output over an input of the same memory needs its strides.
stage_status check_same(const char* a, const Rows& out, const char* b, const Rows& in) {
  if (out.p && out.p == in.p && (out.sb != in.sb || out.ss != in.ss))
    return bad(STAGE_EINVAL, "%s over %s needs the same strides", a, b);
  return STAGE_OK;
}

// Whether the rows of all operands lie as those of one sequence.
bool flat(const layer_norm_shape* s, const Rows* const* r, int n) {
  if (s->batch == 1) return true;
  for (int i = 0; i < n; ++i) {
    if (!r[i]->p) continue;
    if (s->seq > 1 ? r[i]->sb != s->seq * r[i]->ss : false) return false;
  }
  return true;
}
// (of sequences of one row each, the batch's stride is the rows')
void flatten(const layer_norm_shape* s, Rows* const* r, int n) {
  for (int i = 0; i < n; ++i)
    if (s->seq == 1) r[i]->ss = r[i]->sb;
}

}  // namespace

extern "C" {

const char* layer_norm_last_error(void) { return g_err; }

stage_status layer_norm_forward(const layer_norm_shape* s, const void* x, const void* residual,
                                const float* gamma, const float* beta, void* total, void* out,
                                float* mean, float* rstd, void* hip_stream) {
  CK(check_shape(s));
  if (!(s->eps >= 0.0f && std::isfinite(s->eps)))
    return bad(STAGE_EINVAL, "eps must be finite and not negative");
  if (total && !residual) return bad(STAGE_EINVAL, "total without a residual");
  FwdArgs g{};
  CK(check_rows("x", s, x, s->x, false, &g.x));
  if (residual) CK(check_rows("residual", s, residual, s->residual, false, &g.res));
  if (total) CK(check_rows("total", s, total, s->total, true, &g.total));
  CK(check_rows("out", s, out, s->out, true, &g.out));
  if ((uintptr_t)gamma % 4 || (uintptr_t)beta % 4 || (uintptr_t)mean % 4 || (uintptr_t)rstd % 4)
    return bad(STAGE_EINVAL, "gamma, beta, mean or rstd is not aligned");
  const int64_t rows = (int64_t)s->batch * s->seq;
  if (rows == 0) return STAGE_OK;
  if (total && total == out) return bad(STAGE_EINVAL, "total and out have the same memory");
  if (mean && mean == rstd) return bad(STAGE_EINVAL, "mean and rstd have the same memory");
  for (const void* o : {(const void*)total, (const void*)out, (const void*)mean, (const void*)rstd})
    if (o && (o == gamma || o == beta)) return bad(STAGE_EINVAL, "an output may not be written over that input");
  for (const void* o : {(const void*)mean, (const void*)rstd})
    if (o && (o == x || o == residual || o == total || o == out))
      return bad(STAGE_EINVAL, "mean and rstd may not be written over an input or another output");
  CK(check_same("out", g.out, "x", g.x));
  CK(check_same("out", g.out, "residual", g.res));
  CK(check_same("total", g.total, "x", g.x));
  CK(check_same("total", g.total, "residual", g.res));
  Rows* const all[4] = {&g.x, &g.res, &g.total, &g.out};
  const bool one = flat(s, all, 4);
  if (one) flatten(s, all, 4);
  g.gamma = gamma;
  g.beta = beta;
  g.mean = mean;
  g.rstd = rstd;
  g.rows = (int)rows;
  g.batch = one ? 1 : s->batch;
  g.seq = one ? g.rows : s->seq;
  g.w = s->width;
  g.eps = s->eps;
  if (s->dtype == STAGE_BF16) forward<bf16_t>(g, (hipStream_t)hip_stream);
  else forward<float>(g, (hipStream_t)hip_stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return bad(STAGE_EHIP, "layer_norm_forward: %s", hipGetErrorString(e));
  return STAGE_OK;
}

stage_status layer_norm_workspace(const layer_norm_shape* s, size_t* bytes) {
  if (!bytes) return bad(STAGE_EINVAL, "null bytes");
  CK(check_shape(s));
  const int64_t rows = (int64_t)s->batch * s->seq;
  *bytes = rows ? (size_t)bwd_plan((int)rows, s->width).blocks * 2 * s->width * 4 : 0;
  return STAGE_OK;
}

stage_status layer_norm_backward(const layer_norm_shape* s, const void* dy, const void* total,
                                 const float* gamma, const float* mean, const float* rstd,
                                 const void* dtotal, void* dx, float* dgamma, float* dbeta,
                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
  CK(check_shape(s));
  BwdArgs g{};
  CK(check_rows("dy", s, dy, s->dy, false, &g.dy));
  CK(check_rows("total", s, total, s->total, false, &g.z));
  if (dtotal) CK(check_rows("dtotal", s, dtotal, s->dtotal, false, &g.dtotal));
  if (dx) CK(check_rows("dx", s, dx, s->dx, true, &g.dx));
  if ((uintptr_t)gamma % 4 || (uintptr_t)mean % 4 || (uintptr_t)rstd % 4 || (uintptr_t)dgamma % 4 ||
      (uintptr_t)dbeta % 4)
    return bad(STAGE_EINVAL, "gamma, mean, rstd, dgamma or dbeta is not aligned");
  const int64_t rows = (int64_t)s->batch * s->seq;
  if (rows > 0 && (!mean || !rstd)) return bad(STAGE_EINVAL, "null mean or rstd");
  const hipStream_t st = (hipStream_t)hip_stream;
  const void* const outs[2] = {dgamma, dbeta};
  for (const void* o : outs)
    if (o && (o == gamma || (rows > 0 && (o == mean || o == rstd || o == dy || o == total || o == dtotal || o == dx))))
      return bad(STAGE_EINVAL, "a gradient may not be written over an input");
  if (dgamma && dgamma == dbeta) return bad(STAGE_EINVAL, "two gradients have the same memory");
  if (rows > 0 && dx && (dx == gamma || dx == mean || dx == rstd))
    return bad(STAGE_EINVAL, "a gradient may not be written over an input");
  if (rows == 0) {
    if (!dgamma && !dbeta) return STAGE_OK;
    hipLaunchKernelGGL(zero_kernel, dim3((s->width + 255) / 256), dim3(256), 0, st, dgamma, dbeta,
                       s->width);
  } else {
    CK(check_same("dx", g.dx, "dy", g.dy));
    CK(check_same("dx", g.dx, "total", g.z));
    CK(check_same("dx", g.dx, "dtotal", g.dtotal));
    const BwdPlan plan = bwd_plan((int)rows, s->width);
    const bool grads = dgamma || dbeta;
    if (grads) {
      const size_t need = (size_t)plan.blocks * 2 * s->width * 4;
      if (!workspace || workspace_bytes < need)
        return bad(STAGE_EINVAL, "the workspace holds %zu bytes of the %zu needed",
                   workspace ? workspace_bytes : 0, need);
      if ((uintptr_t)workspace % 16) return bad(STAGE_EINVAL, "the workspace is not 16-byte aligned");
    }
    if (!dx && !grads) return STAGE_OK;
    Rows* const all[4] = {&g.dy, &g.z, &g.dtotal, &g.dx};
    const bool one = flat(s, all, 4);
    if (one) flatten(s, all, 4);
    g.gamma = gamma;
    g.mean = mean;
    g.rstd = rstd;
    g.part = (float*)workspace;
    g.dgamma = dgamma;
    g.dbeta = dbeta;
    g.rows = (int)rows;
    g.batch = one ? 1 : s->batch;
    g.seq = one ? g.rows : s->seq;
    g.w = s->width;
    g.rpb = plan.rpb;
    if (s->dtype == STAGE_BF16) backward<bf16_t>(g, plan.blocks, st);
    else backward<float>(g, plan.blocks, st);
    if (grads && !(plan.blocks == 1 && dgamma))
      hipLaunchKernelGGL(reduce_kernel, dim3((2 * s->width + RED_COLS - 1) / RED_COLS), dim3(1024), 0, st,
                         (const float*)workspace, plan.blocks, s->width, dgamma, dbeta);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return bad(STAGE_EHIP, "layer_norm_backward: %s", hipGetErrorString(e));
  return STAGE_OK;
}

}  // extern "C"
