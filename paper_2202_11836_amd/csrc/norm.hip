// Layer norm as an operator of its own (include/norm.h): forward with an optional residual
// addition, backward with the sums of the weights' gradients; plan and argument checks of
// the C ABI.
//
// A few operations a value, so HBM bounds it.  A row stays in the registers of its TPR
// threads (8 to 1024 of them by its width; of fp32 rows beyond 8192 the backward pass that leaves partial
// rows keeps 12 bytes a thread in scratch) from its one read to its one write: forward reads
// x (and the residual) and writes out (and the sum), backward reads dy, z and dtotal and
// writes dx, while every thread adds up dy xh and dy of its columns over the rows of its
// work-group, which leaves one partial row a work-group to a second launch.  bf16 rows of
// 1024, 16384 of them, with residual: forward 27.3 us (4.9 TB/s), backward 27.5 (5.0) and
// 4.6 for the sums; 5000 rows of 5120: 27.2 (3.8), 36.0 (4.9 with the partial rows), 5.4.
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
  int threads;                   // of a row of several wavefronts
  int row_groups;                // COLUMNS: work-groups of rows
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
  // The first n go, zeros come in at the end.
  __device__ __forceinline__ void drop(int n) {
    if (n & 4) r = u32x4_t{r[2], r[3], 0, 0};
    if (n & 2) r = u32x4_t{r[1], r[2], r[3], 0};
    if (n & 1)
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = r[k] >> 16 | (k < 3 ? r[k < 3 ? k + 1 : 3] << 16 : 0);
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
    typedef u32x2_t __attribute__((aligned(2))) four_t;
    typedef uint32_t __attribute__((aligned(2))) two_t;
    if (n & 4) *(four_t*)p = u32x2_t{r[0], r[1]};
    const uint32_t a = n & 4 ? r[2] : r[0], b = n & 4 ? r[3] : r[1];
    if (n & 2) *(two_t*)(p + (n & 4)) = a;
    if (n & 1) p[n - 1] = (bf16_t)(n & 2 ? b : a);
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
  __device__ __forceinline__ void drop(int n) {
    if (n & 4) a = b, b = f32x4_t{0, 0, 0, 0};
    if (n & 2) a = f32x4_t{a[2], a[3], b[0], b[1]}, b = f32x4_t{b[2], b[3], 0, 0};
    if (n & 1) a = f32x4_t{a[1], a[2], a[3], b[0]}, b = f32x4_t{b[1], b[2], b[3], 0};
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
// The eight at place `at` of a row, of which n are left in it (<= 0: none).  A row's last few come as
// the last of the row's last eight, which `trim` puts right once all loads of a thread are on their way
// (loads of single values wait for each other, as does the shift: backward of 868 x 493 in bf16 28.6 us, 20
// with the shift at once, 10.3 so; 868 x 496 9.0).
// TINY: rows may have fewer than eight.
template <bool TINY, typename T>
__device__ __forceinline__ void load_n(Chunk<T>& c, const T* row, int at, int n) {
  if (TINY && n > 0 && n < 8 && at == 0) c.load_part(row, n);
  else if (n > 0) c.load(row + at + min(n - 8, 0));
  else c.zero();
}
template <typename T>
__device__ __forceinline__ void trim(Chunk<T>& c, int at, int n) {
  if (n > 0 && n < 8 && at > 0) c.drop(8 - n);
}
template <typename T>
__device__ __forceinline__ void store_n(const Chunk<T>& c, T* p, int n) {
  if (n >= 8) c.store(p);
  else if (n > 0) c.store_part(p, n);
}
// eight weights (absent: all `none`)
template <bool TINY>
__device__ __forceinline__ void weights(const float* w, int at, int n, float none, float v[8]) {
  Chunk<float> c;
  if (!w) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = none;
    return;
  }
  load_n<TINY>(c, w, at, n);
  trim(c, at, n);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = c.get(k);
}

template <typename T>
__device__ __forceinline__ T* row_at(const Rows& r, int batch, int seq, int row) {
  if (batch == 1) return (T*)r.p + (int64_t)row * r.ss;
  const int b = row / seq;
  return (T*)r.p + b * r.sb + (int64_t)(row - b * seq) * r.ss;
}

// A row has TPR threads, 8 to 64, or (TPR 0) several wavefronts, up to MOST_WAVES in a work-group.
constexpr int MOST_WAVES = 16;
constexpr int BWD_GROUP = 512;  // threads of a backward work-group (rows to 8192)

// Sums over the threads of a row, N of them together: lanes of a wavefront, whose wavefronts meet
// in LDS, twice buffered by `turn` (one barrier a sum).
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float v[N], float* lds, int turn, int row_waves, int slot) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = (TPR ? TPR : 64) / 2; o > 0; o >>= 1) v[i] += __shfl_xor(v[i], o, 64);
  if constexpr (TPR == 0) {
    float* at = lds + turn * N * MOST_WAVES;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) at[i * MOST_WAVES + (threadIdx.x >> 6)] = v[i];
    __syncthreads();
    at += slot * row_waves;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = at[i * MOST_WAVES];
      for (int j = 1; j < row_waves; ++j) t += at[i * MOST_WAVES + j];
      v[i] = t;
    }
  }
}

// What is left of a row at a thread's chunk i of NC, from its first value on: only the last of them can
// lie across the row's end or behind it (the widths that each NC gets make it so).
template <int NC>
__device__ __forceinline__ int left(int w, int at, int i) { return i < NC - 1 ? 8 : w - at; }

// NC chunks of eight values a thread: thread j of a row's T owns chunks j + T i.  EARLY: gamma and
// beta are asked for before the sums, which saves a memory latency, and costs 16 registers a
// chunk.
template <typename T, int TPR, int NC, bool RES, bool EARLY>
__global__ __launch_bounds__(TPR ? 256 : 64 * MOST_WAVES) void fwd_kernel(const FwdArgs g) {
  __shared__ float lds[TPR ? 1 : 2 * MOST_WAVES];
  const int threads = TPR ? TPR : blockDim.x;
  const int lane = TPR ? threadIdx.x % (TPR ? TPR : 1) : threadIdx.x;
  const int row = TPR ? blockIdx.x * (256 / (TPR ? TPR : 256)) + threadIdx.x / (TPR ? TPR : 1) : blockIdx.x;
  if (TPR && row >= g.rows) return;
  const T* x = row_at<T>(g.x, g.batch, g.seq, row);
  Chunk<T> c[NC], r[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i)
    load_n<TPR == 8>(c[i], x, 8 * (lane + threads * i), left<NC>(g.w, 8 * (lane + threads * i), i));
  if constexpr (!RES) {
#pragma unroll
    for (int i = 0; i < NC; ++i) trim(c[i], 8 * (lane + threads * i), left<NC>(g.w, 8 * (lane + threads * i), i));
  } else {
    const T* res = row_at<T>(g.res, g.batch, g.seq, row);
#pragma unroll
    for (int i = 0; i < NC; ++i)
      load_n<TPR == 8>(r[i], res, 8 * (lane + threads * i), left<NC>(g.w, 8 * (lane + threads * i), i));
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      trim(c[i], 8 * (lane + threads * i), left<NC>(g.w, 8 * (lane + threads * i), i));
      trim(r[i], 8 * (lane + threads * i), left<NC>(g.w, 8 * (lane + threads * i), i));
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = c[i].get(k) + r[i].get(k);
      c[i].set(v);  // (what follows sees the sum as it is stored)
    }
    if (g.total.p) {
      T* t = row_at<T>(g.total, g.batch, g.seq, row);
#pragma unroll
      for (int i = 0; i < NC; ++i)
        store_n(c[i], t + 8 * (lane + threads * i), left<NC>(g.w, 8 * (lane + threads * i), i));
    }
  }
  float ga[NC][8], be[NC][8];
  if constexpr (EARLY) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int at = 8 * (lane + threads * i);
      weights<TPR == 8>(g.gamma, at, left<NC>(g.w, at, i), 1.0f, ga[i]);
      weights<TPR == 8>(g.beta, at, left<NC>(g.w, at, i), 0.0f, be[i]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  float s[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) s[0] += c[i].get(k);
  row_sums<TPR, 1>(s, lds, 0, threads / 64, 0);
  const float mean = s[0] / (float)g.w;
  s[0] = 0.0f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int n = left<NC>(g.w, 8 * (lane + threads * i), i);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float d = k < n ? c[i].get(k) - mean : 0.0f;
      s[0] += d * d;
    }
  }
  row_sums<TPR, 1>(s, lds, 1, threads / 64, 0);
  const float rstd = 1.0f / sqrtf(s[0] / (float)g.w + g.eps);
  T* out = row_at<T>(g.out, g.batch, g.seq, row);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int at = 8 * (lane + threads * i), n = left<NC>(g.w, at, i);
    float v[8];
    if constexpr (!EARLY) {
      weights<TPR == 8>(g.gamma, at, n, 1.0f, ga[i]);
      weights<TPR == 8>(g.beta, at, n, 0.0f, be[i]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = fmaf((c[i].get(k) - mean) * rstd, ga[i][k], be[i][k]);
    c[i].set(v);
    store_n(c[i], out + at, n);
  }
  if (lane == 0) {
    if (g.mean) g.mean[row] = mean;
    if (g.rstd) g.rstd[row] = rstd;
  }
}

// dgamma and dbeta of 64 columns over all rows, by a work-group: 8 chunks side by side, an eighth of
// its threads' rows at a time, four of a thread's on their way together.
template <typename T, bool TINY>
__device__ __forceinline__ void column_sums(const BwdArgs& g, int col0) {
  __shared__ float red[2][MOST_WAVES][64];
  const int slots = blockDim.x / 8, waves = blockDim.x / 64;
  const int chunk = threadIdx.x & 7, at = col0 + 8 * chunk, n = g.w - at;
  float pg[8], pb[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) pg[k] = pb[k] = 0.0f;
  for (int first = threadIdx.x >> 3; first < g.rows; first += 4 * slots) {
    Chunk<T> dy[4], z[4];
    float mean[4], rstd[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = first + slots * u;
      const bool live = row < g.rows;
      load_n<TINY>(dy[u], live ? row_at<T>(g.dy, g.batch, g.seq, row) : nullptr, at, live ? n : 0);
      load_n<TINY>(z[u], live ? row_at<T>(g.z, g.batch, g.seq, row) : nullptr, at, live ? n : 0);
      mean[u] = live ? g.mean[row] : 0.0f;
      rstd[u] = live ? g.rstd[row] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      trim(dy[u], at, n);
      trim(z[u], at, n);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        pg[k] += dy[u].get(k) * ((z[u].get(k) - mean[u]) * rstd[u]);
        pb[k] += dy[u].get(k);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) {
      pg[k] += __shfl_xor(pg[k], o, 64);
      pb[k] += __shfl_xor(pb[k], o, 64);
    }
  if ((threadIdx.x & 63) < 8)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      red[0][threadIdx.x >> 6][8 * chunk + k] = pg[k];
      red[1][threadIdx.x >> 6][8 * chunk + k] = pb[k];
    }
  __syncthreads();
  const int which = threadIdx.x >> 6, col = col0 + (threadIdx.x & 63);
  float* const to = which == 0 ? g.dgamma : which == 1 ? g.dbeta : nullptr;
  if (to && col < g.w) {
    float t = red[which][0][threadIdx.x & 63];
    for (int j = 1; j < waves; ++j) t += red[which][j][threadIdx.x & 63];
    to[col] = t;
  }
}

// Values of a row of the partial sums in LDS: whole chunks.
__host__ __device__ __forceinline__ int red_row(int w) { return (w + 7) & ~7; }
typedef f32x4_t __attribute__((aligned(4))) any_f32x4_t;

// What becomes of dy xh and dy: nothing, a partial row of each work-group's, or the sums at once by
// work-groups behind those of the rows, each for 64 columns (few rows, read twice from cache: one
// launch less).
enum Grads { NONE, PARTIAL, COLUMNS };

template <typename T, int TPR, int MAX_THREADS, int NC, Grads G>
__global__ __launch_bounds__(MAX_THREADS) void bwd_kernel(const BwdArgs g) {
  __shared__ float lds[TPR ? 1 : 4 * MOST_WAVES];
  constexpr bool GRADS = G == PARTIAL;
  if constexpr (G == COLUMNS)
    if ((int)blockIdx.x >= g.row_groups) {
      column_sums<T, TPR == 8>(g, 64 * (blockIdx.x - g.row_groups));
      return;
    }
  const int threads = TPR ? TPR : g.threads;
  const int slots = TPR ? BWD_GROUP / (TPR ? TPR : 1) : blockDim.x / g.threads;  // rows side by side
  // (a wavefront is of one row: the slot is the same for all its lanes)
  const int slot = TPR ? threadIdx.x / (TPR ? TPR : 1)
                       : __builtin_amdgcn_readfirstlane(threadIdx.x / g.threads);
  const int lane = threadIdx.x - slot * threads;
  const int r0 = blockIdx.x * g.rpb, r1 = min(g.rows, r0 + g.rpb);
  const float inv_w = 1.0f / (float)g.w;
  float gm[NC][8], pg[GRADS ? NC : 1][8], pb[GRADS ? NC : 1][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int at = 8 * (lane + threads * i);
    weights<TPR == 8>(g.gamma, at, left<NC>(g.w, at, i), 1.0f, gm[i]);
    if constexpr (GRADS)
#pragma unroll
      for (int k = 0; k < 8; ++k) pg[i][k] = pb[i][k] = 0.0f;
  }
  int turn = 0;
  // (the same number of passes for all wavefronts of a row)
  for (int first = r0; first < r1; first += slots) {
    Chunk<T> dy[NC], z[NC], dt[NC];
    const int row = first + slot;
    const bool live = row < r1;
    const T* pd = live ? row_at<T>(g.dy, g.batch, g.seq, row) : nullptr;
    const T* pz = live ? row_at<T>(g.z, g.batch, g.seq, row) : nullptr;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int at = 8 * (lane + threads * i), n = live ? left<NC>(g.w, at, i) : 0;
      load_n<TPR == 8>(dy[i], pd, at, n);
      load_n<TPR == 8>(z[i], pz, at, n);
    }
    if (g.dtotal.p) {
      const T* pt = live ? row_at<T>(g.dtotal, g.batch, g.seq, row) : nullptr;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = 8 * (lane + threads * i);
        load_n<TPR == 8>(dt[i], pt, at, live ? left<NC>(g.w, at, i) : 0);
      }
    }
    const float mean = live ? g.mean[row] : 0.0f, rstd = live ? g.rstd[row] : 0.0f;
    if (g.w & 7)
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = 8 * (lane + threads * i), n = left<NC>(g.w, at, i);
        trim(dy[i], at, n);
        trim(z[i], at, n);
        if (g.dtotal.p) trim(dt[i], at, n);
      }
    float s[2] = {0.0f, 0.0f};
    // (behind a row's end dy is 0, and so is all that comes of it)
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float d = dy[i].get(k), xh = (z[i].get(k) - mean) * rstd;
        const float dg = d * gm[i][k];
        s[0] += dg;
        s[1] += dg * xh;
        if constexpr (GRADS) {
          pg[i][k] += d * xh;
          pb[i][k] += d;
        }
      }
    if (g.dx.p) {
      row_sums<TPR, 2>(s, lds, turn, threads / 64, slot);
      turn ^= 1;
      if (!live) continue;
      T* px = row_at<T>(g.dx, g.batch, g.seq, row);
      const float a = s[0] * inv_w, b = s[1] * inv_w;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = 8 * (lane + threads * i);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float xh = (z[i].get(k) - mean) * rstd;
          v[k] = rstd * (dy[i].get(k) * gm[i][k] - a - xh * b);
          if (g.dtotal.p) v[k] += dt[i].get(k);
        }
        dy[i].set(v);
        store_n(dy[i], px + at, left<NC>(g.w, at, i));
      }
    }
  }
  if constexpr (GRADS) {
    // The work-group's rows side by side: lanes of a wavefront first, then slots in order, one
    // sum after the other through LDS.
    // (LDS rows are whole chunks, so that all of it goes 16 bytes at a time: with rows of w values and
    // one at a time 1200 x 2048 took 10.5 us in bf16, 7.6 so, 5.4 without the sums.)
    extern __shared__ __attribute__((aligned(16))) float red[];  // [TPR 0: slot, else wavefront][wp]
    const int wp = red_row(g.w);
    constexpr bool WAVES = TPR > 0;
    float* const part = g.part + (int64_t)blockIdx.x * 2 * g.w;
    if constexpr (WAVES && TPR < 64) {
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
    const int rows = WAVES ? BWD_GROUP / 64 : slots, mine = WAVES ? threadIdx.x >> 6 : slot;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float* const to = part + which * g.w;
      if (rows > 1) {
        if (!WAVES || (threadIdx.x & 63) < TPR) {
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            const int at = 8 * (lane + threads * i);
            if (at >= g.w) continue;
            const float* v = which ? pb[i] : pg[i];
            f32x4_t* to_lds = (f32x4_t*)(red + mine * wp + at);
            to_lds[0] = f32x4_t{v[0], v[1], v[2], v[3]};
            to_lds[1] = f32x4_t{v[4], v[5], v[6], v[7]};
          }
        }
        __syncthreads();
        for (int e = 4 * threadIdx.x; e < g.w; e += 4 * blockDim.x) {
          const f32x4_t* from = (const f32x4_t*)(red + e);
          f32x4_t t = from[0];
          if constexpr (WAVES) {
#pragma unroll
            for (int j = 1; j < BWD_GROUP / 64; ++j) t += from[j * wp / 4];
          } else {  // (two or four)
            t += from[wp / 4];
            if (rows > 2) {
              t += from[2 * wp / 4];
              t += from[3 * wp / 4];
            }
          }
          if (e + 4 <= g.w) {
            *(any_f32x4_t*)(to + e) = t;
          } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
              if (e + k < g.w) to[e + k] = t[k];
          }
        }
        if (which == 0) __syncthreads();
      } else {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int at = 8 * (lane + threads * i);
          Chunk<float> c;
          c.set(which ? pb[i] : pg[i]);
          store_n(c, to + at, left<NC>(g.w, at, i));
        }
      }
    }
  }
}

// dgamma and dbeta: the sums over the work-groups' partial rows, `parts` of them: 32 stripes of
// rows to 32 columns (a cache line), each in order, then the stripes.
constexpr int RED_COLS = 32, RED_STRIPES = 1024 / RED_COLS;
__global__ __launch_bounds__(1024) void reduce_kernel(const float* __restrict__ part, int parts, int w,
                                                      float* dgamma, float* dbeta) {
  __shared__ float lds[16][RED_COLS];
  const int at = threadIdx.x % RED_COLS, col = blockIdx.x * RED_COLS + at;
  float t = 0.0f;
  if (col < 2 * w) {
    const float* p = part + col;
    const int64_t step = (int64_t)2 * w;
    for (int b = threadIdx.x / RED_COLS; b < parts; b += RED_STRIPES * 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = b + RED_STRIPES * j < parts ? p[(b + RED_STRIPES * j) * step] : 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) t += v[j];
    }
  }
  t += __shfl_xor(t, 32, 64);
  if ((threadIdx.x & 63) < RED_COLS) lds[threadIdx.x >> 6][at] = t;
  __syncthreads();
  if (threadIdx.x < RED_COLS && col < 2 * w) {
    t = lds[0][at];
#pragma unroll
    for (int j = 1; j < 16; ++j) t += lds[j][at];
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
constexpr int FWD_NARROW = 1536, BWD_NARROW = 1024;  // widest rows of one wavefront
constexpr int BWD_MIDDLE = 8192;                      // of eight

int round64(int n) { return (n + 63) / 64 * 64; }
// Threads of a row: a wavefront or less while its row fits (no barriers), then as many
// wavefronts as the row fills with two chunks a thread.  bf16 rows that would leave a third of the lanes
// without a value, or half of the second chunks, have three chunks a thread instead: their instructions
// bound them.  us so / with 64 threads: forward 30000 x 300 11.3 / 17.3, 30000 x 384 13.2 / 15.4, 16384 x
// 768 14.0 / 14.9 (fp32: 21.0 / 21.3, 22.4 / 21.6, 24.0 / 24.2, so it keeps its 64).
bool by_threes(int w, stage_dtype dt) {
  return dt == STAGE_BF16 && ((w > 256 && w <= 384) || (w > 512 && w <= 768));
}
int fwd_threads(int w, stage_dtype dt) {
  if (by_threes(w, dt)) return w <= 384 ? 16 : 32;
  return w <= 64 ? 8 : w <= 128 ? 16 : w <= 256 ? 32 : w <= FWD_NARROW ? 64 : round64((w + 15) / 16);
}
// In the backward pass they take 178 registers for 125, which pays for many rows of the wider ones:
// 40000 x 768 44.2 / 49.0, 22500 x 598 27.1 / 30.7, 16384 x 768 22.9 / 24.0; but 6000 x 768 12.7 / 12.0,
// 30000 x 384 26.8 / 22.9.
bool bwd_by_threes(int rows, int w, stage_dtype dt) { return w > 512 && rows >= 8192 && by_threes(w, dt); }
int bwd_threads(int w) {
  return w <= 64 ? 8 : w <= 128 ? 16 : w <= 256 ? 32 : w <= BWD_NARROW ? 64 : round64((w + 15) / 16);
}
// Threads of a backward work-group: as many rows side by side as fit.
int bwd_group(int w) {
  const int t = bwd_threads(w);
  return w <= BWD_MIDDLE ? BWD_GROUP / t * t : t;
}
// Work-groups, which leave a partial row each: one to a CU, or two where their registers let
// two live there (one chunk a thread, or bf16 rows of more than one wavefront).  us with one and
// two, bf16: 16384 x 1280 43.3 / 33.9, 3000 x 5120 38.5 / 32.5, 2000 x 2048 13.0 / 14.4; rows of up to 1024
// gain or lose 4% with two, and fp32 rows of more than one wavefront lose, 8192 x 2048 50.1 / 54.5.
int bwd_most(int w, stage_dtype dt) {
  return w <= 512 || (w > BWD_NARROW && w <= BWD_MIDDLE && dt == STAGE_BF16) ? 512 : 256;
}
// Up to so many rows the sums are made by work-groups of columns in the same launch, of more by partial
// rows and a launch to sum them: a column's time grows with the rows, that of partial rows with the
// width.  us by columns / partial rows, bf16: 550 x 512 6.3 / 7.8, 650 x 1024 7.3 / 7.8, 800 x 768
// 7.8 / 7.3; 700 x 1280 7.7 / 8.4, 1000 x 1280 9.8 / 9.1; 1100 x 4096 13.2 / 17.0, 1600 x 5120 22.4 / 22.9,
// 2000 x 5120 28.9 / 26.3; fp32 1000 x 1024 10.6 / 8.7, 1100 x 4096 19.3 / 21.4, 1400 x 4096 25.6 / 24.5.
int few_rows(int w) { return w <= BWD_NARROW ? 700 : w < 4096 ? 900 : 1300; }
struct BwdPlan {
  int blocks, rpb;
};
BwdPlan bwd_plan(int rows, int w, stage_dtype dt) {
  const int step = bwd_by_threes(rows, w, dt) ? BWD_GROUP / 32 : bwd_group(w) / bwd_threads(w);  // rows at a time
  const int blocks = std::min(bwd_most(w, dt), (rows + step - 1) / step);
  const int rpb = ((rows + blocks - 1) / blocks + step - 1) / step * step;
  return {(rows + rpb - 1) / rpb, rpb};
}

template <typename T, int TPR, int NC>
void launch_fwd(const FwdArgs& g, hipStream_t st) {
  constexpr int RPB = TPR ? 256 / (TPR ? TPR : 1) : 1;
  const dim3 grid((unsigned)((g.rows + RPB - 1) / RPB)), block(TPR ? 256 : round64((g.w + 15) / 16));
  // Early while all rows run at once: 2000 x 1024 in bf16 5.7 -> 5.1 us; 16384 x 1024 16.7 -> 17.1,
  // in fp32 29.4 -> 32.5.
  const bool early = (int64_t)g.rows * (NC == 3 ? 64 : block.x / RPB) <= 2560 * 64;
  if (g.res.p) {
    if (early) hipLaunchKernelGGL((fwd_kernel<T, TPR, NC, true, true>), grid, block, 0, st, g);
    else hipLaunchKernelGGL((fwd_kernel<T, TPR, NC, true, false>), grid, block, 0, st, g);
  } else {
    if (early) hipLaunchKernelGGL((fwd_kernel<T, TPR, NC, false, true>), grid, block, 0, st, g);
    else hipLaunchKernelGGL((fwd_kernel<T, TPR, NC, false, false>), grid, block, 0, st, g);
  }
}
template <typename T>
void forward(const FwdArgs& g, hipStream_t st) {
  const int w = g.w;
  if constexpr (sizeof(T) == 2)
    if (by_threes(w, STAGE_BF16)) {
      if (w <= 384) launch_fwd<T, 16, 3>(g, st);
      else launch_fwd<T, 32, 3>(g, st);
      return;
    }
  if (w <= 64) launch_fwd<T, 8, 1>(g, st);
  else if (w <= 128) launch_fwd<T, 16, 1>(g, st);
  else if (w <= 256) launch_fwd<T, 32, 1>(g, st);
  else if (w <= 512) launch_fwd<T, 64, 1>(g, st);
  else if (w <= 1024) launch_fwd<T, 64, 2>(g, st);
  else if (w <= FWD_NARROW) launch_fwd<T, 64, 3>(g, st);
  else launch_fwd<T, 0, 2>(g, st);
}

template <typename T, int TPR, int MAX_THREADS, int NC>
void launch_bwd(const BwdArgs& g, int blocks, Grads grads, hipStream_t st) {
  const dim3 grid((unsigned)blocks), block(bwd_group(g.w));
  const int rows = TPR ? BWD_GROUP / 64 : (int)block.x / g.threads;
  const size_t lds = rows > 1 ? (size_t)rows * red_row(g.w) * 4 : 0;
  if (grads == PARTIAL) {
    hipLaunchKernelGGL((bwd_kernel<T, TPR, MAX_THREADS, NC, PARTIAL>), grid, block, lds, st, g);
  } else if (grads == NONE) {
    hipLaunchKernelGGL((bwd_kernel<T, TPR, MAX_THREADS, NC, NONE>), grid, block, 0, st, g);
  } else {
    const dim3 both((unsigned)(blocks + (g.w + 63) / 64));
    hipLaunchKernelGGL((bwd_kernel<T, TPR, MAX_THREADS, NC, COLUMNS>), both, block, 0, st, g);
  }
}
template <typename T>
void backward(const BwdArgs& g, int blocks, Grads grads, hipStream_t st) {
  const int w = g.w;
  if constexpr (sizeof(T) == 2)
    if (grads == PARTIAL && bwd_by_threes(g.rows, w, STAGE_BF16)) {
      hipLaunchKernelGGL((bwd_kernel<T, 32, BWD_GROUP, 3, PARTIAL>), dim3((unsigned)blocks), dim3(BWD_GROUP),
                         BWD_GROUP / 64 * red_row(w) * 4, st, g);
      return;
    }
  if (w <= 64) launch_bwd<T, 8, BWD_GROUP, 1>(g, blocks, grads, st);
  else if (w <= 128) launch_bwd<T, 16, BWD_GROUP, 1>(g, blocks, grads, st);
  else if (w <= 256) launch_bwd<T, 32, BWD_GROUP, 1>(g, blocks, grads, st);
  else if (w <= 512) launch_bwd<T, 64, BWD_GROUP, 1>(g, blocks, grads, st);
  else if (w <= BWD_NARROW) launch_bwd<T, 64, BWD_GROUP, 2>(g, blocks, grads, st);
  else if (w <= BWD_MIDDLE) launch_bwd<T, 0, BWD_GROUP, 2>(g, blocks, grads, st);
  else launch_bwd<T, 0, 1024, 2>(g, blocks, grads, st);
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
  if ((int64_t)s->batch * s->seq > 4294967040LL / fwd_threads(s->width, s->dtype))
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
  *bytes = rows ? (size_t)bwd_plan((int)rows, s->width, s->dtype).blocks * 2 * s->width * 4 : 0;
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
    const BwdPlan plan = bwd_plan((int)rows, s->width, s->dtype);
    Grads grads = dgamma || dbeta ? PARTIAL : NONE;
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
    g.threads = bwd_threads(s->width);
    const auto run = [&](int blocks, Grads how) {
      if (s->dtype == STAGE_BF16) backward<bf16_t>(g, blocks, how, st);
      else backward<float>(g, blocks, how, st);
    };
    if (grads && rows <= few_rows(s->width)) {
      // Work-groups of columns read dy and z while those of rows write dx: over one of them, the
      // columns go first.
      grads = COLUMNS;
      const bool over = dx && (dx == dy || dx == total);
      g.row_groups = dx && !over ? plan.blocks : 0;
      run(g.row_groups, COLUMNS);
      if (over) run(plan.blocks, NONE);
    } else {
      run(plan.blocks, grads);
    }
    if (grads == PARTIAL)
      hipLaunchKernelGGL(reduce_kernel, dim3((2 * s->width + RED_COLS - 1) / RED_COLS), dim3(1024), 0, st,
                         (const float*)workspace, plan.blocks, s->width, dgamma, dbeta);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return bad(STAGE_EHIP, "layer_norm_backward: %s", hipGetErrorString(e));
  return STAGE_OK;
}

}  // extern "C"
