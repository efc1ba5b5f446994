// Forward attention for few queries (single tokens over a long cache): bound by the
// keys and values, which are read once.  A wavefront takes a tile of 32 rows - the
// queries of all query heads that share a key head, so that shared keys are not read
// again - over keys of its own: the 4 wavefronts of a work-group and the splits of
// the keys share the work along the keys, and are joined by their exponents' offsets
// and sums, in LDS and, with several splits, by a second launch.  Each wavefront has
// a two-stage ring of 32-key blocks in LDS to itself and waits for nobody until the
// join: it waits for a block, requests the next one and computes.  (Requesting before the
// wait puts twice as much on its way and was slower for long caches: 16 x 16 heads over
// 8192 keys 105 us against 98, both with ordinary loads.)
// The scores and products are those of xattn.hip: a tile costs 0.3 us of a SIMD's time
// whether one of its rows is in use or all, and a SIMD's share of 5.5 TB/s (256 CUs of 4)
// brings its 8 KB in 1.5 us.  Measured: 16 x 16 heads, one token over 8192 keys, 92 us
// (5.8 TB/s; a plain read of as many bytes takes 88 to 93); where there is less to read,
// the chain of one wavefront's blocks and the join (4 us) are what is left.
#include <algorithm>
#include <cmath>

#include "xattn.h"

namespace {

constexpr int FB = 32;  // keys per block

// x_mma_cols for one 32-key block without the wait for every load in flight that the
// compiler puts before its transposing reads: eight reads and their wait in one
// statement.  tr: this lane's addresses within a tile, by column half and by the
// upper eight of sixteen rows (frag_tr's layout; the second sixteen rows are 2048
// bytes on, with the same swizzle).
struct TrAddr {
  uint32_t a[2][2];
};
__device__ __forceinline__ TrAddr tr_addr(int lane) {
  TrAddr r;
  const int j = lane & 15, row = 4 * (lane >> 5) + (j >> 2);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int d = 32 * t + 16 * ((lane >> 4) & 1) + 4 * (j & 3);
    r.a[t][0] = toff(row, d >> 3) + 2 * (d & 7);
    r.a[t][1] = toff(row + 8, d >> 3) + 2 * (d & 7);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void few_mma_cols(const char* tile, const TrAddr& tr, const f32x16_t& p,
                                             f32x16_t out[2], int lane) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)tile;
    u32x2_t v[2][2][2];  // [16 rows][column half][8 rows]
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n"
        "ds_read_b64_tr_b16 %1, %9\n"
        "ds_read_b64_tr_b16 %2, %10\n"
        "ds_read_b64_tr_b16 %3, %11\n"
        "ds_read_b64_tr_b16 %4, %8 offset:2048\n"
        "ds_read_b64_tr_b16 %5, %9 offset:2048\n"
        "ds_read_b64_tr_b16 %6, %10 offset:2048\n"
        "ds_read_b64_tr_b16 %7, %11 offset:2048\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0][0][0]), "=&v"(v[0][0][1]), "=&v"(v[0][1][0]), "=&v"(v[0][1][1]),
          "=&v"(v[1][0][0]), "=&v"(v[1][0][1]), "=&v"(v[1][1][0]), "=&v"(v[1][1][1])
        : "v"(base + tr.a[0][0]), "v"(base + tr.a[0][1]), "v"(base + tr.a[1][0]),
          "v"(base + tr.a[1][1])
        : "memory");
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const bf16x8_t pb = pack8(p, 8 * ks);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x2_t lo = v[ks][t][0], hi = v[ks][t][1];
        out[t] = mfma32(__builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], hi[0], hi[1]}), pb, out[t]);
      }
    }
  } else {
    x_mma_cols<T>(tile, 0, p, out, lane);
  }
}

// LDS of the near tiles' tables.
size_t few_near_bytes(int nb, int reach) { return nb ? 128 * (size_t)nb + 2 * (reach + XPAD) + 1 : 0; }

template <typename T, bool BIAS, int NW>
__global__ __launch_bounds__(64 * NW, 2) void xattn_few_kernel(XAttnArgs a, int n_rt) {
  constexpr int TILE = FB * XT<T>::ROWB;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  // [NW][2][K, V]; with a bias: the rows' biases [nb][32] and the buckets by distance
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, rr = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* ring = lds + wave * 4 * TILE;
  float* tab = (float*)(lds + NW * 4 * TILE);
  uint8_t* ids = (uint8_t*)(tab + 32 * a.nb);
  int rb, bg;
  attn_block(blockIdx.x, gridDim.x, n_rt * a.few_splits, rb, bg);
  const int split = rb / n_rt, rt = rb % n_rt;
  const int b = bg / a.G, g = bg % a.G;
  const int R = a.Sq * a.rep, row = rt * 32 + rr;  // (row: query i of head h)
  const bool rv = row < R;
  const int i = row / a.rep, h = g * a.rep + row % a.rep;
  const int qp = x_q_pos(a, b);
  const int p_lo = rt * 32 / a.rep + qp, p_hi = min(rt * 32 + 31, R - 1) / a.rep + qp, pos = i + qp;
  const T* K = (const T*)a.k + b * a.sk[0] + g * a.sk[2];
  const T* V = (const T*)a.v + b * a.sv[0] + g * a.sv[2];
  const int lim = a.causal ? max(0, min(a.Sk, p_hi + 1)) : a.Sk;
  // This wavefront's blocks
  const int nblk = (lim + FB - 1) / FB, nw = NW * a.few_splits;
  const int per = (nblk + nw - 1) / nw, first = (NW * split + wave) * per;
  KeyBlocks<FB> blocks;
  blocks.init(a.mask ? a.mask + (int64_t)b * a.Sk : nullptr, lim, min(nblk, first + per), lane);
  auto dma = [&](int kb, int stage) {
    char* to = ring + stage * 2 * TILE;
    if (a.few_stream) {
      x_dma<T, FB, 1, true>(K, a.sk[1], kb * FB, lim, to, 0, lane);
      x_dma<T, FB, 1, true>(V, a.sv[1], kb * FB, lim, to + TILE, 0, lane);
    } else {
      x_dma<T, FB, 1>(K, a.sk[1], kb * FB, lim, to, 0, lane);
      x_dma<T, FB, 1>(V, a.sv[1], kb * FB, lim, to + TILE, 0, lane);
    }
  };
  // The first block is requested before the mask says whether it holds a key.
  if (first < blocks.nblk) dma(first, 0);
  typename XT<T>::Frag qf =
      x_frag((const T*)a.q + b * a.sq[0] + (int64_t)i * a.sq[1] + h * a.sq[2], rv, hf);
  float far_l = 0.0f, far_r = 0.0f;
  const int mid = a.reach + XPAD;
  if constexpr (BIAS) {
    if (rv) {
      far_l = a.table[(int64_t)x_bucket(a, -a.reach) * a.H + h] * XLOG2E;
      far_r = a.table[(int64_t)x_bucket(a, a.reach) * a.H + h] * XLOG2E;
    }
    // The tables of near tiles, where this work-group has any.
    const int k_lo = NW * split * per * FB, k_hi = min(nblk, NW * (split + 1) * per) * FB - 1;
    if (k_hi - p_lo > -a.reach && k_lo - p_hi < a.reach) {
      for (int e = tid; e < 32 * a.nb; e += 64 * NW) {
        const int r = rt * 32 + (e & 31);
        tab[e] = r < R ? a.table[(int64_t)(e >> 5) * a.H + g * a.rep + r % a.rep] * XLOG2E : 0.0f;
      }
      for (int e = tid; e < 2 * mid + 1; e += 64 * NW) ids[e] = (uint8_t)x_bucket(a, e - mid);
      __syncthreads();
    }
  }
  int kb = blocks.nblk;
  if (first < blocks.nblk) {
    blocks.load(first);
    kb = blocks.next(first);
    if (kb > first) wait_all();
    if (kb > first && kb < blocks.nblk) dma(kb, 0);
  }

  float m = -INFINITY, lsum = 0.0f;
  f32x16_t acc[2] = {zero16(), zero16()};
  const TrAddr tr = tr_addr(lane);
  x_arrived(qf);
  if constexpr (BIAS) {
    x_arrived(far_l);
    x_arrived(far_r);
  }
  for (int st = 0; kb < blocks.nblk; st ^= 1) {
    const int k0 = kb * FB;
    const uint32_t bw = blocks.word(kb), hidden = blocks.in_range(kb) & ~bw;
    kb = blocks.next(kb + 1);
    wait_all();
    if (kb < blocks.nblk) dma(kb, st ^ 1);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    char* kv = ring + st * 2 * TILE;
    if (hidden) {
      constexpr int CPR = XT<T>::CPR;
#pragma unroll
      for (int j = 0; j < 2 * FB * CPR / 64; ++j) {
        const int ch = lane + 64 * j;
        if (!((bw >> ((ch / CPR) & (FB - 1))) & 1)) *(u32x4_t*)(kv + 16 * ch) = zero4();
      }
      lds_wait();
      __builtin_amdgcn_wave_barrier();
    }
    f32x16_t s = x_mma_rows(kv, 0, qf, zero16(), lane);
    // Scores in units of log2: s * mul + add, masked; either in one step inside the
    // exponent (a tile with one bias and no hidden key) or here.
    const bool near = BIAS && k0 + FB - 1 - p_lo > -a.reach && k0 - p_hi < a.reach;
    float mul = a.c, add = !BIAS ? 0.0f : k0 > p_hi ? far_r : far_l, mblk = -INFINITY;
    if (bw == 0xffffffffu && !near && (!a.causal || k0 + FB - 1 <= p_lo)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) mblk = fmaxf(mblk, s[r]);
      mblk = fmaf(mblk, mul, add);
    } else {
      uint32_t bits = x_lane_bits(bw, hf);
      if (a.causal) bits &= x_upto(pos - k0 - 4 * hf);
      if (near) {
        // (rows of one tile can lie further apart than the table's margin)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int e = min(max(k0 + acc_row(r, hf) - pos, -mid), mid) + mid;
          s[r] = fmaf(s[r], mul, tab[32 * ids[e] + rr]);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], mul, add);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = x_or_ninf(s[r], bits, r);
        mblk = fmaxf(mblk, s[r]);
      }
      mul = 1.0f;
      add = 0.0f;
    }
    {
      const HalfPair pr = half_pair(mblk);
      mblk = fmaxf(pr.x, pr.y);
    }
    const bool grow = mblk > m + 8.0f;
    if (__any(grow)) {
      const float mn = grow ? mblk : m;
      const float alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
      lsum *= alpha;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] *= alpha;
      m = mn;
    }
    add -= m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, add));
    float ps = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) ps += s[r];
    lsum += ps;
    few_mma_cols<T>(kv + TILE, tr, s, acc, lane);
  }

  // Join the wavefronts: [NW][32][XFEW_ROW] in the place of the rings.
  const HalfPair lp = half_pair(lsum);
  __syncthreads();
  float* J = (float*)lds;
  {
    float* to = J + (wave * 32 + rr) * XFEW_ROW;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4_t*)(to + 32 * t + 8 * q + 4 * hf) =
            f32x4_t{acc[t][4 * q], acc[t][4 * q + 1], acc[t][4 * q + 2], acc[t][4 * q + 3]};
    if (hf == 0) {
      to[64] = m;
      to[65] = lp.x + lp.y;
    }
  }
  __syncthreads();
  const int r0 = tid >> 3, c = (tid & 7) * 8, row0 = rt * 32 + r0;
  if (r0 >= 32 || row0 >= R) return;
  float top = -INFINITY, l = 0.0f, o[8] = {};
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, J[(w * 32 + r0) * XFEW_ROW + 64]);
  // (a NaN or an infinity in m is carried by the sums)
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float* p = J + (w * 32 + r0) * XFEW_ROW;
    const float f = p[64] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(p[64] - top);
    l = fmaf(p[65], f, l);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(p[c + e], f, o[e]);
  }
  if (a.few_splits > 1) {
    float* to = a.part + (((int64_t)split * a.B * a.G + bg) * n_rt * 32 + row0) * XFEW_ROW;
    *(f32x4_t*)(to + c) = f32x4_t{o[0], o[1], o[2], o[3]};
    *(f32x4_t*)(to + c + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
    if (c == 0) {
      to[64] = top;
      to[65] = l;
    }
    return;
  }
  const int i0 = row0 / a.rep, h0 = g * a.rep + row0 % a.rep;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T* to = (T*)a.out + b * a.so[0] + (int64_t)i0 * a.so[1] + h0 * a.so[2] + c;
  if constexpr (sizeof(T) == 2) {
    *(u32x4_t*)to = u32x4_t{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                            pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv)};
  } else {
    *(f32x4_t*)to = f32x4_t{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    *(f32x4_t*)(to + 4) = f32x4_t{o[4] * inv, o[5] * inv, o[6] * inv, o[7] * inv};
  }
  if (a.lse && c == 0)
    a.lse[((int64_t)b * a.H + h0) * a.Sq + i0] =
        l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * XLN2;
}

// The splits of a row, joined in order: 16 threads to a row, 4 columns each.
template <typename T>
__global__ __launch_bounds__(256) void xattn_few_join_kernel(XAttnArgs a, int n_rt) {
  const int R = a.Sq * a.rep;
  const int64_t id = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (id >= (int64_t)a.B * a.G * R) return;
  const int bg = (int)(id / R), row = (int)(id % R), c = (threadIdx.x & 15) * 4;
  const int64_t step = (int64_t)a.B * a.G * n_rt * 32 * XFEW_ROW;
  const float* p = a.part + ((int64_t)bg * n_rt * 32 + row) * XFEW_ROW;
  // Eight splits' values are requested together, none of them waiting for another's.
  float top = -INFINITY, l = 0.0f;
  f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < a.few_splits; s0 += 8) {
    float m[8], ls[8];
    f32x4_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float* ps = p + (int64_t)min(s0 + j, a.few_splits - 1) * step;
      m[j] = ps[64];
      ls[j] = ps[65];
      v[j] = *(const f32x4_t*)(ps + c);
    }
    const float was = top;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (s0 + j >= a.few_splits) {  // (the last one again)
        m[j] = -INFINITY;
        ls[j] = 0.0f;
        v[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      }
      top = fmaxf(top, m[j]);
    }
    const float off = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(was - off);
    l *= keep;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= keep;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float f = __builtin_amdgcn_exp2f(m[j] - off);
      l = fmaf(ls[j], f, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(v[j][e], f, o[e]);
    }
  }
  const int b = bg / a.G, g = bg % a.G, i = row / a.rep, h = g * a.rep + row % a.rep;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T* to = (T*)a.out + b * a.so[0] + (int64_t)i * a.so[1] + h * a.so[2] + c;
  if constexpr (sizeof(T) == 2)
    *(u32x2_t*)to = u32x2_t{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
  else
    *(f32x4_t*)to = f32x4_t{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  if (a.lse && c == 0)
    a.lse[((int64_t)b * a.H + h) * a.Sq + i] =
        l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * XLN2;
}

template <typename T>
hipError_t few_t(const XAttnArgs& a, hipStream_t st) {
  const int n_rt = (int)xattn_few_tiles(a.rep, a.Sq);
  const int64_t grid = (int64_t)a.B * a.G * n_rt * a.few_splits;
  const int nw = a.few_waves;
  const size_t lds = nw * 4 * FB * XT<T>::ROWB + few_near_bytes(a.nb, a.reach);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * nw), lds, st, a, n_rt);
  };
  if constexpr (sizeof(T) == 2) {
    if (nw == 8) a.table ? go(xattn_few_kernel<T, true, 8>) : go(xattn_few_kernel<T, false, 8>);
  }
  if (nw == 4) a.table ? go(xattn_few_kernel<T, true, 4>) : go(xattn_few_kernel<T, false, 4>);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.few_splits == 1) return e;
  const int64_t rows = (int64_t)a.B * a.G * a.Sq * a.rep;
  hipLaunchKernelGGL(xattn_few_join_kernel<T>, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, st, a,
                     n_rt);
  return hipGetLastError();
}

}  // namespace

// A time model of this kernel in us, beside xattn_fwd_time, fitted to 700 timed launches
// (one token to 2500 queries, 51 to 32768 keys; over 40 shapes its choice is on average 2%
// off the best, at worst 12%).  A work-group costs its set-up and, per 32-key block of a
// wavefront, more the more wavefronts share a SIMD.  Splits add a launch and their partial
// results.  For instance 16 heads, one token and 8192 keys: 147 us with the other kernel,
// 38 with one split of 8 wavefronts, 16 with 8; 8 x 8 heads, one token over 700 keys 7.8
// with 8 wavefronts, 8.2 with 4; 32 x 16 heads of 128 queries and 512 keys: 21 with the
// other kernel, 34 with this one.
XFewPlan xattn_few_plan(int B, int G, int rep, int Sq, int Sk, int buckets, int reach,
                        stage_dtype dt) {
  const bool bf16 = dt == STAGE_BF16;
  const double tiles = (double)B * G * (double)xattn_few_tiles(rep, Sq), cus = device_cus();
  // (the model is one of few work-groups: 16 heads of 2500 queries are 1250 tiles and
  // take 60 us with the other kernel, 75 with this one)
  if (tiles == 0.0 || tiles > (bf16 ? 4 : 1) * cus) return {0, 0, 0};
  int ks;
  double best = xattn_fwd_time(B, G * rep, Sq, Sk, 0, dt, &ks);
  // No faster than the memory: of several that are bound by it, the fewest
  // wavefronts (16 x 16 heads over 8192 keys: 97 us with 4, 112 with 8).
  const double floor = 2.0 + 2.0 * B * G * (double)Sk * (bf16 ? 128 : 256) / 5.5e6;
  XFewPlan plan = {0, 0, 0};
  const int blocks = (Sk + FB - 1) / FB;
  for (int waves = 4; waves <= (bf16 ? 8 : 4); waves += 4) {
    const size_t lds = waves * 4 * FB * (bf16 ? 128 : 256) + few_near_bytes(buckets, reach);
    if (lds > 160 * 1024) continue;
    const double wcap = lds <= 80 * 1024 ? 2 : 1;
    for (const int splits :
         {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64, 96, 128, 192}) {
      if (splits > 1 && (splits * waves > blocks || tiles * splits > 2 * cus)) continue;
      const double grid = tiles * splits, n = std::min(wcap, std::ceil(grid / cus));
      const double per = std::ceil((double)blocks / (waves * splits));
      const double rounds = std::ceil(grid / (wcap * cus));
      double t = rounds * (bf16 ? 4.5 + (buckets ? 2.1 : 0.0) + (waves == 8 ? 0.5 : 0.0) +
                                      per * (0.67 + 0.4 * (waves / 4 * n - 1))
                                : 2.6 + per * 2.8);
      if (bf16) t -= 1.3;
      if (splits > 1)
        t += bf16 ? 2.4 + 0.3 * splits + 0.25e-3 * (double)B * G * rep * Sq * splits
                  : 5.3 + 0.025e-3 * (double)B * G * rep * Sq * splits;
      t = std::max(t, floor);
      if (t < best) {
        best = t;
        plan = {waves, splits, 0};
      }
    }
  }
  // One tile of rows over keys and values beyond the caches: loads that leave nothing
  // there let more through (24 x 8 heads over 8192 keys, 403 MB: 90 -> 81 us; 32 x 16
  // over 1024, 134 MB: 31.5 -> 28.1), but 32 x 16 over 512 (67 MB), whose keys the
  // caches can hold, take 14.9 -> 15.9.
  plan.stream = xattn_few_tiles(rep, Sq) == 1 &&
                2.0 * B * G * (double)Sk * (bf16 ? 128 : 256) > 96.0 * (1 << 20);
  return plan;
}

hipError_t xattn_few(const XAttnArgs& a, stage_dtype dt, hipStream_t st) {
  return dt == STAGE_BF16 ? few_t<bf16_t>(a, st) : few_t<float>(a, st);
}
