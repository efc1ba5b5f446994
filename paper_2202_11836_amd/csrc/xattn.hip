// Attention over the keys of another sequence, with a relative position bias by
// buckets (include/attn.h has the formulas).  The kernels are those of the stage's
// self attention (attn.hip) in structure: a wavefront owns 32 queries (forward,
// dQ) or 32 keys (dK, dV), a work-group of 4 shares 64-row blocks of the streamed
// operand in a two-stage LDS ring filled by direct-to-LDS loads, scores are
// produced transposed where a row's statistics are wanted per lane, and
// accumulators go back into the next product as its B operand.  What is added:
//   - fp32 tiles beside the bf16 ones (XT), on v_mfma_f32_32x32x2_f32;
//   - the keys that a mask leaves, as bits (KeyBlocks): blocks without one are
//     skipped, and a block that holds hidden keys has their K and V rows cleared
//     in LDS, so that whatever they hold stays out of the products;
//   - the bias: distances from `reach` on share one value on either side, so a
//     32 x 32 tile that is further adds one scalar inside the exponent; a nearer
//     tile reads a table of the bias by distance that the work-group spread out
//     in LDS (two reads for four scores);
//   - the bias gradient: far tiles sum their dS in a register; a near tile adds
//     its dS along the diagonals (x_diagonals) to the wavefront's sums by distance
//     in LDS; at the end distances of one bucket are summed with a segmented scan
//     over the lanes.  One row of sums per work-group goes to memory; all in a
//     fixed order.

#include <algorithm>
#include <cmath>

#include "xattn.h"

namespace {

constexpr int XQB = 128;  // rows (queries or keys) of a work-group

// Work-group w of n -> (row block, batch * head): as attn_block, or, with `causal`, the
// first row block of every head, then the second of every head, and so on (those with
// the most work first).  Work-groups go round the CUs, and with a head's row blocks in
// a row a CU got the same one of every head: 13 x 16 heads of 387 (with a bias) were as
// slow as without `causal`, forward 25.5 -> 19.7 us, dQ 58.6 -> 41.2, dK and dV 45.4 ->
// 31.7 in this order.  (A head stays on one XCD where the heads are a multiple of 8.)
__device__ __forceinline__ void x_block(const XAttnArgs& a, int w, int n, int nq, int& rb,
                                        int& bh) {
  if (a.causal) {
    const int heads = n / nq;
    rb = w / heads;
    bh = w % heads;
  } else {
    attn_block(w, n, nq, rb, bh);
  }
}

__device__ __forceinline__ int x_dist_n(const XAttnArgs& a) { return 2 * (a.reach + XPAD) + 1; }

// An index into that table, told to be one: only then do the reads' offsets go into
// the instructions.
__device__ __forceinline__ int x_idx(int i) { return i & 0x1fff; }

// The bias of head h by distance, -(reach + XPAD) .. reach + XPAD, in units of
// log2.
__device__ __forceinline__ void x_fill_dist(const XAttnArgs& a, int h, float* dist) {
  const int n = x_dist_n(a), mid = n >> 1;
  for (int e = threadIdx.x; e < n; e += 256)
    dist[e] = a.table[(int64_t)x_bucket(a, e - mid) * a.H + h] * XLOG2E;
}

// Clears the rows of a block's K and V tiles whose key is hidden (word: the keys
// that are not).
template <typename T>
__device__ __forceinline__ void x_clear_hidden(char* kv, uint64_t word) {
  constexpr int CPR = XT<T>::CPR, N = 2 * XKT * CPR;
#pragma unroll
  for (int i = 0; i < N / 256; ++i) {
    const int ch = threadIdx.x + 256 * i;
    if (!((word >> ((ch / CPR) & (XKT - 1))) & 1)) *(u32x4_t*)(kv + 16 * ch) = zero4();
  }
}

// The blocks [first, last) of a pass over the keys, with the first of them on its way
// into stage 0: block `first` is requested before the mask says whether it holds a key (it nearly
// always does), so that the two latencies overlap.  Returns the first block.
template <typename T>
__device__ __forceinline__ int x_start(const XAttnArgs& a, int b, const T* K, const T* V, int lim,
                                       int first, int last, char* kv, int wave, int lane,
                                       KeyBlocks<XKT>& blocks) {
  constexpr int TILE = XKT * XT<T>::ROWB;
  blocks.init(a.mask ? a.mask + (int64_t)b * a.Sk : nullptr, lim, last, lane);
  if (first >= last) return last;
  x_dma<T, XKT, 4>(K, a.sk[1], first * XKT, lim, kv, wave, lane);
  x_dma<T, XKT, 4>(V, a.sv[1], first * XKT, lim, kv + TILE, wave, lane);
  blocks.load(first);
  const int kb = blocks.next(first);
  if (kb > first) wait_all();  // (each wavefront writes its own rows of the tiles)
  if (kb > first && kb < last) {
    x_dma<T, XKT, 4>(K, a.sk[1], kb * XKT, lim, kv, wave, lane);
    x_dma<T, XKT, 4>(V, a.sv[1], kb * XKT, lim, kv + TILE, wave, lane);
  }
  return kb;
}

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
// KS = 2: two wavefronts share 32 queries, one with the first 32 keys of each block and
// one with the others, and are joined at the end; a work-group has 64 queries then.
template <typename T, bool BIAS, int KS>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) void xattn_fwd_kernel(XAttnArgs a) {
  constexpr int TILE = XKT * XT<T>::ROWB, QB = XQB / KS, QW = 4 / KS;
  extern __shared__ __attribute__((aligned(1024))) char lds[];  // [2][K, V], dist
  float* dist = (float*)(lds + 4 * TILE);

  int qb, bh;
  const int nq = (a.Sq + QB - 1) / QB;
  x_block(a, blockIdx.x, gridDim.x, nq, qb, bh);
  if (a.causal) qb = nq - 1 - qb;
  const int b = bh / a.H, h = bh % a.H, g = h / a.rep;
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, rr = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q0 = qb * QB + wave % QW * 32, ks = wave / QW;
  const int qp = x_q_pos(a, b);
  const int p0 = q0 + qp;  // position of the wavefront's first query
  const T* K = (const T*)a.k + b * a.sk[0] + g * a.sk[2];
  const T* V = (const T*)a.v + b * a.sv[0] + g * a.sv[2];
  const int lim =
      a.causal ? max(0, min(a.Sk, min(qb * QB + QB, a.Sq) + qp)) : a.Sk;

  const typename XT<T>::Frag qf =
      x_frag((const T*)a.q + b * a.sq[0] + (int64_t)(q0 + rr) * a.sq[1] + h * a.sq[2],
             q0 + rr < a.Sq, hf);
  KeyBlocks<XKT> blocks;
  int kb = x_start(a, b, K, V, lim, 0, (lim + XKT - 1) / XKT, lds, wave, lane, blocks);
  float far_l = 0.0f, far_r = 0.0f;
  const int mid = a.reach + XPAD;
  if constexpr (BIAS) {
    x_fill_dist(a, h, dist);
    far_l = a.table[(int64_t)x_bucket(a, -a.reach) * a.H + h] * XLOG2E;
    far_r = a.table[(int64_t)x_bucket(a, a.reach) * a.H + h] * XLOG2E;
  }

  float m = -INFINITY, lsum = 0.0f;
  f32x16_t acc[2] = {zero16(), zero16()};
  for (int st = 0; kb < blocks.nblk; st ^= 1) {
    const uint64_t word = blocks.word(kb);
    const uint64_t hidden = blocks.in_range(kb) & ~word;
    const int kn = blocks.next(kb + 1);
    wait_all();
    __syncthreads();
    char* kv = lds + st * 2 * TILE;
    if (kn < blocks.nblk) {
      char* nkv = lds + (st ^ 1) * 2 * TILE;
      x_dma<T, XKT, 4>(K, a.sk[1], kn * XKT, lim, nkv, wave, lane);
      x_dma<T, XKT, 4>(V, a.sv[1], kn * XKT, lim, nkv + TILE, wave, lane);
    }
    if (hidden) {
      x_clear_hidden<T>(kv, word);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2 / KS; ++i) {
      const int sub = KS == 2 ? ks : i;
      const int k0 = kb * XKT + 32 * sub;
      const uint32_t rows = (uint32_t)(word >> (32 * sub));
      if (rows == 0 || q0 >= a.Sq || (a.causal && k0 > p0 + 31)) continue;
      f32x16_t s = x_mma_rows(kv, 32 * sub, qf, zero16(), lane);
      const bool full = rows == 0xffffffffu && (!a.causal || k0 + 31 <= p0);
      const bool near = BIAS && k0 + 31 - p0 > -a.reach && k0 - p0 - 31 < a.reach;
      const float far = !BIAS ? 0.0f : k0 > p0 ? far_r : far_l;  // (of a tile that is not near)
      // Scores in units of log2: s * mul + add, masked; either in one step inside
      // the exponent (a tile with one bias and no hidden key) or here.
      float mul = a.c, add = far, mblk = -INFINITY;
      if (full && !near) {
#pragma unroll
        for (int r = 0; r < 16; ++r) mblk = fmaxf(mblk, s[r]);
        mblk = fmaf(mblk, mul, add);
      } else {
        uint32_t bits = x_lane_bits(rows, hf);
        if (a.causal) bits &= x_upto(p0 + rr - k0 - 4 * hf);
        if (near) {
          const float* d = dist + x_idx(k0 + 4 * hf - p0 - rr + mid);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], mul, d[8 * (r >> 2) + (r & 3)]);
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
      // The offset of the exponents moves only when a tile's maximum exceeds it
      // by more than 8, so most tiles leave the output accumulators alone.
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
      x_mma_cols<T>(kv + TILE, 32 * sub, s, acc, lane);
    }
    kb = kn;
  }
  const HalfPair lp = half_pair(lsum);
  float ltot = lp.x + lp.y;
  if constexpr (KS == 2) {
    // [wavefront][output, offset, sum][lane], in the place of the ring
    float* p = (float*)lds + wave % QW * 34 * 64 + lane;
    __syncthreads();
    if (ks == 1) {
#pragma unroll
      for (int r = 0; r < 32; ++r) p[r * 64] = acc[r >> 4][r & 15];
      p[32 * 64] = m;
      p[33 * 64] = ltot;
    }
    __syncthreads();
    if (ks == 1) return;
    const float m1 = p[32 * 64], top = fmaxf(m, m1), off = top == -INFINITY ? 0.0f : top;
    const float f0 = __builtin_amdgcn_exp2f(m - off), f1 = __builtin_amdgcn_exp2f(m1 - off);
#pragma unroll
    for (int r = 0; r < 32; ++r)
      acc[r >> 4][r & 15] = fmaf(p[r * 64], f1, acc[r >> 4][r & 15] * f0);
    ltot = fmaf(p[33 * 64], f1, ltot * f0);
    m = top;
  }
  if (a.lse && hf == 0 && q0 + rr < a.Sq)
    a.lse[((int64_t)b * a.H + h) * a.Sq + q0 + rr] =
        ltot == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(ltot)) * XLN2;
  if constexpr (KS == 1) __syncthreads();  // the ring becomes the output staging area
  x_store<T>(acc, ltot == 0.0f ? 0.0f : 1.0f / ltot, (T*)(lds + (KS == 2 ? 2 * 34 * 256 : 0)) + wave * 32 * XT<T>::LD,
             (T*)a.out + b * a.so[0] + h * a.so[2], a.so[1], q0, a.Sq);
}

// ---------------------------------------------------------------------------
// Backward, dQ and the bias gradient.  RED: D is formed from P and dP in a pass of
// its own over the keys.  Else it starts as D' = rowsum(dO * out); on bf16 out's
// rounding makes the rows of P (dP - D') sum to D - D' instead of zero, which is of
// the size of dS where few keys take most of P: that sum and P K are kept as well,
// and dQ and D corrected at the end.
// ---------------------------------------------------------------------------

// The sums of a 32 x 32 accumulator along its diagonals (lane = query, registers =
// keys, x_acc order): lane l gets the sum over all (key, query) with key - query =
// 31 - l, lane 63 zero.  Going through the keys upwards, the running sums move one
// lane up per key, as the diagonals do; half a register at a time with zeros above,
// so that diagonals which leave query 31 go on in the upper lanes.  96 vector
// instructions and no LDS: adding the 1024 values to 63 sums in LDS took 190 cycles
// per atomic of a wavefront (the dQ kernel of 32 x 512 tokens and 12 heads 315 us).
__device__ __forceinline__ float x_diagonals(const f32x16_t& s, int lane) {
  // Keys 0-15 and 16-31 in a chain each (a lane move has to wait for the addition
  // before it), joined by moving the first one's sums 16 lanes up.
  float d[2] = {0.0f, 0.0f};
  auto step = [](float& d, uint32_t v) {
    const float up = __uint_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_uint(d), 0x138 /* wave_shr:1 */, 0xf, 0xf, true));
    d = up + __uint_as_float(v);
  };
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t hi[2][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(s[8 * c + 4 * i + e]), 0u, false,
                                                        false);
        step(d[c], r[0]);
        hi[c][e] = r[1];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < 2; ++c) step(d[c], hi[c][e]);
  }
  const float up = __shfl_up(d[0], 16, 64);
  return lane < 16 ? d[1] : d[1] + up;
}

// Adds v of lane l, the sum at distance rel0 + l (lanes from n on have none), to
// its bucket.  Buckets are runs of distances: each run is summed into its last lane.
__device__ __forceinline__ void x_add_buckets(const XAttnArgs& a, float v, int rel0, int n, int lane,
                                              float* bsum) {
  const int bk = lane < n ? x_bucket(a, rel0 + lane) : -1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const float u = __shfl_up(v, o, 64);
    const int ub = __shfl_up(bk, o, 64);
    if (lane >= o && ub == bk) v += u;
  }
  const int nb = __shfl_down(bk, 1, 64);
  if (bk >= 0 && (lane == 63 || nb != bk)) bsum[bk] += v;
  lds_wait();
  __builtin_amdgcn_wave_barrier();
}

// A query that sees no key adds nothing, whatever its dO holds (0 * NaN is NaN): its
// fragment becomes zeros.  lse2: infinite for such a row.
template <typename F>
__device__ __forceinline__ void x_drop_empty(F& dof, float lse2) {
  const bool empty = lse2 == INFINITY;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(dof) / 16); ++i) {
    const u32x4_t w = __builtin_bit_cast(u32x4_t, dof.f[i]);
    dof.f[i] = __builtin_bit_cast(decltype(dof.f[0] + dof.f[0]), empty ? zero4() : w);
  }
}

// KS = 2: two wavefronts share 32 queries, one with the first 32 keys of each block
// and one with the others, and add up at the end; a work-group has 64 queries then.
template <typename T, bool BIAS, bool RED, int KS>
__device__ __forceinline__ void x_dq(const XAttnArgs& a, int w, int n, char* lds) {
  constexpr int TILE = XKT * XT<T>::ROWB, QB = XQB / KS, QW = 4 / KS;
  // [2][K, V]; with a bias: dist, the wavefronts' sums by distance [4][nd] and by
  // bucket [4][nb]
  constexpr bool FIX = sizeof(T) == 2 && !RED;
  float* dist = (float*)(lds + 4 * TILE);
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, rr = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* diag = nullptr;
  float* bsum = nullptr;
  const int nd = x_dist_n(a);
  if constexpr (BIAS) {
    float* p = dist + ((x_dist_n(a) + 3) & ~3);
    diag = p + wave * nd;
    bsum = p + 4 * nd + wave * a.nb;
  }

  int qb, bh;
  const int nq = (a.Sq + QB - 1) / QB;
  x_block(a, w, n, nq * a.dq_splits, qb, bh);
  const int split = qb % a.dq_splits;
  qb /= a.dq_splits;
  if (a.causal) qb = nq - 1 - qb;
  const int b = bh / a.H, h = bh % a.H, g = h / a.rep;
  const int q0 = qb * QB + wave % QW * 32, q = q0 + rr, ks = wave / QW;
  const bool qv = q < a.Sq;
  const int qp = x_q_pos(a, b);
  const int p0 = q0 + qp;
  const T* K = (const T*)a.k + b * a.sk[0] + g * a.sk[2];
  const T* V = (const T*)a.v + b * a.sv[0] + g * a.sv[2];
  const int lim =
      a.causal ? max(0, min(a.Sk, min(qb * QB + QB, a.Sq) + qp)) : a.Sk;

  const int nblk = (lim + XKT - 1) / XKT, per = (nblk + a.dq_splits - 1) / a.dq_splits;
  const int first = min(nblk, split * per), last = min(nblk, first + per);

  const typename XT<T>::Frag qf = x_frag(
      (const T*)a.q + b * a.sq[0] + (int64_t)q * a.sq[1] + h * a.sq[2], qv, hf);
  typename XT<T>::Frag dof = x_frag(
      (const T*)a.dout + b * a.sdo[0] + (int64_t)q * a.sdo[1] + h * a.sdo[2], qv, hf);
  const int64_t row = ((int64_t)b * a.H + h) * a.Sq + q;
  // No key, and lanes behind the last query (whose sums by bucket, over all lanes, a bias
  // beyond 2^128 would make NaN): P = exp2(s - inf) = 0.
  float lse2 = qv ? a.lse[row] * XLOG2E : INFINITY;
  if (lse2 == -INFINITY) lse2 = INFINITY;
  float D = 0.0f;
  typename XT<T>::Frag of;
  if constexpr (!RED)
    of = x_frag((const T*)a.o + b * a.so[0] + (int64_t)q * a.so[1] + h * a.so[2], qv, hf);
  // (the first keys are on their way while D and the tables are formed)
  KeyBlocks<XKT> blocks;
  int kb = x_start(a, b, K, V, lim, first, last, lds, wave, lane, blocks);
  if constexpr (!RED) {
    x_drop_empty(dof, lse2);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(of) / 16); ++i)
#pragma unroll
      for (int e = 0; e < 16 / (int)sizeof(T); ++e) D += (float)dof.f[i][e] * (float)of.f[i][e];
    const HalfPair pr = half_pair(D);
    D = pr.x + pr.y;
  }
  float far_l = 0.0f, far_r = 0.0f;      // far bias
  float gfar_l = 0.0f, gfar_r = 0.0f;    // far sums of dS
  const int mid = a.reach + XPAD;
  if constexpr (BIAS) {
    x_fill_dist(a, h, dist);
    far_l = a.table[(int64_t)x_bucket(a, -a.reach) * a.H + h] * XLOG2E;
    far_r = a.table[(int64_t)x_bucket(a, a.reach) * a.H + h] * XLOG2E;
    for (int i = lane; i < nd; i += 64) diag[i] = 0.0f;
    for (int i = lane; i < a.nb; i += 64) bsum[i] = 0.0f;
  }
  if constexpr (RED) x_drop_empty(dof, lse2);

  // Sum of a value over the wavefronts that share the queries (in the ring's place,
  // after the pass's last barrier), the same in both.
  auto join = [&](float v) {
    if constexpr (KS == 1) return v;
    float* p = (float*)lds + lane;
    p[wave * 64] = v;
    __syncthreads();
    v = p[wave % QW * 64] + p[(wave % QW + QW) * 64];
    __syncthreads();
    return v;
  };
  f32x16_t dq[2] = {zero16(), zero16()};
  f32x16_t pk[2] = {zero16(), zero16()};  // FIX: P K
  float rsum = 0.0f;                      // FIX: row sum of dS; RED: of P
  auto sweep = [&](auto sum_d) {
    constexpr bool SUM_D = decltype(sum_d)::value;
    for (int st = 0; kb < blocks.nblk; st ^= 1) {
      const uint64_t word = blocks.word(kb);
      const uint64_t hidden = blocks.in_range(kb) & ~word;
      const int kn = blocks.next(kb + 1);
      wait_all();
      __syncthreads();
      char* kv = lds + st * 2 * TILE;
      if (kn < blocks.nblk) {
        char* nkv = lds + (st ^ 1) * 2 * TILE;
        x_dma<T, XKT, 4>(K, a.sk[1], kn * XKT, lim, nkv, wave, lane);
        x_dma<T, XKT, 4>(V, a.sv[1], kn * XKT, lim, nkv + TILE, wave, lane);
      }
      if (hidden) {
        x_clear_hidden<T>(kv, word);
        __syncthreads();
      }
#pragma unroll
      for (int i = 0; i < 2 / KS; ++i) {
        const int sub = KS == 2 ? ks : i;
        const int k0 = kb * XKT + 32 * sub;
        const uint32_t rows = (uint32_t)(word >> (32 * sub));
        if (rows == 0 || q0 >= a.Sq || (a.causal && k0 > p0 + 31)) continue;
        f32x16_t s = x_mma_rows(kv, 32 * sub, qf, zero16(), lane);
        // (RED: both passes form the same dP, so that the matrix core's rounding,
        // which is one-sided, cancels in dP - D; from an accumulator that starts at
        // -D the sums over a bucket of 3 million pairs were off by 1e-6)
        f32x16_t dp = x_mma_rows(kv + TILE, 32 * sub, dof, splat16(RED ? 0.0f : -D), lane);
        const bool full = rows == 0xffffffffu && (!a.causal || k0 + 31 <= p0);
        const bool near = BIAS && k0 + 31 - p0 > -a.reach && k0 - p0 - 31 < a.reach;
        if (near) {
          const float* d = dist + x_idx(k0 + 4 * hf - p0 - rr + mid);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, d[8 * (r >> 2) + (r & 3)]) - lse2);
        } else {
          const float add = (!BIAS ? 0.0f : k0 > p0 ? far_r : far_l) - lse2;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, add));
        }
        if (!full) {
          uint32_t bits = x_lane_bits(rows, hf);
          if (a.causal) bits &= x_upto(p0 + rr - k0 - 4 * hf);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = x_or_zero(s[r], bits, r);
        }
        if constexpr (SUM_D) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            D = fmaf(s[r], dp[r], D);
            rsum += s[r];
          }
        } else {
          if constexpr (FIX) x_mma_cols<T>(kv, 32 * sub, s, pk, lane);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[r] *= RED ? dp[r] - D : dp[r];  // dS
            if constexpr (FIX) rsum += s[r];
          }
          // (bf16: the product first, whose rounded copy frees the registers that the
          // diagonals' moves overwrite)
          if constexpr (sizeof(T) == 2) x_mma_cols<T>(kv, 32 * sub, s, dq, lane);
          if constexpr (BIAS) {
            if (a.dtable && near) {
              const float v = x_diagonals(s, lane);
              if (lane < 63) diag[k0 - p0 + 31 - lane + mid] += v;
            } else if (a.dtable) {
              float t = s[0];
#pragma unroll
              for (int r = 1; r < 16; ++r) t += s[r];
              if (k0 > p0) gfar_r += t;
              else gfar_l += t;
            }
          }
          if constexpr (sizeof(T) == 4) x_mma_cols<T>(kv, 32 * sub, s, dq, lane);
        }
      }
      kb = kn;
    }
    __syncthreads();  // (the next pass, or the output, takes the ring)
  };
  if constexpr (RED) {
    sweep(std::true_type());
    // Over the sum of these P, which the log-sum-exp's rounding leaves off 1: the
    // rows of dS then sum to zero to the last bits, as far buckets of long rows
    // need.
    const HalfPair pr = half_pair(D), ps = half_pair(rsum);
    const float top = join(pr.x + pr.y), total = join(ps.x + ps.y);
    D = total == 0.0f ? 0.0f : top / total;
    kb = x_start(a, b, K, V, lim, first, last, lds, wave, lane, blocks);
  }
  sweep(std::false_type());
  if constexpr (KS == 2) {
    // [wavefront][dq, P K][register][lane]
    float* p = (float*)lds + wave % QW * (FIX ? 64 : 32) * 64 + lane;
    if (ks == 1) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[(16 * t + r) * 64] = dq[t][r];
          if constexpr (FIX) p[(32 + 16 * t + r) * 64] = pk[t][r];
        }
    }
    __syncthreads();
    if (ks == 0) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dq[t][r] += p[(16 * t + r) * 64];
          if constexpr (FIX) pk[t][r] += p[(32 + 16 * t + r) * 64];
        }
    }
    __syncthreads();
  }
  if constexpr (FIX) {
    const HalfPair pr = half_pair(rsum);
    const float off = join(pr.x + pr.y);
    if (a.dq_splits > 1) {
      rsum = off;
    } else {
      D += off;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[t][r] = fmaf(-off, pk[t][r], dq[t][r]);
    }
  }
  if (hf == 0 && qv && ks == 0 && split == 0) a.dsum[row] = D;
  if constexpr (!RED) {
    if (a.dq_splits > 1) {
      if (ks == 1) return;
      constexpr int ROW = sizeof(T) == 2 ? 132 : 64;
      float* to = a.part + (((int64_t)split * a.B + b) * a.H + h) * a.Sq * ROW;
      float* stage = (float*)lds + wave * 32 * XT<float>::LD;
      x_store<float>(dq, 1.0f, stage, to, ROW, q0, a.Sq);
      if constexpr (FIX) {
        lds_wait();
        __builtin_amdgcn_wave_barrier();
        x_store<float>(pk, 1.0f, stage, to + XHD, ROW, q0, a.Sq);
        if (hf == 0 && qv) to[(int64_t)q * ROW + 2 * XHD] = rsum;
      }
      return;
    }
  }
  if constexpr (BIAS) {
    if (a.dtable) {
      const float* all = diag - wave * nd;  // (after the pass's last barrier)
      for (int e0 = 64 * wave; e0 < nd; e0 += 256) {
        const int e = e0 + lane;
        const float v =
            e < nd ? (all[e] + all[nd + e]) + (all[2 * nd + e] + all[3 * nd + e]) : 0.0f;
        x_add_buckets(a, v, e0 - mid, nd - e0, lane, bsum);
      }
      gfar_l = wave_sum(gfar_l);
      gfar_r = wave_sum(gfar_r);
      if (lane == 0) {
        bsum[x_bucket(a, -a.reach)] += gfar_l;
        bsum[x_bucket(a, a.reach)] += gfar_r;
      }
      __syncthreads();
      const float* p = bsum - wave * a.nb;
      for (int i = tid; i < a.nb; i += 256)
        a.tpart[(((int64_t)b * a.H + h) * nq + qb) * a.nb + i] =
            (p[i] + p[a.nb + i]) + (p[2 * a.nb + i] + p[3 * a.nb + i]);
    }
  }
  if (ks == 0)
    x_store<T>(dq, a.scale, (T*)lds + wave * 32 * XT<T>::LD,
               (T*)a.dq + b * a.sdq[0] + h * a.sdq[2], a.sdq[1], q0, a.Sq);
}
template <typename T, bool BIAS, bool RED, int KS>
__global__ __launch_bounds__(256, RED ? 3 : 2) void xattn_dq_kernel(XAttnArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  x_dq<T, BIAS, RED, KS>(a, blockIdx.x, gridDim.x, lds);
}

// dQ and D from the splits, in order: 16 threads to a query, 4 columns each.
template <typename T>
__global__ __launch_bounds__(256) void xattn_dq_sum_kernel(XAttnArgs a) {
  constexpr bool FIX = sizeof(T) == 2;
  constexpr int ROW = FIX ? 132 : 64;
  const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), n = (int64_t)a.B * a.H * a.Sq;
  if (row >= n) return;
  const int c = (threadIdx.x & 15) * 4;
  const float* p = a.part + row * ROW;
  f32x4_t dq = {0.0f, 0.0f, 0.0f, 0.0f}, pk = dq;
  float off = 0.0f;
#pragma unroll 4
  for (int i = 0; i < a.dq_splits; ++i, p += n * ROW) {
    dq += *(const f32x4_t*)(p + c);
    if constexpr (FIX) {
      pk += *(const f32x4_t*)(p + XHD + c);
      off += p[2 * XHD];
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) dq[e] = (FIX ? fmaf(-off, pk[e], dq[e]) : dq[e]) * a.scale;
  const int q = (int)(row % a.Sq), bh = (int)(row / a.Sq), b = bh / a.H, h = bh % a.H;
  T* to = (T*)a.dq + b * a.sdq[0] + (int64_t)q * a.sdq[1] + h * a.sdq[2] + c;
  if constexpr (FIX) {
    *(u32x2_t*)to = u32x2_t{pack_bf16x2(dq[0], dq[1]), pack_bf16x2(dq[2], dq[3])};
    if (c == 0) a.dsum[row] += off;
  } else {
    *(f32x4_t*)to = dq;
  }
}

// ---------------------------------------------------------------------------
// Backward, dK and dV: wavefront = 32 keys, loops over blocks of QB queries of
// every query head that shares the keys.  Work-groups from n_kv on sum the bias
// gradient: one to eight buckets of a head.
// ---------------------------------------------------------------------------
template <typename T> constexpr int x_qb() { return sizeof(T) == 2 ? 128 : 64; }
constexpr int XOWN = 256;  // most queries (of all its heads) whose D a work-group forms
// LDS: [2][Q, dO], per stage lse and -D of QB rows, a word per wavefront; with a bias
// its table by distance follows.
template <typename T> constexpr int kv_lds() {
  return 4 * x_qb<T>() * XT<T>::ROWB + 4 * x_qb<T>() * 4 + 16;
}

// The bias gradient of 8 buckets of a head: 32 rows of bucket sums at a time, in a fixed
// order.  (With a work-group to each bucket and head they took turns with those of dK and
// dV for the CUs' LDS: 32 x 12 heads of 512 tokens 78.5 -> 77.3 us, 13 x 16 of 387 31.2 ->
// 30.7.)
__device__ __forceinline__ void x_dtable_sum(const XAttnArgs& a, int w, float* red) {
  const int per = (a.nb + 7) / 8, h = w / per, c = w % per * 8 + (threadIdx.x & 7);
  const int qb = XQB / a.dq_ks, nq = (a.Sq + qb - 1) / qb, rows = a.B * nq;
  const int lane = threadIdx.x & 63;
  float t = 0.0f;
  if (c < a.nb) {
#pragma unroll 4
    for (int i = threadIdx.x >> 3; i < rows; i += 32)
      t += a.tpart[((int64_t)(i / nq * a.H + h) * nq + i % nq) * a.nb + c];
  }
#pragma unroll
  for (int o = 8; o < 64; o <<= 1) t += __shfl_xor(t, o, 64);
  if (lane < 8) red[(threadIdx.x >> 6) * 8 + lane] = t;
  __syncthreads();
  if (threadIdx.x < 8 && c < a.nb)
    a.dtable[(int64_t)c * a.H + h] =
        (red[threadIdx.x] + red[8 + threadIdx.x]) + (red[16 + threadIdx.x] + red[24 + threadIdx.x]);
}

// D of the x_qb<T>() queries of head h from q0 on, into own (0 behind the last, and where
// no key is seen): fp32 rowsum(dO * out); bf16 sum(P dP) / sum(P) over all keys, since out's
// rounding would go into dK (9 queries over 17 keys: its error 1.6 times that of fp32 sums
// rounded once).
// With a bias, dist and far_l, far_r are head h's.
template <typename T, bool BIAS>
__device__ __forceinline__ void x_own_d(const XAttnArgs& a, int b, int g, int h, int q0, int qp,
                                        char* ring, float* own, const float* dist, float far_l,
                                        float far_r, int wave, int lane) {
  constexpr int QB = x_qb<T>(), TILE = XKT * XT<T>::ROWB;
  const int hf = lane >> 5, rr = lane & 31, w0 = q0 + 32 * wave, q = w0 + rr;
  const bool qv = q < a.Sq && 32 * wave < QB;
  const typename XT<T>::Frag dof = x_frag(
      (const T*)a.dout + b * a.sdo[0] + (int64_t)q * a.sdo[1] + h * a.sdo[2], qv, hf);
  float lse2 = qv ? a.lse[((int64_t)b * a.H + h) * a.Sq + q] * XLOG2E : INFINITY;
  if (lse2 == -INFINITY) lse2 = INFINITY;
  float D = 0.0f;
  if constexpr (sizeof(T) == 4) {
    const typename XT<T>::Frag of = x_frag(
        (const T*)a.o + b * a.so[0] + (int64_t)q * a.so[1] + h * a.so[2], qv, hf);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) D += dof.f[i][e] * of.f[i][e];
    const HalfPair pr = half_pair(D);
    D = pr.x + pr.y;
  } else {
    const T* K = (const T*)a.k + b * a.sk[0] + g * a.sk[2];
    const T* V = (const T*)a.v + b * a.sv[0] + g * a.sv[2];
    const int p0 = w0 + qp;
    const int lim = a.causal ? max(0, min(a.Sk, min(q0 + QB, a.Sq) + qp)) : a.Sk;
    const typename XT<T>::Frag qf = x_frag(
        (const T*)a.q + b * a.sq[0] + (int64_t)q * a.sq[1] + h * a.sq[2], qv, hf);
    KeyBlocks<XKT> blocks;
    int kb = x_start(a, b, K, V, lim, 0, (lim + XKT - 1) / XKT, ring, wave, lane, blocks);
    float rsum = 0.0f;
    for (int st = 0; kb < blocks.nblk; st ^= 1) {
      const uint64_t word = blocks.word(kb);
      const uint64_t hidden = blocks.in_range(kb) & ~word;
      const int kn = blocks.next(kb + 1);
      wait_all();
      __syncthreads();
      char* kv = ring + st * 2 * TILE;
      if (kn < blocks.nblk) {
        char* nkv = ring + (st ^ 1) * 2 * TILE;
        x_dma<T, XKT, 4>(K, a.sk[1], kn * XKT, lim, nkv, wave, lane);
        x_dma<T, XKT, 4>(V, a.sv[1], kn * XKT, lim, nkv + TILE, wave, lane);
      }
      if (hidden) {
        x_clear_hidden<T>(kv, word);
        __syncthreads();
      }
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const int k0 = kb * XKT + 32 * sub;
        const uint32_t rows = (uint32_t)(word >> (32 * sub));
        if (rows == 0 || w0 >= a.Sq || (a.causal && k0 > p0 + 31)) continue;
        f32x16_t s = x_mma_rows(kv, 32 * sub, qf, zero16(), lane);
        const f32x16_t dp = x_mma_rows(kv + TILE, 32 * sub, dof, zero16(), lane);
        uint32_t bits = x_lane_bits(rows, hf);
        if (a.causal) bits &= x_upto(p0 + rr - k0 - 4 * hf);
        if (BIAS && k0 + 31 - p0 > -a.reach && k0 - p0 - 31 < a.reach) {
          const float* d = dist + x_idx(k0 + 4 * hf - p0 - rr + a.reach + XPAD);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, d[8 * (r >> 2) + (r & 3)]) - lse2);
        } else {
          const float add = (!BIAS ? 0.0f : k0 > p0 ? far_r : far_l) - lse2;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, add));
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = x_or_zero(s[r], bits, r);
          D = fmaf(s[r], dp[r], D);
          rsum += s[r];
        }
      }
      kb = kn;
    }
    __syncthreads();  // (the next queries' blocks, or the queries themselves, take the ring)
    const HalfPair pr = half_pair(D), ps = half_pair(rsum);
    const float top = pr.x + pr.y, total = ps.x + ps.y;
    D = total == 0.0f ? 0.0f : top / total;
  }
  if (hf == 0 && 32 * wave < QB) own[32 * wave + rr] = lse2 == INFINITY ? 0.0f : D;
}

// The first query from row0 on, of the next 256, that some head of key head g has a
// log-sum-exp for: with `causal`, those further on that meet the work-group's keys are
// behind one of them.  (Loads without conditions, so that they are on their way together.)
__device__ __forceinline__ int x_first_seen(const XAttnArgs& a, int b, int g, int row0, int lane) {
  bool none[4] = {true, true, true, true};
  int at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) at[j] = min(row0 + 64 * j + lane, a.Sq - 1);
  const float* l = a.lse + ((int64_t)b * a.H + g * a.rep) * a.Sq;
#pragma unroll 4
  for (int h = 0; h < a.rep; ++h, l += a.Sq) {
#pragma unroll
    for (int j = 0; j < 4; ++j) none[j] &= l[at[j]] == -INFINITY;
  }
  int n = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint64_t seen = ~__ballot(none[j]);
    if (n == 64 * j) n += seen ? __builtin_ctzll(seen) : 64;
  }
  return row0 + n;
}

// QS = 2: two wavefronts share 32 keys, each with every other tile of queries, and add
// up at the end; a work-group has 64 keys then.
// CAUSAL: a.causal may be set.  OWN_D: D is formed here, for all queries of the work-group,
// and not read.
template <typename T, bool BIAS, int QS, bool CAUSAL, bool OWN_D>
__device__ __forceinline__ void x_dkdv(const XAttnArgs& a, int w, int n_kv, char* lds) {
  constexpr int QB = x_qb<T>(), TILE = QB * XT<T>::ROWB, KB = XQB / QS, KW = 4 / QS;
  const bool causal = CAUSAL && a.causal;
  float* rowv = (float*)(lds + 4 * TILE);
  float* own = (float*)(lds + kv_lds<T>());  // OWN_D: [iteration][QB]
  float* dist = own + (OWN_D ? XOWN : 0);
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, rr = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int kblk, bg;
  x_block(a, w, n_kv, (a.Sk + KB - 1) / KB * a.kv_splits, kblk, bg);
  const int split = kblk % a.kv_splits;
  kblk /= a.kv_splits;
  const int b = bg / a.G, g = bg % a.G;
  const int k0 = kblk * KB + wave % KW * 32, key = k0 + rr, qs = wave / KW;
  const int qp = x_q_pos(a, b);
  // Queries from q_first on see a key of this work-group, those before it none.
  const int q_first = causal ? max(0, kblk * KB - qp) : 0;
  const int qb0 = q_first / QB, nqb = max(0, (a.Sq + QB - 1) / QB - qb0);
  const int it0 = split * a.kv_chunk;
  int n_it = min(nqb * a.rep, it0 + a.kv_chunk);
  if (split > 0 && it0 >= n_it) return;  // (the sum knows which splits there are)
  // A key that the mask hides, or no query sees, may hold anything: its rows are not
  // read, and a work-group without another key only writes zeros.  (The rows wait for
  // the mask this way; but few queries make this a copy of K and V to dK and dV: 32 x
  // 16 heads of 128 queries and 512 keys, half of them hidden, 40 -> 36 us.)
  const int bit = key >= a.Sk ? 0 : a.mask ? a.mask[(int64_t)b * a.Sk + key] : 1;
  // The queries before the first visible key see none and may hold anything: their rows
  // are not read.  (Without `causal` the queries of a sequence without a key are not gone
  // through at all.)
  int q_seen = !causal || nqb == 0 ? 0 : a.mask ? x_first_seen(a, b, g, qb0 * QB, lane) : -qp;
  if (causal) asm volatile("" : "+v"(q_seen));  // (in a vector register: scalar ones are short)
  const bool kvalid = bit != 0 && (!causal || key - qp < a.Sq);
  const bool all_valid = __all(kvalid), any_valid = __any(kvalid);
  const uint32_t kbits = kvalid ? 0xffffffffu : 0u;
  if (a.mask) {
    int* any = (int*)(lds + kv_lds<T>() - 16);
    any[wave] = any_valid;
    __syncthreads();
    if (!(any[0] | any[1] | any[2] | any[3])) n_it = it0;
  }
  const T* Q = (const T*)a.q + b * a.sq[0];
  const T* dO = (const T*)a.dout + b * a.sdo[0];

  auto head = [&](int it) { return g * a.rep + it / nqb; };
  auto qrow = [&](int it) { return (qb0 + it % nqb) * QB; };
  auto dma = [&](int it, char* to) {
    const int h = head(it), r = qrow(it);
    x_dma<T, QB, 4, false, CAUSAL>(Q + h * a.sq[2], a.sq[1], r, a.Sq, to, wave, lane, q_seen - r);
    x_dma<T, QB, 4, false, CAUSAL>(dO + h * a.sdo[2], a.sdo[1], r, a.Sq, to + TILE, wave, lane,
                                 q_seen - r);
  };
  // Thread t < QB carries lse (in log2 units) of row t of a block, the next QB
  // threads -D; rows that are not there have P = exp2(s - inf) = 0.
  const bool row_thread = tid < 2 * QB;
  auto row_raw = [&](int it) {
    const int r = qrow(it) + (tid & (QB - 1));
    if (!row_thread || r >= a.Sq) return tid < QB ? INFINITY : 0.0f;
    if (OWN_D && tid >= QB) return own[(it - it0) * QB + (tid & (QB - 1))];
    return (tid < QB ? a.lse : a.dsum)[((int64_t)b * a.H + head(it)) * a.Sq + r];
  };
  auto row_store = [&](float raw, int st) {
    if (row_thread)
      rowv[st * 2 * QB + tid] = tid >= QB ? -raw : raw == -INFINITY ? INFINITY : raw * XLOG2E;
  };
  float raw = 0.0f;
  const typename XT<T>::Frag kf = x_frag(
      (const T*)a.k + b * a.sk[0] + (int64_t)key * a.sk[1] + g * a.sk[2], kvalid && it0 < n_it, hf);
  const typename XT<T>::Frag vf = x_frag(
      (const T*)a.v + b * a.sv[0] + (int64_t)key * a.sv[1] + g * a.sv[2], kvalid && it0 < n_it, hf);
  if (it0 < n_it) dma(it0, lds);
  const int mid = a.reach + XPAD;
  float far_l = 0.0f, far_r = 0.0f;
  int cur_h = -1;  // whose tables are there
  auto tables = [&](int h) {
    cur_h = h;
    x_fill_dist(a, h, dist);
    far_l = a.table[(int64_t)x_bucket(a, -a.reach) * a.H + h] * XLOG2E;
    far_r = a.table[(int64_t)x_bucket(a, a.reach) * a.H + h] * XLOG2E;
  };
  if constexpr (OWN_D) {
    for (int it = it0; it < n_it; ++it) {
      if constexpr (BIAS && sizeof(T) == 2) {
        if (cur_h != head(it)) tables(head(it));
      }
      x_own_d<T, BIAS>(a, b, g, head(it), qrow(it), qp, lds + 2 * TILE, own + (it - it0) * QB, dist,
                       far_l, far_r, wave, lane);
    }
    __syncthreads();
  }
  if (it0 < n_it) {
    row_store(row_raw(it0), 0);
    if (it0 + 1 < n_it) raw = row_raw(it0 + 1);
  }
  f32x16_t dv[2] = {zero16(), zero16()}, dk[2] = {zero16(), zero16()};
  for (int it = it0; it < n_it; ++it) {
    const int st = (it - it0) & 1;
    const int h = head(it), qr = qrow(it);
    wait_all();
    __syncthreads();
    if constexpr (BIAS) {
      if (h != cur_h) {
        // (every wavefront is past its last use of the previous head's table)
        tables(h);
        __syncthreads();
      }
    }
    if (it + 1 < n_it) dma(it + 1, lds + (st ^ 1) * 2 * TILE);
    const float raw2 = it + 2 < n_it ? row_raw(it + 2) : 0.0f;
    const char* Qs = lds + st * 2 * TILE;
    const char* dOs = Qs + TILE;
    const float* lv = rowv + st * 2 * QB;
#pragma unroll
    for (int i = 0; i < QB / 32 / QS; ++i) {
      const int sub = QS == 2 ? 2 * i + qs : i;
      const int r0 = qr + 32 * sub;   // first query
      const int p0 = r0 + qp;         // its position
      if (!any_valid || r0 >= a.Sq || (causal && k0 > p0 + 31)) continue;
      f32x16_t dp;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4_t d4 = *(const f32x4_t*)(lv + QB + 32 * sub + 8 * j + 4 * hf);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * j + e] = d4[e];
      }
      f32x16_t s = x_mma_rows(Qs, 32 * sub, kf, zero16(), lane);
      dp = x_mma_rows(dOs, 32 * sub, vf, dp, lane);
      const bool full = all_valid && (!causal || k0 + 31 <= p0);
      const bool near = BIAS && k0 + 31 - p0 > -a.reach && k0 - p0 - 31 < a.reach;
      // Key rr is seen by the queries from rr + k0 - p0 on.
      uint32_t bits = kbits;
      if (causal) bits &= ~x_upto(k0 + rr - p0 - 4 * hf - 1);
      if constexpr (!BIAS) {
      } else if (near) {
        const float* d = dist + x_idx(k0 + rr - p0 - 4 * hf + mid - 27);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.c, d[27 - (8 * (r >> 2) + (r & 3))]);
      } else {
        const float far = k0 > p0 ? far_r : far_l;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.c, far);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4_t l4 = *(const f32x4_t*)(lv + 32 * sub + 8 * j + 4 * hf);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = s[4 * j + e];
          s[4 * j + e] = __builtin_amdgcn_exp2f(BIAS ? x - l4[e] : fmaf(x, a.c, -l4[e]));
        }
      }
      if (!full) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = x_or_zero(s[r], bits, r);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] *= s[r];  // dS
      x_mma_cols<T>(dOs, 32 * sub, s, dv, lane);
      x_mma_cols<T>(Qs, 32 * sub, dp, dk, lane);
    }
    if (it + 1 < n_it) row_store(raw, st ^ 1);
    raw = raw2;
  }
  __syncthreads();  // the ring becomes the output staging area
  if constexpr (QS == 2) {
    // [wavefront][dK, dV][register][lane]
    float* p = (float*)lds + wave % KW * 64 * 64 + lane;
    if (qs == 1) {
#pragma unroll
      for (int r = 0; r < 32; ++r) {
        p[r * 64] = dk[r >> 4][r & 15];
        p[(32 + r) * 64] = dv[r >> 4][r & 15];
      }
    }
    __syncthreads();
    if (qs == 0) {
#pragma unroll
      for (int r = 0; r < 32; ++r) {
        dk[r >> 4][r & 15] += p[r * 64];
        dv[r >> 4][r & 15] += p[(32 + r) * 64];
      }
    }
    __syncthreads();
    if (qs == 1) return;
  }
  if (a.kv_splits > 1) {
    float* to = a.part + ((int64_t)split * a.B * a.G + bg) * a.Sk * 2 * XHD;
    float* stage = (float*)lds + wave * 32 * XT<float>::LD;
    x_store<float>(dk, a.scale, stage, to, 2 * XHD, k0, a.Sk);
    lds_wait();
    __builtin_amdgcn_wave_barrier();
    x_store<float>(dv, 1.0f, stage, to + XHD, 2 * XHD, k0, a.Sk);
    return;
  }
  T* stage = (T*)lds + wave * 32 * XT<T>::LD;
  x_store<T>(dk, a.scale, stage, (T*)a.dk + b * a.sdk[0] + g * a.sdk[2], a.sdk[1], k0, a.Sk);
  lds_wait();
  __builtin_amdgcn_wave_barrier();
  x_store<T>(dv, 1.0f, stage, (T*)a.dv + b * a.sdv[0] + g * a.sdv[2], a.sdv[1], k0, a.Sk);
}
template <typename T, bool BIAS, int QS, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void xattn_dkdv_kernel(XAttnArgs a, int n_kv) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  if ((int)blockIdx.x < n_kv) x_dkdv<T, BIAS, QS, CAUSAL, false>(a, blockIdx.x, n_kv, lds);
  else x_dtable_sum(a, blockIdx.x - n_kv, (float*)lds);
}

// The whole backward pass in one launch: work-groups from n_kv on make dQ.
template <typename T, bool BIAS, int QS, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void xattn_bwd_kernel(XAttnArgs a, int n_kv) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  if ((int)blockIdx.x < n_kv) x_dkdv<T, BIAS, QS, CAUSAL, true>(a, blockIdx.x, n_kv, lds);
  else x_dq<T, BIAS, BIAS && sizeof(T) == 2, 2>(a, blockIdx.x - n_kv, gridDim.x - n_kv, lds);
}

// dK and dV from their splits, in order: 32 threads to a key, 4 values each.  Work-groups
// from n_sum on sum the bias gradient.
template <typename T>
__global__ __launch_bounds__(256) void xattn_kv_sum_kernel(XAttnArgs a, int n_sum) {
  constexpr int QB = x_qb<T>();
  __shared__ float red[32];
  if ((int)blockIdx.x >= n_sum) {
    x_dtable_sum(a, blockIdx.x - n_sum, red);
    return;
  }
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), n = (int64_t)a.B * a.G * a.Sk;
  if (row >= n) return;
  const int key = (int)(row % a.Sk), bg = (int)(row / a.Sk), b = bg / a.G, g = bg % a.G;
  const int c = (threadIdx.x & 31) * 4;
  const int qp = x_q_pos(a, b);
  const int kb = XQB / a.kv_qs;
  const int q_first = a.causal ? max(0, key / kb * kb - qp) : 0;
  const int n_it = max(0, (a.Sq + QB - 1) / QB - q_first / QB) * a.rep;
  const int splits = max(1, (n_it + a.kv_chunk - 1) / a.kv_chunk);
  f32x4_t t = {0.0f, 0.0f, 0.0f, 0.0f};
  const float* p = a.part + row * 2 * XHD + c;
  // (four loads on their way at a time: 2 x 8 heads over 1, fp32, 8 splits and more, 6.8 -> 4
  // us)
  for (int i = 0; i < splits; i += 4) {
    f32x4_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = *(const f32x4_t*)(p + (int64_t)min(i + j, splits - 1) * n * 2 * XHD);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < splits) t += v[j];
  }
  T* to = c < XHD ? (T*)a.dk + b * a.sdk[0] + (int64_t)key * a.sdk[1] + g * a.sdk[2] + c
                  : (T*)a.dv + b * a.sdv[0] + (int64_t)key * a.sdv[1] + g * a.sdv[2] + c - XHD;
  if constexpr (sizeof(T) == 2)
    *(u32x2_t*)to = u32x2_t{pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
  else
    *(f32x4_t*)to = t;
}

template <typename K>
hipError_t launch(K kernel, int64_t grid, size_t lds, hipStream_t st, const XAttnArgs& a) {
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), lds, st, a);
  return hipGetLastError();
}

size_t dist_bytes(const XAttnArgs& a) {
  return a.table ? (size_t)((2 * (a.reach + XPAD) + 1 + 3) & ~3) * 4 : 0;
}

template <typename T>
hipError_t forward_t(const XAttnArgs& a, hipStream_t st) {
  if (a.few_splits > 0) return xattn_few(a, sizeof(T) == 2 ? STAGE_BF16 : STAGE_F32, st);
  constexpr int KS2 = sizeof(T) == 4 ? 2 : 1;
  const int qb = XQB / a.fwd_ks;
  const int64_t grid = (int64_t)a.B * a.H * ((a.Sq + qb - 1) / qb);
  const size_t lds = 4 * XKT * XT<T>::ROWB + dist_bytes(a);
  if (grid == 0) return hipSuccess;
  if (a.fwd_ks == 1)
    return a.table ? launch(xattn_fwd_kernel<T, true, 1>, grid, lds, st, a)
                   : launch(xattn_fwd_kernel<T, false, 1>, grid, lds, st, a);
  return a.table ? launch(xattn_fwd_kernel<T, true, KS2>, grid, lds, st, a)
                 : launch(xattn_fwd_kernel<T, false, KS2>, grid, lds, st, a);
}

// Kernels that take `causal` keep the first query that sees a key beside what the others
// keep: dK and dV of 32 x 16 heads of 128 over 512 without `causal` 37.2 us with such a
// kernel, 34.8 with one of its own.  (fp32 has none: 8 x 12 heads of 128 with a bias take
// 33.3 either way.)
typedef void (*KvKernel)(XAttnArgs, int);
template <typename T, int QS>
KvKernel dkdv_kernel(const XAttnArgs& a) {
  if constexpr (sizeof(T) == 2) {
    if (!a.causal)
      return a.table ? xattn_dkdv_kernel<T, true, QS, false> : xattn_dkdv_kernel<T, false, QS, false>;
  }
  return a.table ? xattn_dkdv_kernel<T, true, QS, true> : xattn_dkdv_kernel<T, false, QS, true>;
}
template <typename T, int QS>
KvKernel bwd_kernel(const XAttnArgs& a) {
  if constexpr (sizeof(T) == 2) {
    if (!a.causal)
      return a.table ? xattn_bwd_kernel<T, true, QS, false> : xattn_bwd_kernel<T, false, QS, false>;
  }
  return a.table ? xattn_bwd_kernel<T, true, QS, true> : xattn_bwd_kernel<T, false, QS, true>;
}

// Floats of 32 fp32 rows for each of a work-group's wavefronts (x_store<float>).
constexpr size_t XSTAGE = 4 * 32 * XT<float>::LD;

template <typename T>
hipError_t backward_t(const XAttnArgs& a, hipStream_t st) {
  hipError_t e = hipSuccess;
  const int qb = XQB / a.dq_ks;
  const int kb = XQB / a.kv_qs;
  const int64_t n_kv = (int64_t)a.B * a.G * ((a.Sk + kb - 1) / kb) * a.kv_splits;
  const int64_t gq = (int64_t)a.B * a.H * ((a.Sq + qb - 1) / qb) * a.dq_splits;
  const int64_t n_red = a.dtable ? (int64_t)((a.nb + 7) / 8) * a.H : 0;
  const int64_t n_sum = a.kv_splits > 1 ? ((int64_t)a.B * a.G * a.Sk + 7) / 8 : 0;
  // dQ: [2][K, V], with splits as large as the wavefronts' fp32 rows; with a bias: dist,
  // sums by distance and by bucket of 4 wavefronts
  size_t dq_lds = 4 * XKT * XT<T>::ROWB;
  if (a.dq_splits > 1) dq_lds = std::max<size_t>(dq_lds, XSTAGE * 4);
  if (a.table) dq_lds += dist_bytes(a) + 4 * (size_t)(2 * (a.reach + XPAD) + 1 + a.nb) * 4;
  auto sums = [&](int64_t red) {
    hipLaunchKernelGGL(xattn_kv_sum_kernel<T>, dim3((unsigned)(n_sum + red)), dim3(256), 0, st, a,
                       (int)n_sum);
    return hipGetLastError();
  };
  constexpr int QS2 = sizeof(T) == 4 ? 2 : 1;
  if (a.one_launch) {
    const dim3 grid((unsigned)(n_kv + gq));
    const size_t lds = std::max(kv_lds<T>() + XOWN * 4 + dist_bytes(a), dq_lds);
    hipLaunchKernelGGL(a.kv_qs == 1 ? (bwd_kernel<T, 1>(a)) : (bwd_kernel<T, QS2>(a)), grid, dim3(256),
                       lds, st, a, (int)n_kv);
    if ((e = hipGetLastError()) != hipSuccess || n_sum + n_red == 0) return e;
    return sums(n_red);
  }
  if (gq > 0) {
    // The bias gradient is a sum of many dS that nearly cancel, in fp32: with D from
    // a bf16 out it would be off by out's rounding.
    constexpr bool BF = sizeof(T) == 2;
    const bool red = BF && a.dtable;
    const size_t lds = dq_lds;
    if (a.dq_ks == 1)
      e = !a.table ? launch(xattn_dq_kernel<T, false, false, 1>, gq, lds, st, a)
          : red    ? launch(xattn_dq_kernel<T, true, BF, 1>, gq, lds, st, a)
                   : launch(xattn_dq_kernel<T, true, false, 1>, gq, lds, st, a);
    else
      e = !a.table ? launch(xattn_dq_kernel<T, false, false, 2>, gq, lds, st, a)
          : red    ? launch(xattn_dq_kernel<T, true, BF, 2>, gq, lds, st, a)
                   : launch(xattn_dq_kernel<T, true, false, 2>, gq, lds, st, a);
    if (e == hipSuccess && a.dq_splits > 1)
      e = launch(xattn_dq_sum_kernel<T>, ((int64_t)a.B * a.H * a.Sq + 15) / 16, 0, st, a);
    if (e != hipSuccess) return e;
  }
  if (n_kv + n_red == 0) return e;
  const size_t lds = kv_lds<T>() + dist_bytes(a);
  const dim3 grid((unsigned)(n_kv + n_red));
  hipLaunchKernelGGL(a.kv_qs == 1 ? (dkdv_kernel<T, 1>(a)) : (dkdv_kernel<T, QS2>(a)), grid, dim3(256),
                     lds, st, a, (int)n_kv);
  if ((e = hipGetLastError()) != hipSuccess || a.kv_splits == 1) return e;
  return sums(0);
}

}  // namespace

// Half as many queries to a work-group fill more CUs and waste fewer rows of the last
// block, but read the keys twice as often.  us of both for 512 keys by work-groups per
// CU, fitted to 30 shapes: 2 x 16 heads of 512 queries with bias 34 -> 26, 12 x 16 heads
// 57 -> 67; under `causal`, where the long rows decide, 13 x 16 heads of 387 58 -> 50;
// fp32, 8 x 12 heads of 128: 26 -> 19.
XDqPlan xattn_dq_plan(int B, int H, int Sq, int Sk, int causal, bool bias, stage_dtype dt) {
  const double cus = device_cus(), bh = (double)B * H;
  const double n1 = std::max(1.0, bh * ((Sq + XQB - 1) / XQB) / cus);
  const double n2 = std::max(1.0, bh * ((Sq + XQB / 2 - 1) / (XQB / 2)) / cus);
  double t1, t2;
  if (dt == STAGE_F32) {
    t1 = 11 + 52 * std::ceil(n1);
    t2 = 8 + 26.5 * std::ceil(n2);
  } else {
    t1 = bias ? 24 + 10.8 * n1 : 8.5 + 8.5 * n1;
    t2 = bias ? 15.5 + 8.4 * n2 : 8 + 6 * n2;
  }
  const int ks = t2 * (causal ? 0.8 : 1.0) < t1 ? 2 : 1;
  // Few queries over many keys: split the keys too, as far as CUs are free (two work-
  // groups on one take turns).  A block of 64 keys takes 0.75 us, fp32 3.3, the sum of
  // the splits a launch of 5: 16 x 4 heads of 25 queries over 4045 keys 54 -> 20 + 5 us
  // in 4 splits, fp32 221 -> 64 + 5; 4 x 16 heads of 64 over 1024 keys 18.6 -> 13.4 +
  // 4.8.  (A bias gradient needs D before the pass: one split.)
  const double wgs = bh * ((Sq + XQB / ks - 1) / (XQB / ks)), blocks = (Sk + XKT - 1) / XKT;
  int splits = 1;
  if (!bias && wgs > 0)
    splits = std::max(1, (int)std::min(std::floor(cus / wgs), std::floor(blocks / 2)));
  if (blocks * (dt == STAGE_F32 ? 3.3 : 0.75) * (1.0 - 1.0 / splits) < 8.0) splits = 1;
  return {ks, splits};
}

// bf16: see xattn_few_plan.  fp32, fitted to 60 launches of 1 to 32 x 8 to 16 heads with 32
// to 512 queries and keys: 4 x 8 heads of 512 44 us with a wavefront to 32 queries, 28
// with two, 8 x 12 of 300 50 and 31, 8 x 12 of 128 13.4 and 10.4; 16 x 12 of 512, where
// every CU has several work-groups, 115 and 124.  (Under `causal` the shares of a
// work-group's rows differ, which the smaller ones even out.)
double xattn_fwd_time(int B, int H, int Sq, int Sk, int causal, stage_dtype dt, int* ks) {
  const double cus = device_cus(), blocks = (Sk + XKT - 1) / XKT;
  const double n1 = (double)B * H * ((Sq + XQB - 1) / XQB);
  *ks = 1;
  if (dt == STAGE_BF16) {
    const double at_once = std::min(4.0, std::ceil(n1 / cus));
    return std::ceil(n1 / (4 * cus)) * (2.1 + blocks * (1.15 + 0.63 * (at_once - 1)));
  }
  const double n2 = (double)B * H * ((Sq + XQB / 2 - 1) / (XQB / 2));
  const double t1 = (3.5 + 5.05 * blocks) * (0.18 + 0.82 * std::ceil(n1 / cus));
  const double t2 = (3.7 + 3.05 * blocks) * (0.3 + 0.7 * std::ceil(n2 / cus));
  if (t2 * (causal ? 0.78 : 1.0) < 0.93 * t1) *ks = 2;
  return std::min(t1, t2);
}

// Few work-groups: both parts of the backward in one launch, which saves the second one and
// the wait for the first; a bias's gradient is then summed in the next launch, beside the
// sums of the chunks.  us in two launches and in one (with a bias, in one more each): 2 x 8
// heads of 64 queries and keys 12.1 and 9.4, fp32 22.6 and 13.9; 3 x 12 of 77 over 201 16.5
// and 14; fp32, 10 x 16 of 128 47.9 and 35.9; with a bias 2 x 8 of 128 21.6 and 16.9, fp32
// 36.9 and 23.6, 10 x 16 of 128 25 and 20.2 (without the bias's gradient, whose launch then
// falls away, 21.3 and 16).  bf16 work-groups go through all keys for D:
// 4 x 16 of 32 over 300 15.6 and 14.5, of 100 over 700 26 and 33.6; two blocks of queries
// (4 x 16 of 256) 20.6 and 26.5.
int xattn_one_launch(int B, int H, int G, int Sq, int Sk, const XDqPlan& dq, const XKvPlan& kv,
                     stage_dtype dt) {
  if (dq.splits != 1 || dq.ks != 2 || B == 0 || Sq == 0 || Sk == 0) return 0;
  if (kv.chunk * kv.rows > XOWN) return 0;
  if (dt == STAGE_BF16 && (kv.chunk > 1 || Sk > 6 * XKT)) return 0;
  const int kb = XQB / kv.qs;
  const int64_t n = (int64_t)B * G * ((Sk + kb - 1) / kb) * kv.splits +
                    (int64_t)B * H * ((Sq + XQB / 2 - 1) / (XQB / 2));
  // (bf16, chunks that each go through many keys: 11 x 8 heads over 2 of 32 over 300, 352
  // work-groups, 24.9 in one launch, 17.8 in two; 4 x 8 over 2 of 77 over 201, 128, 17 and 22)
  const bool long_d = dt == STAGE_BF16 && kv.splits > 1 && Sk > 2 * XKT;
  return n <= (long_d ? 1 : 2) * device_cus();
}

XKvPlan xattn_kv_plan(int B, int G, int rep, int Sq, int Sk, int causal, bool bias,
                      const XDqPlan& dq, stage_dtype dt) {
  const int rows = dt == STAGE_BF16 ? x_qb<bf16_t>() : x_qb<float>();
  const int64_t its = (int64_t)((Sq + rows - 1) / rows) * rep;
  const int64_t wgs = (int64_t)B * G * ((Sk + XQB - 1) / XQB);
  const int64_t cus = device_cus(), slots = 2 * cus;
  XKvPlan plan = {rows, (int)std::max<int64_t>(its, 1), 1, 1};
  // The sum of the splits is a launch and a pass over them (5 us and more), a block of
  // queries 3 us: 1 x 4 key heads of 4 x 2500 queries and 2500 keys 369 us in one piece
  // (80 work-groups), 96 + 8 in chunks; 8 x 12 heads of 128 (two blocks, fp32) 29 and
  // 22 + 5.
  // (A block of few queries costs less, so four full ones: 8 x 16 heads over 4, 32 queries
  // over 300 keys, 30 us in four chunks, 19 in one.  But with a bias each head's table is
  // made: 3 x 8 over 2, 56 queries and keys, 20 and 9.6 + 3.9; and what one launch holds
  // runs beside dQ: 4 x 8 over 2, 22 over 27, dQ and all 14.3 and 10.4, fp32 26 and 13.
  // Two or three blocks for that alone: bf16 with a bias, 1 x 6 over 3 of 128, 25.7 and 17.4,
  // 2 x 8 of 200 28.5 and 21.3; without, 16.9 and 14.2, but 8 x 12 over 6 of 128, more
  // work-groups than CUs, 17 and 18.9.)
  if (wgs * 2 <= slots && wgs > 0 && its >= 2) {
    const int64_t full = (int64_t)((std::min(Sq, rows) + 31) / 32) * 32 * its;
    const int64_t all = wgs * its / (causal ? 2 : 1);
    const int64_t chunk = std::max<int64_t>((all + slots - 1) / slots, 1);
    const XKvPlan split = {rows, (int)chunk, (int)((its + chunk - 1) / chunk), 1};
    const int64_t both = wgs * split.splits +
                         (int64_t)B * G * rep * ((Sq + XQB / 2 - 1) / (XQB / 2));
    const bool one = xattn_one_launch(B, G * rep, G, Sq, Sk, dq, split, dt);
    if (its >= 4 ? bias || full >= 4 * rows || one : one && (bias || both <= cus))
      plan = split;
  }
  // fp32: half as many keys to a work-group, two wavefronts to 32 of them, where that
  // leaves at most two to a CU.  us by work-groups per CU and blocks of queries, fitted
  // to 60 launches: 8 x 12 heads of 128 24 -> 18.7, of 300 90 -> 61, 8 x 8 of 300 (else in
  // 3 chunks) 61 -> 58; 16 x 12 of 128 25 -> 33, 16 x 12 of 512 209 -> 249.  (bf16: no
  // gain for few work-groups, 84 -> 106 at 32 x 12 of 512.)
  const int64_t halves = (int64_t)B * G * ((Sk + XQB / 2 - 1) / (XQB / 2));
  if (dt == STAGE_F32 && wgs > 0 && Sq > 32 && halves <= slots) {
    const int64_t n = wgs * plan.splits;
    const double t1 = (5.0 + 8.1 * plan.chunk) * ((n + cus - 1) / cus) + (plan.splits > 1 ? 6.0 : 0.0);
    const double t2 = halves <= cus ? 5.0 + 6.5 * its : 2.0 * (6.0 + 4.6 * its);
    if (t2 < t1) plan = {rows, (int)std::max<int64_t>(its, 1), 1, 2};
  }
  return plan;
}

hipError_t xattn_forward(const XAttnArgs& a, stage_dtype dt, hipStream_t st) {
  return dt == STAGE_BF16 ? forward_t<bf16_t>(a, st) : forward_t<float>(a, st);
}
hipError_t xattn_backward(const XAttnArgs& a, stage_dtype dt, hipStream_t st) {
  return dt == STAGE_BF16 ? backward_t<bf16_t>(a, st) : backward_t<float>(a, st);
}
