// Attention with keys of a sequence of their own and a relative position bias
// (include/attn.h): kernel arguments, host-side launchers, and the device pieces
// that its kernels share.
#pragma once
#include "../../include/attn.h"
#include "attn_tile.h"

#include <climits>

struct XAttnArgs {
  const void* q;
  const void* k;
  const void* v;
  const void* o;     // backward: the forward's out
  const void* dout;
  void* out;
  void* dq;
  void* dk;
  void* dv;
  const uint8_t* mask;     // [B, Sk] or null
  const int32_t* q_pos;    // [B] or null
  const float* table;      // [nb, H] or null
  float* lse;              // [B, H, Sq], natural logarithm (forward: may be null)
  float* dtable;           // [nb, H] or null
  float* dsum;             // workspace [B, H, Sq]: D of the backward
  float* tpart;            // workspace [B, H, ceil(Sq * dq_ks / 128)][nb]: sums of dS by bucket
  float* part;             // workspace: partial results of the splits
  int64_t sq[3], sk[3], sv[3], so[3], sdo[3], sdq[3], sdk[3], sdv[3];
  int B, Sq, Sk, H, G, rep;  // G key heads, rep = H / G query heads to each
  int causal;
  int kv_chunk, kv_splits, kv_qs;         // XKvPlan
  int few_waves, few_splits, few_stream;  // XFewPlan
  int dq_ks, dq_splits;                   // XDqPlan
  int fwd_ks;                             // xattn_fwd_time
  int one_launch;                         // xattn_one_launch
  float c;      // scale * log2(e)
  float scale;
  // Buckets (attn_relpos): nb in all, nbd to a direction, `one` of them with one
  // distance each.
  int nb, nbd, one, both, reach, n_borders;
  int border[ATTN_MAX_BUCKETS / 2];  // INT_MAX from n_borders on
};

// How the dK / dV kernel goes through the query blocks (of XKvPlan::rows queries of
// one head) that a block of 128 / qs keys meets: `chunk` of them to a work-group, whose
// wavefronts share 32 keys by qs (1 or 2), and with splits > 1 each chunk's fp32 sums go
// to the workspace, [split][B, G][Sk][dK | dV].
struct XKvPlan {
  int rows, chunk, splits, qs;
};

// About how long the forward kernel for many queries takes, in us, and by how many (1 or
// 2) of its wavefronts 32 queries are shared.
double xattn_fwd_time(int B, int H, int Sq, int Sk, int causal, stage_dtype dt, int* ks);

// How the dQ kernel goes along the keys: ks wavefronts (1 or 2) of a work-group share
// 32 queries, and `splits` work-groups the keys.  With several splits each leaves, per
// query, xattn_dq_row floats in the workspace, [split][B, H][Sq]: 64 of dQ, on bf16
// also 64 of P K and the sum of its dS.
struct XDqPlan {
  int ks, splits;
};
XDqPlan xattn_dq_plan(int B, int H, int Sq, int Sk, int causal, bool bias, stage_dtype dt);
XKvPlan xattn_kv_plan(int B, int G, int rep, int Sq, int Sk, int causal, bool bias,
                      const XDqPlan& dq, stage_dtype dt);
// Whether one kernel makes all of a backward's results, up to the sums of dK's splits and of
// the bias's gradient.
int xattn_one_launch(int B, int H, int G, int Sq, int Sk, const XDqPlan& dq, const XKvPlan& kv,
                     stage_dtype dt);
inline int xattn_dq_row(stage_dtype dt) { return dt == STAGE_BF16 ? 132 : 64; }

// The forward kernel that serves few queries (xattn_few.hip): wavefronts of a
// work-group and splits of the keys, 0 splits where the other kernel is faster; stream:
// keys and values are marked as read once.  With
// more than one split it leaves, in the workspace, per split and row (query and query
// head of a key head, in tiles of 32) XFEW_ROW floats: 64 sums of P v, the exponents'
// offset and the sum of P.  buckets, reach: of the bias, 0 without one.
constexpr int XFEW_ROW = 68;
struct XFewPlan {
  int waves, splits, stream;
};
XFewPlan xattn_few_plan(int B, int G, int rep, int Sq, int Sk, int buckets, int reach,
                        stage_dtype dt);
inline int64_t xattn_few_tiles(int rep, int Sq) { return ((int64_t)Sq * rep + 31) / 32; }
hipError_t xattn_few(const XAttnArgs& a, stage_dtype dt, hipStream_t st);

hipError_t xattn_forward(const XAttnArgs& a, stage_dtype dt, hipStream_t st);
hipError_t xattn_backward(const XAttnArgs& a, stage_dtype dt, hipStream_t st);

namespace {

constexpr int XHD = 64;        // head width
constexpr int XKT = 64;        // keys per block
constexpr float XLOG2E = 1.4426950408889634f;
constexpr float XLN2 = 0.6931471805599453f;

// Distances within a 32 x 32 tile that has a pair nearer than `reach` are below
// reach + XPAD, so that a table of the bias by distance over +-(reach + XPAD)
// serves such a tile without a bounds test.
constexpr int XPAD = 62;

__device__ __forceinline__ int x_bucket(const XAttnArgs& a, int rel) {
  const int base = a.both && rel > 0 ? a.nbd : 0;
  const int n = rel <= 0 ? -rel : (a.both ? rel : 0);
  if (n < a.one) return base + n;
  int b = base + a.one;
  for (int i = 0; i < a.n_borders; i += 8) {  // (padded; eight to a scalar load)
#pragma unroll
    for (int j = 0; j < 8; ++j) b += n >= a.border[i + j];
  }
  return b;
}

// q_pos within +-2^30: sequences are shorter than 2^29, so positions beyond that
// are beyond every key (or before it) by more than any reach all the same, and
// differences of positions fit 32 bits.
__device__ __forceinline__ int x_q_pos(const XAttnArgs& a, int b) {
  return a.q_pos ? min(max(a.q_pos[b], -(1 << 30)), 1 << 30) : 0;
}

// Tiles of [rows][64] in LDS: rows of ROWB bytes in 16-byte chunks, chunk c of row
// r stored at chunk c ^ swz(r), so that fragment reads of 16 rows fall on distinct
// banks.
template <typename T> struct XT;
template <> struct XT<bf16_t> {
  static constexpr int ROWB = 128, CPR = 8, LD = XHD + 8;
  struct Frag {
    bf16x8_t f[4];
  };
  static __device__ __forceinline__ int swz(int r) { return tswz(r); }
};
template <> struct XT<float> {
  static constexpr int ROWB = 256, CPR = 16, LD = XHD + 4;
  struct Frag {
    f32x4_t f[8];
  };
  static __device__ __forceinline__ int swz(int r) { return r & 15; }
};
template <typename T>
__device__ __forceinline__ int x_off(int r, int c) {
  return r * XT<T>::ROWB + 16 * (c ^ XT<T>::swz(r));
}

// Rows [row0, row0 + NR) of a [lim][64] operand into a tile with direct-to-LDS
// loads by NW wavefronts; rows from lim on are zero.  The buffer resource starts at
// row0, so the operand may be of any length.  STREAM: marked as read once.  SKIP: the
// tile's rows before `skip` are not read, and zero.
template <typename T, int NR, int NW, bool STREAM = false, bool SKIP = false>
__device__ __forceinline__ void x_dma(const T* base, int64_t ld, int row0, int lim, char* tile,
                                      int wave, int lane, int skip = 0) {
  constexpr int RPI = 1024 / XT<T>::ROWB, CPR = XT<T>::CPR;
  const int n = min(NR, lim - row0);
  const int bytes = n > 0 ? ((n - 1) * (int)ld + XHD) * (int)sizeof(T) : 0;
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(base + (int64_t)row0 * ld), (short)0, bytes, 0x00020000);
#pragma unroll
  for (int i = 0; i < NR / RPI / NW; ++i) {
    const int q = NR / RPI / NW * wave + i;
    const int r = RPI * q + lane / CPR;
    const int c = (lane % CPR) ^ XT<T>::swz(r);
    // (`bytes` is below 2^31)
    const int at = SKIP && r < skip ? INT_MIN : r * (int)ld * (int)sizeof(T) + 16 * c;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_t*)(tile + q * 1024), 16, at, 0, 0,
                                             STREAM ? 2 /* nt */ : 0);
  }
}

// Row p as an MFMA operand held in registers: lane l has, of row l % 32, the
// columns that pair with the tile rows x_mma_rows reads (bf16: 16 ks + 8 (l / 32)
// .. +7; fp32: 8 c + 4 (l / 32) .. +3).
template <typename T>
__device__ __forceinline__ typename XT<T>::Frag x_frag(const T* p, bool valid, int hf) {
  typename XT<T>::Frag r;
  constexpr int N = sizeof(r) / 16, W = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const u32x4_t w = valid ? *(const u32x4_t*)(p + W * (2 * i + hf)) : zero4();
    r.f[i] = __builtin_bit_cast(decltype(r.f[0] + r.f[0]), w);
  }
  return r;
}

// Waits for values that were loaded, here: with the wait left to their first use inside a
// loop, the compiler has every iteration wait for every load in flight.
template <typename F>
__device__ __forceinline__ void x_arrived(F& r) {
  constexpr int N = sizeof(r) / 16;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4_t w = __builtin_bit_cast(u32x4_t, r.f[i]);
    asm volatile("" : "+v"(w));
    r.f[i] = __builtin_bit_cast(decltype(r.f[0] + r.f[0]), w);
  }
}
__device__ __forceinline__ void x_arrived(float& v) { asm volatile("" : "+v"(v)); }

__device__ __forceinline__ f32x16_t mfma32_f32(float a, float b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// acc += tile[r0 .. r0 + 31] . b^T over the 64 columns.
__device__ __forceinline__ f32x16_t x_mma_rows(const char* tile, int r0, const XT<bf16_t>::Frag& b,
                                               f32x16_t acc, int lane) {
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) acc = mfma32(frag_rows(tile, r0, ks, lane), b.f[ks], acc);
  return acc;
}
__device__ __forceinline__ f32x16_t x_mma_rows(const char* tile, int r0, const XT<float>::Frag& b,
                                               f32x16_t acc, int lane) {
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const f32x4_t v =
        *(const f32x4_t*)(tile + x_off<float>(r0 + (lane & 31), 2 * c + (lane >> 5)));
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = mfma32_f32(v[e], b.f[c][e], acc);
  }
  return acc;
}

// out[t] (32 columns each) += tile[rb .. rb + 31]^T p, p a 32 x 32 accumulator
// whose rows are the tile's; bf16: p rounded to bf16.
template <typename T>
__device__ __forceinline__ void x_mma_cols(const char* tile, int rb, const f32x16_t& p,
                                           f32x16_t out[2], int lane) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const bf16x8_t pb = pack8(p, 8 * ks);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        out[t] = mfma32(frag_tr(tile, 32 * t, rb + 16 * ks, lane), pb, out[t]);
    }
  } else {
    const int hf = lane >> 5, rr = lane & 31;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = rb + acc_row(r, hf);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float v = *(const float*)(tile + x_off<float>(row, 8 * t + (rr >> 2)) + 4 * (rr & 3));
        out[t] = mfma32_f32(v, p[r], out[t]);
      }
    }
  }
}

// A wavefront's 32 x 64 result, held transposed in two accumulators (lane = row),
// times mul, to dst rows [row0, row0 + 32) clipped to nrows, through the
// wavefront's LDS area (32 x LD).
template <typename T>
__device__ __forceinline__ void x_store(const f32x16_t acc[2], float mul, T* stage,
                                        T* __restrict__ dst, int64_t ld, int row0, int nrows) {
  constexpr int LD = XT<T>::LD, CPR = XT<T>::CPR, W = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, hf = lane >> 5, rr = lane & 31;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = 32 * t + 8 * q + 4 * hf;
      f32x4_t w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = acc[t][4 * q + e] * mul;
      if constexpr (sizeof(T) == 2)
        *(u32x2_t*)(stage + rr * LD + col) = u32x2_t{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
      else
        *(f32x4_t*)(stage + rr * LD + col) = w;
    }
  lds_wait();
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < CPR / 2; ++i) {
    const int ch = lane + 64 * i;
    const int row = ch / CPR, col = (ch % CPR) * W;
    if (row0 + row < nrows)
      *(u32x4_t*)(dst + (int64_t)(row0 + row) * ld + col) = *(const u32x4_t*)(stage + row * LD + col);
  }
}

// The blocks of BK keys that a wavefront goes through: those of [0, nblk) that
// hold a key below lim which the mask leaves.  A window of 64 blocks is held at a
// time, lane i with the mask bits of its block base + i, so that a block's bits
// come from one lane and the next block to visit from one ballot, and blocks
// without a key cost nothing.  Every call is made by all lanes, with uniform
// arguments.
template <int BK>
struct KeyBlocks {
  typedef typename std::conditional<BK == 64, uint64_t, uint32_t>::type Word;
  const uint8_t* m;
  int lim, nblk, base, lane;
  Word w;
  uint64_t live;

  // (load(first) comes before the first next())
  __device__ __forceinline__ void init(const uint8_t* mask_row, int lim_, int last, int lane_) {
    m = mask_row;
    lim = lim_;
    nblk = last;
    lane = lane_;
  }
  // Bits of the keys of block b that are below lim.
  __device__ __forceinline__ Word in_range(int b) const {
    const int n = lim - b * BK;
    return n >= BK ? ~(Word)0 : n <= 0 ? (Word)0 : (((Word)1 << n) - 1);
  }
  __device__ __forceinline__ void load(int b) {
    base = b;
    w = b + lane < nblk ? in_range(b + lane) : 0;
    if (m) {
      Word bits = 0;
      const int ng = min(BK, ((nblk - base) * BK + 63) / 64);  // groups of 64 keys
      for (int g0 = 0; g0 < ng; g0 += 8) {
        int v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int key = base * BK + (g0 + j) * 64 + lane;
          v[j] = key < lim ? m[key] : 0;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint64_t bal = __ballot(v[j] != 0);
          if constexpr (BK == 64) {
            if (lane == g0 + j) bits = bal;
          } else {
            if ((lane >> 1) == g0 + j) bits = (Word)(bal >> (32 * (lane & 1)));
          }
        }
      }
      w &= bits;
    }
    live = __ballot(w != 0);
  }
  // First block from b on with a key, nblk if there is none.
  __device__ __forceinline__ int next(int b) {
    while (b < nblk) {
      if (b >= base + 64) load(b);
      const uint64_t l = live >> (b - base);
      if (l) return b + __builtin_ctzll(l);
      b = base + 64;
    }
    return nblk;
  }
  // Bits of block b, the last one that next() gave.
  __device__ __forceinline__ Word word(int b) const {
    const int i = b - base;
    if constexpr (BK == 64) {
      const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)w, i);
      const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(w >> 32), i);
      return ((uint64_t)hi << 32) | lo;
    } else {
      return (uint32_t)__builtin_amdgcn_readlane((int)w, i);
    }
  }
};

// A lane's bits of a 32 x 32 tile whose rows have bits `rows`: that of register r is
// bit 8 (r / 4) + r % 4.
__device__ __forceinline__ uint32_t x_lane_bits(uint32_t rows, int hf) { return rows >> (4 * hf); }
// All ones or zeros by the bit of register r, and v where it is set, else 0 or -inf
// (one instruction each; a compare and a select would be three).
__device__ __forceinline__ uint32_t x_mask(uint32_t bits, int r) {
  return (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (r >> 2) + (r & 3), 1);
}
__device__ __forceinline__ float x_or_zero(float v, uint32_t bits, int r) {
  return __uint_as_float(__float_as_uint(v) & x_mask(bits, r));
}
__device__ __forceinline__ float x_or_ninf(float v, uint32_t bits, int r) {
  const uint32_t m = x_mask(bits, r);
  return __uint_as_float((__float_as_uint(v) & m) | (0xff800000u & ~m));
}
// The low n + 1 bits (none for n < 0, all from 31 on).
__device__ __forceinline__ uint32_t x_upto(int n) {
  return n >= 31 ? 0xffffffffu : n < 0 ? 0u : (2u << n) - 1u;
}

}  // namespace
