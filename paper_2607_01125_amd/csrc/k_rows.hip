// The adapted linear of a few rows with packed INT4 weights (zoact_linear_rows).
//
//   y[t][n] = epi(res + b + sum_g s[n][g] sum_{k in g} q[n][k] x[t][k] + sum_i p[t][i] bf16(C[n][i]))
//
// Bound by the weights' bytes, each read once.  A lane's 16 bytes of an operand are 32 of the 128 columns
// of one scale group of one weight row.  A nibble becomes a bf16 number without arithmetic: its bits
// (with the sign bit turned over, u = q + 8) are put at the top of the mantissa of 16, which gives
// 16 + u = q + 24 exactly; the surplus 24 sum x is taken out by starting the group's sum from a product
// of x with a constant -24, which costs one product for all weight rows of the wave.  The group's sum is
// then scaled: one multiply-add a lane and group, no rounding of q s.  The columns of a word come as
// pairs (i, i + 4), so x is put in that order as it is staged.
// The surplus passes fp32's range where x is infinite (inf - inf) or 24 x is past it, which the formula does not:
// a sum that has come out infinite or NaN is formed again from the codes themselves (plain_sum).
#include <math.h>

#include "common.hpp"

namespace zoact {
namespace {

struct RowsArgs {
  const uint8_t* w;
  const uint16_t* sc;
  const uint16_t* bias;
  const uint16_t* x;
  const uint16_t* p;
  const uint16_t* res;
  const void* c;       // coefficients of the layer's first row (F32 or BF16)
  int c_f32, r;
  int64_t plain0, plain1;
  int rows;
  int64_t N;
  int K, groups;       // groups = K / 128
  int per_split;       // groups of one part of the depth
  float* part;         // partial sums, or NULL for one part
  void* y;
  int y_f32;
  uint32_t flags;
};

// Eight codes of a word as 16 + u: each pair is shifted to the mantissas' top and, in one operation, masked
// and combined with 16 and the turned sign bit.  `base` is kBase held in a vector register: an instruction
// reads one constant, the mask, from the scalar ones.
constexpr uint32_t kBase = 0x41C041C0u;
__device__ __forceinline__ bf16x8 nibbles(uint32_t v, uint32_t base) {
  constexpr uint32_t mask = 0x00780078u, and_xor = 0x6A;
  uint4 o;
  o.x = __builtin_amdgcn_bitop3_b32(v << 3, mask, base, and_xor);
  o.y = __builtin_amdgcn_bitop3_b32(v >> 1, mask, base, and_xor);
  o.z = __builtin_amdgcn_bitop3_b32(v >> 5, mask, base, and_xor);
  o.w = __builtin_amdgcn_bitop3_b32(v >> 9, mask, base, and_xor);
  return __builtin_bit_cast(bf16x8, o);
}
// Eight consecutive values in the order of a word's nibble pairs: (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ uint4 pair_order(uint4 u) {
  uint4 o;
  o.x = __builtin_amdgcn_perm(u.z, u.x, 0x05040100);
  o.y = __builtin_amdgcn_perm(u.z, u.x, 0x07060302);
  o.z = __builtin_amdgcn_perm(u.w, u.y, 0x05040100);
  o.w = __builtin_amdgcn_perm(u.w, u.y, 0x07060302);
  return o;
}

// Eight coefficients (or values of p) as bf16 from column i0 on, zeros past r.
template <typename T>
__device__ __forceinline__ bf16x8 tail8(const T* row, int i0, int r, bool in) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const T x = in && i0 + e < r ? row[i0 + e] : (T)0;
    if constexpr (sizeof(T) == 2)
      v[e] = __builtin_bit_cast(__bf16, x);
    else
      v[e] = (__bf16)x;
  }
  return v;
}
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bf16x8 keep_if(const u32x4& u, bool c) {
  return __builtin_bit_cast(bf16x8, u & (c ? 0xFFFFFFFFu : 0u));
}

// What is added to the sums of four rows of x, from `row` on, and one feature (SwiGLU: and the up feature,
// 16 further).  What there is none of is loaded from x instead and dropped at the end: a branch around a load
// would wait for it where the branches meet.
struct Extras {
  uint16_t b[2], res[2][4];
  bool has_b[2], has_res[2];
};
__device__ __forceinline__ Extras load_extras(const RowsArgs& a, int row, int64_t n) {
  Extras e;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t f = n + 16 * h;
    const bool in = f < a.N && (h == 0 || a.flags & ZOACT_EPI_SWIGLU);
    e.has_b[h] = in && a.bias;
    e.has_res[h] = in && a.res;
    e.b[h] = *(e.has_b[h] ? a.bias + f : a.x);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      e.res[h][k] = *(e.has_res[h] && row + k < a.rows ? a.res + (int64_t)(row + k) * a.N + f : a.x);
  }
  return e;
}

__device__ __forceinline__ float plus(float y, bool has, uint16_t v) { return has ? y + bf2f(v) : y; }
// y of those rows and the feature from the sums (SwiGLU: z the gate's, up the up feature's).
__device__ __forceinline__ void finish(const RowsArgs& a, int row, int64_t n, const floatx4& z, const floatx4& up,
                                       const Extras& e) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (row + k >= a.rows) return;
    float y = plus(plus(z[k], e.has_b[0], e.b[0]), e.has_res[0], e.res[0][k]);
    int64_t at = (int64_t)(row + k) * a.N + n;
    if (a.flags & ZOACT_EPI_SWIGLU) {
      y = y / (1.f + __expf(-y)) * plus(plus(up[k], e.has_b[1], e.b[1]), e.has_res[1], e.res[1][k]);
      at = (int64_t)(row + k) * (a.N / 2) + n / 32 * 16 + (n & 15);
    } else if (a.flags & ZOACT_EPI_RELU) {
      y = y > 0.f ? y : y != y ? y : 0.f;
    }
    if (a.y_f32)
      static_cast<float*>(a.y)[at] = y;
    else
      static_cast<uint16_t*>(a.y)[at] = f2bf(y);
  }
}

// Coefficient row of feature n, or -1 where it has none.
__device__ __forceinline__ int64_t coef_row(const RowsArgs& a, int64_t n) {
  return n >= a.N || (n >= a.plain0 && n < a.plain1) ? -1 : n >= a.plain1 ? n - (a.plain1 - a.plain0) : n;
}

// 32 ranks of the correction, from i0 on, for the first `tiles` of TW tiles of features from n0 on and NB blocks
// of 16 rows of x.  All operands are asked for before one is used, and without branches, as above (one after
// another they cost 4096 x 6144, 48 rows, 3 us).  Only where rows of p and C are whole 16-byte pieces
// (elsewhere it adds nothing, see add_odd_ranks).
__device__ __forceinline__ bool whole_ranks(const RowsArgs& a) {
  return (a.r & 7) == 0 && ((uintptr_t)a.c & 15) == 0;
}
template <int TW, int NB>
struct Correction {
  u32x4 p[NB], c[TW], c_hi[TW];        // as loaded (c_hi: the second half of F32 coefficients)
  bool in, has[TW];
  __device__ __forceinline__ void load(const RowsArgs& a, int64_t n0, int b0, int i0, int tiles) {
    const int l16 = threadIdx.x & 15, i = i0 + 8 * ((threadIdx.x & 63) >> 4);
    in = i < a.r && whole_ranks(a);
    const u32x4* const other = reinterpret_cast<const u32x4*>(a.x);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int t = (b0 + b) * 16 + l16;               // (rows past the last take row 0)
      p[b] = *(in ? reinterpret_cast<const u32x4*>(a.p + (int64_t)(t < a.rows ? t : 0) * a.r + i) : other);
    }
#pragma unroll
    for (int t = 0; t < TW; ++t) {
      const int64_t row = coef_row(a, n0 + t * 16 + l16);
      has[t] = in && row >= 0 && t < tiles;
      const char* const at = static_cast<const char*>(a.c) + ((row * a.r + i) << (a.c_f32 ? 2 : 1));
      const u32x4* const cr = has[t] ? reinterpret_cast<const u32x4*>(at) : other;
      c[t] = cr[0];
      c_hi[t] = cr[a.c_f32];
    }
  }
  __device__ __forceinline__ void apply(const RowsArgs& a, floatx4 (&tot)[TW][NB]) const {
    bf16x8 cf[TW];
#pragma unroll
    for (int t = 0; t < TW; ++t) {
      if (a.c_f32) {
        #pragma unroll
        for (int e = 0; e < 8; ++e)
          cf[t][e] = (__bf16)(has[t] ? __uint_as_float(e < 4 ? c[t][e & 3] : c_hi[t][e & 3]) : 0.f);
      } else {
        cf[t] = keep_if(c[t], has[t]);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const bf16x8 pf = keep_if(p[b], in);
#pragma unroll
      for (int t = 0; t < TW; ++t) tot[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf, cf[t], tot[t][b], 0, 0, 0);
    }
  }
};

// The correction where r is not a multiple of 8 or C not aligned: `step` is the waves' share, as above.
template <int TW, int NB>
__device__ __forceinline__ void add_odd_ranks(const RowsArgs& a, int64_t n0, int b0, int i0, int step,
                                              floatx4 (&tot)[TW][NB]) {
  const int l16 = threadIdx.x & 15;
  for (i0 += 8 * ((threadIdx.x & 63) >> 4); __any(i0 < a.r); i0 += step) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int row = (b0 + b) * 16 + l16;
      const bf16x8 pf = tail8(a.p + (int64_t)(row < a.rows ? row : 0) * a.r, i0, a.r, true);
#pragma unroll
      for (int t = 0; t < TW; ++t) {
        const int64_t c = coef_row(a, n0 + t * 16 + l16), at = (c < 0 ? 0 : c) * a.r;
        const bf16x8 cf = a.c_f32 ? tail8(static_cast<const float*>(a.c) + at, i0, a.r, c >= 0)
                                  : tail8(static_cast<const uint16_t*>(a.c) + at, i0, a.r, c >= 0);
        tot[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf, cf, tot[t][b], 0, 0, 0);
      }
    }
  }
}

// The sum of one output over groups gbeg .. gend - 1 (and the correction, of one part), code by code, with x times
// 2^-16: sums of codes times finite values do not overflow then.  Once NaN it stays that.  (A call with an
// infinite x takes 100 to 120 us, with a NaN 14 to 35 for 12 to 23 without.)
__device__ float plain_sum(const RowsArgs& a, int64_t t, int64_t n, int gbeg, int gend) {
  float y = 0.f;
#pragma unroll 1
  for (int gr = gbeg; gr < gend && y == y; ++gr) {
    const uint32_t* const w = reinterpret_cast<const uint32_t*>(a.w + n * (a.K / 2) + gr * 64);
    const uint16_t* const x = a.x + t * a.K + gr * 128;
    float s = 0.f;
#pragma unroll 1
    for (int i = 0; i < 16; ++i) {
      const uint32_t v = w[i];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        s = fmaf((float)((int32_t)(v << (28 - 4 * e)) >> 28), bf2f(x[8 * i + e]) * 0x1p-16f, s);
    }
    y = fmaf(bf2f(a.sc[n * a.groups + gr]), s, y);
  }
  y *= 0x1p16f;
  const int64_t c = coef_row(a, n);
  if (!a.part && c >= 0) {
#pragma unroll 1
    for (int i = 0; i < a.r; ++i) {
      const float f = a.c_f32 ? (float)(__bf16)static_cast<const float*>(a.c)[c * a.r + i]
                              : bf2f(static_cast<const uint16_t*>(a.c)[c * a.r + i]);
      y = fmaf(bf2f(a.p[t * a.r + i]), f, y);
    }
  }
  return y;
}

// RT tiles of 16 weight rows and NB blocks of 16 rows of x a workgroup (XR rows of x in LDS: 4, or 16 NB),
// depth in stages of WK groups.  Weights and x come in whole rows' pieces (a quad of lanes reads 64
// contiguous bytes), a stage ahead in registers (two stages ahead: the same times), and go through LDS to the
// operands' order; read from memory in that order, where a quad touches four rows, 4096 x 28672 took 23 us at
// one row and 27 at 13.  16-byte pieces are swapped by the row's number, so that neither side of LDS has bank
// conflicts (counted: none in the forms of 1, 13 and 48 rows).  x, whose quarter-waves read pieces four apart, is
// swapped by the row's number less four: lanes 0-3 and 12-15 of a quarter are served with 4-11 of the next, and
// without the four they meet on the same banks (20 and 28% of the cycles at 13 and 48 rows; 64 rows of 5120 x
// 20480 41.9 us, now 39.9).  Scales come 32 groups at a time, so that they too are read in pieces of rows.
// Wave w takes group w % WK of a stage and the tiles from w / WK on; the waves' sums meet in LDS in a
// fixed order.  blockIdx.y: the part of the depth (partial sums go to part, rows_join_kernel adds them).
// (Tried and left: one workgroup of 16 waves a compute unit with all of x in LDS and weights streamed
// past it, 7.0 us for 4096 x 4096 at one row, 11.4 at 16; dot products on the vector units for one row,
// 23 us for 4096 x 28672.)
constexpr int kWindow = 32;
template <int RT, int NB, int XR, int NW, int WK>
__global__ void __launch_bounds__(64 * NW) rows_kernel(RowsArgs a) {
  constexpr int WR = NW / WK, TW = RT / WR;              // waves along the tiles, tiles of a wave
  constexpr int WP = 4 * WK, XP = 16 * WK;               // 16-byte pieces of a stage's weight row and x row
  constexpr int WN = RT * 16 * WP, XN = XR * XP;         // pieces of a stage
  constexpr int TH = 64 * NW, WL = (WN + TH - 1) / TH, XL = (XN + TH - 1) / TH;
  constexpr int STAGE = WN + XN;
  constexpr int SUMS = WK * RT * NB * 64;                // floatx4 of the waves' sums
  constexpr int LDS = 2 * STAGE > SUMS ? 2 * STAGE : SUMS;
  constexpr int BN = RT * 16, SL = BN * kWindow / TH;
  __shared__ uint4 lds[LDS];
  __shared__ uint16_t scl[2][BN][kWindow + 2];
  __shared__ int any_large;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15,
            g = lane >> 4;
  const int wk = wave % WK, wr = wave / WK;
  const int64_t n0 = (int64_t)blockIdx.x * BN;
  const int gbeg = blockIdx.y * a.per_split, gend = gbeg + a.per_split < a.groups ? gbeg + a.per_split : a.groups;
  const int stages = (gend - gbeg + WK - 1) / WK;
  const int64_t rows_here = a.N - n0 < BN ? a.N - n0 : BN;
  const __amdgpu_buffer_rsrc_t wrs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(a.w) + n0 * (a.K / 2), 0, (int)(rows_here * (a.K / 2)), 0x00020000);
  const __amdgpu_buffer_rsrc_t xrs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(a.x), 0, a.rows * a.K * 2, 0x00020000);
  const uint16_t* const srow = a.sc + n0 * a.groups;
  // pieces swapped within 16 (8)
  auto swap = [](int row, int piece) { return WK >= 4 ? piece ^ (row & 15) : piece ^ ((row >> 1) & 7); };
  auto swap_x = [](int row, int piece) { return piece ^ ((row - 4) & 15); };

  uint4 wv[WL], xv[XL];
  uint16_t sv[SL];
  // (past the part's last group there is nothing: such pieces are asked for outside the descriptor)
  auto load = [&](int st) {
    const int gr = gbeg + st * WK;
#pragma unroll
    for (int j = 0; j < WL; ++j) {
      const int u = tid + j * TH, row = u / WP, piece = u % WP;
      if (WN % TH == 0 || u < WN)
        wv[j] = __builtin_bit_cast(
            uint4, __builtin_amdgcn_raw_buffer_load_b128(
                       wrs, gr + piece / 4 < gend ? row * (a.K / 2) + gr * 64 + piece * 16 : 0x7FFF0000, 0, 0));
    }
#pragma unroll
    for (int j = 0; j < XL; ++j) {
      const int u = tid + j * TH, row = u / XP, piece = u % XP;
      if ((XN % TH == 0 || u < XN) && row < a.rows)
        xv[j] = __builtin_bit_cast(
            uint4, __builtin_amdgcn_raw_buffer_load_b128(
                       xrs, gr + piece / 16 < gend ? row * a.K * 2 + gr * 256 + piece * 16 : 0x7FFF0000, 0, 0));
    }
  };
  auto load_scales = [&](int g0) {
#pragma unroll
    for (int j = 0; j < SL; ++j) {
      const int u = tid + j * TH, row = u / kWindow, gr = g0 + u % kWindow;
      sv[j] = row < rows_here && gr < gend ? srow[(int64_t)row * a.groups + gr] : (uint16_t)0;
    }
  };
  floatx4 tot[TW][NB];
#pragma unroll
  for (int t = 0; t < TW; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) tot[t][b] = floatx4{0.f, 0.f, 0.f, 0.f};
  const uint32_t m24 = 0xC1C0C1C0u;                  // (-24, -24)
  uint32_t base = kBase;
  asm("" : "+v"(base));
  const bf16x8 minus24 = __builtin_bit_cast(bf16x8, make_uint4(m24, m24, m24, m24));
  load_scales(gbeg);
  load(0);
  // (a thread's share of the outputs, where it is one: what is added to them is on its way from here on)
  constexpr bool kEarly = RT * NB * 64 <= TH;
  Extras ex{};
  if (kEarly && tid < RT * NB * 64 && !a.part)
    ex = load_extras(a, (tid >> 6) % NB * 16 + 4 * (lane >> 4), n0 + (tid >> 6) / NB * 16 + l16);
  // the correction (of one part; else rows_join_kernel's), 32 ranks a step, the steps shared out over the
  // waves of a tile; here its loads come with the first stage's
  if (!a.part) {
    if (whole_ranks(a)) {
      for (int i0 = 32 * wk; i0 < a.r; i0 += 32 * WK) {
        Correction<TW, NB> corr;
        corr.load(a, n0 + wr * TW * 16, 0, i0, TW);
        corr.apply(a, tot);
      }
    } else {
      add_odd_ranks<TW, NB>(a, n0 + wr * TW * 16, 0, 32 * wk, 32 * WK, tot);
    }
  }
  if (tid == 0) any_large = 0;
  // rows of x past the last are never loaded: both buffers start with zeros there
  for (int u = tid; u < XN; u += TH)
    if (u / XP >= a.rows) lds[WN + u] = lds[STAGE + WN + u] = make_uint4(0, 0, 0, 0);
  for (int st = 0; st < stages; ++st) {
    uint4* const wb = lds + (st & 1) * STAGE;
    uint4* const xb = wb + WN;
    const int win = st / (kWindow / WK), in_win = st % (kWindow / WK);
    if (in_win == 0) {
#pragma unroll
      for (int j = 0; j < SL; ++j) {
        const int u = tid + j * TH;
        scl[win & 1][u / kWindow][u % kWindow] = sv[j];
      }
      if (st + kWindow / WK < stages) load_scales(gbeg + (win + 1) * kWindow);
    }
#pragma unroll
    for (int j = 0; j < WL; ++j) {
      const int u = tid + j * TH, row = u / WP, piece = u % WP;
      if (WN % TH == 0 || u < WN) wb[row * WP + swap(row, piece)] = wv[j];
    }
#pragma unroll
    for (int j = 0; j < XL; ++j) {
      const int u = tid + j * TH, row = u / XP, piece = u % XP;
      if ((XN % TH == 0 || u < XN) && row < a.rows) xb[row * XP + swap_x(row, piece)] = pair_order(xv[j]);
    }
    if (st + 1 < stages) load(st + 1);
    __syncthreads();
    if (gbeg + st * WK + wk >= gend) continue;
    bf16x8 xf[NB][4];
    floatx4 off[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int xrow = XR < 16 ? l16 & (XR - 1) : b * 16 + l16;
      off[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        xf[b][j] = __builtin_bit_cast(bf16x8, xb[xrow * XP + swap_x(xrow, wk * 16 + g * 4 + j)]);
        off[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[b][j], minus24, off[b], 0, 0, 0);
      }
    }
#pragma unroll
    for (int t = 0; t < TW; ++t) {
      const int row = (wr * TW + t) * 16 + l16;
      const uint4 v = wb[row * WP + swap(row, wk * 4 + g)];
      const uint32_t wd[4] = {v.x, v.y, v.z, v.w};
      const float sc = bf2f(scl[win & 1][row][in_win * WK + wk]);
      floatx4 acc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = off[b];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8 wf = nibbles(wd[j], base);
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[b][j], wf, acc[b], 0, 0, 0);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) tot[t][b][k] = fmaf(sc, acc[b][k], tot[t][b][k]);
    }
  }
  // (the squares' sum is finite while all sums are below 2^61, and then those over the waves are finite too)
  float squares = 0.f;
#pragma unroll
  for (int t = 0; t < TW; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int k = 0; k < 4; ++k) squares = fmaf(tot[t][b][k], tot[t][b][k], squares);
  __syncthreads();
  floatx4* const sum = reinterpret_cast<floatx4*>(lds);      // [WK][RT][NB][64]
#pragma unroll
  for (int t = 0; t < TW; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) sum[((wk * RT + wr * TW + t) * NB + b) * 64 + lane] = tot[t][b];
  if (!(squares < INFINITY)) any_large = 1;
  __syncthreads();
  if (__builtin_expect(any_large, 0)) {
    // each thread adds the waves' sums of its outputs, puts right those that are not finite, and leaves them as
    // the first wave's
#pragma unroll 1
    for (int u = tid; u < RT * NB * 64; u += TH) {
      const int row = (u >> 6) % NB * 16 + 4 * ((u & 63) >> 4);
      const int64_t n = n0 + (u >> 6) / NB * 16 + (u & 15);
#pragma unroll 1
      for (int k = 0; k < 4; ++k) {
        float* const z = reinterpret_cast<float*>(sum + u) + k;
        float y = 0.f;
        for (int w = 0; w < WK; ++w) {
          y += z[w * RT * NB * 256];
          z[w * RT * NB * 256] = 0.f;
        }
        if (!(fabsf(y) < INFINITY) && row + k < a.rows && n < a.N) y = plain_sum(a, row + k, n, gbeg, gend);
        *z = y;
      }
    }
    __syncthreads();
  }
  // lane (g, l16) of a tile: rows 4 g + k of x, feature l16
  const bool swiglu = a.flags & ZOACT_EPI_SWIGLU;
  for (int u = tid; u < RT * NB * 64; u += TH) {
    const int ul = u & 63, b = (u >> 6) % NB, t = (u >> 6) / NB;
    floatx4 z{0.f, 0.f, 0.f, 0.f}, up{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WK; ++w) z += sum[((w * RT + t) * NB + b) * 64 + ul];
    if (a.part) {
      if (n0 + t * 16 < a.N)
        reinterpret_cast<floatx4*>(a.part)[(blockIdx.y * (a.N / 16) + n0 / 16 + t) * (NB * 64) + b * 64 + ul] = z;
      continue;
    }
    const int64_t n = n0 + t * 16 + (ul & 15);
    if (n >= a.N || (swiglu && (t & 1))) continue;
    if (swiglu) {
#pragma unroll
      for (int w = 0; w < WK; ++w) up += sum[((w * RT + t + (RT > 1 ? 1 : 0)) * NB + b) * 64 + ul];
    }
    const int row = b * 16 + 4 * (ul >> 4);
    finish(a, row, n, z, up, kEarly ? ex : load_extras(a, row, n));
  }
}

// Adds the parts of the depth in order and the correction, and finishes: a wave per tile of 16 features and
// block of 16 rows of x, whose sums lie as a product's do.  4 us after a product that took 8 to 15, most of
// it the launch and one trip to memory: bias, residual, correction and sums are all asked for at once.
template <int NB>
__global__ void __launch_bounds__(256) rows_join_kernel(RowsArgs a, int splits, int64_t tiles) {
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, tile = u / (NB * 64);
  const int lane = threadIdx.x & 63, b = (int)(u / 64 % NB), row = b * 16 + 4 * (lane >> 4);
  const int64_t n = tile * 16 + (lane & 15);
  const bool swiglu = a.flags & ZOACT_EPI_SWIGLU;
  if (tile >= tiles || (swiglu && (tile & 1))) return;
  const Extras ex = load_extras(a, row, n);
  Correction<2, 1> corr;
  corr.load(a, tile * 16, b, 0, swiglu ? 2 : 1);
  const floatx4* const part = reinterpret_cast<const floatx4*>(a.part);
  floatx4 z[2][1] = {{floatx4{0.f, 0.f, 0.f, 0.f}}, {floatx4{0.f, 0.f, 0.f, 0.f}}};
  const int up = swiglu ? NB * 64 : 0;     // (without SwiGLU the second sum repeats the first and is not used)
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const floatx4* const p = part + s * tiles * (NB * 64) + u;
    z[0][0] += p[0];
    z[1][0] += p[up];
  }
  corr.apply(a, z);
  if (whole_ranks(a)) {
    for (int i0 = 32; i0 < a.r; i0 += 32) {
      corr.load(a, tile * 16, b, i0, swiglu ? 2 : 1);
      corr.apply(a, z);
    }
  } else {
    add_odd_ranks<2, 1>(a, tile * 16, b, 0, 32, z);
  }
  finish(a, row, n, z[0][0], z[1][0], ex);
}

// Parts of the depth: as many as wanted, of at least `least` groups, and as the workspace holds.
int splits_of(const RowsArgs& a, int64_t want, int least, int NB, size_t ws_bytes) {
  const int64_t deep = a.groups / least, room = (int64_t)(ws_bytes / ((size_t)(a.N / 16) * NB * 1024));
  int64_t n = want < deep ? want : deep;
  n = n < room ? n : room;
  return n < 1 ? 1 : n > 64 ? 64 : (int)n;
}

template <int RT, int NB, int XR, int NW, int WK>
hipError_t go(RowsArgs a, int splits, void* ws, hipStream_t s) {
  const unsigned tiles = (unsigned)((a.N + 16 * RT - 1) / (16 * RT));
  const int stages = (a.groups + WK - 1) / WK, per = (stages + splits - 1) / splits;
  a.per_split = per * WK;
  splits = (stages + per - 1) / per;
  a.part = splits > 1 ? static_cast<float*>(ws) : nullptr;
  rows_kernel<RT, NB, XR, NW, WK><<<dim3(tiles, (unsigned)splits), 64 * NW, 0, s>>>(a);
  if (splits > 1) rows_join_kernel<NB><<<(unsigned)((a.N / 16 * NB + 3) / 4), 256, 0, s>>>(a, splits, a.N / 16);
  return hipGetLastError();
}

// One block of 16 rows.  What counts is the weights in flight on a compute unit and how few workgroups read x
// again, so layers of few tiles get eight waves on a tile, deep ones parts of the depth (of six stages at
// least), wide ones larger tiles, and with more than four rows, whose x weighs more than the tile, those
// also where parts fill the chip.  us on cold weights (columns x features, 1 / 13 rows; the bytes alone,
// read in one piece, take the first figure):
//   4096 x 4096   3.0: 16 weight rows, 8 waves  6.0 /  8.1;  32, 8 waves  7.2 /  8.9;  64, 4 parts  8.3 /  8.6
//   4096 x 6144   3.7:                          6.8 / 14.2;               7.5 /  9.3;               9.3 /  9.9
//   4096 x 28672 10.2: 32 weight rows, 4 waves 14.9 / 23.9;  64, 8 waves 14.6 / 17.8
//   5120 x 20480  9.6:                         14.8 / 19.2;              16.4 / 19.4
//   14336 x 4096  6.0: 1 part                  22.6 / 27.7;              25.0 / 27.7
//                      4 parts                 12.5 / 14.4;              12.7 / 13.6;  8 parts     12.6 / 14.0
//   20480 x 5120  9.6: 1 part                  31.0 / 38.7;              33.4 / 38.7
//                      4 parts                 16.7 / 21.1;              18.3 / 21.6
//                      6 parts                 16.3 / 22.9;              16.6 / 18.3;  8 parts     18.4 / 19.7
// The turn at 8192 columns lies where the sides meet for few rows; 4096 features, what is taken and the other side:
// 8192 columns 9.0 / 11.9 (four parts 9.6 / 10.7), 10240 12.1 / 13.5 (one part of 16 weight rows 10.1 / 13.5),
// 12288 11.7 / 12.9 (11.4 / 15.4).
template <int XR>
hipError_t pick16(const RowsArgs& a, int cus, void* ws, size_t ws_bytes, hipStream_t s) {
  const bool swiglu = a.flags & ZOACT_EPI_SWIGLU;
  const int64_t t16 = a.N / 16, t32 = (t16 + 1) / 2, t64 = (t16 + 3) / 4;
  if (a.K <= 8192 && t16 <= 2 * cus) {
    if (t16 <= (XR == 4 ? 2 : 1) * cus && !swiglu) return go<1, 1, XR, 8, 8>(a, 1, nullptr, s);
    return go<2, 1, XR, 8, 8>(a, 1, nullptr, s);
  }
  if constexpr (XR == 4)
    if (t32 <= 3 * cus) return go<2, 1, XR, 4, 4>(a, splits_of(a, 4 * cus / t32, 24, 1, ws_bytes), ws, s);
  return go<4, 1, XR, 8, 4>(a, splits_of(a, 2 * cus / t64, 24, 1, ws_bytes), ws, s);
}

// 17 rows and more: 128 weight rows a workgroup, so that x, which every workgroup reads whole, is read
// rarely; one workgroup a compute unit (4096 x 28672 at 64 rows 34 us, with 64 weight rows 48; 20480 x 5120
// 33 us in 6 parts, 70 in 2).  Up to 32 rows layers of few tiles take 32, whose stages are shorter: 4096 x 4096
// 9.8 us in two parts, with 128 in eight 11.9, 4096 x 6144 11.8 and 13.2, 8192 x 4096 14.0 and 14.4, 10240 x 4096
// 16.3 and 15.3 (but 4096 x 28672 42 and 23; at 48 rows 4096 x 4096 12.9 and 13.9, 4096 x 6144 15.3 and 15.7).
template <int NB>
hipError_t pick_more(const RowsArgs& a, int cus, void* ws, size_t ws_bytes, hipStream_t s) {
  const int64_t t16 = a.N / 16;
  if constexpr (NB == 2)
    if (a.K <= 8192 && t16 <= 2 * cus)
      return go<2, NB, 16 * NB, 8, 4>(a, splits_of(a, cus / ((t16 + 1) / 2), 8, NB, ws_bytes), ws, s);
  return go<8, NB, 16 * NB, 8, 2>(a, splits_of(a, cus / ((t16 + 7) / 8), 4, NB, ws_bytes), ws, s);
}

hipError_t pick(const RowsArgs& a, void* ws, size_t ws_bytes, hipStream_t s) {
  const int cus = cu_count() > 0 ? cu_count() : 256;
  if (a.rows <= 4) return pick16<4>(a, cus, ws, ws_bytes, s);
  if (a.rows <= 16) return pick16<16>(a, cus, ws, ws_bytes, s);
  if (a.rows <= 32) return pick_more<2>(a, cus, ws, ws_bytes, s);
  if (a.rows <= 48) return pick_more<3>(a, cus, ws, ws_bytes, s);
  return pick_more<4>(a, cus, ws, ws_bytes, s);
}

}  // namespace

hipError_t launch_linear_rows(const zoact_linear& L, const zoact_arena* A, const void* x, int64_t rows, const void* p,
                              const void* residual, uint32_t flags, void* y, int32_t y_dtype, hipStream_t s) {
  RowsArgs a{};
  a.w = static_cast<const uint8_t*>(L.w);
  a.sc = static_cast<const uint16_t*>(L.w_scales);
  a.bias = static_cast<const uint16_t*>(L.bias);
  a.x = static_cast<const uint16_t*>(x);
  a.p = static_cast<const uint16_t*>(p);
  a.res = static_cast<const uint16_t*>(residual);
  a.r = L.r;
  if (L.r > 0) {
    a.c_f32 = A->c_dtype == ZOACT_F32;
    a.c = static_cast<const char*>(A->c) + L.coef_offset * (a.c_f32 ? 4 : 2);
    a.plain0 = L.plain_begin;
    a.plain1 = L.plain_end;
  }
  a.rows = (int)rows;
  a.N = L.d_out;
  a.K = (int)L.d_in;
  a.groups = (int)(L.d_in / 128);
  a.y = y;
  a.y_f32 = y_dtype == ZOACT_F32;
  a.flags = flags;
  return pick(a, L.ws, L.ws ? L.ws_bytes : 0, s);
}

}  // namespace zoact
