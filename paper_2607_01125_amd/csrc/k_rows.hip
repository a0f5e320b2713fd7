// The adapted linear of a few rows with packed INT4 weights (zoact_linear_rows).
//
//   y[t][n] = epi(res + b + sum_g s[n][g] sum_{k in g} q[n][k] x[t][k] + sum_i p[t][i] bf16(C[n][i]))
//
// Bound by the weights' bytes: each is read once, 16 bytes a lane, straight into the registers that
// feed the matrix unit.  A lane's 16 bytes are 32 of the 128 columns of one scale group of one weight
// row, so one load instruction covers 16 rows and one group.  A nibble becomes a bf16 number without
// arithmetic: its bits (with the sign bit turned over, u = q + 8) are put at the top of the mantissa
// of 16, which gives 16 + u = q + 24 exactly; the surplus 24 sum x is taken out by starting the
// group's sum from a product of x with a constant -24, which costs one product for all weight rows
// of the wave.  The group's sum is then scaled: one multiply-add a lane and group, no rounding of
// q s.  The columns of a word come as pairs (i, i + 4), so x is put in that order instead.
// The waves of a workgroup share out the groups; their sums meet in LDS in a fixed order.
#include <string>

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
  void* y;
  int y_f32;
  uint32_t flags;
};

__device__ __forceinline__ bf16x8 nibbles(uint32_t v) {
  v ^= 0x88888888u;
  uint4 o;
  o.x = ((v << 3) & 0x00780078u) | 0x41804180u;
  o.y = ((v >> 1) & 0x00780078u) | 0x41804180u;
  o.z = ((v >> 5) & 0x00780078u) | 0x41804180u;
  o.w = ((v >> 9) & 0x00780078u) | 0x41804180u;
  return __builtin_bit_cast(bf16x8, o);
}
// Eight consecutive values in the order of a word's nibble pairs: (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ bf16x8 pair_order(uint4 u) {
  uint4 o;
  o.x = __builtin_amdgcn_perm(u.z, u.x, 0x05040100);
  o.y = __builtin_amdgcn_perm(u.z, u.x, 0x07060302);
  o.z = __builtin_amdgcn_perm(u.w, u.y, 0x05040100);
  o.w = __builtin_amdgcn_perm(u.w, u.y, 0x07060302);
  return __builtin_bit_cast(bf16x8, o);
}

// Eight coefficients (or values of p) from column i0 on, zeros past r.
__device__ __forceinline__ bf16x8 tail8(const uint16_t* row, int i0, int r, bool in) {
  uint16_t v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = in && i0 + e < r ? row[i0 + e] : (uint16_t)0;
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<uint4*>(v));
}
__device__ __forceinline__ bf16x8 tail8(const float* row, int i0, int r, bool in) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (__bf16)(in && i0 + e < r ? row[i0 + e] : 0.f);
  return v;
}

// RT: tiles of 16 weight rows of a workgroup (2 with SwiGLU: a gate and its up tile); NB: blocks
// of 16 rows of x; NW: waves.
template <int RT, int NB, int NW>
__global__ void __launch_bounds__(64 * NW) rows_kernel(RowsArgs a) {
  __shared__ floatx4 sum[NW][RT][NB][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * RT * 16;
  floatx4 tot[RT][NB];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) tot[t][b] = floatx4{0.f, 0.f, 0.f, 0.f};

  // weight rows of the lane (rows past the last repeat it; they are not stored)
  const uint8_t* wrow[RT];
  const uint16_t* srow[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    int64_t n = n0 + t * 16 + l16;
    if (n >= a.N) n = a.N - 1;
    wrow[t] = a.w + n * (a.K / 2) + 16 * g;
    srow[t] = a.sc + n * a.groups;
  }
  const uint16_t* xrow[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int t = b * 16 + l16;
    xrow[b] = a.x + (int64_t)(t < a.rows ? t : a.rows - 1) * a.K + 32 * g;
  }
  const uint32_t m24 = 0xC1C0C1C0u;                  // (-24, -24)
  const bf16x8 minus24 = __builtin_bit_cast(bf16x8, make_uint4(m24, m24, m24, m24));

#pragma unroll 2
  for (int gr = wave; gr < a.groups; gr += NW) {
    uint4 wv[RT];
    float s[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      wv[t] = *reinterpret_cast<const uint4*>(wrow[t] + (int64_t)gr * 64);
      s[t] = bf2f(srow[t][gr]);
    }
    bf16x8 xf[NB][4];
    floatx4 off[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        xf[b][j] = pair_order(*reinterpret_cast<const uint4*>(xrow[b] + (int64_t)gr * 128 + 8 * j));
      off[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j) off[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[b][j], minus24, off[b], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const uint32_t wd[4] = {wv[t].x, wv[t].y, wv[t].z, wv[t].w};
      floatx4 acc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = off[b];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8 wf = nibbles(wd[j]);
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[b][j], wf, acc[b], 0, 0, 0);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) tot[t][b][i] = fmaf(s[t], acc[b][i], tot[t][b][i]);
    }
  }
  // the correction, 32 ranks a step, the steps shared out over the waves
  for (int i0 = 32 * wave; i0 < a.r; i0 += 32 * NW) {
    bf16x8 pf[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int t = b * 16 + l16;
      pf[b] = tail8(a.p + (int64_t)(t < a.rows ? t : a.rows - 1) * a.r, i0 + 8 * g, a.r, true);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t n = n0 + t * 16 + l16;
      const bool in = n < a.N && !(n >= a.plain0 && n < a.plain1);
      const int64_t row = !in ? 0 : n >= a.plain1 ? n - (a.plain1 - a.plain0) : n;
      const bf16x8 cf = a.c_f32 ? tail8(static_cast<const float*>(a.c) + row * a.r, i0 + 8 * g, a.r, in)
                                : tail8(static_cast<const uint16_t*>(a.c) + row * a.r, i0 + 8 * g, a.r, in);
#pragma unroll
      for (int b = 0; b < NB; ++b) tot[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[b], cf, tot[t][b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) sum[wave][t][b][lane] = tot[t][b];
  __syncthreads();
  // lane (g, l16) of a tile: rows 4 g + i of x, feature l16
  const bool swiglu = a.flags & ZOACT_EPI_SWIGLU;
  constexpr int UNITS = RT * NB * 64;
  for (int u = threadIdx.x; u < UNITS; u += 64 * NW) {
    const int ul = u & 63, b = (u >> 6) % NB, t = (u >> 6) / NB;
    if (swiglu && (t & 1)) continue;
    const int64_t n = n0 + t * 16 + (ul & 15);
    if (n >= a.N) continue;
    floatx4 z[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k && !swiglu) break;
      const int tt = RT > 1 ? t + k : t;
      floatx4 v = sum[0][tt][b][ul];
#pragma unroll
      for (int w = 1; w < NW; ++w) v += sum[w][tt][b][ul];
      z[k] = v;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = b * 16 + 4 * (ul >> 4) + i;
      if (row >= a.rows) continue;
      float y = z[0][i];
      if (a.bias) y += bf2f(a.bias[n]);
      if (a.res) y += bf2f(a.res[(int64_t)row * a.N + n]);
      int64_t at = (int64_t)row * a.N + n;
      if (swiglu) {
        float up = z[1][i];
        if (a.bias) up += bf2f(a.bias[n + 16]);
        if (a.res) up += bf2f(a.res[(int64_t)row * a.N + n + 16]);
        y = y / (1.f + __expf(-y)) * up;
        at = (int64_t)row * (a.N / 2) + n / 32 * 16 + (n & 15);
      } else if (a.flags & ZOACT_EPI_RELU) {
        y = y > 0.f ? y : y != y ? y : 0.f;
      }
      if (a.y_f32)
        static_cast<float*>(a.y)[at] = y;
      else
        static_cast<uint16_t*>(a.y)[at] = f2bf(y);
    }
  }
}

template <int RT, int NB, int NW>
hipError_t go(const RowsArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)((a.N + 16 * RT - 1) / (16 * RT));
  rows_kernel<RT, NB, NW><<<grid, 64 * NW, 0, s>>>(a);
  return hipGetLastError();
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
  if (rows <= 16) return go<2, 1, 8>(a, s);
  if (rows <= 32) return go<2, 2, 8>(a, s);
  return go<2, 4, 8>(a, s);
}

}  // namespace zoact
