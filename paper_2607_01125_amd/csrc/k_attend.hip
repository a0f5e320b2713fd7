// Attention over the paged 8-bit cache (zoact_cache.h).
//
// One wave works on one page (64 tokens) of one key/value head at a time, for 16 query columns:
// the heads that share the key/value head times the new rows.  Scores are formed transposed,
// S^T = K Q^T, so that a lane holds, of one query column (lane % 16), the tokens 16 n + 4 g + i
// (g = lane / 16; n, i < 4) of the page: the softmax statistics stay in the lane (two shuffles
// per page join the four lanes of a column), and those 16 probabilities are, as they stand, the
// right operand of O^T = V^T P^T -- the page keeps V's tokens in that order, so nothing moves
// between lanes and K and V go from memory to the matrix unit in whole 16-byte loads.
// Codes become f16 without rounding; a K scale multiplies its block's scores, a V scale its block's
// probabilities.  q (brought to f16's range by a power of two for each column) and the probabilities
// enter as NT f16 terms: one carries 11 bits (bf16 activations: the output has 8), two carry 22 and
// more (fp32).  bf16 terms would need two and three for this.
#include <math.h>

#include <string>

#include "cache.hpp"

namespace zoact {
namespace {

struct AttendArgs {
  zoact_cache c;
  zoact_cache_batch b;
  int layer, H, G, S, pps;     // splits, pages per split (the last split takes the rest)
  const void* q;
  int64_t ldq;
  float scale;                 // scale * log2(e)
  const float *ct, *st;
  int64_t n_pos;
  void* out;
  float* part;                 // [n * max_new * H][S][HD], each split's weighted mean of values
  float2* ml;                  // [n * max_new * H][S] maximum (log2 domain) and sum of weights
};

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Four int8 codes as f16, exactly: with its sign bit turned over a code is u = code + 128, and the bytes
// (u, 0x64) are the f16 number 1024 + u.
__device__ __forceinline__ void codes4(uint32_t w, uint32_t (&o)[2]) {
  w ^= 0x80808080u;
  const f16x2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
  o[0] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400)) + off);
  o[1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402)) + off);
}
__device__ __forceinline__ f16x8 codes8(uint32_t a, uint32_t b) {
  uint32_t x[2], y[2];
  codes4(a, x);
  codes4(b, y);
  return __builtin_bit_cast(f16x8, make_uint4(x[0], x[1], y[0], y[1]));
}
// x as NT f16 terms, each the nearest to what the ones before it leave.  What a term is taken from is held in a
// register: where the compiler forms one rounding from x's own product and another from its fp32 value, the two
// differ by a step now and then, and the second term would belong to a first that is not the one used.
template <int NT>
__device__ __forceinline__ void terms8(const float (&x)[8], f16x8 (&t)[NT]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int k = 0; k < NT; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (NT > 1) asm("" : "+v"(r[e]));
      t[k][e] = (_Float16)r[e];
      if (k + 1 < NT) r[e] -= (float)t[k][e];
    }
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  } else {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}

// Loads of what all lanes share and no one writes meanwhile (scales, page numbers): through the scalar
// cache, into scalar registers.
__device__ __forceinline__ floatx4 scalar4(const float* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) floatx4*>(reinterpret_cast<uintptr_t>(p));
}
__device__ __forceinline__ int scalar1(const int* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int*>(reinterpret_cast<uintptr_t>(p));
}

// A page of one head on its way to the wave, 16 bytes a lane and load (HD 32: K's upper half is not used).
// Through a descriptor of the page: the lane's part of the address stays, the rest is scalar.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_rsrc(const int8_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(p), 0, bytes, 0x00020000);
}
template <int HD>
__device__ __forceinline__ uint4 load_keys(__amdgpu_buffer_rsrc_t rs, int lane, int n, int h) {
  const int vo = (lane & 15) * HD + (HD == 32 ? 8 : 16) * (lane >> 4), so = n * 16 * HD + 64 * h;
  if constexpr (HD == 32) {
    const uint2 t = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rs, vo, so, 0));
    return make_uint4(t.x, t.y, 0, 0);
  } else {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, vo, so, 0));
  }
}
__device__ __forceinline__ uint4 load_values(__amdgpu_buffer_rsrc_t rs, int lane, int d) {
  return __builtin_bit_cast(
      uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, (lane & 15) * kPage + 16 * (lane >> 4), d * 16 * kPage, 0));
}
template <int HD>
struct KeyLoad {
  static constexpr int H = HD == 32 ? 1 : HD / 64, N = 4 * H;
  uint4 u[N];
  __device__ __forceinline__ void go(const int8_t* kp, int lane) {
    const __amdgpu_buffer_rsrc_t rs = page_rsrc(kp, kPage * HD);
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = load_keys<HD>(rs, lane, i / H, i % H);
  }
};
template <int HD>
struct ValueLoad {
  uint4 u[HD / 16];
  __device__ __forceinline__ void go(const int8_t* vp, int lane) {
    const __amdgpu_buffer_rsrc_t rs = page_rsrc(vp, kPage * HD);
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) u[d] = load_values(rs, lane, d);
  }
};

constexpr int kPExp = 14;         // probabilities enter their product times 2^14: f16 then keeps 11 bits
                                  // of them down to 2^-28, and something down to 2^-38
constexpr int kNoScale = -200;    // below every exponent of an fp32 number

// V scales of a page's blocks that hold a token up to `last`, the column's own, times a power of two that keeps
// p vsc below 2^14; vexp follows, and o's unit 2^(vexp - 14) with it.  Each column has its own vexp: later tokens'
// scales, which columns of the same wave may see, take none of its bits.
__device__ __forceinline__ void value_scales(const floatx4& vs, int t0, int last, int& vexp, float (&vsc)[4]) {
  const float v[4] = {vs[0], vs[1], vs[2], vs[3]};
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    vsc[n] = t0 + 16 * n > last ? 0.f : v[n];
    const int ex = vsc[n] > 0.f ? __builtin_amdgcn_frexp_expf(vsc[n]) : kNoScale;   // (NaN stays NaN)
    vexp = ex > vexp ? ex : vexp;
  }
#pragma unroll
  for (int n = 0; n < 4; ++n) vsc[n] = __builtin_amdgcn_ldexpf(vsc[n], kPExp - vexp);
}

// One page's scores of a lane's column, s times its block's f >= 0 (log2 domain): masks tokens past lim (edge:
// there may be some), updates the running maximum and sum, and gives the factor of what was summed before and
// the probabilities times V's scales as terms.  The maximum is taken before the factor, a product a block, and
// the factor and the maximum's subtraction are one multiply-add a score.  That one does not round the product
// as the maximum's was, which scores below 2^20 allow (a probability stays below 2^(1/16)): |s| < 2^29 (128
// values below 2^15 times 127), so f <= 2^-9 will do, and larger ones are multiplied first, as masked pages are.
template <int NT>
__device__ __forceinline__ void soft_page(float (&s)[4][4], float (&f)[4], int t0, int lim, bool edge, int g,
                                          const float (&vsc)[4], float& m, float& l, float& alpha,
                                          f16x8 (&pf)[2][NT]) {
  if (edge || __any(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])) > 0x1p-9f)) {
#pragma unroll
    for (int n = 0; n < 4; ++n) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][i] = t0 + 16 * n + 4 * g + i > lim ? -INFINITY : s[n][i] * f[n];
      f[n] = 1.f;
    }
  }
  float mx = m;
#pragma unroll
  for (int n = 0; n < 4; ++n) mx = fmaxf(mx, fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3])) * f[n]);
  mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
  mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
  const float base = mx == -INFINITY ? 0.f : mx;
  alpha = __builtin_amdgcn_exp2f(m - base);
  m = mx;
  l *= alpha;
  float lsum = 0.f;
#pragma unroll
  for (int n2 = 0; n2 < 2; ++n2) {
    float p8[8];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[2 * n2 + n][i], f[2 * n2 + n], -base));
        p8[4 * n + i] = p[i] * vsc[2 * n2 + n];
      }
      lsum += (p[0] + p[1]) + (p[2] + p[3]);
    }
    terms8<NT>(p8, pf[n2]);
  }
  l += lsum;
}

// What a sum of weights is divided by, as a factor: 0 for the sum of nothing.  (A sum is no less than 2^(-1/16), the
// weight of its own maximum.)
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.f ? 0.f : 1.f / l; }

// q of one column as right operands: step s of a lane holds dims 64 (s / 2) + 16 g + 8 (s % 2) + 0..7 (HD 32:
// 8 g + 0..7), rotated, times a power of two that brings the column's largest to [2^14, 2^15).
template <typename T, int HD>
__device__ __forceinline__ void query_step(const AttendArgs& a, int64_t row, int h, int64_t pos, int g, int s,
                                           float (&x)[8]) {
  constexpr int HALF = HD / 2;
  const T* const qr = static_cast<const T*>(a.q) + row * a.ldq + (int64_t)h * HD;
  const int d = HD == 32 ? 8 * g : 64 * (s >> 1) + 16 * g + 8 * (s & 1);
  load8(qr + d, x);
  if (a.ct) {
#pragma clang fp contract(off)
    const bool up = d >= HALF;
    const int64_t base = (pos < a.n_pos ? pos : a.n_pos - 1) * HALF + (up ? d - HALF : d);
    float y[8], cs[8], sn[8];
    load8(qr + (up ? d - HALF : d + HALF), y);
    load8(a.ct + base, cs);
    load8(a.st + base, sn);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = up ? x[k] * cs[k] + y[k] * sn[k] : x[k] * cs[k] - y[k] * sn[k];
  }
}
// Largest magnitude of a column in a lane's values and its three partners'.
__device__ __forceinline__ float column_top(const float (&x)[8], float top) {
#pragma unroll
  for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(x[k]));
  return top;
}
// Factor of the values, and of the scores (log2 domain) in return, that one not negative; both powers of two
// stay normal numbers.
__device__ __forceinline__ float column_shift(const AttendArgs& a, float top, float& factor) {
  int sh = 14 - ((int)(__float_as_uint(top) >> 23) - 127);
  sh = top == 0.f ? 0 : sh > 120 ? 120 : sh < -113 ? -113 : sh;
  factor = copysignf(__uint_as_float((uint32_t)(127 + sh) << 23), a.scale);
  return __uint_as_float((uint32_t)(127 - sh) << 23) * fabsf(a.scale);
}
template <typename T, int HD, int NT>
__device__ __forceinline__ float load_query(const AttendArgs& a, int64_t row, int h, int64_t pos, int g,
                                            f16x8 (&qf)[HD / 32][NT]) {
  constexpr int KS = HD / 32;
  float x[KS][8], top = 0.f, factor;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    query_step<T, HD>(a, row, h, pos, g, s, x[s]);
    top = column_top(x[s], top);
  }
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  const float qs = column_shift(a, top, factor);
#pragma unroll
  for (int s = 0; s < KS; ++s) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[s][k] *= factor;
    terms8<NT>(x[s], qf[s]);
  }
  return qs;
}

// A workgroup's key/value head, split and column tile.  Workgroups go to the eight XCDs in turn, so heads,
// which all have the same work, come first in the order, and an entry's splits start at its number:
// the late ones, which short sequences leave empty, do not meet on one XCD (with splits first the
// 48-sequence batch took 113 us, with heads first 71).
struct Place {
  int hk, split, tile;
};
__device__ __forceinline__ Place place_of(const AttendArgs& a) {
  const unsigned x = blockIdx.x, hkv = (unsigned)a.c.n_kv_heads, q = x / hkv;
  Place p;
  p.hk = (int)(x % hkv);
  p.tile = (int)(q / a.S);
  p.split = (int)((q % a.S + blockIdx.z) % a.S);
  return p;
}

struct Range {
  int last, pbeg, pend;     // last visible token, pages of the split
};
__device__ __forceinline__ Range split_range(const AttendArgs& a, const CacheEntry& e, int jmax, int split) {
  Range r;
  r.last = e.ok ? e.pos + jmax : -1;
  const int pages = (r.last + kPage) / kPage;
  r.pbeg = split * a.pps;
  r.pend = split == a.S - 1 ? pages : (r.pbeg + a.pps < pages ? r.pbeg + a.pps : pages);
  return r;
}

// Decoding: at most 16 columns, each wave its own pages.  Bound by the pages' bytes: one row behind 131071 tokens,
// 8 key/value heads of 128 (268 MB), 51 us and 5 for the join, 5.3 TB/s; the same pages read in the same way
// and nothing done with them, 45 us.  48 rows behind 70 to 8000 tokens (271 MB): 60 and 5.  35 to 43% of a wave's
// cycles wait for memory, a third issue vector instructions.  (Pages through LDS in whole rows' order: 67 us
// where this order took 61.)
template <typename T, int HD, int NT>
__global__ void __launch_bounds__(256, NT == 1 ? 3 : 2) attend_kernel(AttendArgs a) {
  constexpr int KS = HD / 32;           // 32-deep products of a score
  constexpr int DT = HD / 16;           // 16-wide tiles of the output
  constexpr int LD = HD + 4;
  __shared__ __align__(16) char lds[4 * 16 * LD * 4];
  float(*const so)[16][LD] = reinterpret_cast<float(*)[16][LD]>(lds);      // at the end
  f16x8(*const sq)[NT][64] = reinterpret_cast<f16x8(*)[NT][64]>(lds);      // q, until the waves have read it
  static_assert(KS * NT * 1024 <= 4 * 16 * LD * 4, "q fits");
  __shared__ float sm[4][16], sl[4][16];
  const zoact_cache& c = a.c;
  const Place at = place_of(a);
  const int hk = at.hk, split = at.split, c0 = at.tile * 16;
  const CacheEntry e = read_entry(c, a.b, blockIdx.z, threadIdx.x == 0 && blockIdx.x == 0);
  const int ncol = e.count * a.G;
  if (c0 >= ncol) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4;
  const Range rg = split_range(a, e, (c0 + 15 < ncol ? c0 + 15 : ncol - 1) / a.G, split);

  floatx4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  int vexp = kNoScale;   // V scales the column has seen are below 2^vexp; o is kept in units of 2^(vexp - 14)

  if (rg.pbeg < rg.pend) {
    // the first page's keys are on their way before q is ready, each next page's before this one's softmax
    const int* const trow = c.table + (int64_t)e.slot * c.max_pages;
    const int64_t lbase = (int64_t)a.layer * c.n_pages;
    auto head_of = [&](int pid, bool& bad) {
      bad = pid < 0 || pid >= c.n_pages;
      return (lbase + (bad ? 0 : pid)) * c.n_kv_heads + hk;
    };
    int pg = rg.pbeg + wave;
    const bool any = pg < rg.pend;
    bool bad = false;
    int64_t head = 0;
    KeyLoad<HD> kl;
    ValueLoad<HD> vl;
    floatx4 ks;
    int pid1 = 0;
    if (any) {
      head = head_of(scalar1(trow + pg), bad);
      kl.go(c.k + head * (kPage * HD), lane);
      ks = scalar4(c.k_scale + head * 4);
      if (pg + 4 < rg.pend) pid1 = scalar1(trow + pg + 4);
    }
    // the columns are the same in all waves: each prepares one step of q for all
    const int col = c0 + (lane & 15), cq = col < ncol ? col : ncol - 1;   // (columns past the last repeat it)
    const int tcol = e.pos + cq / a.G;                                    // the column's last token
    float x[8], top = 0.f, factor;
    if (wave < KS) {
      query_step<T, HD>(a, e.row0 + cq / a.G, hk * a.G + cq % a.G, tcol, g, wave, x);
      top = column_top(x, 0.f);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
    }
    if (g == 0) sm[wave][lane] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sm[0][lane & 15], sm[1][lane & 15]), fmaxf(sm[2][lane & 15], sm[3][lane & 15]));
    const float qs = column_shift(a, top, factor);
    if (wave < KS) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= factor;
      f16x8 t[NT];
      terms8<NT>(x, t);
#pragma unroll
      for (int q = 0; q < NT; ++q) sq[wave][q][lane] = t[q];
    }
    __syncthreads();
    f16x8 qf[KS][NT];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int q = 0; q < NT; ++q) qf[s][q] = sq[s][q][lane];

    while (any) {
      vl.go(c.v + head * (kPage * HD), lane);
      const floatx4 vs = scalar4(c.v_scale + head * 4);
      const float ksc[4] = {ks[0], ks[1], ks[2], ks[3]};
      float s[4][4], f[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        floatx4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint4 u = kl.u[n * (KeyLoad<HD>::N / 4) + k / 2];
          const f16x8 kf = k & 1 ? codes8(u.z, u.w) : codes8(u.x, u.y);
#pragma unroll
          for (int q = 0; q < NT; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[k][q], acc, 0, 0, 0);
        }
        f[n] = ksc[n] * qs;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = acc[i];
        __builtin_amdgcn_sched_barrier(0);      // (codes converted early would not fit three waves' registers)
      }
      const int t0 = pg * kPage, next = pg + 4;
      const bool now_bad = bad;
      if (next < rg.pend) {
        head = head_of(pid1, bad);
        kl.go(c.k + head * (kPage * HD), lane);
        ks = scalar4(c.k_scale + head * 4);
        pid1 = next + 4 < rg.pend ? scalar1(trow + next + 4) : 0;
      }
      // a page number that is none counts as if its tokens were masked
      if (now_bad && lane == 0) raise_status(a.b.status, ZOACT_STATUS_BAD_ENTRY);
      const bool edge = now_bad || t0 + kPage > e.pos + c0 / a.G + 1;    // some column ends inside the page
      float vsc[4], alpha;
      const int vold = vexp;
      value_scales(vs, t0, now_bad ? -1 : tcol, vexp, vsc);
      f16x8 pf[2][NT];
      soft_page<NT>(s, f, t0, now_bad ? -1 : tcol, edge, g, vsc, m, l, alpha, pf);
      alpha = __builtin_amdgcn_ldexpf(alpha, vold - vexp);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f16x8 v0 = codes8(vl.u[d].x, vl.u[d].y), v1 = codes8(vl.u[d].z, vl.u[d].w);
        floatx4 acc = o[d] * alpha;
#pragma unroll
        for (int q = 0; q < NT; ++q) {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[0][q], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[1][q], acc, 0, 0, 0);
        }
        o[d] = acc;
        if (d & 1) __builtin_amdgcn_sched_barrier(0);
      }
      if (next >= rg.pend) break;
      pg = next;
    }
  }
  // the four waves' results (q and its maxima have been read by all), means: sums of large values would overflow
  __syncthreads();
  constexpr int DV = HD / 16;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  const float inverse = inverse_sum(l);
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    floatx4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_ldexpf(o[d][i] * inverse, vexp - kPExp);
    *reinterpret_cast<floatx4*>(&so[wave][lane & 15][d * 16 + 4 * g]) = r;
  }
  if (g == 0) {
    sm[wave][lane] = m;
    sl[wave][lane] = l;
  }
  __syncthreads();
  const int oc = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * DV, col = c0 + oc;
  if (col >= ncol) return;
  float M = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w][oc]);
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f, r[DV], f[4];
#pragma unroll
  for (int k = 0; k < DV; ++k) r[k] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = __builtin_amdgcn_exp2f(sm[w][oc] - base) * sl[w][oc];
    L += f[w];
  }
  const float share = inverse_sum(L);
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int k = 0; k < DV; ++k) r[k] += f[w] * share * so[w][oc][d0 + k];
  const int oj = col / a.G, oh = hk * a.G + col % a.G;
  if (a.S == 1) {
    T* const op = static_cast<T*>(a.out) + ((int64_t)(e.row0 + oj) * a.H + oh) * HD + d0;
#pragma unroll
    for (int k = 0; k < DV; ++k) {
      if constexpr (sizeof(T) == 2)
        op[k] = f2bf(r[k]);
      else
        op[k] = r[k];
    }
  } else {
    const int64_t R = (((int64_t)blockIdx.z * a.b.max_new + oj) * a.H + oh) * a.S + split;
    if (d0 == 0) a.ml[R] = make_float2(M, L);
    if (L != 0.f) {
#pragma unroll
      for (int k = 0; k < DV; ++k) a.part[R * HD + d0 + k] = r[k];
    }
  }
}

// Chunks of new rows: 64 columns a workgroup, 16 a wave; the waves walk the pages together.  Each converts a
// quarter of a page to f16 in LDS, as operands in the order they are read (1 KB apart and contiguous, so
// neither side has bank conflicts), the next page's codes on their way meanwhile.  Two buffers and one barrier
// a page, or one buffer and two where that lets a compute unit hold a third workgroup.
// Bound by the vector units' share (16 scores a lane and page: scale, maximum, exponential, rounding), the LDS
// reads and the products in turn: 333 rows of three sequences behind 500 to 1500, 40 heads of 128, 56 us, 356
// TFLOP/s (with two buffers 63; alone on the card 62, in fp32 82); 4 times 2048 rows, 32/8 heads, 210 us.  128
// columns a workgroup, which halve the LDS reads but take 248 registers, are no faster: 71 us and 213.
// One form and one number of splits serve a batch, by its longest entry's rows: a single token behind 131070 beside
// a chunk of 512 rows walks its pages in one workgroup a head, 3.5 ms for the batch; apart they take 52 and 22 us.
constexpr int chunk_buffers(int HD, int NT) { return HD == 128 && NT == 1 ? 1 : 2; }
template <typename T, int HD, int NT>
__global__ void __launch_bounds__(256, chunk_buffers(HD, NT) == 1 ? 3 : 2) attend_chunk_kernel(AttendArgs a) {
  constexpr int KS = HD / 32, DT = HD / 16;
  constexpr int KL = HD == 32 ? 1 : HD / 64;          // K loads of a wave (its 16 tokens)
  constexpr int VL = (DT + 3) / 4;                    // V tiles of a wave
  constexpr int NBUF = chunk_buffers(HD, NT);
  __shared__ f16x8 kb[NBUF][4][KS][64];
  __shared__ f16x8 vb[NBUF][DT][2][64];
  const zoact_cache& c = a.c;
  const Place at = place_of(a);
  const int hk = at.hk, split = at.split, c0 = at.tile * 64;
  const CacheEntry e = read_entry(c, a.b, blockIdx.z, threadIdx.x == 0 && blockIdx.x == 0);
  const int ncol = e.count * a.G;
  if (c0 >= ncol) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4;
  const Range rg = split_range(a, e, (c0 + 63 < ncol ? c0 + 63 : ncol - 1) / a.G, split);
  const int w0 = c0 + 16 * wave;                 // the wave's first column
  // (a wave past the last column repeats it, so that every wave reaches every barrier)
  const int wfirst = e.pos + (w0 < ncol ? w0 : ncol - 1) / a.G;
  const int wlast = e.pos + (w0 + 15 < ncol ? w0 + 15 : ncol - 1) / a.G;

  const int col = w0 + (lane & 15), cq = col < ncol ? col : ncol - 1;
  floatx4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  int vexp = kNoScale;
  if (rg.pbeg < rg.pend) {
    const int* const trow = c.table + (int64_t)e.slot * c.max_pages;
    const int64_t lbase = (int64_t)a.layer * c.n_pages;
    uint4 kr[KL], vr[VL];
    floatx4 ks, vs;
    bool bad;
    auto load = [&](int pid) {
      bad = pid < 0 || pid >= c.n_pages;
      const int64_t head = (lbase + (bad ? 0 : pid)) * c.n_kv_heads + hk;
      const __amdgpu_buffer_rsrc_t krs = page_rsrc(c.k + head * (kPage * HD), kPage * HD);
      const __amdgpu_buffer_rsrc_t vrs = page_rsrc(c.v + head * (kPage * HD), kPage * HD);
#pragma unroll
      for (int h = 0; h < KL; ++h) kr[h] = load_keys<HD>(krs, lane, wave, h);
#pragma unroll
      for (int d = 0; d < VL; ++d) {
        const int dt = wave * VL + d;
        if (DT % 4 == 0 || dt < DT) vr[d] = load_values(vrs, lane, dt);
      }
      ks = scalar4(c.k_scale + head * 4);
      vs = scalar4(c.v_scale + head * 4);
    };
    load(scalar1(trow + rg.pbeg));
    int pid1 = rg.pbeg + 1 < rg.pend ? scalar1(trow + rg.pbeg + 1) : 0;
    const int tcol = e.pos + cq / a.G;
    f16x8 qf[KS][NT];
    const float qs = load_query<T, HD, NT>(a, e.row0 + cq / a.G, hk * a.G + cq % a.G, tcol, g, qf);
    for (int pg = rg.pbeg, buf = 0; pg < rg.pend; ++pg, buf ^= NBUF - 1) {
      if (NBUF == 1 && pg > rg.pbeg) __syncthreads();
#pragma unroll
      for (int k = 0; k < KS; ++k)
        kb[buf][wave][k][lane] = k & 1 ? codes8(kr[k / 2].z, kr[k / 2].w) : codes8(kr[k / 2].x, kr[k / 2].y);
#pragma unroll
      for (int d = 0; d < VL; ++d) {
        const int dt = wave * VL + d;
        if (DT % 4 == 0 || dt < DT) {
          vb[buf][dt][0][lane] = codes8(vr[d].x, vr[d].y);
          vb[buf][dt][1][lane] = codes8(vr[d].z, vr[d].w);
        }
      }
      const float ksc[4] = {ks[0], ks[1], ks[2], ks[3]};
      const floatx4 vsn = vs;
      const bool now_bad = bad;
      if (pg + 1 < rg.pend) {
        load(pid1);
        pid1 = pg + 2 < rg.pend ? scalar1(trow + pg + 2) : 0;
      }
      __syncthreads();
      const int t0 = pg * kPage;
      if (now_bad && threadIdx.x == 0) raise_status(a.b.status, ZOACT_STATUS_BAD_ENTRY);
      if (now_bad || t0 > wlast) continue;            // nothing here that the wave's columns see
      const bool edge = t0 + kPage > wfirst + 1;
      float vsc[4];
      const int vold = vexp;
      value_scales(vsn, t0, tcol, vexp, vsc);
      float s[4][4], f[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        floatx4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const f16x8 kf = kb[buf][n][k][lane];
#pragma unroll
          for (int q = 0; q < NT; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[k][q], acc, 0, 0, 0);
        }
        f[n] = ksc[n] * qs;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = acc[i];
      }
      f16x8 pf[2][NT];
      float alpha;
      soft_page<NT>(s, f, t0, tcol, edge, g, vsc, m, l, alpha, pf);
      alpha = __builtin_amdgcn_ldexpf(alpha, vold - vexp);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f16x8 v0 = vb[buf][d][0][lane], v1 = vb[buf][d][1][lane];
        floatx4 acc = o[d] * alpha;
#pragma unroll
        for (int q = 0; q < NT; ++q) {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[0][q], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[1][q], acc, 0, 0, 0);
        }
        o[d] = acc;
      }
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (col >= ncol) return;
  const int oj = col / a.G, oh = hk * a.G + col % a.G;
  const float inverse = inverse_sum(l);
  const int64_t R = (((int64_t)blockIdx.z * a.b.max_new + oj) * a.H + oh) * a.S + split;
  if (a.S > 1 && g == 0) a.ml[R] = make_float2(m, l);
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    float r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_ldexpf(o[d][i] * inverse, vexp - kPExp);
    const int d0 = d * 16 + 4 * g;
    if (a.S > 1) {
      if (l != 0.f) *reinterpret_cast<float4*>(a.part + R * HD + d0) = make_float4(r[0], r[1], r[2], r[3]);
    } else {
      T* const op = static_cast<T*>(a.out) + ((int64_t)(e.row0 + oj) * a.H + oh) * HD + d0;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint2*>(op) = make_uint2((uint32_t)f2bf(r[0]) | (uint32_t)f2bf(r[1]) << 16,
                                                   (uint32_t)f2bf(r[2]) | (uint32_t)f2bf(r[3]) << 16);
      } else {
        *reinterpret_cast<float4*>(op) = make_float4(r[0], r[1], r[2], r[3]);
      }
    }
  }
}

constexpr int kMaxSplits = 128;
// Weight of a split with sum l and maximum m in a row whose maximum is the base.  An empty one (l == 0) has written
// no mean; any other counts with its mean, even where the weight is 0, so that a NaN among its values
// reaches the row as it does unsplit: the joins mark the empty ones' shares by -1.
__device__ __forceinline__ float split_weight(float m, float l, float base) {
  return l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - base) * l;
}
// Joins up to eight splits of a row and head in half a wave, HD / 32 columns a lane; sums and statistics (a lane
// holds those of split lane % 8) are asked for at once.  Bound by the launch and one trip to memory: 48 rows of 32
// heads in eight splits 5 us; for 512 rows in three, a workgroup a row and head took 13 us more.
constexpr int kFewSplits = 8;
template <typename T, int HD>
__global__ void __launch_bounds__(256) attend_join_few_kernel(AttendArgs a) {
  constexpr int DV = HD / 32;
  typedef float vec __attribute__((ext_vector_type(DV)));
  const CacheEntry e = read_entry(a.c, a.b, blockIdx.z, false);
  const int lane = threadIdx.x & 63, d0 = (lane & 31) * DV;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int64_t R = ((int64_t)blockIdx.z * a.b.max_new * a.H + row) * a.S;
  if (row >= (int64_t)e.count * a.H) return;
  const int k0 = lane & 7;
  const float2 got = a.ml[R + (k0 < a.S ? k0 : 0)];
  vec v[kFewSplits];
#pragma unroll
  for (int k = 0; k < kFewSplits; ++k)
    v[k] = *reinterpret_cast<const vec*>(a.part + (R + (k < a.S ? k : 0)) * HD + d0);
  const float m = k0 < a.S ? got.x : -INFINITY, l = k0 < a.S ? got.y : 0.f;
  float M = m;
#pragma unroll
  for (int k = 1; k < 8; k <<= 1) M = fmaxf(M, __shfl_xor(M, k, 64));
  const float base = M == -INFINITY ? 0.f : M;
  float f = split_weight(m, l, base), L = f;
#pragma unroll
  for (int k = 1; k < 8; k <<= 1) L += __shfl_xor(L, k, 64);
  f = l == 0.f ? -1.f : f * inverse_sum(L);
  vec r = 0.f;
#pragma unroll
  for (int k = 0; k < kFewSplits; ++k) {
    const float w = __shfl(f, (lane & ~7) | k, 64);
    if (!(w < 0.f)) r += w * v[k];      // (a NaN weight counts)
  }
  T* const op = static_cast<T*>(a.out) + ((int64_t)e.row0 * a.H + row) * HD + d0;
#pragma unroll
  for (int d = 0; d < DV; ++d) {
    if constexpr (sizeof(T) == 2)
      op[d] = f2bf(r[d]);
    else
      op[d] = r[d];
  }
}

// Joins more splits of one row and head: 32 lanes of HD / 32 columns, eight groups of splits, up to NI each.
// A thread's sums are on their way while the statistics, a thread a split, give the weights.  32 heads of one row
// in 96 splits: 5 us.
template <typename T, int HD>
__global__ void __launch_bounds__(256) attend_join_kernel(AttendArgs a) {
  constexpr int DV = HD / 32, NG = 8, NI = kMaxSplits / NG;
  typedef float vec __attribute__((ext_vector_type(DV)));
  __shared__ float wt[kMaxSplits], red[2], redl[2];
  __shared__ vec sr[NG][32];
  const int i = blockIdx.z, j = blockIdx.y, h = blockIdx.x;
  const CacheEntry e = read_entry(a.c, a.b, i, false);
  if (j >= e.count) return;
  const int64_t R = (((int64_t)i * a.b.max_new + j) * a.H + h) * a.S;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, grp = tid >> 5;
  float2 ml = make_float2(-INFINITY, 0.f);
  if (tid < a.S) ml = a.ml[R + tid];
  vec v[NI];
#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int at = grp + k * NG < a.S ? grp + k * NG : 0;
    v[k] = *reinterpret_cast<const vec*>(a.part + (R + at) * HD + (tid & 31) * DV);
  }
  if (wave < kMaxSplits / 64) {
    float M = ml.x;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) M = fmaxf(M, __shfl_xor(M, k, 64));
    if (lane == 0) red[wave] = M;
  }
  __syncthreads();
  if (wave < kMaxSplits / 64) {
    const float M = fmaxf(red[0], red[1]), base = M == -INFINITY ? 0.f : M;
    float L = split_weight(ml.x, ml.y, base);
    wt[tid] = ml.y == 0.f ? -1.f : L;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) L += __shfl_xor(L, k, 64);
    if (lane == 0) redl[wave] = L;
  }
  __syncthreads();
  const float share = inverse_sum(redl[0] + redl[1]);
  vec r = 0.f;
#pragma unroll
  for (int k = 0; k < NI; ++k)
    if (grp + k * NG < a.S) {
      const float w = wt[grp + k * NG];
      if (!(w < 0.f)) r += w * share * v[k];    // (a NaN weight counts)
    }
  sr[grp][tid & 31] = r;
  __syncthreads();
  if (tid >= HD) return;
  float y = 0.f;
#pragma unroll
  for (int k = 0; k < NG; ++k) y += reinterpret_cast<const float*>(sr[k])[tid];
  T* const op = static_cast<T*>(a.out) + ((int64_t)(e.row0 + j) * a.H + h) * HD + tid;
  if constexpr (sizeof(T) == 2)
    *op = f2bf(y);
  else
    *op = y;
}

// Query columns of a workgroup: 16 while that holds an entry's (decoding), 64 for chunks of rows.
int attend_cols(const zoact_cache_batch& b, int G) { return (int64_t)b.max_new * G <= 16 ? 16 : 64; }

template <typename T, int HD, int NT>
void run_attend(const AttendArgs& a, int w, hipStream_t s) {
  const int tiles = (int)(((int64_t)a.b.max_new * a.G + w - 1) / w);
  const dim3 grid((unsigned)(tiles * a.S * a.c.n_kv_heads), 1, (unsigned)a.b.n);
  if (w == 16)
    attend_kernel<T, HD, NT><<<grid, 256, 0, s>>>(a);
  else
    attend_chunk_kernel<T, HD, NT><<<grid, 256, 0, s>>>(a);
  if (a.S > kFewSplits) {
    const dim3 join((unsigned)a.H, (unsigned)a.b.max_new, (unsigned)a.b.n);
    attend_join_kernel<T, HD><<<join, 256, 0, s>>>(a);
  } else if (a.S > 1) {
    const dim3 join((unsigned)(((int64_t)a.b.max_new * a.H + 7) / 8), 1, (unsigned)a.b.n);
    attend_join_few_kernel<T, HD><<<join, 256, 0, s>>>(a);
  }
}

// Splits of the length.  Decoding: sixteen pages each (four a wave) where that gives two workgroups a compute
// unit, else as few as four pages, so that sequences of unequal length end together and a single one fills the
// chip; the join reads 2 KB for 256 KB of such a split.  Chunks: one round of the workgroups that compute
// units hold (three in bf16, two in fp32), of eight pages at least, as their partial results weigh more: 512
// rows, 32/8 heads of 128, behind 4000 tokens 115 us unsplit, 88 in two, 79 in three, 83 in six; behind none
// 19, 26, 25 and 30.  Chunks of up to 16 rows may go down to four pages too: 16 rows behind 9000 tokens 25 us
// in 16 splits, 20 in 32.
int attend_splits(const zoact_cache& c, const zoact_cache_batch& b, int n_heads, int w, int32_t dtype,
                  int64_t max_len) {
  const int G = n_heads / c.n_kv_heads;
  const int64_t tiles = ((int64_t)b.max_new * G + w - 1) / w;
  const int64_t groups = tiles * c.n_kv_heads * b.n;
  const int64_t pages = (max_len + kPage - 1) / kPage, cus = cu_count() > 0 ? cu_count() : 256;
  int64_t s, most = (pages + 3) / 4;
  if (w > 16) {
    s = (dtype == ZOACT_BF16 ? 3 : 2) * cus / groups;
    if (b.max_new > 16) most = pages / 8;
  } else {
    const int64_t want = 2 * cus;
    s = (pages + 15) / 16;
    if (groups * s < want) s = (want + groups - 1) / groups;
    // (between one and two rounds of three workgroups a compute unit: one)
    if (groups * s > want + want / 2 && groups * s < 3 * want && groups <= want) s = (want + want / 2) / groups;
  }
  if (s > most) s = most;
  if (s > kMaxSplits) s = kMaxSplits;
  // (the second pass has a grid row per new row)
  if (b.max_new > 65535) s = 1;
  return s < 1 ? 1 : (int)s;
}

size_t attend_ws(const zoact_cache& c, const zoact_cache_batch& b, int n_heads, int S) {
  return S > 1 ? (size_t)b.n * b.max_new * n_heads * S * (c.head_dim + 2) * sizeof(float) : 0;
}

int64_t within(const zoact_cache& c, int64_t max_len) {
  const int64_t most = (int64_t)c.max_pages * kPage;
  return max_len < most ? max_len : most;
}

bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace
}  // namespace zoact

using namespace zoact;

#define ZA(cond, msg) \
  if (!(cond)) return set_error(ZOACT_E_INVALID, msg)

extern "C" size_t zoact_attention_cache_workspace_bytes(const zoact_cache* c, const zoact_cache_batch* b,
                                                        int32_t n_heads, int64_t max_len) {
  if (check_cache(c) != ZOACT_OK || check_batch(b, c) != ZOACT_OK || n_heads < 1 || n_heads % c->n_kv_heads != 0 ||
      max_len < 1)
    return 0;
  max_len = within(*c, max_len);
  // (of the types the one with more splits: bf16, see attend_splits)
  const int w = attend_cols(*b, n_heads / c->n_kv_heads);
  return attend_ws(*c, *b, n_heads, attend_splits(*c, *b, n_heads, w, ZOACT_BF16, max_len));
}

extern "C" zoact_status zoact_attention_cache(const zoact_cache* c, int32_t layer, const void* q, int64_t ldq,
                                              int32_t dtype, int32_t n_heads, const zoact_cache_batch* b, float scale,
                                              int64_t max_len, const float* cos_t, const float* sin_t, int64_t n_pos,
                                              void* out, void* ws, size_t ws_bytes, zoact_stream stream) {
  zoact_status st = check_cache(c);
  if (st == ZOACT_OK) st = check_batch(b, c);
  if (st != ZOACT_OK) return st;
  ZA(layer >= 0 && layer < c->n_layers, "attention_cache: layer outside the cache");
  ZA(dtype == ZOACT_F32 || dtype == ZOACT_BF16, "attention_cache: dtype must be F32 or BF16");
  ZA((q && out) || b->rows == 0, "attention_cache: NULL pointer");
  ZA(n_heads >= 1 && n_heads % c->n_kv_heads == 0, "attention_cache: n_heads must be a multiple of n_kv_heads");
  const int vec = dtype == ZOACT_BF16 ? 8 : 4;
  ZA(ldq >= (int64_t)n_heads * c->head_dim && ldq % vec == 0 && al16(q) && al16(out),
     "attention_cache: rows must hold the heads; q, its rows and out must be 16-byte aligned");
  ZA(max_len >= 1, "attention_cache: max_len must be at least 1");
  ZA((cos_t == nullptr) == (sin_t == nullptr), "attention_cache: both rotary tables or neither");
  ZA(cos_t == nullptr || n_pos >= 1, "attention_cache: empty rotary table");
  ZA(al16(cos_t) && al16(sin_t), "attention_cache: rotary tables must be 16-byte aligned");
  if (b->rows == 0) return ZOACT_OK;
  max_len = within(*c, max_len);
  AttendArgs a{};
  a.c = *c;
  a.b = *b;
  a.layer = layer;
  a.H = n_heads;
  a.G = n_heads / c->n_kv_heads;
  ZA((int64_t)b->max_new * n_heads < INT32_MAX / kMaxSplits, "attention_cache: too many new rows");
  const int w = attend_cols(*b, a.G);
  a.S = attend_splits(*c, *b, n_heads, w, dtype, max_len);
  const size_t need = attend_ws(*c, *b, n_heads, a.S);
  if (ws == nullptr || ws_bytes < need) a.S = 1;
  if (a.S > 1) ZA(al16(ws), "attention_cache: ws must be 16-byte aligned");
  a.pps = (int)(((max_len + kPage - 1) / kPage + a.S - 1) / a.S);
  a.q = q;
  a.ldq = ldq;
  a.scale = scale * 1.44269504088896340736f;
  a.ct = cos_t;
  a.st = sin_t;
  a.n_pos = n_pos;
  a.out = out;
  if (a.S > 1) {
    a.part = static_cast<float*>(ws);
    a.ml = reinterpret_cast<float2*>(a.part + (size_t)b->n * b->max_new * n_heads * a.S * c->head_dim);
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
#define ZO_ATTEND(T, NT)                                       \
  if (c->head_dim == 128) run_attend<T, 128, NT>(a, w, s);        \
  else if (c->head_dim == 64) run_attend<T, 64, NT>(a, w, s);     \
  else run_attend<T, 32, NT>(a, w, s);
  if (dtype == ZOACT_BF16) {
    ZO_ATTEND(uint16_t, 1)
  } else {
    ZO_ATTEND(float, 2)
  }
#undef ZO_ATTEND
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return set_error(ZOACT_E_HIP, (std::string("attention_cache: ") + hipGetErrorString(err)).c_str());
  return ZOACT_OK;
}
