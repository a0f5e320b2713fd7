// Attention over the paged 8-bit cache (zoact_cache.h).
//
// One wave works on one page (64 tokens) of one key/value head at a time, for 16 query columns:
// the heads that share the key/value head times the new rows.  Scores are formed transposed,
// S^T = K Q^T, so that a lane holds, of one query column (lane % 16), the tokens 16 n + 4 g + i
// (g = lane / 16; n, i < 4) of the page: the softmax statistics stay in the lane (two shuffles
// per page join the four lanes of a column), and those 16 probabilities are, as they stand, the
// right operand of O^T = V^T P^T -- the page keeps V's tokens in that order, so nothing moves
// between lanes and K and V go from memory to the matrix unit in whole 16-byte loads.
// Codes become bf16 without rounding (magnitudes up to 127 need 7 bits); a K scale multiplies its
// block's scores, a V scale its block's probabilities.  q and the probabilities enter as NT bf16
// terms: two carry 16 bits (bf16 activations: beside the output's 8 nothing shows), three carry
// fp32's 24.
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
  float* part;                 // [n * max_new * H][S][HD], unnormalised
  float2* ml;                  // [n * max_new * H][S] maximum (log2 domain) and sum
};

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {   // exact: the lower halves are zero
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
}
// Eight int8 codes as bf16.
__device__ __forceinline__ bf16x8 codes8(uint32_t a, uint32_t b) {
  uint32_t o[4];
  const uint32_t w[2] = {a, b};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t x = w[e >> 1] >> (16 * (e & 1));
    o[e] = pack2((float)(int8_t)x, (float)(int8_t)(x >> 8));
  }
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<uint4*>(o));
}
// x as NT bf16 terms, each the nearest to what the ones before it leave.
template <int NT>
__device__ __forceinline__ void terms8(const float (&x)[8], bf16x8 (&t)[NT]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int k = 0; k < NT; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[k][e] = (__bf16)r[e];
      r[e] -= (float)t[k][e];
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

template <typename T, int HD, int NT>
__global__ void __launch_bounds__(256, 2) attend_kernel(AttendArgs a) {
  constexpr int KS = HD / 32;           // 32-deep products of a score
  constexpr int DT = HD / 16;           // 16-wide tiles of the output
  constexpr int LD = HD + 4;
  __shared__ float so[4][16][LD];
  __shared__ float sm[4][16], sl[4][16];
  const zoact_cache& c = a.c;
  const int hk = blockIdx.y, split = blockIdx.x % a.S, tile = blockIdx.x / a.S;
  const CacheEntry e = read_entry(c, a.b, blockIdx.z, threadIdx.x == 0 && blockIdx.x == 0 && hk == 0);
  const int ncol = e.count * a.G, c0 = tile * 16;
  if (c0 >= ncol) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4;
  const int col = c0 + (lane & 15);
  // (columns past the last repeat it; they are not stored)
  const int cq = col < ncol ? col : ncol - 1;
  const int j = cq / a.G, h = hk * a.G + cq % a.G;
  const int tcol = e.pos + j;                                        // the column's last token
  const int jmax = (c0 + 15 < ncol ? c0 + 15 : ncol - 1) / a.G;
  const int last = e.ok ? e.pos + jmax : -1;
  const int pages = (last + kPage) / kPage;
  const int pbeg = split * a.pps, pend = split == a.S - 1 ? pages : (pbeg + a.pps < pages ? pbeg + a.pps : pages);

  floatx4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  if (pbeg + wave < pend) {
    // q of the column, dims 64 (s / 2) + 16 g + 8 (s % 2) + 0..7 of step s (HD 32: 8 g + 0..7)
    bf16x8 qf[KS][NT];
    {
      const T* const row = static_cast<const T*>(a.q) + (int64_t)(e.row0 + j) * a.ldq + (int64_t)h * HD;
      const int64_t tp = tcol < a.n_pos ? tcol : a.n_pos - 1;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = HD == 32 ? 8 * g : 64 * (s >> 1) + 16 * g + 8 * (s & 1);
        float x[8];
        load8(row + d, x);
        if (a.ct) {
#pragma clang fp contract(off)
          constexpr int half = HD / 2;
          const bool up = d >= half;
          float y[8], cs[8], sn[8];
          load8(row + (up ? d - half : d + half), y);
          const int64_t base = tp * half + (up ? d - half : d);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            cs[k] = a.ct[base + k];
            sn[k] = a.st[base + k];
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = up ? x[k] * cs[k] + y[k] * sn[k] : x[k] * cs[k] - y[k] * sn[k];
        }
        terms8<NT>(x, qf[s]);
      }
    }
    const int* const trow = c.table + (int64_t)e.slot * c.max_pages;
    const int64_t lbase = (int64_t)a.layer * c.n_pages;
    for (int pg = pbeg + wave; pg < pend; pg += 4) {
      int pid = __builtin_amdgcn_readfirstlane(trow[pg]);
      const bool bad = pid < 0 || pid >= c.n_pages;
      if (bad) {
        if (lane == 0) raise_status(a.b.status, ZOACT_STATUS_BAD_ENTRY);
        continue;                                 // as if its tokens were masked
      }
      const int64_t head = (lbase + pid) * c.n_kv_heads + hk;
      const int8_t* const kp = c.k + head * (kPage * HD);
      const int8_t* const vp = c.v + head * (kPage * HD);
      const float4 ks = *reinterpret_cast<const float4*>(c.k_scale + head * 4);
      const float4 vs = *reinterpret_cast<const float4*>(c.v_scale + head * 4);
      const float ksc[4] = {ks.x * a.scale, ks.y * a.scale, ks.z * a.scale, ks.w * a.scale};
      const float vsc[4] = {vs.x, vs.y, vs.z, vs.w};
      float s[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        floatx4 acc{0.f, 0.f, 0.f, 0.f};
        const int8_t* const kr = kp + (n * 16 + (lane & 15)) * HD;
        if constexpr (HD == 32) {
          const uint2 u = *reinterpret_cast<const uint2*>(kr + 8 * g);
          const bf16x8 kf = codes8(u.x, u.y);
#pragma unroll
          for (int t = 0; t < NT; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[0][t], acc, 0, 0, 0);
        } else {
#pragma unroll
          for (int sl2 = 0; sl2 < KS / 2; ++sl2) {
            const uint4 u = *reinterpret_cast<const uint4*>(kr + 64 * sl2 + 16 * g);
            const bf16x8 k0 = codes8(u.x, u.y), k1 = codes8(u.z, u.w);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[2 * sl2][t], acc, 0, 0, 0);
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[2 * sl2 + 1][t], acc, 0, 0, 0);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = acc[i] * ksc[n];
      }
      const int t0 = pg * kPage;
      const bool edge = t0 + kPage > e.pos + c0 / a.G + 1;      // some column ends inside the page
      if (edge) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (t0 + 16 * n + 4 * g + i > tcol) s[n][i] = -INFINITY;
      }
      float mx = m;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[n][i]);
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float base = mx == -INFINITY ? 0.f : mx;
      const float alpha = __builtin_amdgcn_exp2f(m - base);
      m = mx;
      l *= alpha;
      bf16x8 pf[2][NT];
#pragma unroll
      for (int n2 = 0; n2 < 2; ++n2) {
        float p8[8];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = s[2 * n2 + n][i];
            const float p = __builtin_amdgcn_exp2f(x - base);
            l += p;
            // (a masked token's block may hold no scale yet)
            p8[4 * n + i] = edge && t0 + 16 * (2 * n2 + n) + 4 * g + i > tcol ? 0.f : p * vsc[2 * n2 + n];
          }
        terms8<NT>(p8, pf[n2]);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const uint4 u = *reinterpret_cast<const uint4*>(vp + (d * 16 + (lane & 15)) * kPage + 16 * g);
        const bf16x8 v0 = codes8(u.x, u.y), v1 = codes8(u.z, u.w);
        floatx4 acc = o[d] * alpha;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf[0][t], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf[1][t], acc, 0, 0, 0);
        }
        o[d] = acc;
      }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
  }
  // the four waves' results
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) so[wave][lane & 15][d * 16 + 4 * g + i] = o[d][i];
  if (g == 0) {
    sm[wave][lane] = m;
    sl[wave][lane] = l;
  }
  __syncthreads();
  constexpr int DV = HD / 16;
  const int oc = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * DV;
  if (c0 + oc >= ncol) return;
  float M = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w][oc]);
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f, r[DV];
#pragma unroll
  for (int k = 0; k < DV; ++k) r[k] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(sm[w][oc] - base);
    L += f * sl[w][oc];
#pragma unroll
    for (int k = 0; k < DV; ++k) r[k] += f * so[w][oc][d0 + k];
  }
  const int oj = (c0 + oc) / a.G, oh = hk * a.G + (c0 + oc) % a.G;
  if (a.S == 1) {
    const float div = L == 0.f ? 1.f : L;
    T* const op = static_cast<T*>(a.out) + ((int64_t)(e.row0 + oj) * a.H + oh) * HD + d0;
#pragma unroll
    for (int k = 0; k < DV; ++k) {
      if constexpr (sizeof(T) == 2)
        op[k] = f2bf(r[k] / div);
      else
        op[k] = r[k] / div;
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

// Joins the splits of one row and head: HD lanes along the columns, 256 / HD groups of splits.
template <typename T, int HD>
__global__ void __launch_bounds__(256) attend_join_kernel(AttendArgs a) {
  constexpr int NG = 256 / HD;
  __shared__ float sr[NG][HD], sw[NG];
  const int i = blockIdx.z, j = blockIdx.y, h = blockIdx.x;
  const CacheEntry e = read_entry(a.c, a.b, i, false);
  if (j >= e.count) return;
  const int d = threadIdx.x % HD, grp = threadIdx.x / HD;
  const int64_t R = (((int64_t)i * a.b.max_new + j) * a.H + h) * a.S;
  float M = -INFINITY;
  for (int s = 0; s < a.S; ++s) M = fmaxf(M, a.ml[R + s].x);
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f, r = 0.f;
  for (int s = grp; s < a.S; s += NG) {
    const float2 ml = a.ml[R + s];
    if (ml.y == 0.f) continue;
    const float f = __builtin_amdgcn_exp2f(ml.x - base);
    L += f * ml.y;
    r += f * a.part[(R + s) * HD + d];
  }
  sr[grp][d] = r;
  if (d == 0) sw[grp] = L;
  __syncthreads();
  if (grp) return;
#pragma unroll
  for (int k = 1; k < NG; ++k) {
    r += sr[k][d];
    L += sw[k];
  }
  const float y = L == 0.f ? 0.f : r / L;
  T* const op = static_cast<T*>(a.out) + ((int64_t)(e.row0 + j) * a.H + h) * HD + d;
  if constexpr (sizeof(T) == 2)
    *op = f2bf(y);
  else
    *op = y;
}

template <typename T, int HD, int NT>
void run_attend(const AttendArgs& a, hipStream_t s) {
  const int tiles = (int)(((int64_t)a.b.max_new * a.G + 15) / 16);
  const dim3 grid((unsigned)(tiles * a.S), (unsigned)a.c.n_kv_heads, (unsigned)a.b.n);
  attend_kernel<T, HD, NT><<<grid, 256, 0, s>>>(a);
  if (a.S > 1) {
    const dim3 join((unsigned)a.H, (unsigned)a.b.max_new, (unsigned)a.b.n);
    attend_join_kernel<T, HD><<<join, 256, 0, s>>>(a);
  }
}

constexpr int kMaxSplits = 128;

// Splits of the length: about four workgroups a compute unit, at least four pages each.
int attend_splits(const zoact_cache& c, const zoact_cache_batch& b, int n_heads, int64_t max_len) {
  const int ncu = cu_count();
  const int64_t tiles = ((int64_t)b.max_new * (n_heads / c.n_kv_heads) + 15) / 16;
  const int64_t groups = tiles * c.n_kv_heads * b.n;
  const int64_t pages = (max_len + kPage - 1) / kPage;
  int64_t s = (4 * (ncu > 0 ? ncu : 256) + groups - 1) / groups;
  if (s > (pages + 3) / 4) s = (pages + 3) / 4;
  if (s > kMaxSplits) s = kMaxSplits;
  // (the second pass has a grid row per new row)
  if (b.max_new > 65535) s = 1;
  return s < 1 ? 1 : (int)s;
}

size_t attend_ws(const zoact_cache& c, const zoact_cache_batch& b, int n_heads, int S) {
  return S > 1 ? (size_t)b.n * b.max_new * n_heads * S * (c.head_dim + 2) * sizeof(float) : 0;
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
  return attend_ws(*c, *b, n_heads, attend_splits(*c, *b, n_heads, max_len));
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
  ZA(q && out, "attention_cache: NULL pointer");
  ZA(n_heads >= 1 && n_heads % c->n_kv_heads == 0, "attention_cache: n_heads must be a multiple of n_kv_heads");
  const int vec = dtype == ZOACT_BF16 ? 8 : 4;
  ZA(ldq >= (int64_t)n_heads * c->head_dim && ldq % vec == 0 && al16(q) && al16(out),
     "attention_cache: rows must hold the heads; q, its rows and out must be 16-byte aligned");
  ZA(max_len >= 1, "attention_cache: max_len must be at least 1");
  ZA((cos_t == nullptr) == (sin_t == nullptr), "attention_cache: both rotary tables or neither");
  ZA(cos_t == nullptr || n_pos >= 1, "attention_cache: empty rotary table");
  AttendArgs a{};
  a.c = *c;
  a.b = *b;
  a.layer = layer;
  a.H = n_heads;
  a.G = n_heads / c->n_kv_heads;
  ZA((int64_t)b->max_new * a.G < INT32_MAX / kMaxSplits, "attention_cache: too many new rows");
  a.S = attend_splits(*c, *b, n_heads, max_len);
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
  if (c->head_dim == 128) run_attend<T, 128, NT>(a, s);        \
  else if (c->head_dim == 64) run_attend<T, 64, NT>(a, s);     \
  else run_attend<T, 32, NT>(a, s);
  if (dtype == ZOACT_BF16) {
    ZO_ATTEND(uint16_t, 2)
  } else {
    ZO_ATTEND(float, 3)
  }
#undef ZO_ATTEND
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return set_error(ZOACT_E_HIP, (std::string("attention_cache: ") + hipGetErrorString(err)).c_str());
  return ZOACT_OK;
}
