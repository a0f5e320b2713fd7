// Causal attention over packed sequences on the matrix cores (zoact_packed.h): head_dim 32, 64 or
// 128, rows of 16-byte aligned heads.
//
// One pass over the keys with the running maximum m and sum l of each row's softmax:
//   S^T = K Q^T (32 keys x 32 queries an MFMA),  P^T = 2^(S^T c - m),  O^T += V^T P^T,
// c = scale log2(e) (a negative one's sign goes into q).  A lane holds one query of each tile, so
// maxima and sums need one exchange between the wave's halves, O^T is rescaled by a factor of the
// lane's own, and P^T, packed, is the B operand of the second product as it stands: the keys of one
// MFMA may come in any order if V^T has the same.  m follows the maximum only where that passes it
// by 2^8, so that most tiles rescale nothing; probabilities are then up to 2^8, with the same
// relative rounding.
//
// A workgroup of four waves takes up to four query heads that read one key/value head, 32 QB rows
// of a head a wave; K and V tiles go through LDS for all four, chunks of 16 bytes swizzled so that
// neither the K rows nor the V columns (read transposed by ds_read_tr16) meet in a bank.
//
// Keys that some of a wave's rows may not see are in its last tiles only, from its first row's tile
// of 32 on; there the scores are masked, and where a masked V is not finite (0 * inf is NaN) the
// product runs on the vector unit, for the rows that see each key.
#include <math.h>

#include <type_traits>

#include "packed.hpp"

namespace zoact {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// Place of a workgroup: sequence, first row in it, rows from its beginning on.
struct Place {
  int64_t row0;    // the sequence's first row
  int len, q0;     // its length, the workgroup's first row in it; len 0: nothing to do
};

// Sequences own numbered slots, sequence i those from begin[i] / R + i on: at least as many as it has
// tiles of R rows, so that no list of them is needed.  Late (long) tiles come first.
__device__ __forceinline__ Place place_of(const zoact_packed& s, int64_t slot, int R) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = s.n;                            // the last i in [lo, hi) whose slots begin at or before slot
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    bool at = false;
    if (i < hi) {
      const int b = s.begin[i];
      at = (int64_t)((b > 0 ? b : 0) / R) + i <= slot;
    }
    const int c = __popcll(__ballot(at));
    lo += (c > 0 ? c - 1 : 0) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  Place p{0, 0, 0};
  const int b = s.begin[lo], e = s.begin[lo + 1];
  if (b < 0 || e <= b || e > s.rows) return p;
  const int64_t k = slot - ((int64_t)(b / R) + lo);
  const int tiles = (e - b + R - 1) / R;
  if (k < 0 || k >= tiles) return p;
  p.row0 = b;
  p.len = e - b;
  p.q0 = (tiles - 1 - (int)k) * R;
  return p;
}

template <typename T, int HD>
struct Tile {
  static constexpr bool BF = std::is_same<T, uint16_t>::value;
  static constexpr int KT = BF ? 64 : 32;                    // keys of a staged tile
  static constexpr int SUBS = KT / 32;
  static constexpr int ROW = HD * (int)sizeof(T), CH = ROW / 16;
  static constexpr int BYTES = KT * ROW;
  static constexpr int PER = KT * CH / 256;                  // 16-byte chunks a thread of K, and of V
  static constexpr int NB = HD / 32;                         // 32-column blocks of O
  // Chunk c of a row lies at c ^ swz(row): the 16 lanes of a read of K's chunk (rows in turn), and the
  // lanes of a transposed read of V (4 rows of 64 bytes), then cover all banks (256 bytes) once.
  __device__ static int kswz(int row) { return CH >= 16 ? row & 15 : CH == 8 ? (row >> 1) & 7 : (row >> 2) & 3; }
  __device__ static int vswz(int row) { return !BF ? 0 : CH == 16 ? (row & 3) << 2 : CH == 8 ? ((row >> 1) & 1) << 2 : 0; }
};

template <typename T, int HD, int QB>
__global__ void __launch_bounds__(256, QB == 1 ? 2 : 1)
    attention_packed_kernel(zoact_packed s, const T* __restrict__ q, int64_t ldq, const T* __restrict__ k, int64_t ldk,
                            const T* __restrict__ v, int64_t ldv, int heads, int kv_heads, int gh, float scale,
                            T* __restrict__ out) {
  using C = Tile<T, HD>;
  constexpr bool BF = C::BF;
  constexpr int KT = C::KT, SUBS = C::SUBS, ROW = C::ROW, CH = C::CH, PER = C::PER, NB = C::NB;
  constexpr int QF = BF ? HD / 16 : HD / 8;                  // 16-byte pieces of a lane's query
  // (arrays of their own, so that a read of one does not wait for the loads into another)
  __shared__ __align__(16) char k0[C::BYTES], k1[C::BYTES], v0[C::BYTES], v1[C::BYTES];
  __shared__ T pw[4][32][32];                                // a wave's probabilities for the vector product
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lq = lane & 31,
            lh = lane >> 5;
  const int hgs = heads / gh, R = (4 / gh) * 32 * QB;
  const int64_t slot = blockIdx.x / hgs;
  const int hg = blockIdx.x - (int)slot * hgs;
  const Place pl = place_of(s, slot, R);
  if (pl.len == 0) return;
  const int h = hg * gh + wave % gh, g = hg * gh / (heads / kv_heads);
  const int len = pl.len, w0 = pl.q0 + wave / gh * 32 * QB;  // the wave's first row
  const int last = pl.q0 + R < len ? pl.q0 + R : len;        // keys the workgroup needs
  const int n_tiles = (last + KT - 1) / KT;

  // queries: lane's own row of each block, pieces of 8 (4) values by halves
  u32x4 qf[QB][QF];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int r = w0 + b * 32 + lq < len ? w0 + b * 32 + lq : len - 1;
    const char* qp = reinterpret_cast<const char*>(q + (pl.row0 + r) * ldq + (int64_t)h * HD);
#pragma unroll
    for (int c = 0; c < QF; ++c) qf[b][c] = *reinterpret_cast<const u32x4*>(qp + (2 * c + lh) * 16);
    if (scale < 0.f) {
#pragma unroll
      for (int c = 0; c < QF; ++c) qf[b][c] ^= BF ? 0x80008000u : 0x80000000u;
    }
  }
  const float c2 = fabsf(scale) * 1.4426950408889634f;

  // Tiles go from global memory straight to LDS, a wave's 64 chunks side by side; the swizzle is in the
  // choice of each lane's chunk.  Rows past the sequence read as its last.
  const int row_t = threadIdx.x / CH, ch_t = threadIdx.x % CH;
  const int kstep = (int)(ldk * (int64_t)sizeof(T)), vstep = (int)(ldv * (int64_t)sizeof(T));
  const char* const kb = reinterpret_cast<const char*>(k + pl.row0 * ldk + (int64_t)g * HD);
  const char* const vb = reinterpret_cast<const char*>(v + pl.row0 * ldv + (int64_t)g * HD);
  auto load = [&](const char* from, int step, int (*swz)(int), char* to, int t) {
    typedef __attribute__((address_space(3))) void lds_t;
    const int left = len - t * KT < KT ? len - t * KT : KT;
    const uint64_t a = reinterpret_cast<uint64_t>(from + (int64_t)t * KT * step);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(((uint64_t)hi << 32) | lo), (short)0, (left - 1) * step + ROW, 0x00020000);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      int row = row_t + u * (256 / CH);
      const int chunk = ch_t ^ swz(row);
      row = row < left ? row : left - 1;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_t*)(to + wave * 1024 + u * 4096), 16, row * step + chunk * 16, 0,
                                               0, 0);
    }
  };
  auto load_k = [&](char* to, int t) { load(kb, kstep, C::kswz, to, t); };
  auto load_v = [&](char* to, int t) { load(vb, vstep, C::vswz, to, t); };
  auto arrived = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0): this wave's part; then everybody's
    __syncthreads();
  };

  floatx16 o[QB][NB];
  float m[QB], l[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    m[b] = -1.0e38f;                     // (finite: a score of -inf has weight 0 also where nothing else came before)
    l[b] = 0.f;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][n][i] = 0.f;
  }

  // keys of register i of a 32-key block: 8 (i / 4) + 4 half + i % 4
  auto scores = [&](const char* kt, int sub, floatx16 (&st)[QB]) {
#pragma unroll
    for (int b = 0; b < QB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) st[b][i] = 0.f;
    const int key = sub * 32 + lq;
    const char* kp = kt + key * ROW;
#pragma unroll
    for (int c = 0; c < QF; ++c) {
      const u32x4 kf = *reinterpret_cast<const u32x4*>(kp + ((2 * c + lh) ^ C::kswz(key)) * 16);
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        if constexpr (BF) {
          st[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf),
                                                          __builtin_bit_cast(bf16x8, qf[b][c]), st[b], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            st[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qf[b][c][e]), st[b], 0,
                                                         0, 0);
        }
      }
    }
  };
  // a row's maximum over both halves of the wave
  auto both = [&](float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  };
  // moves m where the maximum mx of the coming scores has passed it
  auto follow = [&](int b, float mx) {
    mx *= c2;
    if (__ballot(mx > m[b] + 8.f)) {
      const float mn = fmaxf(m[b], mx), a = __builtin_amdgcn_exp2f(m[b] - mn);
      m[b] = mn;
      l[b] *= a;
#pragma unroll
      for (int n = 0; n < NB; ++n) o[b][n] *= a;
    }
  };
  // (diag: keys behind the lane's row have no weight, whatever their score)
  auto weigh = [&](int b, floatx16& st, bool diag) {
    float t0 = 0.f, t1 = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      st[i] = __builtin_amdgcn_exp2f(fmaf(st[i], c2, -m[b]));
      if (diag && 8 * (i / 4) + 4 * lh + i % 4 > lq) st[i] = 0.f;
      (i & 1 ? t1 : t0) += st[i];
    }
    l[b] += t0 + t1;
  };
  // V^T of block n, keys 16 c .. + 15 of sub (BF16): the order of the packed probabilities
  const int gl = lane & 15, g1 = (lane >> 4) & 1, vrow = gl >> 2;
  auto v_frag = [&](const char* vt, int sub, int c, int n) {
    typedef __attribute__((address_space(3))) bf16x4* lp;
    const int row = sub * 32 + 16 * c + 4 * lh + vrow;       // (vswz(row) = vswz(row + 8))
    const char* p = vt + row * ROW + (((4 * n + 2 * g1) ^ C::vswz(row)) * 16) + (gl & 3) * 8;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lp)(p)));
    const u32x2 z = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lp)(p + 8 * ROW)));
    return u32x4{a.x, a.y, z.x, z.y};
  };
  auto packed_p = [&](const floatx16& st, int c) {
    return u32x4{pack2(st[8 * c], st[8 * c + 1]), pack2(st[8 * c + 2], st[8 * c + 3]),
                 pack2(st[8 * c + 4], st[8 * c + 5]), pack2(st[8 * c + 6], st[8 * c + 7])};
  };
  // blocks [b0, QB) with a sub-tile of 32 keys
  auto add = [&](const char* vt, int sub, const floatx16 (&st)[QB], int b0) {
    if constexpr (BF) {
      u32x4 pb[QB][2];
#pragma unroll
      for (int b = 0; b < QB; ++b)
#pragma unroll
        for (int c = 0; c < 2; ++c) pb[b][c] = packed_p(st[b], c);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const u32x4 va = v_frag(vt, sub, c, n);
#pragma unroll
          for (int b = 0; b < QB; ++b)
            if (b >= b0)
              o[b][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va),
                                                                __builtin_bit_cast(bf16x8, pb[b][c]), o[b][n], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float* vp = reinterpret_cast<const float*>(vt + (sub * 32 + 8 * (i / 4) + 4 * lh + i % 4) * ROW) + lq;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int b = 0; b < QB; ++b)
            if (b >= b0) o[b][n] = __builtin_amdgcn_mfma_f32_32x32x2f32(vp[n * 32], st[b][i], o[b][n], 0, 0, 0);
      }
    }
  };
  // whether a sub-tile of V holds something that is not finite (its rows spread over the wave)
  auto v_broken = [&](const char* vt, int sub) {
    bool bad = false;
    for (int c = lane; c < 32 * CH; c += 64) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(vt + sub * 32 * ROW + c * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bad |= (x[e] & 0x7F800000u) == 0x7F800000u;
        if (BF) bad |= (x[e] & 0x7F80u) == 0x7F80u;
      }
    }
    return __ballot(bad) != 0;
  };
  // block b with its diagonal sub-tile, key by key for the rows from it on
  auto add_by_rows = [&](const char* vt, int sub, int b, const floatx16& st) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = 8 * (i / 4) + 4 * lh + i % 4;
      if constexpr (BF) pw[wave][lq][key ^ lq] = f2bf(st[i]);
      else pw[wave][lq][key ^ lq] = st[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
    for (int t = 0; t < 32; ++t) {
      const int row = sub * 32 + t;
      float p;
      if constexpr (BF) p = bf2f(pw[wave][lq][t ^ lq]);
      else p = pw[wave][lq][t ^ lq];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int col = 32 * n + 8 * (i / 4) + 4 * lh + i % 4, at = col * (int)sizeof(T);
          const T* x = reinterpret_cast<const T*>(vt + row * ROW + ((at / 16) ^ C::vswz(row)) * 16 + at % 16);
          float xv;
          if constexpr (BF) xv = bf2f(*x);
          else xv = *x;
          o[b][n][i] = t <= lq ? fmaf(p, xv, o[b][n][i]) : o[b][n][i];
        }
    }
  };

  const int d0 = w0 / 32;                                    // sub-tiles d0 + b are the blocks' diagonals
  const int n_full = pl.q0 / KT;                             // tiles that every row of the workgroup sees
  floatx16 st[SUBS][QB];
  float mx[QB];
  auto maxima = [&] {
#pragma unroll
    for (int b = 0; b < QB; ++b) {
      mx[b] = -INFINITY;
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx[b] = fmaxf(mx[b], st[u][b][i]);
      mx[b] = both(mx[b]);
    }
  };
  // One tile t: its scores are in st; the next one's are formed while these become probabilities, then
  // the product with V, the next maxima under it.  K of t + 2 and V of t + 1 are on their way meanwhile.
  auto full = [&](char* kt, char* kn, char* vt, char* vn, int t) {
    if (t + 2 < n_tiles) load_k(kt, t + 2);
    load_v(vn, t + 1);
#pragma unroll
    for (int b = 0; b < QB; ++b) follow(b, mx[b]);
    floatx16 nx[SUBS][QB];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) scores(kn, u, nx[u]);
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int b = 0; b < QB; ++b) weigh(b, st[u][b], false);
#pragma unroll
    for (int u = 0; u < SUBS; ++u) add(vt, u, st[u], 0);
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int b = 0; b < QB; ++b) st[u][b] = nx[u][b];
    maxima();
    arrived();
  };
  load_k(k0, 0);
  load_v(v0, 0);
  if (n_tiles > 1) load_k(k1, 1);
  arrived();
#pragma unroll
  for (int u = 0; u < SUBS; ++u) scores(k0, u, st[u]);
  if (n_full > 0) maxima();
  __syncthreads();                                           // (K of tile 0 is overwritten next)
#pragma unroll 1
  for (int t = 0; t < n_full; t += 2) {
    full(k0, k1, v0, v1, t);
    if (t + 1 == n_full) break;
    full(k1, k0, v1, v0, t + 1);
  }
  // tiles that some rows of the workgroup do not see, or not whole
#pragma unroll 1
  for (int t = n_full; t < n_tiles; ++t) {
    char* const vt = t & 1 ? v1 : v0;
    if (t + 1 < n_tiles) load_v(t & 1 ? v0 : v1, t + 1);
    if (t + 2 < n_tiles) load_k(t & 1 ? k1 : k0, t + 2);
#pragma unroll 1
    for (int u = 0; u < SUBS; ++u) {
      const int over = t * SUBS + u - d0;                    // block `over` is on the diagonal, those before are past it
      if (over >= QB || w0 + over * 32 >= len) break;
      floatx16 x[QB];
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        x[b] = st[0][b];
        if (SUBS > 1 && u > 0) x[b] = st[SUBS - 1][b];
      }
      const bool broken = over >= 0 && v_broken(vt, u);
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        if (b < over) continue;
        float mb = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool seen = b > over || 8 * (i / 4) + 4 * lh + i % 4 <= lq;
          mb = fmaxf(mb, seen ? x[b][i] : -INFINITY);
        }
        follow(b, both(mb));
        weigh(b, x[b], b == over);
      }
      add(vt, u, x, over + (broken ? 1 : 0));
      if (broken) {
#pragma unroll
        for (int b = 0; b < QB; ++b)
          if (b == over) add_by_rows(vt, u, b, x[b]);
      }
    }
    if (t + 1 == n_tiles) break;
    const char* const kn = t & 1 ? k0 : k1;
#pragma unroll
    for (int u = 0; u < SUBS; ++u) scores(kn, u, st[u]);
    arrived();
  }

#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int r = w0 + b * 32 + lq;
    const float total = l[b] + __shfl_xor(l[b], 32, 64), inv = 1.f / total;
    if (r >= len) continue;
    T* op = out + (pl.row0 + r) * (int64_t)heads * HD + (int64_t)h * HD + 4 * lh;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a0 = o[b][n][4 * i] * inv, a1 = o[b][n][4 * i + 1] * inv, a2 = o[b][n][4 * i + 2] * inv,
                    a3 = o[b][n][4 * i + 3] * inv;
        if constexpr (BF) *reinterpret_cast<uint2*>(op + n * 32 + 8 * i) = make_uint2(pack2(a0, a1), pack2(a2, a3));
        else *reinterpret_cast<float4*>(op + n * 32 + 8 * i) = make_float4(a0, a1, a2, a3);
      }
  }
}

}  // namespace

hipError_t launch_attention_packed(const zoact_packed& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                   const void* v, int64_t ldv, int32_t heads, int32_t kv_heads, int32_t hd, float scale,
                                   int32_t dtype, void* out, hipStream_t hs) {
  const int64_t vec = dtype == ZOACT_BF16 ? 8 : 4;
  if ((hd != 32 && hd != 64 && hd != 128) || ldq % vec || ldk % vec || ldv % vec || !aligned_to(q, 16) ||
      !aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(out, 16))
    return hipErrorNotSupported;
  // (a tile's rows are addressed with 32 bits)
  if (ldk >= (int64_t(1) << 22) || ldv >= (int64_t(1) << 22)) return hipErrorNotSupported;
  const int G = heads / kv_heads, gh = G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1;
  const int qb = 1, R = (4 / gh) * 32 * qb;
  const int64_t slots = s.rows / R + s.n, grid = slots * (heads / gh);
  if (grid >= (int64_t(1) << 31)) return hipErrorNotSupported;
#define ZO_ATT(T, HD)                                                                                                \
  attention_packed_kernel<T, HD, 1><<<(unsigned)grid, 256, 0, hs>>>(s, (const T*)q, ldq, (const T*)k, ldk,            \
                                                                    (const T*)v, ldv, heads, kv_heads, gh, scale,     \
                                                                    (T*)out)
  if (dtype == ZOACT_BF16) {
    if (hd == 128) ZO_ATT(uint16_t, 128);
    else if (hd == 64) ZO_ATT(uint16_t, 64);
    else ZO_ATT(uint16_t, 32);
  } else {
    if (hd == 128) ZO_ATT(float, 128);
    else if (hd == 64) ZO_ATT(float, 64);
    else ZO_ATT(float, 32);
  }
#undef ZO_ATT
  return hipGetLastError();
}

}  // namespace zoact
