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
// A workgroup of four waves takes up to four query heads that read one key/value head, 32 rows of a
// head a wave; K and V tiles go through LDS for all four, chunks of 16 bytes swizzled so that
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

__device__ __forceinline__ float ld1(const float* p) { return *p; }
__device__ __forceinline__ float ld1(const uint16_t* p) { return bf2f(*p); }
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
  int lo = 0, hi = s.n, b, e;                      // the last i in [lo, hi) whose slots begin at or before slot
  for (;;) {                                       // (each round reads 64 bounds; 63 sequences take one)
    const int step = (hi - lo + 62) / 63, i = lo + lane * step;
    const int x = s.begin[i < s.n ? i : s.n];
    const int c = __popcll(__ballot(i < hi && (int64_t)((x > 0 ? x : 0) / R) + i <= slot)), k = c > 0 ? c - 1 : 0;
    lo += k * step;
    hi = lo + step < hi ? lo + step : hi;
    if (step > 1) continue;
    b = __builtin_amdgcn_readlane(x, k);
    e = __builtin_amdgcn_readlane(x, k + 1);
    break;
  }
  Place p{0, 0, 0};
  if (b < 0 || e <= b || e > s.rows) return p;
  const int64_t k = slot - ((int64_t)(b / R) + lo);
  const int tiles = (e - b + R - 1) / R;
  if (k < 0 || k >= tiles) return p;
  p.row0 = b;
  p.len = e - b;
  p.q0 = (tiles - 1 - (int)k) * R;
  return p;
}

template <typename T, int HD, int KT_>
struct Tile {
  static constexpr bool BF = std::is_same<T, uint16_t>::value;
  static constexpr int KT = KT_;                             // keys of a staged tile
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

template <typename T, int HD, int KT_, int OCC>
__global__ void __launch_bounds__(256, OCC)
    attention_packed_kernel(zoact_packed s, const T* __restrict__ q, int64_t ldq, const T* __restrict__ k, int64_t ldk,
                            const T* __restrict__ v, int64_t ldv, int heads, int kv_heads, int gh, float scale,
                            T* __restrict__ out) {
  using C = Tile<T, HD, KT_>;
  constexpr bool BF = C::BF;
  constexpr int KT = C::KT, SUBS = C::SUBS, ROW = C::ROW, CH = C::CH, PER = C::PER, NB = C::NB;
  constexpr int QF = BF ? HD / 16 : HD / 8;                  // 16-byte pieces of a lane's query
  // (arrays of their own, so that a read of one does not wait for the loads into another)
  __shared__ __align__(16) char k0[C::BYTES], k1[C::BYTES], v0[C::BYTES], v1[C::BYTES];
  __shared__ T pw[4][32][32];                                // a wave's probabilities for the vector product
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lq = lane & 31,
            lh = lane >> 5;
  const int hgs = heads / gh, R = (4 / gh) * 32;
  const int64_t slot = blockIdx.x / hgs;
  const int hg = blockIdx.x - (int)slot * hgs;
  const Place pl = place_of(s, slot, R);
  if (pl.len == 0) return;
  const int h = hg * gh + wave % gh, g = hg * gh / (heads / kv_heads);
  const int len = pl.len, w0 = pl.q0 + wave / gh * 32;       // the wave's first row
  const int last = pl.q0 + R < len ? pl.q0 + R : len;        // keys the workgroup needs
  const int n_tiles = (last + KT - 1) / KT;

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
    constexpr int NEXT = 256 / CH;                           // rows between a thread's chunks
    if (NEXT % 16 == 0 && left == KT) {                      // (the swizzles are the same there: one offset for all)
      const int off = row_t * step + (ch_t ^ swz(row_t)) * 16;
#pragma unroll
      for (int u = 0; u < PER; ++u)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_t*)(to + wave * 1024 + u * 4096), 16, off, u * NEXT * step, 0, 0);
      return;
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      int row = row_t + u * NEXT;
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
  load_k(k0, 0);

  // queries: lane's own row, pieces of 8 (4) values by halves
  u32x4 qf[QF];
  {
    const int r = w0 + lq < len ? w0 + lq : len - 1;
    const char* qp = reinterpret_cast<const char*>(q + (pl.row0 + r) * ldq + (int64_t)h * HD);
#pragma unroll
    for (int c = 0; c < QF; ++c) qf[c] = *reinterpret_cast<const u32x4*>(qp + (2 * c + lh) * 16);
  }
  load_v(v0, 0);
  if (n_tiles > 1) load_k(k1, 1);
  if (scale < 0.f) {
#pragma unroll
    for (int c = 0; c < QF; ++c) qf[c] ^= BF ? 0x80008000u : 0x80000000u;
  }
  const float c2 = fabsf(scale) * 1.4426950408889634f;

  floatx16 o[NB];
  float l = 0.f, m = -1.0e38f;           // (finite: a score of -inf has weight 0 also where nothing else came before)
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = 0.f;

  // keys of register i of a 32-key block: 8 (i / 4) + 4 half + i % 4
  auto scores = [&](const char* kt, int sub) {
    floatx16 st;
#pragma unroll
    for (int i = 0; i < 16; ++i) st[i] = 0.f;
    const int key = sub * 32 + lq;
    const char* kp = kt + key * ROW;
#pragma unroll
    for (int c = 0; c < QF; ++c) {
      const u32x4 kf = *reinterpret_cast<const u32x4*>(kp + ((2 * c + lh) ^ C::kswz(key)) * 16);
      if constexpr (BF) {
        st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[c]), st,
                                                     0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          st = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qf[c][e]), st, 0, 0, 0);
      }
    }
    return st;
  };
  // a row's maximum over both halves of the wave
  auto both = [&](float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  };
  // moves m where the maximum mx of the coming scores has passed it
  auto follow = [&](float mx) {
    mx *= c2;
    if (__ballot(mx > m + 8.f)) {
      const float mn = fmaxf(m, mx), a = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= a;
#pragma unroll
      for (int n = 0; n < NB; ++n) o[n] *= a;
    }
  };
  // probabilities of a block's scores; with CUT keys behind `lim` (numbered as the registers are, without the
  // half's 4) have none, whatever their scores
  auto weigh = [&](floatx16& st, auto cut, int lim) {
    float t0 = 0.f, t1 = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      st[i] = __builtin_amdgcn_exp2f(fmaf(st[i], c2, -m));
      if (decltype(cut)::value && 8 * (i / 4) + i % 4 > lim) st[i] = 0.f;
      (i & 1 ? t1 : t0) += st[i];
    }
    l += t0 + t1;
  };
  // V^T of block n, keys 16 c .. + 15 of sub (BF16): the order of the packed probabilities
  const int gl = lane & 15, g1 = (lane >> 4) & 1, vrow = gl >> 2;
  auto v_frag = [&](const char* vt, int sub, int c, int n) {
    typedef __attribute__((address_space(3))) bf16x4* lp;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const int row = sub * 32 + 16 * c + 4 * lh + vrow;       // (vswz(row) = vswz(row + 8))
    const char* p = vt + row * ROW + (((4 * n + 2 * g1) ^ C::vswz(row)) * 16) + (gl & 3) * 8;
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lp)(p)));
    const u32x2 z = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lp)(p + 8 * ROW)));
    return u32x4{a.x, a.y, z.x, z.y};
  };
  auto add = [&](const char* vt, int sub, const floatx16& st) {
    if constexpr (BF) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const u32x4 pb = u32x4{pack2(st[8 * c], st[8 * c + 1]), pack2(st[8 * c + 2], st[8 * c + 3]),
                               pack2(st[8 * c + 4], st[8 * c + 5]), pack2(st[8 * c + 6], st[8 * c + 7])};
#pragma unroll
        for (int n = 0; n < NB; ++n)
          o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_frag(vt, sub, c, n)),
                                                         __builtin_bit_cast(bf16x8, pb), o[n], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float* vp = reinterpret_cast<const float*>(vt + (sub * 32 + 8 * (i / 4) + 4 * lh + i % 4) * ROW) + lq;
#pragma unroll
        for (int n = 0; n < NB; ++n) o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(vp[n * 32], st[i], o[n], 0, 0, 0);
      }
    }
  };
  // whether a sub-tile of V holds something that is not finite (its rows spread over the wave)
  auto v_broken = [&](const char* vt, int sub) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};
#pragma unroll
    for (int c = 0; c < 32 * CH / 64; ++c) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(vt + sub * 32 * ROW + (c * 64 + lane) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[e] & (BF ? 0x7FFF7FFFu : 0x7FFF0000u)));
    }
    return __ballot(most.x >= 0x7F80 || most.y >= 0x7F80) != 0;
  };
  // the diagonal sub-tile key by key, for the rows from each on
  auto add_by_rows = [&](const char* vt, int sub, const floatx16& st) {
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
      const float p = ld1(&pw[wave][lq][t ^ lq]);
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = (32 * n + 8 * (i / 4) + 4 * lh + i % 4) * (int)sizeof(T);
          const float x = ld1(reinterpret_cast<const T*>(vt + row * ROW + ((at / 16) ^ C::vswz(row)) * 16 + at % 16));
          o[n][i] = t <= lq ? fmaf(p, x, o[n][i]) : o[n][i];
        }
    }
  };

  const int n_full = pl.q0 / KT;                             // tiles that every row of the workgroup sees
  floatx16 st[SUBS];
  float mx;
  auto maximum = [&] {
    mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[u][i]);
    mx = both(mx);
  };
  // One tile t: its scores are in st; the next one's are formed while these become probabilities, then
  // the product with V, the next maximum under it.  K of t + 2 and V of t + 1 are on their way meanwhile.
  auto full = [&](char* kt, char* kn, char* vt, char* vn, int t) {
    if (t + 2 < n_tiles) load_k(kt, t + 2);
    load_v(vn, t + 1);
    follow(mx);
    floatx16 nx[SUBS];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) nx[u] = scores(kn, u);
#pragma unroll
    for (int u = 0; u < SUBS; ++u) weigh(st[u], std::false_type{}, 0);
#pragma unroll
    for (int u = 0; u < SUBS; ++u) add(vt, u, st[u]);
#pragma unroll
    for (int u = 0; u < SUBS; ++u) st[u] = nx[u];
    maximum();
    arrived();
  };
  arrived();
#pragma unroll
  for (int u = 0; u < SUBS; ++u) st[u] = scores(k0, u);
  maximum();
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
    const int ahead = (w0 - t * KT) / 32;                    // this wave's diagonal sub-tile (all above 0 are past it)
    if (t * KT <= w0 && w0 < len) {
      const int lim = w0 + lq - t * KT - 4 * lh;
      float mb = -INFINITY;
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) mb = fmaxf(mb, u * 32 + 8 * (i / 4) + i % 4 <= lim ? st[u][i] : -INFINITY);
      follow(both(mb));
      const bool broken = ahead < SUBS && v_broken(vt, ahead);
#pragma unroll
      for (int u = 0; u < SUBS; ++u) {
        if (u > ahead) break;
        weigh(st[u], std::true_type{}, lim - u * 32);
        if (u == ahead && broken) add_by_rows(vt, u, st[u]);
        else add(vt, u, st[u]);
      }
    }
    if (t + 1 == n_tiles) break;
    const char* const kn = t & 1 ? k0 : k1;
#pragma unroll
    for (int u = 0; u < SUBS; ++u) st[u] = scores(kn, u);
    arrived();
  }

  // O^T has four columns of a row in a lane: rows are put together in the tiles' LDS, so that whole
  // lines are written
  const float inv = 1.f / (l + __shfl_xor(l, 32, 64));
  __syncthreads();
  const int at = wave / SUBS;
  char* const mine = (at == 0 ? k0 : at == 1 ? k1 : at == 2 ? v0 : v1) + wave % SUBS * 32 * ROW;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a0 = o[n][4 * i] * inv, a1 = o[n][4 * i + 1] * inv, a2 = o[n][4 * i + 2] * inv,
                  a3 = o[n][4 * i + 3] * inv;
      if constexpr (BF)
        *reinterpret_cast<uint2*>(mine + lq * ROW + ((4 * n + i) ^ C::kswz(lq)) * 16 + lh * 8) =
            make_uint2(pack2(a0, a1), pack2(a2, a3));
      else
        *reinterpret_cast<float4*>(mine + lq * ROW + ((8 * n + 2 * i + lh) ^ C::kswz(lq)) * 16) =
            make_float4(a0, a1, a2, a3);
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  char* const op = reinterpret_cast<char*>(out + ((pl.row0 + w0) * heads + h) * HD);
#pragma unroll
  for (int u = 0; u < 32 * CH / 64; ++u) {
    const int row = (u * 64 + lane) / CH, c = lane % CH;
    const u32x4 x = *reinterpret_cast<const u32x4*>(mine + row * ROW + (c ^ C::kswz(row)) * 16);
    if (w0 + row < len) *reinterpret_cast<u32x4*>(op + (int64_t)row * heads * ROW + c * 16) = x;
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
  const int R = (4 / gh) * 32;
  const int64_t slots = s.rows / R + s.n, grid = slots * (heads / gh);
  if (grid >= (int64_t(1) << 31)) return hipErrorNotSupported;
#define ZO_ATT(T, HD, KT, OCC)                                                                                          \
  attention_packed_kernel<T, HD, KT, OCC><<<(unsigned)grid, 256, 0, hs>>>(s, (const T*)q, ldq, (const T*)k, ldk,        \
                                                                          (const T*)v, ldv, heads, kv_heads, gh, scale, \
                                                                          (T*)out)
  if (dtype == ZOACT_BF16) {
    if (hd == 128) ZO_ATT(uint16_t, 128, 64, 2);
    else if (hd == 64) ZO_ATT(uint16_t, 64, 64, 2);
    else ZO_ATT(uint16_t, 32, 64, 2);
  } else {
    if (hd == 128) ZO_ATT(float, 128, 32, 2);
    else if (hd == 64) ZO_ATT(float, 64, 32, 2);
    else ZO_ATT(float, 32, 32, 2);
  }
#undef ZO_ATT
  return hipGetLastError();
}

}  // namespace zoact
