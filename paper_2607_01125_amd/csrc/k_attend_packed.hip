// Causal attention over packed sequences on the matrix cores (zoact_packed.h): rows of 16-byte
// aligned heads of 32, 64 or 128 values, or fewer with zeros in place of the rest.
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
// Keys that some of a wave's rows may not see are in its last tiles only, from its first row's tile of 32 on; there
// the scores are masked.  Three things make a wave take its rows one by one in the end: a masked V that is not finite
// (0 * inf is NaN) and values whose weighted sum, or scores whose product with c, passes the range though their mean, or
// score, does not, both looked for where an output is not finite; and a maximum past 2^27, where S^T c - m, fused, is off
// by the rounding of the product that became m, which 2^x no longer bears.
//
// Long sequences are bound by the matrix cores (60% busy at 1.7 GHz) and as many cycles of exponentials, sums and
// conversions beside them: 12001 tokens and 30 short sequences, 32/8 heads of 128, in 1.09 ms, 1080 TFLOP/s.  Short
// ones are bound by a workgroup's ends, its place, first tiles and rows out: 32 sequences up to 510 tokens in 46 us,
// 2.8 TB/s.  64 rows a wave were slower (2.3 against 1.27 ms, at that time), tiles of 32 keys with three workgroups a
// compute unit spilled (95 against 53 us); scores of the next tile beside the probabilities of this one, and tiles
// straight to LDS, took the first kernel's 2.23 ms to 1.18.
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
  const int tiles = (int)(((int64_t)e - b + R - 1) / R);
  if (k < 0 || k >= tiles) return p;
  p.row0 = b;
  p.len = e - b;
  p.q0 = (tiles - 1 - (int)k) * R;
  return p;
}

// The same with the tiles of 64 sequences at a time (a lane each) in the order of the keys before them, most
// first, whichever sequence they are of: the last to start are then short.  Sequences 64 g on have the slots
// from begin[64 g] / R + 64 g on.  For fp32, which the products bind (8 sequences of 700 tokens 105 -> 85 us);
// in bf16 what tiles of one sequence find in the cache weighs more (OPT's heads 190 -> 200 us).
__device__ __forceinline__ Place longest_first(const zoact_packed& s, int64_t slot, int R) {
  const int lane = threadIdx.x & 63, sh = 31 - __builtin_clz(R);       // (R is a power of two)
  int lo = 0, hi = (s.n + 63) >> 6;                // the last group in [lo, hi) whose slots begin at or before slot
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6, i = lo + lane * step;
    bool at = false;
    if (i < hi) {
      const int x = s.begin[i << 6];
      at = (int64_t)((x > 0 ? x : 0) >> sh) + (i << 6) <= slot;
    }
    const int c = __popcll(__ballot(at));
    lo += (c > 0 ? c - 1 : 0) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  const int i = (lo << 6) + lane;
  const int b = s.begin[i < s.n ? i : s.n], e = s.begin[i < s.n ? i + 1 : s.n];
  const int tiles = b >= 0 && e > b && e <= s.rows ? (int)(((int64_t)e - b + R - 1) >> sh) : 0;
  const int b0 = __builtin_amdgcn_readfirstlane(b);
  const int64_t k64 = slot - ((int64_t)((b0 > 0 ? b0 : 0) >> sh) + (lo << 6));
  Place p{0, 0, 0};
  if (k64 < 0 || k64 >= wave_sum(tiles)) return p;
  // the highest tile number t of which, and of higher ones, there are more than k
  const int k = (int)k64;
  int t = 0, top = 1;
  while (__ballot(tiles > top)) top <<= 1;         // (all tile numbers are below top)
  while (top - t > 1) {
    const int mid = (t + top) >> 1;
    if (wave_sum(tiles > mid ? tiles - mid : 0) > k) t = mid;
    else top = mid;
  }
  const int above = wave_sum(tiles > t + 1 ? tiles - t - 1 : 0);
  const int rank = __popcll(__ballot(tiles > t) & ((1ull << lane) - 1));
  const int who = __ffsll((unsigned long long)__ballot(tiles > t && rank == k - above)) - 1;
  const int row0 = __builtin_amdgcn_readlane(b, who), end = __builtin_amdgcn_readlane(e, who);
  // (nobody where bounds that do not ascend count more tiles than 32 bits hold)
  if (row0 < 0 || end <= row0 || end > s.rows || ((int64_t)t << sh) >= end - row0) return p;
  p.row0 = row0;
  p.len = end - row0;
  p.q0 = t << sh;
  return p;
}

// A workgroup's number in the order of its work.  Where all workgroups of a launch find room at once, those that
// share a compute unit are 256 apart: every second 256 are taken backwards (by eights, each of which goes to its own
// XCD), so that long ones share with short ones (2 sequences of 1000 tokens 35.7 -> 29.7 us, one of 4000 in fp32
// 349 -> 314).
__device__ __forceinline__ unsigned turn_about() {
  const unsigned turn = blockIdx.x >> 8;
  return (turn & 1) && (turn + 1) << 8 <= gridDim.x
             ? (turn << 8) + ((31 - ((blockIdx.x & 255) >> 3)) << 3) + (blockIdx.x & 7) : blockIdx.x;
}

__device__ __forceinline__ int no_swizzle(int) { return 0; }

// Bits of what a value is that is not finite.
enum { IS_NAN = 1, IS_POS = 2, IS_NEG = 4 };
__device__ __forceinline__ int kind_of(float x) { return x - x == 0.f ? 0 : x != x ? IS_NAN : x > 0.f ? IS_POS : IS_NEG; }

// Whether the formula may have others in place of a wave's outputs that are not finite (outs(c): what those of column
// c are): not where V holds their cause in a row that all of the wave's rows see, 0 .. seen.  It may where that cause
// is in a row that some do not see (0 * inf is NaN), or where the weighted sum passed the range and the mean does not.
template <typename T, typename Outs>
__device__ __forceinline__ bool in_doubt(Outs outs, const T* v, int64_t ldv, int seen, int hd) {
  bool doubt = false;
  for (int c = threadIdx.x & 63; c < hd; c += 64) {
    const int got = outs(c);
    if (got == 0) continue;
    int have = 0;
    for (int r = 0; r <= seen && !(have & IS_NAN); r += 8)
#pragma unroll
      for (int u = 0; u < 8; ++u) have |= kind_of(ld1(v + (r + u < seen ? r + u : seen) * ldv + c));
    doubt |= !(have & IS_NAN) && have != (IS_POS | IS_NEG) && have != got;
  }
  return __ballot(doubt) != 0;
}

// Rows of a K or V tile from global memory straight to LDS, 256 threads with PER chunks of 16 bytes each, a
// wave's 64 side by side; the swizzle is in the choice of each lane's chunk.  Rows past the sequence read as its
// last.  With PAD rows hold `chunks` chunks only, and the lanes of others load nothing.
template <int CH, int PER, bool PAD>
struct TileLoad {
  int wave, len, chunks;
  __device__ __forceinline__ void run(const char* from, int step, int (*swz)(int), char* to, int first, int rows) const {
    typedef __attribute__((address_space(3))) void lds_t;
    const int row_t = threadIdx.x / CH, ch_t = threadIdx.x % CH;
    const int left = len - first < rows ? len - first : rows;
    const uint64_t a = reinterpret_cast<uint64_t>(from + (int64_t)first * step);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(((uint64_t)hi << 32) | lo), (short)0, (left - 1) * step + (PAD ? chunks : CH) * 16, 0x00020000);
    constexpr int NEXT = 256 / CH;                           // rows between a thread's chunks
    if (NEXT % 16 == 0 && left == rows) {                    // (the swizzles are the same there: one offset for all)
      const int off = row_t * step + (ch_t ^ swz(row_t)) * 16;
      if (PAD && (ch_t ^ swz(row_t)) >= chunks) return;
#pragma unroll
      for (int u = 0; u < PER; ++u)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_t*)(to + wave * 1024 + u * 4096), 16, off, u * NEXT * step, 0, 0);
      return;
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      int row = row_t + u * NEXT;
      const int chunk = ch_t ^ swz(row);
      if (PAD && chunk >= chunks) continue;
      row = row < left ? row : left - 1;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_t*)(to + wave * 1024 + u * 4096), 16, row * step + chunk * 16, 0,
                                               0, 0);
    }
  }
};

// The chunks of a tile that PAD loads leave out, as zeros.
template <int CH, int ROWS>
__device__ __forceinline__ void clear_rest(char* tile, int (*swz)(int), int chunks) {
  for (int i = threadIdx.x; i < ROWS * CH; i += 256) {
    const int row = i / CH, c = i % CH;
    if (c >= chunks) *reinterpret_cast<u32x4*>(tile + (row * CH + (c ^ swz(row))) * 16) = u32x4{0, 0, 0, 0};
  }
}

template <int HD>
struct Tile {
  static constexpr int KT = 64;                              // keys of a staged tile
  static constexpr int SUBS = KT / 32;
  static constexpr int ROW = HD * 2, CH = ROW / 16;
  static constexpr int BYTES = KT * ROW;
  static constexpr int PER = KT * CH / 256;                  // 16-byte chunks a thread of K, and of V
  static constexpr int NB = HD / 32;                         // 32-column blocks of O
  // Chunk c of a row lies at c ^ swz(row): the 16 lanes of a read of K's chunk (rows in turn), and the
  // lanes of a transposed read of V (4 rows of 64 bytes), then cover all banks (256 bytes) once.
  __device__ static int kswz(int row) { return CH >= 16 ? row & 15 : CH == 8 ? (row >> 1) & 7 : (row >> 2) & 3; }
  __device__ static int vswz(int row) { return CH == 16 ? (row & 3) << 2 : CH == 8 ? ((row >> 1) & 1) << 2 : 0; }
};

// PAD: heads are hd < HD values wide, a multiple of 8; the rest of HD is zero in q, K and V.
template <int HD, bool PAD>
__global__ void __launch_bounds__(256, HD == 128 ? 2 : 3)
    attention_packed_bf16_kernel(zoact_packed s, const uint16_t* __restrict__ q, int64_t ldq,
                                 const uint16_t* __restrict__ k, int64_t ldk, const uint16_t* __restrict__ v, int64_t ldv,
                                 int heads, int kv_heads, int hd, int gh, float scale,
                                 uint16_t* __restrict__ out) {
  using C = Tile<HD>;
  constexpr int KT = C::KT, SUBS = C::SUBS, ROW = C::ROW, CH = C::CH, PER = C::PER, NB = C::NB;
  constexpr int QF = HD / 16;                                // 16-byte pieces of a lane's query
  const int WD = PAD ? hd : HD, chunks = WD / 8;
  // (arrays of their own, so that a read of one does not wait for the loads into another)
  __shared__ __align__(16) char k0[C::BYTES], k1[C::BYTES], v0[C::BYTES], v1[C::BYTES];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lq = lane & 31,
            lh = lane >> 5;
  const int hgs = heads / gh, R = (4 / gh) * 32;
  const unsigned id = turn_about(), slot = id / hgs;
  const int hg = (int)(id - slot * hgs);
  const Place pl = place_of(s, slot, R);
  if (pl.len == 0) return;
  const int h = hg * gh + wave % gh, g = hg * gh / (heads / kv_heads);
  const int len = pl.len, w0 = pl.q0 + wave / gh * 32;       // the wave's first row
  const int last = pl.q0 + R < len ? pl.q0 + R : len;        // keys the workgroup needs
  const int n_tiles = (last + KT - 1) / KT;

  const int kstep = (int)(ldk * 2), vstep = (int)(ldv * 2);
  const char* const kb = reinterpret_cast<const char*>(k + pl.row0 * ldk + (int64_t)g * WD);
  const char* const vb = reinterpret_cast<const char*>(v + pl.row0 * ldv + (int64_t)g * WD);
  const TileLoad<CH, PER, PAD> tl{wave, len, chunks};
  auto load_k = [&](char* to, int t) { tl.run(kb, kstep, C::kswz, to, t * KT, KT); };
  auto load_v = [&](char* to, int t) { tl.run(vb, vstep, C::vswz, to, t * KT, KT); };
  auto arrived = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0): this wave's part; then everybody's
    __syncthreads();
  };
  if (PAD) {
    clear_rest<CH, KT>(k0, C::kswz, chunks);
    clear_rest<CH, KT>(k1, C::kswz, chunks);
    clear_rest<CH, KT>(v0, C::vswz, chunks);
    clear_rest<CH, KT>(v1, C::vswz, chunks);
  }
  load_k(k0, 0);

  // queries: lane's own row, pieces of 8 values by halves
  u32x4 qf[QF];
  {
    const int r = w0 + lq < len ? w0 + lq : len - 1;
    const char* qp = reinterpret_cast<const char*>(q + (pl.row0 + r) * ldq + (int64_t)h * WD);
#pragma unroll
    for (int c = 0; c < QF; ++c)
      qf[c] = !PAD || 2 * c + lh < chunks ? *reinterpret_cast<const u32x4*>(qp + (2 * c + lh) * 16) : u32x4{0, 0, 0, 0};
  }
  load_v(v0, 0);
  if (n_tiles > 1) load_k(k1, 1);
  if (scale < 0.f) {
#pragma unroll
    for (int c = 0; c < QF; ++c) qf[c] ^= 0x80008000u;
  }
  const float c2 = fabsf(scale) * 1.4426950408889634f;

  bool far = false;                      // the wave's scores are too large for all this
  floatx16 o[NB];
  float l = 0.f, m = -3.4028235e38f;     // (finite: a score of -inf has weight 0 also where nothing else came before)
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
      st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[c]), st, 0,
                                                   0, 0);
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
      if (__ballot(fabsf(m) > 0x1p27f && m < INFINITY)) far = true;
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
  // V^T of block n, keys 16 c .. + 15 of sub: the order of the packed probabilities
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
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const u32x4 pb = u32x4{pack2(st[8 * c], st[8 * c + 1]), pack2(st[8 * c + 2], st[8 * c + 3]),
                             pack2(st[8 * c + 4], st[8 * c + 5]), pack2(st[8 * c + 6], st[8 * c + 7])};
#pragma unroll
      for (int n = 0; n < NB; ++n)
        o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_frag(vt, sub, c, n)),
                                                       __builtin_bit_cast(bf16x8, pb), o[n], 0, 0, 0);
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
    for (int u = 0; u < SUBS; ++u) {
      weigh(st[u], std::false_type{}, 0);
      nx[u] = scores(kn, u);
      add(vt, u, st[u]);
    }
#pragma unroll
    for (int u = 0; u < SUBS; ++u) st[u] = nx[u];
    maximum();
    arrived();
  };
  // (V of tile 0 and K of tile 1 may still be on their way)
  if (n_tiles > 1) __builtin_amdgcn_s_waitcnt(0x0F70 | 2 * PER);
  else __builtin_amdgcn_s_waitcnt(0x0F70 | PER);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < SUBS; ++u) st[u] = scores(k0, u);
  maximum();
  arrived();                                                 // (K of tile 0 is overwritten next)
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
#pragma unroll
      for (int u = 0; u < SUBS; ++u) {
        if (u > ahead) break;
        weigh(st[u], std::true_type{}, lim - u * 32);
        add(vt, u, st[u]);
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
  l += __shfl_xor(l, 32, 64);
  const float inv = 1.f / l;
  float any = 0.f;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) any += o[n][i] *= inv;
  __syncthreads();
  char* const mine = (wave < 2 ? k0 : k1) + wave % 2 * 32 * ROW;
  auto put_rows = [&] {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<uint2*>(mine + lq * ROW + ((4 * n + i) ^ C::kswz(lq)) * 16 + lh * 8) =
            make_uint2(pack2(o[n][4 * i], o[n][4 * i + 1]), pack2(o[n][4 * i + 2], o[n][4 * i + 3]));
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  // (of a row whose l is not finite nothing is, whatever V holds)
  if (!far && w0 < len && __ballot(any - any != 0.f && l - l == 0.f)) {
    put_rows();
    const uint32_t sums = (uint32_t)__ballot(l - l == 0.f);
    far = in_doubt([&](int c) {
      int got = 0;
      for (int r = 0; r < 32; ++r) {
        const char* const at = mine + r * ROW + ((c >> 3) ^ C::kswz(r)) * 16 + (c & 7) * 2;
        got |= sums >> r & 1 ? kind_of(bf2f(*reinterpret_cast<const uint16_t*>(at))) : 0;
      }
      return got;
    }, v + pl.row0 * ldv + (int64_t)g * WD, ldv, w0, WD);
  }
  if (far) {
    for (int r = w0; r < w0 + 32 && r < len; ++r)
      attend_row(q + (pl.row0 + r) * ldq + (int64_t)h * WD, k + pl.row0 * ldk + (int64_t)g * WD, ldk,
                 v + pl.row0 * ldv + (int64_t)g * WD, ldv, r, WD, scale, reinterpret_cast<float*>(mine),
                 out + ((pl.row0 + r) * heads + h) * WD);
    return;
  }
  put_rows();
  char* const op = reinterpret_cast<char*>(out + ((pl.row0 + w0) * heads + h) * WD);
#pragma unroll
  for (int u = 0; u < 32 * CH / 64; ++u) {
    const int row = (u * 64 + lane) / CH, c = lane % CH;
    const u32x4 x = *reinterpret_cast<const u32x4*>(mine + row * ROW + (c ^ C::kswz(row)) * 16);
    if (w0 + row < len && (!PAD || c < chunks))
      *reinterpret_cast<u32x4*>(op + (int64_t)row * heads * WD * 2 + c * 16) = x;
  }
}


// ---------------------------------------------------------------- fp32
// The same on v_mfma_f32_16x16x4_f32 with 16 rows a wave: the products, 64 flops a cycle and SIMD, take
// nearly all of the time, so that short workgroups matter more than what LDS gives (16 rows instead of 32: 131 ->
// 109 us).  6 sequences up to 1501 tokens, 16 heads of 64, in 87 us; one of 4000 in 285, 115 TFLOP/s.
template <int HD>
struct TileF {
  static constexpr int KT = 32, ROW = HD * 4, CH = HD / 4, BYTES = KT * ROW;
  static constexpr int QF = HD / 16;                         // 16-byte pieces of a lane's query
  static constexpr int W = HD >= 64 ? 4 : 2, NV = HD / (16 * W); // columns of V a lane reads at once, and how often
  __device__ static int kswz(int row) { return CH >= 16 ? row & 15 : (row >> 1) & 7; }
};

// (PAD: a multiple of 4)
template <int HD, bool PAD>
__global__ void __launch_bounds__(256, HD == 128 ? 2 : 4)
    attention_packed_f32_kernel(zoact_packed s, const float* __restrict__ q, int64_t ldq, const float* __restrict__ k,
                                int64_t ldk, const float* __restrict__ v, int64_t ldv, int heads, int kv_heads, int hd,
                                int gh, float scale, float* __restrict__ out) {
  using C = TileF<HD>;
  constexpr int KT = C::KT, ROW = C::ROW, CH = C::CH, QF = C::QF, W = C::W, NV = C::NV;
  const int WD = PAD ? hd : HD, chunks = WD / 4;
  typedef float floatw __attribute__((ext_vector_type(W)));
  __shared__ __align__(16) char k0[C::BYTES], k1[C::BYTES], v0[C::BYTES], v1[C::BYTES];
  __shared__ float qs[4][HD];                                // a row's query, where rows are taken one by one
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lq = lane & 15,
            lg = lane >> 4;
  const int hgs = heads / gh, R = 4 / gh * 16;
  const unsigned id = turn_about(), slot = id / hgs;
  const int hg = (int)(id - slot * hgs);
  Place pl = longest_first(s, slot, R);
  if (__builtin_amdgcn_readfirstlane(pl.len) == 0) return;
  // (the same in all lanes, which the compiler does not see through the search)
  pl = Place{__builtin_amdgcn_readfirstlane((int)pl.row0), __builtin_amdgcn_readfirstlane(pl.len),
             __builtin_amdgcn_readfirstlane(pl.q0)};
  const int h = hg * gh + wave % gh, g = hg * gh / (heads / kv_heads);
  const int len = pl.len, w0 = pl.q0 + wave / gh * 16;       // the wave's first row
  const int last = pl.q0 + R < len ? pl.q0 + R : len;        // keys the workgroup needs
  const int n_tiles = (last + KT - 1) / KT;

  const int kstep = (int)(ldk * 4), vstep = (int)(ldv * 4);
  const char* const kb = reinterpret_cast<const char*>(k + pl.row0 * ldk + (int64_t)g * WD);
  const char* const vb = reinterpret_cast<const char*>(v + pl.row0 * ldv + (int64_t)g * WD);
  const TileLoad<CH, KT * CH / 256, PAD> tl{wave, len, chunks};
  auto load_k = [&](char* to, int t) { tl.run(kb, kstep, C::kswz, to, t * KT, KT); };
  auto load_v = [&](char* to, int t) { tl.run(vb, vstep, no_swizzle, to, t * KT, KT); };
  auto arrived = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0): this wave's part; then everybody's
    __syncthreads();
  };
  if (PAD) {
    clear_rest<CH, KT>(k0, C::kswz, chunks);
    clear_rest<CH, KT>(k1, C::kswz, chunks);
    clear_rest<CH, KT>(v0, no_swizzle, chunks);
    clear_rest<CH, KT>(v1, no_swizzle, chunks);
  }
  load_k(k0, 0);
  // queries: lane's own row, chunks 4 c + lg
  u32x4 qf[QF];
  {
    const int r = w0 + lq < len ? w0 + lq : len - 1;
    const char* qp = reinterpret_cast<const char*>(q + (pl.row0 + r) * ldq + (int64_t)h * WD);
#pragma unroll
    for (int c = 0; c < QF; ++c)
      qf[c] = !PAD || 4 * c + lg < chunks ? *reinterpret_cast<const u32x4*>(qp + (4 * c + lg) * 16) : u32x4{0, 0, 0, 0};
  }
  load_v(v0, 0);
  if (n_tiles > 1) load_k(k1, 1);
  if (scale < 0.f) {
#pragma unroll
    for (int c = 0; c < QF; ++c) qf[c] ^= 0x80000000u;
  }
  const float c2 = fabsf(scale) * 1.4426950408889634f;

  bool far = false;                                          // the wave's scores are too large for all this
  floatx4 o[NV][W];                                          // o[n][e][i]: column 16 W n + W (4 lg + i) + e
  float l = 0.f, m = -3.4028235e38f;     // (finite: a score of -inf has weight 0 also where nothing else came before)
#pragma unroll
  for (int n = 0; n < NV; ++n)
#pragma unroll
    for (int e = 0; e < W; ++e) o[n][e] = floatx4{0.f, 0.f, 0.f, 0.f};

  // scores of a block of 16 keys; register i: key 4 lg + i.  One product takes a value of each of four chunks.
  auto scores = [&](const char* kt, int blk) {
    floatx4 st = {0.f, 0.f, 0.f, 0.f};
    const int key = blk * 16 + lq;
#pragma unroll
    for (int c = 0; c < QF; ++c) {
      const u32x4 kf = *reinterpret_cast<const u32x4*>(kt + key * ROW + ((4 * c + lg) ^ C::kswz(key)) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        st = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[e]), __uint_as_float(qf[c][e]), st, 0, 0, 0);
    }
    return st;
  };
  // a row's maximum over the four parts of the wave
  auto all = [&](float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto z = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(z[0]), __uint_as_float(z[1]));
  };
  auto follow = [&](float mx) {
    mx *= c2;
    if (__ballot(mx > m + 8.f)) {
      const float mn = fmaxf(m, mx), a = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      if (__ballot(fabsf(m) > 0x1p27f && m < INFINITY)) far = true;
      l *= a;
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < W; ++e) o[n][e] *= a;
    }
  };
  auto weigh = [&](floatx4& st, auto cut, int lim) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      st[i] = __builtin_amdgcn_exp2f(fmaf(st[i], c2, -m));
      if (decltype(cut)::value && i > lim) st[i] = 0.f;
    }
    l += (st[0] + st[1]) + (st[2] + st[3]);
  };
  auto add = [&](const char* vt, int blk, const floatx4& st) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const char* vp = vt + (blk * 16 + 4 * lg + i) * ROW + lq * W * 4;
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const floatw x = *reinterpret_cast<const floatw*>(vp + n * 16 * W * 4);
#pragma unroll
        for (int e = 0; e < W; ++e) o[n][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], st[i], o[n][e], 0, 0, 0);
      }
    }
  };
  const int n_full = pl.q0 / KT;                             // tiles that every row of the workgroup sees
  floatx4 st[2];
  float mx;
  auto maximum = [&] {
    mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, fmaxf(st[0][i], st[1][i]));
    mx = all(mx);
  };
  auto full = [&](char* kt, char* kn, char* vt, char* vn, int t) {
    if (t + 2 < n_tiles) load_k(kt, t + 2);
    load_v(vn, t + 1);
    follow(mx);
    const floatx4 n0 = scores(kn, 0), n1 = scores(kn, 1);
    weigh(st[0], std::false_type{}, 0);
    weigh(st[1], std::false_type{}, 0);
    add(vt, 0, st[0]);
    add(vt, 1, st[1]);
    st[0] = n0;
    st[1] = n1;
    maximum();
    arrived();
  };
  arrived();
  st[0] = scores(k0, 0);
  st[1] = scores(k0, 1);
  maximum();
  __syncthreads();                                           // (K of tile 0 is overwritten next)
#pragma unroll 1
  for (int t = 0; t < n_full; t += 2) {
    full(k0, k1, v0, v1, t);
    if (t + 1 == n_full) break;
    full(k1, k0, v1, v0, t + 1);
  }
#pragma unroll 1
  for (int t = n_full; t < n_tiles; ++t) {
    char* const vt = t & 1 ? v1 : v0;
    if (t + 1 < n_tiles) load_v(t & 1 ? v0 : v1, t + 1);
    if (t + 2 < n_tiles) load_k(t & 1 ? k1 : k0, t + 2);
    if (t * KT <= w0 && w0 < len) {
      const int lim = w0 + lq - t * KT;
      float mb = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) mb = fmaxf(mb, 16 * u + i <= lim - 4 * lg ? st[u][i] : -INFINITY);
      follow(all(mb));
      weigh(st[0], std::true_type{}, lim - 4 * lg);
      weigh(st[1], std::true_type{}, lim - 4 * lg - 16);
      add(vt, 0, st[0]);
      if (w0 - t * KT >= 16) add(vt, 1, st[1]);
    }
    if (t + 1 == n_tiles) break;
    const char* const kn = t & 1 ? k0 : k1;
    st[0] = scores(kn, 0);
    st[1] = scores(kn, 1);
    arrived();
  }

  l += __shfl_xor(l, 32, 64);
  l += __shfl_xor(l, 16, 64);
  const float inv = 1.f / l;
  float any = 0.f;
#pragma unroll
  for (int n = 0; n < NV; ++n)
#pragma unroll
    for (int e = 0; e < W; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) any += o[n][e][i] *= inv;
  // (of a row whose l is not finite nothing is, whatever V holds)
  if (!far && w0 < len && __ballot(any - any != 0.f && l - l == 0.f)) {
    int* const cols = reinterpret_cast<int*>(qs[wave]);
    for (int c = lane; c < HD; c += 64) cols[c] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (l - l == 0.f) {
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < W; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (const int x = kind_of(o[n][e][i])) atomicOr(cols + 16 * W * n + W * (4 * lg + i) + e, x);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    far = in_doubt([&](int c) { return cols[c]; }, v + pl.row0 * ldv + (int64_t)g * WD, ldv, w0, WD);
  }
  if (far) {
    for (int r = w0; r < w0 + 16 && r < len; ++r)
      attend_row(q + (pl.row0 + r) * ldq + (int64_t)h * WD, k + pl.row0 * ldk + (int64_t)g * WD, ldk,
                 v + pl.row0 * ldv + (int64_t)g * WD, ldv, r, WD, scale, qs[wave],
                 out + ((pl.row0 + r) * heads + h) * WD);
    return;
  }
  if (w0 + lq >= len) return;
  float* const op = out + ((pl.row0 + w0 + lq) * heads + h) * WD;
#pragma unroll
  for (int n = 0; n < NV; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      floatw x;
#pragma unroll
      for (int e = 0; e < W; ++e) x[e] = o[n][e][i];
      const int col = 16 * W * n + W * (4 * lg + i);
      if (!PAD || col < hd) *reinterpret_cast<floatw*>(op + col) = x;
    }
}

}  // namespace

hipError_t launch_attention_packed(const zoact_packed& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                   const void* v, int64_t ldv, int32_t heads, int32_t kv_heads, int32_t hd, float scale,
                                   int32_t dtype, void* out, hipStream_t hs) {
  const int64_t vec = dtype == ZOACT_BF16 ? 8 : 4;
  if (hd > 128 || hd % vec || ldq % vec || ldk % vec || ldv % vec || !aligned_to(q, 16) ||
      !aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(out, 16))
    return hipErrorNotSupported;
  if (!isfinite(fabsf(scale) * 1.4426950408889634f)) return hipErrorNotSupported;
  // (a tile's rows are addressed with 32 bits)
  if (ldk >= (int64_t(1) << 22) || ldv >= (int64_t(1) << 22)) return hipErrorNotSupported;
  const int G = heads / kv_heads, gh = G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1;
  const int R = 4 / gh * (dtype == ZOACT_BF16 ? 32 : 16);
  const int64_t grid = (s.rows / R + s.n) * (heads / gh);
  if (grid >= (int64_t(1) << 24)) return hipErrorNotSupported;    // (a launch has less than 2^32 threads)
#define ZO_ATT(T, KERNEL, HD)                                                                                       \
  do {                                                                                                              \
    if (hd == HD)                                                                                                   \
      KERNEL<HD, false><<<(unsigned)grid, 256, 0, hs>>>(s, (const T*)q, ldq, (const T*)k, ldk, (const T*)v, ldv, heads, \
                                                        kv_heads, hd, gh, scale, (T*)out);                          \
    else                                                                                                            \
      KERNEL<HD, true><<<(unsigned)grid, 256, 0, hs>>>(s, (const T*)q, ldq, (const T*)k, ldk, (const T*)v, ldv, heads, \
                                                       kv_heads, hd, gh, scale, (T*)out);                           \
  } while (0)
  if (dtype == ZOACT_BF16) {
    if (hd > 64) ZO_ATT(uint16_t, attention_packed_bf16_kernel, 128);
    else if (hd > 32) ZO_ATT(uint16_t, attention_packed_bf16_kernel, 64);
    else ZO_ATT(uint16_t, attention_packed_bf16_kernel, 32);
  } else {
    if (hd > 64) ZO_ATT(float, attention_packed_f32_kernel, 128);
    else if (hd > 32) ZO_ATT(float, attention_packed_f32_kernel, 64);
    else ZO_ATT(float, attention_packed_f32_kernel, 32);
  }
#undef ZO_ATT
  return hipGetLastError();
}

}  // namespace zoact
