// The paged 8-bit key/value cache (zoact_cache.h): rotary and quantisation of new rows, and
// the operations on pages -- extend (with copy on write), fork, free, compact.
#include <math.h>

#include <string>

#include "cache.hpp"

namespace zoact {
namespace {

// ---------------------------------------------------------------- append
// One workgroup per (page of an entry's new tokens, keys or values of a head, entry); wave w holds the
// page's block w.  The four lanes of a token take its 16-byte pieces in turn (a quad reads 64 contiguous
// bytes), so the partner of a rotated value lies in the same lane, and the block's maximum is a reduction
// over the wave.  V goes through LDS to its transposed place.  Bound by bytes, each read and written once: four
// prompts of 2011 tokens, 40 heads of 128 (216 MB), 62 us, 3.5 TB/s (on the same inputs again and again 49, in fp32
// 74); 32 single tokens, 8 heads, 8 us of launch and trips to memory (batch, page number, rows).
// Value i of a lane is dim ((i / V) * 4 + quarter) * V + i % V, V values a piece.
template <typename T, int HD>
struct Quarter {
  static constexpr int Q = HD / 4, V = 16 / (int)sizeof(T), HALF = HD / 2;
  static constexpr bool kInLane = Q / V >= 2;      // (bf16, HD 32: one piece a lane, the partner two lanes on)
  __device__ static int dim(int i, int q) { return ((i / V) * 4 + q) * V + i % V; }
  __device__ static void load_piece(const T* p, float* o) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if constexpr (sizeof(T) == 2)
        o[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
      else
        o[e] = __uint_as_float(w[e]);
    }
  }
  __device__ static void load(const T* row, int q, float (&x)[Q]) {
#pragma unroll
    for (int i = 0; i < Q; i += V) load_piece(row + dim(i, q), &x[i]);
  }
  // (lo, hi) -> (lo c - hi s, hi c + lo s), one rounding per operation
  __device__ static void rotate(float (&x)[Q], int q, const float* ct, const float* st) {
#pragma clang fp contract(off)
    if constexpr (kInLane) {
#pragma unroll
      for (int i = 0; i < Q / 2; i += 4) {
        const float4 c4 = *reinterpret_cast<const float4*>(ct + dim(i, q));
        const float4 s4 = *reinterpret_cast<const float4*>(st + dim(i, q));
        const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float lo = x[i + e], hi = x[Q / 2 + i + e];
          x[i + e] = lo * c[e] - hi * s[e];
          x[Q / 2 + i + e] = hi * c[e] + lo * s[e];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        const float y = __shfl_xor(x[i], 2, 64);
        const int d = dim(i, q) % HALF;
        x[i] = q >= 2 ? x[i] * ct[d] + y * st[d] : x[i] * ct[d] - y * st[d];
      }
    }
  }
};

// Codes of four values of a lane under their block's scale (the same in all lanes; NaN: 0, s == 0: every value
// is 0), rint(x / s).  A division is a dozen instructions (32 single tokens 9.5 us with them, 8.4 without); x times
// inverse is off by no more than 3 half steps of 127, 2^-15.4, so the quotients are formed only where it comes
// within 2^-14 of the middle between two codes.  Scales near the smallest numbers (inverse 0) always take
// them, and only there a quotient passes 127.
__device__ __forceinline__ void quantise4(const float* x, float s, float inverse, int (&q)[4]) {
  float off = inverse > 0.f ? 0.f : 1.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float t = x[j] * inverse, n = rintf(t);
    off = fmaxf(off, fabsf(t - n));
    q[j] = (int)n;
  }
  if (__any(off > 0.5f - 0x1p-14f)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = (int)fminf(fmaxf(s > 0.f ? rintf(x[j] / s) : 0.f, -127.f), 127.f);
  }
}
__device__ __forceinline__ float inverse_of(float s) { return s > 0x1p-100f ? 1.f / s : 0.f; }
__device__ __forceinline__ int requantise(int q, float ratio) { return (int)rintf((float)q * ratio); }
__device__ __forceinline__ uint32_t requantise4(uint32_t w, float ratio) {
  uint32_t o = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) o |= (uint32_t)(requantise((int8_t)(w >> (8 * e)), ratio) & 255) << (8 * e);
  return o;
}

// Largest magnitude of a wave's values; NaN if one is not finite.
template <int Q>
__device__ __forceinline__ float wave_absmax(const float (&x)[Q], bool in) {
  uint32_t m = 0;      // (magnitudes order as their bits do, infinities and NaN last)
#pragma unroll
  for (int j = 0; j < Q; ++j) m = max(m, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  if (!in) m = 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  return m >= 0x7F800000u ? NAN : __uint_as_float(m);
}

// Scale of a block with `held` earlier tokens, and the ratio their codes are multiplied by.
__device__ __forceinline__ float block_scale(float amax, bool held, float old, float& ratio) {
  float s = amax * (1.f / 127.f);
  ratio = 1.f;
  if (held) {
    if (s != s || old != old)
      s = NAN;
    else if (s > old)
      ratio = old / s;
    else
      s = old;
  }
  return s;
}

template <typename T, int HD>
__global__ void __launch_bounds__(256) append_kernel(zoact_cache c, int layer, const T* __restrict__ k, int64_t ldk,
                                                     const T* __restrict__ v, int64_t ldv, zoact_cache_batch b,
                                                     const float* __restrict__ ct, const float* __restrict__ st,
                                                     int64_t n_pos) {
  typedef Quarter<T, HD> Qt;
  constexpr int Q = Qt::Q;
  __shared__ uint32_t tile[HD * kPage / 4];      // V's page as stored: [HD][64]
  const bool is_v = blockIdx.y >= (unsigned)c.n_kv_heads;
  const int hk = is_v ? blockIdx.y - c.n_kv_heads : blockIdx.y;
  const CacheEntry e = read_entry(c, b, blockIdx.z, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0);
  if (!e.ok || e.count == 0) return;
  const int pg = e.pos / kPage + blockIdx.x, end = e.pos + e.count;
  if ((int64_t)pg * kPage >= end) return;
  const int pid = c.table[(int64_t)e.slot * c.max_pages + pg];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane & 3;
  const int t0 = pg * kPage + wave * kBlock;     // the block's first token
  const bool live = t0 + kBlock > e.pos && t0 < end;
  const int tok = t0 + (lane >> 2);
  const bool in = tok >= e.pos && tok < end, held = t0 < e.pos;
  float x[Q];
  if (live) {
    // (lanes without a new token take one that there is)
    const int64_t row = e.row0 + (tok < e.pos ? 0 : tok >= end ? e.count - 1 : tok - e.pos);
    Qt::load((is_v ? v + row * ldv : k + row * ldk) + (int64_t)hk * HD, q, x);
  }
  if (pid < 0 || pid >= c.n_pages) {
    if (threadIdx.x == 0 && blockIdx.y == 0) raise_status(b.status, ZOACT_STATUS_BAD_ENTRY);
    return;
  }
  const int64_t head = ((int64_t)layer * c.n_pages + pid) * c.n_kv_heads + hk;
  float* const sp = (is_v ? c.v_scale : c.k_scale) + head * kPageBlocks + wave;
  if (!is_v) {
    if (!live) return;
    const float before = held ? *sp : 0.f;
    if (ct) {
      const int64_t ti = tok < n_pos ? tok : n_pos - 1;
      Qt::rotate(x, q, ct + ti * (HD / 2), st + ti * (HD / 2));
    }
    float ratio;
    const float s = block_scale(wave_absmax<Q>(x, in), held, before, ratio);
    const float inverse = inverse_of(s);
    int8_t* const kp = c.k + (head * kPage + wave * kBlock + (lane >> 2)) * HD;
#pragma unroll
    for (int i = 0; i < Q; i += 4) {
      uint32_t* const at = reinterpret_cast<uint32_t*>(kp + Qt::dim(i, q));
      int code[4];
      quantise4(&x[i], s, inverse, code);
      if (in) {
        *at = (uint32_t)(code[0] & 255) | (uint32_t)(code[1] & 255) << 8 | (uint32_t)(code[2] & 255) << 16 |
              (uint32_t)code[3] << 24;
      } else if (tok < e.pos && ratio != 1.f) {
        *at = requantise4(*at, ratio);
      }
    }
    if (lane == 0 && !(held && s == before)) *sp = s;
    return;
  }
  uint32_t* const vp = reinterpret_cast<uint32_t*>(c.v + head * kPage * HD);
  if (live) {
    const float before = held ? *sp : 0.f;
    // the block's words of old codes, unless all are new
    constexpr int W = HD / 16;
    const bool whole = t0 >= e.pos && t0 + kBlock <= end;
    uint32_t w[W];
    if (!whole) {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = vp[((lane >> 2) + i * 16) * 16 + q * 4 + wave];
    }
    float ratio;
    const float s = block_scale(wave_absmax<Q>(x, in), held, before, ratio);
    if (!whole) {
      // word (d, g) holds tokens 4 g .. 4 g + 3 of the block; only those before pos are the sequence's
      const int n = e.pos - (t0 + 4 * q);
      const uint32_t keep = n <= 0 ? 0u : n >= 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
#pragma unroll
      for (int i = 0; i < W; ++i)
        tile[((lane >> 2) + i * 16) * 16 + q * 4 + wave] =
            ratio != 1.f && keep ? (requantise4(w[i], ratio) & keep) | (w[i] & ~keep) : w[i];
      __builtin_amdgcn_wave_barrier();
      __threadfence_block();
    }
    // the new codes over them
    const float inverse = inverse_of(s);
    const int i = lane >> 2;                       // token of the block: group i >> 2, byte i & 3
    uint8_t* const tb = reinterpret_cast<uint8_t*>(tile) + (i >> 2) * 16 + wave * 4 + (i & 3);
#pragma unroll
    for (int j = 0; j < Q; j += 4) {
      int code[4];
      quantise4(&x[j], s, inverse, code);
      if (in) {
#pragma unroll
        for (int e2 = 0; e2 < 4; ++e2) tb[Qt::dim(j + e2, q) * kPage] = (uint8_t)code[e2];
      }
    }
    if (lane == 0 && !(held && s == before)) *sp = s;
  }
  __syncthreads();
  if (pg * kPage + kPage <= end && e.pos < pg * kPage + kBlock) {   // all four blocks
    for (int i = threadIdx.x; i < HD * kPage / 16; i += 256)
      reinterpret_cast<uint4*>(vp)[i] = reinterpret_cast<const uint4*>(tile)[i];
  } else if (live) {
    for (int i = lane; i < HD * 4; i += 64) {
      const int at = (i >> 2) * 16 + (i & 3) * 4 + wave;
      vp[at] = tile[at];
    }
  }
}

// ---------------------------------------------------------------- pages
__device__ __forceinline__ bool good_page(const zoact_cache& c, int p) { return p >= 0 && p < c.n_pages; }
__device__ __forceinline__ bool good_len(const zoact_cache& c, int L) {
  return L >= 0 && L <= (int64_t)c.max_pages * kPage;
}
__device__ __forceinline__ int page_count(int L) { return (int)(((int64_t)L + kPage - 1) / kPage); }

// Inclusive scan over a workgroup of TH threads: within the rows of 16 lanes, over a wave's four rows, then over
// the waves through sh (TH / 64 ints); `total` is the last value.  One barrier: a scan that follows takes other
// words of LDS, the one after it may take these again.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_lane(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
template <int TH>
__device__ __forceinline__ int scan(int v, int* sh, int& total) {
  constexpr int NW = TH / 64;
  const int w = threadIdx.x >> 6;
  v = add_lane<0x111, 0xF>(v);     // from one, two, four, eight lanes before
  v = add_lane<0x112, 0xF>(v);
  v = add_lane<0x114, 0xF>(v);
  v = add_lane<0x118, 0xF>(v);
  v = add_lane<0x142, 0xA>(v);     // the first row's last to the second, the third's to the fourth
  v = add_lane<0x143, 0xC>(v);     // the second's last to the third and fourth
  if ((threadIdx.x & 63) == 63) sh[w] = v;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < NW; i += 4) {
    const int4 q = *reinterpret_cast<const int4*>(sh + i);
    const int t[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      base += i + k < w ? t[k] : 0;
      total += t[k];
    }
  }
  return base + v;
}

// How many of v[0 .. i - 1] (LDS, n of them set) are x: four a load and no branches, as a thread's loop of
// tests one by one is a branch and a wait each.
__device__ __forceinline__ int count_before(const int* v, int i, int x, int n) {
  const int end = n < (int)(threadIdx.x | 63) ? n : (int)(threadIdx.x | 63);      // (the wave's last)
  int k = 0;
#pragma unroll 4
  for (int j = 0; j < end; j += 4) {
    const int4 q = *reinterpret_cast<const int4*>(v + j);
    k += (q.x == x && j < i) + (q.y == x && j + 1 < i) + (q.z == x && j + 2 < i) + (q.w == x && j + 3 < i);
  }
  return k;
}

// Bookkeeping of extend: one workgroup, a thread per entry.  ws: pairs[n] (source and target of a
// page to copy, source -1 for none), then the free pages handed out past the first kFresh, which stay in LDS.
// Bound by the trips to memory that wait for each other (slot, length, page, its holders)
// and the scans: 5.8 us for 32 entries (on 1024 threads 8.1); the first free pages are asked for meanwhile.
constexpr int kFresh = 2048;
template <int TH>
__global__ void __launch_bounds__(TH) extend_kernel(zoact_cache c, zoact_cache_batch b, int2* __restrict__ pairs,
                                                      int* __restrict__ more) {
  __shared__ __align__(16) int slot_of[TH], last_of[TH], sh[3][TH / 64];
  __shared__ int upto[TH], first[kFresh];
  const int i = threadIdx.x;
  const int64_t n_pages = c.n_pages;
  auto holders = [&](int64_t p) { return c.refs[p < n_pages ? p : n_pages - 1]; };
  int held[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) held[q] = holders(4 * i + q);
  CacheEntry e{};
  e.slot = -1;
  int L = 0, last = -1, holding = 0;
  bool ok = false;
  if (i < b.n) {
    entry_rows(b, i, e);
    ok = e.rows_ok && e.slot >= 0 && e.slot < c.n_slots;
    if (ok) {
      L = c.len[e.slot];
      ok = good_len(c, L) && (int64_t)L + e.count <= (int64_t)c.max_pages * kPage;
    }
    if (ok && e.count > 0 && L % kPage) {
      last = c.table[(int64_t)e.slot * c.max_pages + L / kPage];
      ok = good_page(c, last);
      if (ok) holding = c.refs[last];
    }
  }
  slot_of[i] = i < b.n ? e.slot : -1;
  __syncthreads();
  if (count_before(slot_of, i, e.slot, b.n) > 0) ok = false;               // named before in the batch
  if (!ok) last = -1;
  last_of[i] = last;
  __syncthreads();
  // a shared last page is copied by every entry that writes to it but its last holder
  const int before = count_before(last_of, i, last, b.n);
  bool cow = false;
  if (last >= 0) {
    cow = before < holding - 1;
  }
  const int grow = ok ? page_count(L + e.count) - page_count(L) : 0;
  const int need = grow + (cow ? 1 : 0);
  int total;
  const int incl = scan<TH>(need, sh[2], total);
  upto[i] = incl;
  // free pages, lowest number first
  int found = 0;
  auto fresh = [&](int at) { return at < kFresh ? first[at] : more[at]; };
  for (int64_t p0 = 0, round = 0; p0 < n_pages && found < total; p0 += 4 * TH, ++round) {
    const int64_t p = p0 + 4 * i;
    int f[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f[q] = p + q < n_pages && held[q] == 0;
      held[q] = holders(p + 4 * TH + q);       // (of the next round, if there is one)
    }
    const int mine = f[0] + f[1] + f[2] + f[3];
    int n;
    int at = found + scan<TH>(mine, sh[round & 1], n) - mine;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (f[q]) {
        if (at < total && at < kFresh) first[at] = (int)(p + q);
        if (at < total && at >= kFresh) more[at] = (int)(p + q);
        ++at;
      }
    found += n;
  }
  const bool enough = found >= total;      // (the same in every thread)
  if (i == 0 && !enough) raise_status(b.status, ZOACT_STATUS_NO_PAGES);
  if (i < b.n && !ok) raise_status(b.status, ZOACT_STATUS_BAD_ENTRY);
  __threadfence_block();
  __syncthreads();
  if (i < b.n) {
    int2 pair = make_int2(-1, -1);
    const bool served = ok && enough;
    b.pos[i] = served ? L : -1;
    if (served) {
      c.len[e.slot] = L + e.count;
      if (cow) {
        const int p = fresh(incl - need);
        pair = make_int2(last, p);
        atomicSub(&c.refs[last], 1);
        c.table[(int64_t)e.slot * c.max_pages + L / kPage] = p;
      }
    }
    pairs[i] = pair;
    last_of[i] = served ? page_count(L) - (cow ? 1 : 0) : 0;   // table index of the entry's page 0, less a copied one
  }
  __syncthreads();
  if (!enough) return;
  // tables and counts, a thread per page handed out
  for (int t = i; t < total; t += TH) {
    int lo = 0, hi = b.n - 1;              // the entry whose pages hold t
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (upto[mid] > t) hi = mid; else lo = mid + 1;
    }
    const int p = fresh(t), j = t - (lo ? upto[lo - 1] : 0);
    c.refs[p] = 1;
    // (a copied page is j = 0: the same entry of the table as written above)
    c.table[(int64_t)slot_of[lo] * c.max_pages + last_of[lo] + j] = p;
  }
}

// Bytes of page `src` over page `dst`, one layer, one of k and v with its scales.
__device__ __forceinline__ void copy_page(const zoact_cache& c, int64_t src, int64_t dst, int layer, int is_v, int part,
                                          int parts) {
  const int64_t per = (int64_t)c.n_kv_heads * kPage * c.head_dim / 16;     // 16-byte units of a page
  const int64_t base = (int64_t)layer * c.n_pages;
  uint4* const pool = reinterpret_cast<uint4*>(is_v ? c.v : c.k);
  const uint4* const s = pool + (base + src) * per;
  uint4* const d = pool + (base + dst) * per;
  for (int64_t i = part * 256 + threadIdx.x; i < per; i += 256 * parts) d[i] = s[i];
  if (part == 0) {
    float* const sc = is_v ? c.v_scale : c.k_scale;
    const int n = c.n_kv_heads * kPageBlocks;
    for (int i = threadIdx.x; i < n; i += 256) sc[(base + dst) * n + i] = sc[(base + src) * n + i];
  }
}

// Four workgroups a page, layer and kind: 16 KB each of 8 heads of 128 (32 pages of two layers 4.8 us).
constexpr int kCopyParts = 4;
__global__ void __launch_bounds__(256) copy_pairs_kernel(zoact_cache c, const int2* __restrict__ pairs) {
  const int2 p = pairs[blockIdx.x];
  if (p.x < 0) return;
  copy_page(c, p.x, p.y, blockIdx.y >> 1, blockIdx.y & 1, blockIdx.z, kCopyParts);
}

// Whether v[i] is among the values before it: by the W threads of an entry (a workgroup of 256, or half a wave).
template <int W>
__device__ __forceinline__ bool named_before(const int* v, int i, int lane) {
  const int x = v[i];
  bool again = false;
  for (int j = lane; j < i; j += W) again |= v[j] == x;
  if constexpr (W == 32)
    return (__ballot(again) >> (threadIdx.x & 32)) & 0xFFFFFFFFull;
  else
    return __syncthreads_or(again);
}

// Fork, first half, by an entry's W threads: stages its source's length and pages in ws and adds the
// destination as a holder (integer sums: any order gives the same counts).
template <int W>
__device__ __forceinline__ void fork_read(const zoact_cache& c, const int* src, const int* dst, int n, int i, int lane,
                                          int* ws, uint32_t* status) {
  const int s = src[i], d = dst[i];
  bool ok = s >= 0 && s < c.n_slots && d >= 0 && d < c.n_slots;
  ok = !named_before<W>(dst, i, lane) && ok;
  const int L = ok ? c.len[s] : 0;
  ok = ok && good_len(c, L) && good_len(c, c.len[d]);
  if (lane == 0) {
    ws[i] = ok ? L : -1;
    if (!ok) raise_status(status, ZOACT_STATUS_BAD_ENTRY);
  }
  if (!ok) return;
  int* const row = ws + n + (int64_t)i * c.max_pages;
  for (int j = lane; j < page_count(L); j += W) {
    const int p = c.table[(int64_t)s * c.max_pages + j];
    row[j] = p;
    if (good_page(c, p))
      atomicAdd(&c.refs[p], 1);
    else
      raise_status(status, ZOACT_STATUS_BAD_ENTRY);
  }
}

template <int W>
__device__ __forceinline__ void release_slot(const zoact_cache& c, int slot, int lane, uint32_t* status) {
  const int n = page_count(c.len[slot]);
  for (int j = lane; j < n; j += W) {
    const int p = c.table[(int64_t)slot * c.max_pages + j];
    if (good_page(c, p))
      atomicSub(&c.refs[p], 1);
    else
      raise_status(status, ZOACT_STATUS_BAD_ENTRY);
  }
}

// Second half: the destination gives back what it held and takes the staged row.  (A thread gives back and
// writes the same places of the row; the length is written when all have read it.)
template <int W>
__device__ __forceinline__ void fork_write(const zoact_cache& c, const int* dst, int n, int i, int lane, const int* ws,
                                           uint32_t* status) {
  const int L = ws[i];
  if (L < 0) return;
  const int d = dst[i];
  release_slot<W>(c, d, lane, status);
  const int* const row = ws + n + (int64_t)i * c.max_pages;
  for (int j = lane; j < page_count(L); j += W) c.table[(int64_t)d * c.max_pages + j] = row[j];
  if constexpr (W > 64) __syncthreads();
  if (lane == 0) c.len[d] = L;
}

__global__ void __launch_bounds__(256) fork_read_kernel(zoact_cache c, const int* __restrict__ src,
                                                        const int* __restrict__ dst, int n, int* __restrict__ ws,
                                                        uint32_t* status) {
  fork_read<256>(c, src, dst, n, blockIdx.x, threadIdx.x, ws, status);
}
__global__ void __launch_bounds__(256) fork_write_kernel(zoact_cache c, const int* __restrict__ dst, int n,
                                                         const int* __restrict__ ws, uint32_t* status) {
  fork_write<256>(c, dst, n, blockIdx.x, threadIdx.x, ws, status);
}
// Both halves in one workgroup, half a wave per entry, up to 32 entries of 64 pages: 8 full slots of 16 pages 3.3
// us and 5.4 in two launches, 32 of 16 pages 4.2 and 5.7, 32 of 60 5.4 and 5.5, 32 of 120 7.4 and 5.5, 64 of 60
// 8.8 and 5.6.
__global__ void __launch_bounds__(1024) fork_kernel(zoact_cache c, const int* __restrict__ src,
                                                    const int* __restrict__ dst, int n, int* ws, uint32_t* status) {
  const int lane = threadIdx.x & 31, i = threadIdx.x >> 5;
  if (i < n) fork_read<32>(c, src, dst, n, i, lane, ws, status);
  __threadfence_block();
  __syncthreads();
  if (i < n) fork_write<32>(c, dst, n, i, lane, ws, status);
}

__global__ void __launch_bounds__(256) free_kernel(zoact_cache c, const int* __restrict__ slots, uint32_t* status) {
  const int i = blockIdx.x, s = slots[i];
  if (named_before<256>(slots, i, threadIdx.x)) return;
  if (s < 0 || s >= c.n_slots || !good_len(c, c.len[s])) {
    if (threadIdx.x == 0) raise_status(status, ZOACT_STATUS_BAD_ENTRY);
    return;
  }
  release_slot<256>(c, s, threadIdx.x, status);
  __syncthreads();
  if (threadIdx.x == 0) c.len[s] = 0;
}

// Compact, first half (one workgroup): counts the used pages, pairs those at or past the count
// with the free ones below it, and moves their reference counts.  ws: head (pairs, used count),
// map [n_pages] from a moved page to its new number, sources, targets.  3.6 us for 1600 pages.
__global__ void __launch_bounds__(1024) compact_plan_kernel(zoact_cache c, int* __restrict__ head,
                                                            int* __restrict__ map, int* __restrict__ src,
                                                            int* __restrict__ dst, int* __restrict__ n_used) {
  __shared__ __align__(16) int sh[3][16];
  const int i = threadIdx.x;
  const int64_t N = c.n_pages;
  int mine = 0, used;
  for (int64_t p = i; p < N; p += 1024) mine += c.refs[p] > 0;
  scan<1024>(mine, sh[2], used);
  int ns = 0, nd = 0;
  for (int64_t p0 = 0, round = 0; p0 < N; p0 += 1024, ++round) {
    const int64_t p = p0 + i;
    const bool in = p < N, u = in && c.refs[p] > 0;
    const int move = u && p >= used, hole = in && !u && p < used;
    int tot;
    // (both ranks in one scan: at most 1024 of each)
    const int r = scan<1024>(move | hole << 16, sh[round & 1], tot);
    if (move) src[ns + (r & 0xFFFF) - 1] = (int)p;
    if (hole) dst[nd + (r >> 16) - 1] = (int)p;
    ns += tot & 0xFFFF;
    nd += tot >> 16;
  }
  __threadfence_block();
  __syncthreads();
  for (int k = i; k < ns; k += 1024) {
    const int s = src[k], d = dst[k];
    map[s] = d;
    c.refs[d] = c.refs[s];
    c.refs[s] = 0;
  }
  if (i == 0) {
    head[0] = ns;
    head[1] = used;
    if (n_used) *n_used = used;
  }
}

// Second half: the pages' bytes and the tables, near the rate of a copy (142 MB read and written in 32 us, 4.4
// TB/s).  Blocks walk (pair, layer, k or v) work items; no target is a source, so the copies need no order.
__global__ void __launch_bounds__(256) compact_move_kernel(zoact_cache c, const int* __restrict__ head,
                                                           const int* __restrict__ map, const int* __restrict__ src,
                                                           const int* __restrict__ dst) {
  const int n = head[0], used = head[1];
  if (n == 0) return;
  const int64_t items = (int64_t)n * c.n_layers * 2 * kCopyParts;
  for (int64_t w = blockIdx.x; w < items; w += gridDim.x) {
    const int part = (int)(w % kCopyParts);
    const int64_t q = w / kCopyParts;
    const int64_t pair = q / (2 * c.n_layers);
    const int lv = (int)(q % (2 * c.n_layers));
    copy_page(c, src[pair], dst[pair], lv >> 1, lv & 1, part, kCopyParts);
  }
  const int64_t cells = (int64_t)c.n_slots * c.max_pages;
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < cells; w += (int64_t)gridDim.x * 256) {
    const int64_t slot = w / c.max_pages;
    const int L = c.len[slot];
    if (!good_len(c, L) || w % c.max_pages >= page_count(L)) continue;
    const int p = c.table[w];
    if (p >= used && p < c.n_pages) c.table[w] = map[p];
  }
}

size_t cache_ws(const zoact_cache& c) {
  const size_t fork = (size_t)c.n_slots * ((size_t)c.max_pages + 1);
  const size_t extend = 2 * ZOACT_CACHE_MAX_BATCH + (size_t)c.n_pages;
  const size_t compact = 4 + 3 * (size_t)c.n_pages;
  const size_t m = fork > extend ? fork : extend;
  return 4 * (m > compact ? m : compact) + 64;
}

bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool al4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

#define ZC(cond, msg) \
  if (!(cond)) return set_error(ZOACT_E_INVALID, msg)

zoact_status check_cache(const zoact_cache* c) {
  ZC(c != nullptr, "cache: NULL cache");
  ZC(c->k && c->v && c->k_scale && c->v_scale && c->table && c->len && c->refs, "cache: NULL pointer in the cache");
  ZC(al16(c->k) && al16(c->v) && al16(c->k_scale) && al16(c->v_scale),
     "cache: pools and scales must be 16-byte aligned");
  ZC(al4(c->table) && al4(c->len) && al4(c->refs),
     "cache: table, len and refs must be 4-byte aligned");
  ZC(c->head_dim == 32 || c->head_dim == 64 || c->head_dim == 128, "cache: head_dim must be 32, 64 or 128");
  ZC(c->n_layers >= 1 && c->n_layers <= 32767, "cache: n_layers outside [1, 32767]");
  ZC(c->n_kv_heads >= 1 && c->n_kv_heads <= 32767, "cache: n_kv_heads outside [1, 32767]");
  ZC(c->n_slots >= 1 && c->max_pages >= 1 && c->n_pages >= 1, "cache: empty table or pool");
  ZC(c->n_pages < INT32_MAX - 4096, "cache: too many pages");
  ZC((int64_t)c->max_pages * kPage < INT32_MAX, "cache: max_pages * 64 must be below 2^31");
  return ZOACT_OK;
}

zoact_status check_batch(const zoact_cache_batch* b, const zoact_cache* c) {
  ZC(b != nullptr, "cache batch: NULL batch");
  ZC(b->n >= 1 && b->n <= ZOACT_CACHE_MAX_BATCH, "cache batch: n outside [1, 1024]");
  ZC(b->max_new >= 1 && b->rows >= 0 && b->rows < INT32_MAX, "cache batch: bad max_new or rows");
  ZC(b->pos != nullptr, "cache batch: NULL pos");
  ZC((((uintptr_t)b->pos | (uintptr_t)b->slots | (uintptr_t)b->row_begin | (uintptr_t)b->status) & 3) == 0,
     "cache batch: slots, row_begin, pos and status must be 4-byte aligned");
  ZC(b->slots != nullptr || b->n <= c->n_slots, "cache batch: more entries than slots");
  ZC(b->row_begin != nullptr || (int64_t)b->n * b->max_new <= b->rows, "cache batch: n * max_new exceeds rows");
  return ZOACT_OK;
}

namespace {
zoact_status done(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ZOACT_OK
                         : set_error(ZOACT_E_HIP, (std::string(who) + ": " + hipGetErrorString(e)).c_str());
}

template <typename T, int HD>
void run_append(const zoact_cache& c, int layer, const void* k, int64_t ldk, const void* v, int64_t ldv,
                const zoact_cache_batch& b, const float* ct, const float* st, int64_t n_pos, hipStream_t s) {
  // (an entry that touches more pages than a slot has does not fit, and is left out)
  const int64_t pages = ((int64_t)b.max_new + kPage - 2) / kPage + 1;
  const dim3 grid((unsigned)(pages < c.max_pages ? pages : c.max_pages), (unsigned)(2 * c.n_kv_heads), (unsigned)b.n);
  append_kernel<T, HD><<<grid, 256, 0, s>>>(c, layer, (const T*)k, ldk, (const T*)v, ldv, b, ct, st, n_pos);
}
}  // namespace

}  // namespace zoact

using namespace zoact;

extern "C" size_t zoact_cache_workspace_bytes(const zoact_cache* c) {
  return c && c->n_slots >= 1 && c->max_pages >= 1 && c->n_pages >= 1 ? cache_ws(*c) : 0;
}

static zoact_status check_ws(const zoact_cache& c, const void* ws, size_t bytes, const char* who) {
  if (ws == nullptr || bytes < cache_ws(c))
    return set_error(ZOACT_E_WORKSPACE, (std::string(who) + ": workspace missing or too small").c_str());
  if (!al16(ws)) return set_error(ZOACT_E_INVALID, (std::string(who) + ": ws must be 16-byte aligned").c_str());
  return ZOACT_OK;
}

extern "C" zoact_status zoact_cache_extend(const zoact_cache* c, const zoact_cache_batch* b, void* ws, size_t ws_bytes,
                                           zoact_stream stream) {
  zoact_status st = check_cache(c);
  if (st == ZOACT_OK) st = check_batch(b, c);
  if (st == ZOACT_OK) st = check_ws(*c, ws, ws_bytes, "cache_extend");
  if (st != ZOACT_OK) return st;
  ZC((int64_t)b->n * (b->max_new / kPage + 2) < INT32_MAX, "cache_extend: n * max_new too large");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  int2* const pairs = static_cast<int2*>(ws);
  int* const more = reinterpret_cast<int*>(pairs + ZOACT_CACHE_MAX_BATCH);
  if (b->n <= 256)
    extend_kernel<256><<<1, 256, 0, s>>>(*c, *b, pairs, more);
  else
    extend_kernel<1024><<<1, 1024, 0, s>>>(*c, *b, pairs, more);
  const dim3 grid((unsigned)b->n, (unsigned)(2 * c->n_layers), kCopyParts);
  copy_pairs_kernel<<<grid, 256, 0, s>>>(*c, pairs);
  return done("cache_extend");
}

extern "C" zoact_status zoact_cache_fork(const zoact_cache* c, const int32_t* src, const int32_t* dst, int32_t n,
                                         void* ws, size_t ws_bytes, uint32_t* status, zoact_stream stream) {
  zoact_status st = check_cache(c);
  if (st != ZOACT_OK) return st;
  ZC(src && dst, "cache_fork: NULL slots");
  ZC(al4(src) && al4(dst) && al4(status), "cache_fork: src, dst and status must be 4-byte aligned");
  ZC(n >= 1 && n <= c->n_slots, "cache_fork: n outside [1, n_slots]");
  st = check_ws(*c, ws, ws_bytes, "cache_fork");
  if (st != ZOACT_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (n <= 32 && c->max_pages <= 64) {
    fork_kernel<<<1, 1024, 0, s>>>(*c, src, dst, n, static_cast<int*>(ws), status);
  } else {
    fork_read_kernel<<<(unsigned)n, 256, 0, s>>>(*c, src, dst, n, static_cast<int*>(ws), status);
    fork_write_kernel<<<(unsigned)n, 256, 0, s>>>(*c, dst, n, static_cast<const int*>(ws), status);
  }
  return done("cache_fork");
}

extern "C" zoact_status zoact_cache_free(const zoact_cache* c, const int32_t* slots, int32_t n, uint32_t* status,
                                         zoact_stream stream) {
  const zoact_status st = check_cache(c);
  if (st != ZOACT_OK) return st;
  ZC(slots, "cache_free: NULL slots");
  ZC(al4(slots) && al4(status), "cache_free: slots and status must be 4-byte aligned");
  ZC(n >= 1 && n <= c->n_slots, "cache_free: n outside [1, n_slots]");
  free_kernel<<<(unsigned)n, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(*c, slots, status);
  return done("cache_free");
}

extern "C" zoact_status zoact_cache_compact(const zoact_cache* c, void* ws, size_t ws_bytes, int32_t* n_used,
                                            zoact_stream stream) {
  zoact_status st = check_cache(c);
  if (st == ZOACT_OK) st = check_ws(*c, ws, ws_bytes, "cache_compact");
  if (st != ZOACT_OK) return st;
  ZC(al4(n_used), "cache_compact: n_used must be 4-byte aligned");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  int* const head = static_cast<int*>(ws);
  int* const map = head + 4;
  int* const src = map + c->n_pages;
  int* const dst = src + c->n_pages;
  compact_plan_kernel<<<1, 1024, 0, s>>>(*c, head, map, src, dst, n_used);
  compact_move_kernel<<<2048, 256, 0, s>>>(*c, head, map, src, dst);
  return done("cache_compact");
}

extern "C" zoact_status zoact_cache_append(const zoact_cache* c, int32_t layer, const void* k, int64_t ldk,
                                           const void* v, int64_t ldv, int32_t dtype, const zoact_cache_batch* b,
                                           const float* cos_t, const float* sin_t, int64_t n_pos, zoact_stream stream) {
  zoact_status st = check_cache(c);
  if (st == ZOACT_OK) st = check_batch(b, c);
  if (st != ZOACT_OK) return st;
  ZC(layer >= 0 && layer < c->n_layers, "cache_append: layer outside the cache");
  ZC(dtype == ZOACT_F32 || dtype == ZOACT_BF16, "cache_append: dtype must be F32 or BF16");
  ZC((k && v) || b->rows == 0, "cache_append: NULL pointer");
  const int64_t width = (int64_t)c->n_kv_heads * c->head_dim;
  const int vec = dtype == ZOACT_BF16 ? 8 : 4;
  ZC(ldk >= width && ldv >= width && ldk % vec == 0 && ldv % vec == 0 && al16(k) && al16(v),
     "cache_append: rows must hold the heads and be 16-byte aligned");
  ZC((cos_t == nullptr) == (sin_t == nullptr), "cache_append: both rotary tables or neither");
  ZC(cos_t == nullptr || n_pos >= 1, "cache_append: empty rotary table");
  ZC(al16(cos_t) && al16(sin_t), "cache_append: rotary tables must be 16-byte aligned");
  if (b->rows == 0) return ZOACT_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
#define ZO_APPEND(T, HD) run_append<T, HD>(*c, layer, k, ldk, v, ldv, *b, cos_t, sin_t, n_pos, s)
  if (dtype == ZOACT_BF16) {
    if (c->head_dim == 128) ZO_APPEND(uint16_t, 128);
    else if (c->head_dim == 64) ZO_APPEND(uint16_t, 64);
    else ZO_APPEND(uint16_t, 32);
  } else {
    if (c->head_dim == 128) ZO_APPEND(float, 128);
    else if (c->head_dim == 64) ZO_APPEND(float, 64);
    else ZO_APPEND(float, 32);
  }
#undef ZO_APPEND
  return done("cache_append");
}
