// Selection of a beam search's candidates over beams and vocabulary (zoact_packed.h).
//
// Two launches: beam_rows reads the logits once, 4096 of a row a workgroup, and leaves of each such
// part the maximum, the sum of exponentials relative to it and its `beams` largest logits in order
// (within one beam the order of the values is that of the logits); beam_pick joins a prompt's sums
// to log sums, ranks the parts' candidates by value and copies the kept candidates' histories.
// Where a prompt has one part only, beam_pick's workgroup reads it itself, in one launch (one row of
// 512 logits 7.6 -> 6.7 us; with four rows of 4096 that would be 9.6 -> 10.3).
//
// Bound by the logits' bytes for many rows (128 of 128256: 19 us of beam_rows, 3.5 TB/s, loads 12 of them, then a wave's
// threshold by ballots and its short list), by chains of trips to memory and LDS for few (48 rows of 50272, 16 kept:
// 9 + 7).
#include <math.h>

#include "packed.hpp"

namespace zoact {
namespace {

constexpr int PART = 4096;               // logits of a workgroup
constexpr int NT = 256, PER = PART / NT;
constexpr int NP = 1024;                 // threads of a prompt's workgroup
constexpr int KMAX = ZOACT_BEAMS_MAX;
constexpr int WCAP = 512;                // candidates a wave gathers before it takes the slow way
constexpr int FEW_GROUPS = 48;           // beams of which 64 groups' maxima give a threshold

// Order of fp32 (fp64) values as that of unsigned numbers above 0.
__device__ __forceinline__ uint32_t order32(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);          // (-0 counts as 0)
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t order64(double x) {
  if (x != x) return ~0ull;
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return (b >> 63) ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ float from_order32(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

struct Cand {
  float x;
  int32_t v;             // token, -1: none
};

// Workspace: [rows][splits] (maximum, sum), then [rows][splits][beams] candidates.
struct Layout {
  int64_t rows;
  int splits;
  size_t cand_at, bytes;
};
Layout layout_of(int32_t n, int32_t beams_in, int32_t beams, int64_t vocab) {
  Layout l;
  l.rows = (int64_t)n * beams_in;
  l.splits = (int)((vocab + PART - 1) / PART);
  const size_t parts = (size_t)l.rows * (size_t)l.splits;
  l.cand_at = (parts * sizeof(float2) + 255) & ~(size_t)255;
  l.bytes = l.cand_at + parts * (size_t)beams * sizeof(Cand);
  return l;
}

__device__ __forceinline__ void ld4(const float* p, float (&x)[4]) {
  const float4 u = *reinterpret_cast<const float4*>(p);
  x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
}
__device__ __forceinline__ void ld4(const uint16_t* p, float (&x)[4]) {
  const ushort4 u = *reinterpret_cast<const ushort4*>(p);
  x[0] = bf2f(u.x), x[1] = bf2f(u.y), x[2] = bf2f(u.z), x[3] = bf2f(u.w);
}

// Key of a candidate within a row: larger values first, then lower tokens; 0: none.
__device__ __forceinline__ uint64_t row_key(uint32_t ord, int v) { return ((uint64_t)ord << 32) | (0xFFFFFFFFu - (uint32_t)v); }

struct PartLds {
  uint64_t list[4][WCAP];
  uint64_t best[4][KMAX];
  float2 sum[4];
};

__device__ __forceinline__ bool has_ended(const zoact_beams& b, int64_t row) {
  return b.eos >= 0 && b.length > 0 && b.hist[row * b.ld_hist + b.length - 1] == b.eos;
}

// What each of a part's four waves finds in its 1024 logits, by 256 threads (tid).  VEC: rows start on 16 bytes
// (fp32; 8 in bf16) and hold a multiple of four values.
template <typename T, bool VEC>
__device__ __forceinline__ void part_of_row(const T* lr, int V, int part, int K, int tid, PartLds& lds) {
  auto& list = lds.list;
  auto& best = lds.best;
  const int wave = tid >> 6, lane = tid & 63;
  const int v0 = part * PART + tid * 4;  // this thread: v0 + 1024 j + e
  const bool whole = (part + 1) * (int64_t)PART <= V;
  float x[PER], mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    const int64_t v = (int64_t)v0 + j * (NT * 4);
    if (VEC) {
      if (v < V) ld4(lr + v, t);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v + e < V) t[e] = ld1(lr + v + e);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[j * 4 + e] = t[e];
      mx = fmaxf(mx, t[e]);
    }
  }
  // maximum and sum of the wave's 1024 (a NaN stays out of the maximum and goes into the sum)
  const float wm = wave_max(mx);
  const float base = wm == -INFINITY ? 0.f : wm;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += __expf(x[i] - base);
  sum = wave_sum(sum);
  if (lane == 0) lds.sum[wave] = make_float2(wm, sum);
  if (!whole) {                          // what is behind the row is no candidate: NaN is above no threshold
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if ((int64_t)v0 + (i >> 2) * (NT * 4) + (i & 3) >= V) x[i] = NAN;
  }

  // The K-th largest of the lanes' maxima, or a little less (its upper 20 bits): at least K of the wave's
  // values reach it, and few others.
  uint32_t to = 0;
  const uint32_t ord = order32(mx);
#pragma unroll
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t t = to | (1u << bit);
    if (__popcll(__ballot(ord >= t)) >= K) to = t;
  }
  const float thr = from_order32(to > order32(-INFINITY) ? to : order32(-INFINITY));
  // gather what lies above it, and of what equals it (-inf in a masked vocabulary) the K lowest tokens
  int cnt = 0, eq = 0;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float m4 = fmaxf(fmaxf(x[j * 4], x[j * 4 + 1]), fmaxf(x[j * 4 + 2], x[j * 4 + 3]));
    if (__ballot(m4 >= thr) == 0) continue;
    uint64_t at[4];
    int lower = 0, all = 0;               // equal ones of lower lanes, of all lanes
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      at[e] = __ballot(x[j * 4 + e] == thr);
      lower += __popcll(at[e] & below);
      all += __popcll(at[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = x[j * 4 + e];
      const bool take = y > thr || (y == thr && eq + lower < K);
      if (y == thr) ++lower;
      const uint64_t m = __ballot(take);
      const int p = cnt + __popcll(m & below);
      if (take && p < WCAP) list[wave][p] = row_key(order32(y), v0 + j * (NT * 4) + e);
      cnt += __popcll(m);
    }
    eq += all;
  }
  // the wave's K largest, in order (best[][i] = 0: fewer)
  if (lane < K) best[wave][lane] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (cnt <= WCAP) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (every lane's entries)
    if (cnt > 128) {
      // only what reaches the K-th largest is ranked (64 of 16000 logits: 57 -> 23 us)
      uint32_t have[WCAP / 64], kth = 0;
#pragma unroll
      for (int u = 0; u < WCAP / 64; ++u) have[u] = u * 64 + lane < cnt ? (uint32_t)(list[wave][u * 64 + lane] >> 32) : 0;
#pragma unroll 1
      for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
        int reach = 0;
#pragma unroll
        for (int u = 0; u < WCAP / 64; ++u) reach += __popcll(__ballot(have[u] >= (kth | bit)));
        if (reach >= K) kth |= bit;
      }
      int kept = 0;
#pragma unroll
      for (int u = 0; u < WCAP / 64; ++u) {                  // (an entry moves down, over ones that were read)
        const uint64_t mine = list[wave][u * 64 + lane];
        const bool take = have[u] >= kth;
        const uint64_t m = __ballot(take);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (take) list[wave][kept + __popcll(m & below)] = mine;
        kept += __popcll(m);
      }
      cnt = kept;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    for (int i = lane; i < cnt; i += 64) {
      const uint64_t mine = list[wave][i];
      int rank = 0;
      for (int t = 0; t < cnt; ++t) rank += list[wave][t] > mine;
      if (rank < K) best[wave][rank] = mine;
    }
  } else {
    uint64_t last = ~0ull;
    for (int r = 0; r < K; ++r) {
      uint64_t mine = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint64_t c = x[i] == x[i] ? row_key(order32(x[i]), v0 + (i >> 2) * (NT * 4) + (i & 3)) : 0;
        if (c < last && c > mine) mine = c;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const uint64_t c = __shfl_xor((unsigned long long)mine, o, 64);
        mine = c > mine ? c : mine;
      }
      if (lane == 0) best[wave][r] = mine;
      last = mine;
      if (mine == 0) break;
    }
  }
}

// The part's sum and its largest logits (each wave's list is in order).
__device__ __forceinline__ void join_part(const PartLds& lds, int K, int tid, float2* sum, Cand* out) {
  const auto& best = lds.best;
  for (int i = tid; i < 4 * K; i += NT) {
    const int w = i / K;
    const uint64_t mine = best[w][i - w * K];
    int rank = 0, any = 0;
    for (int u = 0; u < 4; ++u)
      for (int t = 0; t < K; ++t) {
        const uint64_t c = best[u][t];
        rank += c > mine;
        any += c != 0;
      }
    if (mine && rank < K) out[rank] = Cand{from_order32((uint32_t)(mine >> 32)), (int)(0xFFFFFFFFu - (uint32_t)mine)};
    if (i < K && i >= any) out[i] = Cand{0.f, -1};
  }
  if (tid == 0) {
    float M = lds.sum[0].x;
    for (int u = 1; u < 4; ++u) M = fmaxf(M, lds.sum[u].x);
    const float mb = M == -INFINITY ? 0.f : M;
    float S = 0.f;
    for (int u = 0; u < 4; ++u) S += lds.sum[u].y * (lds.sum[u].x == -INFINITY ? 1.f : expf(lds.sum[u].x - mb));
    *sum = make_float2(M, S);            // (a NaN among the values is in S)
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(NT) beam_rows(const T* __restrict__ logits, int64_t ldl, zoact_beams b, int splits,
                                                float2* __restrict__ sums, Cand* __restrict__ cand) {
  __shared__ PartLds lds;
  const int row = blockIdx.y, part = blockIdx.x;
  if (has_ended(b, row)) return;
  part_of_row<T, VEC>(logits + (int64_t)row * ldl, (int)b.vocab, part, b.beams, threadIdx.x, lds);
  __syncthreads();
  const int64_t at = (int64_t)row * splits + part;
  join_part(lds, b.beams, threadIdx.x, sums + at, cand + at * b.beams);
}

enum { BEAM_PLAIN, BEAM_ENDED, BEAM_NAN, BEAM_LOST };   // LOST: every value is -inf

// One workgroup a prompt.  Candidates are compared as (key, place, logit): the value's order, then the lower beam, then
// the larger logit (which 64 bits may not resolve beside the log sum: the parts' lists are in its order), then the lower
// token.  OWN: the prompt's part, its only one, is not there yet.
template <typename T, bool VEC, bool OWN>
__global__ void __launch_bounds__(NP) beam_pick(const T* __restrict__ logits, int64_t ldl, zoact_beams b, int splits,
                                                float2* sums, Cand* cand) {
  constexpr int CAP = 1024, WAVES = NP / 64;
  __shared__ double lse[KMAX], sc[KMAX];
  __shared__ float top[KMAX];
  __shared__ int kind[KMAX];
  __shared__ uint64_t key[CAP], place[CAP];
  __shared__ uint32_t logit[CAP];
  __shared__ uint64_t wkey[WAVES], wplace[WAVES];
  __shared__ uint32_t wlogit[WAVES];
  __shared__ uint32_t tops[WAVES][64];
  __shared__ int n_got;
  __shared__ int parent[KMAX];
  const int i0 = blockIdx.x, BI = b.beams_in, K = b.beams;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (OWN) {
    __shared__ PartLds lds;
    const bool live = threadIdx.x < NT && !has_ended(b, i0);
    if (live) part_of_row<T, VEC>(logits + i0 * ldl, (int)b.vocab, 0, K, threadIdx.x, lds);
    __syncthreads();
    if (live) join_part(lds, K, threadIdx.x, sums + i0, cand + (int64_t)i0 * K);
    __syncthreads();
  }
  if (threadIdx.x == 0) n_got = 0;
  // (asked for before the sums are joined)
  const bool mine_j = (int)threadIdx.x < BI;
  const int64_t row_j = (int64_t)i0 * BI + (mine_j ? threadIdx.x : 0);
  const float score_j = b.score[row_j];
  const bool ended_j = has_ended(b, row_j);
  const uint32_t per = (uint32_t)splits * (uint32_t)K, total = (uint32_t)BI * per;      // (at most 2^30)
  constexpr int KEEP = 4;                // candidates that a thread keeps from the first look to the second
  // A thread's q-th candidate: each time 7 further round, so that a thread meets all ranks of the parts' lists (1031 is
  // prime), not the first of each list or the last.
  auto nth = [](int q) { return (uint32_t)q * NP + ((threadIdx.x + 7 * q) & (NP - 1)); };
  const int rounds = (int)((total + NP - 1) / NP);
  Cand raw[KEEP];
#pragma unroll
  for (int q = 0; q < KEEP; ++q) {
    const uint32_t c = nth(q);
    raw[q] = c < total ? cand[(int64_t)i0 * total + c] : Cand{0.f, -1};
  }
  for (int j = wave; j < BI; j += WAVES) {
    const float2* const p = sums + ((int64_t)i0 * BI + j) * splits;
    const float2 first = lane < splits ? p[lane] : make_float2(-INFINITY, 0.f);
    float M = first.x;
    for (int t = lane + 64; t < splits; t += 64) M = fmaxf(M, p[t].x);
    M = wave_max(M);
    // (a part of nothing but -inf has the sum 0, or NaN)
    auto part = [&](float2 y) { return y.x == -INFINITY ? y.y : y.y * expf(y.x - M); };
    float S = part(first);
    for (int t = lane + 64; t < splits; t += 64) S += part(p[t]);
    S = wave_sum(S);
    if (lane == 0) lse[j] = (double)S, top[j] = M;
  }
  __syncthreads();
  if (mine_j) {
    const int j = threadIdx.x;
    const double s = (double)score_j, l = (double)top[j] + log(lse[j]);
    int kd = BEAM_PLAIN;
    if (s != s || s == INFINITY) kd = BEAM_NAN;
    else if (ended_j) kd = s == -INFINITY ? BEAM_LOST : BEAM_ENDED;      // (nothing was left of its row)
    else if (!(l - l == 0.0)) kd = BEAM_NAN;
    else if (s == -INFINITY) kd = BEAM_LOST;
    lse[j] = l, sc[j] = s, kind[j] = kd;
  }
  __syncthreads();
  // Candidate c of the prompt: beam j's part and place, or for beams whose values do not follow the
  // logits the lowest tokens (an ended one's eos first).
  auto place_at = [](uint32_t j, int v) { return ~(((uint64_t)j << 32) | (uint32_t)v); };
  auto rate = [&](uint32_t c, Cand d, uint64_t& k, uint64_t& f, uint32_t& x) {
    const uint32_t j = c / per, t = c - j * per;
    k = f = x = 0;
    if (kind[j] == BEAM_PLAIN) {
      if (d.v < 0) return;
      x = order32(d.x);
      k = order64(sc[j] + ((double)d.x - lse[j]));
      f = place_at(j, d.v);
    } else if (t < (uint32_t)K) {
      int v = (int)t;
      double val = kind[j] == BEAM_NAN ? (double)NAN : -INFINITY;
      if (kind[j] == BEAM_ENDED) {
        if (t == 0) v = b.eos, val = sc[j];
        else v = (int)t - 1 < b.eos ? (int)t - 1 : (int)t;
      }
      k = order64(val);
      f = place_at(j, v);
    }
  };
  auto read = [&](uint32_t c, uint64_t& k, uint64_t& f, uint32_t& x) { rate(c, cand[(int64_t)i0 * total + c], k, f, x); };
  // (of equal keys)
  auto before = [](uint64_t f, uint32_t x, uint64_t f2, uint32_t x2) {
    return f >> 32 == f2 >> 32 && x != x2 ? x > x2 : f > f2;
  };
  auto better = [&](uint64_t k, uint64_t f, uint32_t x, uint64_t k2, uint64_t f2, uint32_t x2) {
    return k > k2 || (k == k2 && before(f, x, f2, x2));
  };
  auto emit = [&](int m, uint64_t k, uint64_t f) {
    const int j = (int)(~f >> 32), v = (int)(uint32_t)~f;
    const int64_t o = (int64_t)i0 * K + m;
    b.score_out[o] = k == ~0ull ? NAN : (float)__longlong_as_double((long long)((k >> 63) ? k & ~(1ull << 63) : ~k));
    if (b.token) b.token[o] = v;
    if (b.src) b.src[o] = i0 * K + j;
    b.hist_out[o * b.ld_hist_out + b.length] = v;
    parent[m] = j;
  };
  const bool few = total <= 128;         // all of them are ranked then
  uint64_t kk[KEEP], kf[KEEP], mine = 0;
  uint32_t kx[KEEP];
#pragma unroll
  for (int q = 0; q < KEEP; ++q) {
    kk[q] = kf[q] = kx[q] = 0;
    const uint32_t c = nth(q);
    if (c < total) rate(c, raw[q], kk[q], kf[q], kx[q]);
    mine = kk[q] > mine ? kk[q] : mine;
  }
#pragma unroll 8
  for (int q = KEEP; q < rounds; ++q) {
    const uint32_t c = nth(q);
    uint64_t k = 0, f;
    uint32_t x;
    if (c < total) read(c, k, f, x);
    mine = k > mine ? k : mine;
  }
  // The threshold is reached by K candidates at least, and few others: of the maxima of 64 groups (a lane's in all
  // waves) the K-th largest (24 bits of it: scores of -1500 still differ by a quarter), or with many beams of those of
  // all threads, since K of 64 groups are nearly all then and more than CAP candidates, where there are as many, may
  // reach the least of them.  (32 of 32 x 16000 logits: groups 18 to 20 us, threads 25 to 27; 48 of 48 x 128256: 112,
  // 120; 64 of 64 x 16000: 54 to 99, 48; 64 of 64 x 128256: 227 to 4485, 225.)
  uint64_t thr = 1;
  if (!few) {
    tops[wave][lane] = (uint32_t)(mine >> 32);
    __syncthreads();
    uint32_t to = 0, part[WAVES];
#pragma unroll
    for (int u = 0; u < WAVES; ++u) part[u] = tops[u][lane];
    if (K <= FEW_GROUPS || total <= CAP) {
      uint32_t upper = 0;
#pragma unroll
      for (int u = 0; u < WAVES; ++u) upper = part[u] > upper ? part[u] : upper;
#pragma unroll
      for (int bit = 31; bit >= 8; --bit) {
        const uint32_t x = to | (1u << bit);
        if (__popcll(__ballot(upper >= x)) >= K) to = x;
      }
    } else {
#pragma unroll 1
      for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
        int reach = 0;
#pragma unroll
        for (int u = 0; u < WAVES; ++u) reach += __popcll(__ballot(part[u] >= (to | bit)));
        if (reach >= K) to |= bit;
        if (reach == K) break;
      }
    }
    thr = to ? (uint64_t)to << 32 : 1;
  }
  auto gather = [&](uint64_t k, uint64_t f, uint32_t x) {
    if (k < thr) return;
    const int p = atomicAdd(&n_got, 1);  // (the order of arrival changes nothing: ranks decide)
    if (p < CAP) key[p] = k, place[p] = f, logit[p] = x;
  };
#pragma unroll
  for (int q = 0; q < KEEP; ++q) gather(kk[q], kf[q], kx[q]);
#pragma unroll 8
  for (int q = KEEP; q < rounds; ++q) {
    const uint32_t c = nth(q);
    uint64_t k = 0, f = 0;
    uint32_t x = 0;
    if (c < total) read(c, k, f, x);
    gather(k, f, x);
  }
  __syncthreads();
  const int got = n_got;
  if (got <= CAP) {
    // (a candidate's rank is counted by as many neighbouring threads as there are for each, up to 16)
    int each = 16;
    while (each * got > NP) each >>= 1;
    const int c = threadIdx.x / each;
    int rank = 0;
    uint64_t k = 0, f = 0;
    if (c < got) {
      k = key[c], f = place[c];
      for (int t = threadIdx.x & (each - 1); t < got; t += each) {
        const uint64_t other = key[t];
        rank += other > k;
        if (other == k && t != c) rank += before(place[t], logit[t], f, logit[c]);
      }
    }
    for (int o = each >> 1; o > 0; o >>= 1) rank += __shfl_xor(rank, o, 64);
    if (c < got && rank < K && (threadIdx.x & (each - 1)) == 0) emit(rank, k, f);
  } else {
    // very many equal ones: one at a time, each behind the one before (a NaN of the first beam and token has the
    // highest key and place that there are: nothing is behind what the first would start from)
    uint64_t lk = 0, lf = 0;
    uint32_t lx = 0;
    for (int m = 0; m < K; ++m) {
      uint64_t bk = 0, bf = 0;
      uint32_t bx = 0;
      for (uint32_t c = threadIdx.x; c < total; c += NP) {
        uint64_t k, f;
        uint32_t x;
        read(c, k, f, x);
        if (k && (m == 0 || better(lk, lf, lx, k, f, x)) && better(k, f, x, bk, bf, bx)) bk = k, bf = f, bx = x;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const uint64_t k = __shfl_xor((unsigned long long)bk, o, 64), f = __shfl_xor((unsigned long long)bf, o, 64);
        const uint32_t x = __shfl_xor(bx, o, 64);
        if (better(k, f, x, bk, bf, bx)) bk = k, bf = f, bx = x;
      }
      if (lane == 0) wkey[wave] = bk, wplace[wave] = bf, wlogit[wave] = bx;
      __syncthreads();
      for (int u = 0; u < WAVES; ++u)
        if (better(wkey[u], wplace[u], wlogit[u], bk, bf, bx)) bk = wkey[u], bf = wplace[u], bx = wlogit[u];
      if (threadIdx.x == 0) emit(m, bk, bf);
      lk = bk, lf = bf, lx = bx;
      __syncthreads();
    }
  }
  __syncthreads();
  const uint32_t len = (uint32_t)b.length;
  for (uint64_t c = threadIdx.x; c < (uint64_t)K * len; c += NP) {
    const uint32_t m = (uint64_t)K * len >> 32 ? (uint32_t)(c / len) : (uint32_t)c / len, t = (uint32_t)(c - (uint64_t)m * len);
    b.hist_out[((int64_t)i0 * K + m) * b.ld_hist_out + t] = b.hist[((int64_t)i0 * BI + parent[m]) * b.ld_hist + t];
  }
}

}  // namespace
}  // namespace zoact

using namespace zoact;

extern "C" size_t zoact_beam_workspace_bytes(int32_t n, int32_t beams_in, int32_t beams, int64_t vocab) {
  if (n < 1 || beams_in < 1 || beams_in > ZOACT_BEAMS_MAX || beams < 1 || beams > ZOACT_BEAMS_MAX || vocab < 1 ||
      vocab > (int64_t(1) << 30) || (int64_t)n * beams_in > 65535)
    return 0;
  return layout_of(n, beams_in, beams, vocab).bytes;
}

extern "C" zoact_status zoact_beam_select(const zoact_beams* b, const void* logits, int64_t ldl, int32_t dtype, void* ws,
                                          size_t ws_bytes, zoact_stream stream) {
  ZP_CHECK(b && logits && b->score && b->score_out && b->hist_out, "beam_select: NULL pointer");
  ZP_CHECK(dtype == ZOACT_F32 || dtype == ZOACT_BF16, "beam_select: dtype must be F32 or BF16");
  ZP_CHECK(b->n >= 1 && b->beams_in >= 1 && b->beams_in <= ZOACT_BEAMS_MAX && b->beams >= 1 &&
               b->beams <= ZOACT_BEAMS_MAX && (int64_t)b->n * b->beams_in <= 65535,
           "beam_select: n, beams_in or beams out of range");
  ZP_CHECK((int64_t)b->n * b->beams < (int64_t(1) << 31), "beam_select: n * beams past 32 bits");
  ZP_CHECK(b->vocab >= b->beams && b->vocab <= (int64_t(1) << 30), "beam_select: vocab outside [beams, 2^30]");
  ZP_CHECK(ldl >= b->vocab, "beam_select: rows of logits overlap");
  ZP_CHECK(b->eos >= -1 && b->eos < b->vocab, "beam_select: eos outside [-1, vocab)");
  ZP_CHECK(b->length >= 0 && (b->length == 0 || (b->hist && b->length <= b->ld_hist)) && b->length < b->ld_hist_out &&
               b->length < (int64_t(1) << 31),
           "beam_select: histories do not hold the tokens");
  ZP_CHECK(aligned_to(logits, dtype == ZOACT_F32 ? 4 : 2) && aligned_to(b->score, 4) && aligned_to(b->score_out, 4) &&
               aligned_to(b->hist, 4) && aligned_to(b->hist_out, 4) && aligned_to(b->token, 4) && aligned_to(b->src, 4),
           "beam_select: pointers must be aligned to their types");
  ZP_CHECK(b->score_out != b->score && b->hist_out != b->hist, "beam_select: candidates selected into themselves");
  const Layout l = layout_of(b->n, b->beams_in, b->beams, b->vocab);
  if (ws == nullptr || ws_bytes < l.bytes) return set_error(ZOACT_E_WORKSPACE, "beam_select: workspace too small");
  ZP_CHECK(aligned_to(ws, 16), "beam_select: ws must be 16-byte aligned");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  float2* const sums = static_cast<float2*>(ws);
  Cand* const cand = reinterpret_cast<Cand*>(static_cast<char*>(ws) + l.cand_at);
  const dim3 grid((unsigned)l.splits, (unsigned)l.rows);
  const bool vec = b->vocab % 4 == 0 && ldl % 4 == 0 && aligned_to(logits, dtype == ZOACT_F32 ? 16 : 8);
  const bool own = b->beams_in == 1 && l.splits == 1;
#define ZO_ROWS(T, VEC)                                                                               \
  do {                                                                                                \
    if (own) {                                                                                        \
      beam_pick<T, VEC, true><<<(unsigned)b->n, NP, 0, s>>>((const T*)logits, ldl, *b, l.splits, sums, cand); \
      break;                                                                                          \
    }                                                                                                 \
    beam_rows<T, VEC><<<grid, NT, 0, s>>>((const T*)logits, ldl, *b, l.splits, sums, cand);           \
    beam_pick<float, true, false><<<(unsigned)b->n, NP, 0, s>>>(nullptr, 0, *b, l.splits, sums, cand); \
  } while (0)
  if (dtype == ZOACT_F32) {
    if (vec) ZO_ROWS(float, true);
    else ZO_ROWS(float, false);
  } else {
    if (vec) ZO_ROWS(uint16_t, true);
    else ZO_ROWS(uint16_t, false);
  }
#undef ZO_ROWS
  return launched_or("beam_select");
}
