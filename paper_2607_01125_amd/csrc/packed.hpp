// What the kernels of packed sequences and of the beam search share (zoact_packed.h).
#pragma once
#include <string>

#include "common.hpp"
#include "zoact_packed.h"

#define ZP_CHECK(cond, msg)                                 \
  do {                                                      \
    if (!(cond)) return zoact::set_error(ZOACT_E_INVALID, msg); \
  } while (0)

namespace zoact {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline zoact_status launched_or(const char* who) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ZOACT_OK;
  const std::string m = std::string(who) + ": " + hipGetErrorString(e);
  return set_error(ZOACT_E_HIP, m.c_str());
}

inline zoact_status check_packed(const zoact_packed* s) {
  ZP_CHECK(s && s->begin, "packed: NULL pointer");
  ZP_CHECK(aligned_to(s->begin, 4), "packed: begin must be 4-byte aligned");
  ZP_CHECK(s->n >= 1 && s->n <= (1 << 24), "packed: n outside [1, 2^24]");
  // (a tile that begins in the last row still numbers its keys in 32 bits)
  ZP_CHECK(s->rows >= 0 && s->rows <= (int64_t(1) << 31) - 1024, "packed: rows outside [0, 2^31 - 1024]");
  return ZOACT_OK;
}

// Matrix-core form of zoact_attention_packed; hipErrorNotSupported outside its shapes.
hipError_t launch_attention_packed(const zoact_packed& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                   const void* v, int64_t ldv, int32_t heads, int32_t kv_heads, int32_t hd, float scale,
                                   int32_t dtype, void* out, hipStream_t hs);

// Lane 63 of the wave gets op over all lanes (`none` where a lane has no partner), every lane the result.
template <typename Op>
__device__ __forceinline__ int wave_reduce(int x, int none, Op op) {
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x111, 0xf, 0xf, false));   // row_shr:1
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x112, 0xf, 0xf, false));   // row_shr:2
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x114, 0xf, 0xf, false));   // row_shr:4
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x118, 0xf, 0xf, false));   // row_shr:8
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x142, 0xa, 0xf, false));   // row_bcast:15
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x143, 0xc, 0xf, false));   // row_bcast:31
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int wave_sum(int x) {
  return wave_reduce(x, 0, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ float wave_sum(float x) {
  return __int_as_float(wave_reduce(__float_as_int(x), 0, [](int a, int b) {
    return __float_as_int(__int_as_float(a) + __int_as_float(b));
  }));
}
// (NaN stays out)
__device__ __forceinline__ float wave_max(float x) {
  return __int_as_float(wave_reduce(__float_as_int(x), (int)0xFF800000u, [](int a, int b) {
    return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b)));
  }));
}

// The last i with begin[i] <= row, or -1: row's sequence if row < begin[i + 1].
__device__ __forceinline__ int packed_find(const int32_t* __restrict__ begin, int n, int row) {
  int lo = -1, hi = n;                  // begin[lo] <= row < begin[hi + 1], as far as they exist
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (begin[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float ld1(const float* p) { return *p; }
__device__ __forceinline__ float ld1(const uint16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(uint16_t* p, float v) { *p = f2bf(v); }

// Attention of one row and head by one wave: q over the keys 0 .. row, 64 at a time, a key a lane for the scores and
// a column a lane for the means, with the running maximum m and sum l of the softmax; head_dim at most 256, which qs
// (in LDS, the wave's own) holds in fp32.  What is carried is the mean of the values so far, not their weighted sum,
// which large values would take past the range.
template <typename T>
__device__ __forceinline__ void attend_row(const T* q, const T* k, int64_t ldk, const T* v, int64_t ldv, int row, int hd,
                                           float scale, float* qs, T* out) {
  const int lane = threadIdx.x & 63;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");     // (qs was read for another row)
  for (int d = lane; d < hd; d += 64) qs[d] = ld1(q + d);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // (-inf scores, which a formula's softmax gives weight 0, stay below every m)
  float m = -3.4028235e38f, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int key0 = 0; key0 <= row; key0 += 64) {
    const int key = key0 + lane;
    float sc = -INFINITY;
    if (key <= row) {
      const T* kr = k + key * ldk;
      float t = 0.f;
      for (int d = 0; d < hd; ++d) t = fmaf(qs[d], ld1(kr + d), t);
      sc = t * scale;
    }
    const float mn = fmaxf(m, wave_max(sc));
    const float p = key <= row ? expf(sc - mn) : 0.f, was = l * expf(m - mn);
    m = mn;
    l = was + wave_sum(p);
    const float unit = l != 0.f ? 1.f / l : 0.f, share = was * unit, w = p * unit;
    const int cnt = row - key0 + 1 < 64 ? row - key0 + 1 : 64;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= share;
    for (int t = 0; t < cnt; ++t) {
      const float wt = __shfl(w, t, 64);
      const T* vr = v + (key0 + t) * ldv;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e * 64 + lane < hd) o[e] = fmaf(wt, ld1(vr + e * 64 + lane), o[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e * 64 + lane < hd) st1(out + e * 64 + lane, l != 0.f ? o[e] : NAN);
}

// Whether row has a next row in its own sequence.
__device__ __forceinline__ bool packed_has_next(const int32_t* __restrict__ begin, int n, int64_t rows, int row) {
  const int i = packed_find(begin, n, row);
  if (i < 0 || i >= n) return false;
  const int64_t end = begin[i + 1];
  return row + 1 < (end < rows ? end : rows);
}

}  // namespace zoact
