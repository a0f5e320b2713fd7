// Rotary positions and causal attention over packed sequences (zoact_packed.h).
#include <math.h>

#include "packed.hpp"

namespace zoact {
namespace {

// ---------------------------------------------------------------- rotary positions
// One thread a pair or a copied value: any head_dim, rot_dim, stride and alignment (16411 rows of 40 heads of 128 bf16
// values, 64 of them turned: 215 us where pieces of 16 bytes take 61 to 65).
template <typename T>
__global__ void __launch_bounds__(256) rope_at_kernel(const T* x, int64_t ldx, T* out, int64_t ldo, int64_t rows,
                                                      int heads, int hd, int rot, int layout,
                                                      const int32_t* __restrict__ pos, const float* __restrict__ cos_t,
                                                      const float* __restrict__ sin_t, int64_t n_pos) {
  const int half = rot / 2, per = half + (hd - rot);        // units of a head: pairs, then single values
  const int64_t total = rows * heads * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / ((int64_t)heads * per);
    const int u = (int)(i - row * heads * per), h = u / per, j = u - h * per;
    const T* xr = x + row * ldx + (int64_t)h * hd;
    T* yr = out + row * ldo + (int64_t)h * hd;
    if (j >= half) {
      if (out != x) yr[rot + j - half] = xr[rot + j - half];
      continue;
    }
    int64_t p = pos ? pos[row] : row;
    p = p < 0 ? 0 : (p >= n_pos ? n_pos - 1 : p);
    const float c = cos_t[p * half + j], s = sin_t[p * half + j];
    const int ja = layout == ZOACT_ROPE_HALF ? j : 2 * j, jb = layout == ZOACT_ROPE_HALF ? j + half : 2 * j + 1;
    const float a = ld1(xr + ja), b = ld1(xr + jb);
    st1(yr + ja, a * c - b * s);
    st1(yr + jb, b * c + a * s);
  }
}

// Pieces of 16 bytes: a thread takes one place of a row -- a pair of pieces half the turned part apart (HALF), a
// piece of whole pairs (INTERLEAVED), or a piece to copy -- in RT rows, all of whose loads are on their way before
// the first is used.  Bound by memory: 16411 rows of 40 heads of 128 bf16 values, 64 of them turned in pairs, 65 us,
// 5.2 TB/s; torch's copy of the same 337 MB takes 66.
template <typename T, bool HALF, int RT>
__global__ void __launch_bounds__(1024) rope_at_vec_kernel(const T* x, int64_t ldx, T* out, int64_t ldo, int64_t rows,
                                                           int heads, int hd, int rot, const int32_t* __restrict__ pos,
                                                           const float* __restrict__ cos_t,
                                                           const float* __restrict__ sin_t, int64_t n_pos) {
  constexpr int V = 16 / sizeof(T), NT = HALF ? V : V / 2;   // values of a piece, angles of it
  typedef T piece __attribute__((ext_vector_type(V)));
  typedef float angles __attribute__((ext_vector_type(NT)));
  const int turned = HALF ? rot / (2 * V) : rot / V, copied = out == x ? 0 : (hd - rot) / V, n_turned = heads * turned;
  const int units = n_turned + heads * copied, half = rot / 2;
  const int64_t row0 = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * RT;
  for (int u = threadIdx.x; u < units; u += blockDim.x) {
    // (all heads' turned pieces first, so that lanes do the same)
    const bool turn = u < n_turned;
    const int w = turn ? u : u - n_turned, per = turn ? turned : copied, h = w / per, j = w - h * per;
    const int64_t col = (int64_t)h * hd + (turn ? j * V : rot + j * V);
    piece a[RT], b[RT];
    angles c[RT], s[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int64_t row = row0 + r < rows ? row0 + r : rows - 1;
      a[r] = *reinterpret_cast<const piece*>(x + row * ldx + col);
      if (turn) {
        int64_t p = pos ? pos[row] : row;
        p = p < 0 ? 0 : (p >= n_pos ? n_pos - 1 : p);
        if (HALF) b[r] = *reinterpret_cast<const piece*>(x + row * ldx + col + half);
        c[r] = *reinterpret_cast<const angles*>(cos_t + p * half + j * NT);
        s[r] = *reinterpret_cast<const angles*>(sin_t + p * half + j * NT);
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if (row0 + r >= rows) break;
      T* const y = out + (row0 + r) * ldo + col;
      if (turn) {
        piece m, n;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          T ea = a[r][HALF ? i : 2 * i], eb = HALF ? b[r][i] : a[r][2 * i + 1];
          const float fa = ld1(&ea), fb = ld1(&eb);
          T ma, mb;
          st1(&ma, fa * c[r][i] - fb * s[r][i]);
          st1(&mb, fb * c[r][i] + fa * s[r][i]);
          if (HALF) m[i] = ma, n[i] = mb;
          else m[2 * i] = ma, m[2 * i + 1] = mb;
        }
        *reinterpret_cast<piece*>(y) = m;
        if (HALF) *reinterpret_cast<piece*>(y + half) = n;
      } else {
        *reinterpret_cast<piece*>(y) = a[r];
      }
    }
  }
}

// Where less than half a head is turned, and not in whole pieces: a thread forms a piece of out, value by value where
// it is turned, so that rows are still written in whole lines; in place, where a pair belongs to one thread, it turns a
// head's pairs (16411 rows of 40 heads of 128, 10 of them turned: 128 us, 250 value by
// value throughout).
template <typename T>
__global__ void __launch_bounds__(512) rope_at_part_kernel(const T* x, int64_t ldx, T* out, int64_t ldo, int64_t rows,
                                                           int heads, int hd, int rot, int layout,
                                                           const int32_t* __restrict__ pos,
                                                           const float* __restrict__ cos_t,
                                                           const float* __restrict__ sin_t, int64_t n_pos) {
  constexpr int V = 16 / sizeof(T);
  typedef T piece __attribute__((ext_vector_type(V)));
  const int half = rot / 2, sa = layout == ZOACT_ROPE_HALF ? 1 : 2, sb = layout == ZOACT_ROPE_HALF ? half : 1;
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= rows) return;
  int64_t p = pos ? pos[row] : row;
  p = p < 0 ? 0 : (p >= n_pos ? n_pos - 1 : p);
  if (out == x) {
    for (int h = threadIdx.x; h < heads; h += blockDim.x) {
      T* const y = out + row * ldo + (int64_t)h * hd;
#pragma unroll 4
      for (int i = 0; i < half; ++i) {
        const float c = cos_t[p * half + i], s = sin_t[p * half + i];
        const float a = ld1(y + i * sa), b = ld1(y + i * sa + sb);
        st1(y + i * sa, a * c - b * s);
        st1(y + i * sa + sb, b * c + a * s);
      }
    }
    return;
  }
  const int per = hd / V;
  for (int u = threadIdx.x; u < heads * per; u += blockDim.x) {
    const int h = u / per, first = (u - h * per) * V;
    const T* const xr = x + row * ldx + (int64_t)h * hd;
    piece y = *reinterpret_cast<const piece*>(xr + first);
    if (first < rot) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int at = first + e;
        if (at >= rot) break;
        const int i = layout == ZOACT_ROPE_HALF ? (at < half ? at : at - half) : at >> 1;
        const float c = cos_t[p * half + i], s = sin_t[p * half + i];
        const float a = ld1(xr + i * sa), b = ld1(xr + i * sa + sb);
        T r;
        st1(&r, at == i * sa ? a * c - b * s : b * c + a * s);
        y[e] = r;
      }
    }
    *reinterpret_cast<piece*>(out + row * ldo + (int64_t)h * hd + first) = y;
  }
}

template <typename T>
bool rope_at_vec(const T* x, int64_t ldx, T* out, int64_t ldo, int64_t rows, int heads, int hd, int rot, int layout,
                 const int32_t* pos, const float* cos_t, const float* sin_t, int64_t n_pos, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool halves = layout == ZOACT_ROPE_HALF;
  if (hd % V || ldx % V || ldo % V || !aligned_to(x, 16) || !aligned_to(out, 16)) return false;
  const bool whole = rot % (halves ? 2 * V : V) == 0 && aligned_to(cos_t, 16) && aligned_to(sin_t, 16);
  if (!whole && rot > hd / 2) return false;
  const int64_t units = whole ? (int64_t)heads * (rot / (halves ? 2 * V : V) + (out == x ? 0 : (hd - rot) / V))
                              : (int64_t)heads * (out == x ? 1 : hd / V);
  const int bx = (int)(units < 512 ? units : 512), by = bx < 256 ? 256 / bx : 1;
  // (two rows a thread in pairs once there are workgroups enough: 65 us at the size above, 69 with one, 80 with four;
  // halves keep twice the loads on their way with one: 62 us where all 128 values are turned, 71 with two)
  const bool many = !halves && whole && rows * units >= (int64_t)512 * 1024 * 4;
  const int64_t step = (int64_t)by * (many ? 2 : 1), grid = (rows + step - 1) / step;
  if (grid * bx * by >= (int64_t(1) << 32)) return false;    // (more threads than a launch has)
  if (!whole) {
    rope_at_part_kernel<T><<<(unsigned)grid, dim3(bx, by), 0, s>>>(x, ldx, out, ldo, rows, heads, hd, rot, layout, pos,
                                                                   cos_t, sin_t, n_pos);
    return true;
  }
#define ZO_ROPE(HALF, RT)                                                                                             \
  rope_at_vec_kernel<T, HALF, RT><<<(unsigned)grid, dim3(bx, by), 0, s>>>(x, ldx, out, ldo, rows, heads, hd, rot, pos, \
                                                                          cos_t, sin_t, n_pos)
  if (halves) ZO_ROPE(true, 1);
  else if (many) ZO_ROPE(false, 2);
  else ZO_ROPE(false, 1);
#undef ZO_ROPE
  return true;
}

// ---------------------------------------------------------------- attention, any shape
// One wave a (row, head): what the tiles' kernels do not take.  Bound by latency and by K and V read again for every
// row: 2018 tokens in 8 sequences, 8 heads of 80, 986 us (16 in tiles).
template <typename T>
__global__ void __launch_bounds__(256) attention_packed_any(zoact_packed s, const T* __restrict__ q, int64_t ldq,
                                                            const T* __restrict__ k, int64_t ldk,
                                                            const T* __restrict__ v, int64_t ldv, int heads,
                                                            int kv_heads, int hd, float scale, T* __restrict__ out) {
  __shared__ float qs[4][256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t total = s.rows * heads;
  for (int64_t w0 = (int64_t)blockIdx.x * 4; w0 < total; w0 += (int64_t)gridDim.x * 4) {
    const int64_t w = w0 + wave;
    bool live = w < total;
    const int row = live ? (int)(w / heads) : 0, h = live ? (int)(w - (int64_t)row * heads) : 0;
    int64_t b0 = 0;
    if (live) {
      const int i = packed_find(s.begin, s.n, row);
      live = i >= 0 && i < s.n && row < s.begin[i + 1];
      if (live) b0 = s.begin[i];
      live = live && b0 >= 0;
    }
    if (!live) continue;
    const int g = h / (heads / kv_heads);
    attend_row(q + (int64_t)row * ldq + (int64_t)h * hd, k + b0 * ldk + (int64_t)g * hd, ldk,
               v + b0 * ldv + (int64_t)g * hd, ldv, row - b0, hd, scale, qs[wave],
               out + (int64_t)row * heads * hd + (int64_t)h * hd);
  }
}

}  // namespace
}  // namespace zoact

using namespace zoact;

extern "C" zoact_status zoact_rope_at(const void* x, int64_t ldx, void* out, int64_t ldo, int32_t dtype, int64_t rows,
                                      int32_t n_heads, int32_t head_dim, int32_t rot_dim, int32_t layout,
                                      const int32_t* pos, const float* cos_t, const float* sin_t, int64_t n_pos,
                                      zoact_stream stream) {
  ZP_CHECK(dtype == ZOACT_F32 || dtype == ZOACT_BF16, "rope_at: dtype must be F32 or BF16");
  ZP_CHECK(rows >= 0 && rows < (int64_t(1) << 31), "rope_at: rows outside [0, 2^31)");
  ZP_CHECK(n_heads >= 1 && n_heads <= 65535 && head_dim >= 1 && head_dim <= 65535, "rope_at: bad heads");
  ZP_CHECK(rot_dim >= 2 && rot_dim % 2 == 0 && rot_dim <= head_dim, "rope_at: rot_dim must be even, 2 .. head_dim");
  ZP_CHECK(layout == ZOACT_ROPE_HALF || layout == ZOACT_ROPE_INTERLEAVED, "rope_at: unknown layout");
  ZP_CHECK((x && out) || rows == 0, "rope_at: NULL pointer");
  ZP_CHECK(cos_t && sin_t, "rope_at: NULL rotary table");
  ZP_CHECK(n_pos >= 1, "rope_at: empty rotary table");
  const int64_t width = (int64_t)n_heads * head_dim;
  ZP_CHECK(width < (int64_t(1) << 31), "rope_at: n_heads * head_dim past 32 bits");
  ZP_CHECK(ldx >= width && ldo >= width, "rope_at: heads exceed the row");
  ZP_CHECK(out != x || ldo == ldx, "rope_at: in place with another row stride");
  const size_t esize = dtype == ZOACT_F32 ? 4 : 2;
  ZP_CHECK(aligned_to(x, esize) && aligned_to(out, esize), "rope_at: x and out must be aligned to their type");
  ZP_CHECK(aligned_to(cos_t, 4) && aligned_to(sin_t, 4) && aligned_to(pos, 4),
           "rope_at: tables and pos must be 4-byte aligned");
  if (rows == 0) return ZOACT_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == ZOACT_BF16 ? rope_at_vec((const uint16_t*)x, ldx, (uint16_t*)out, ldo, rows, n_heads, head_dim, rot_dim,
                                        layout, pos, cos_t, sin_t, n_pos, s)
                          : rope_at_vec((const float*)x, ldx, (float*)out, ldo, rows, n_heads, head_dim, rot_dim, layout,
                                        pos, cos_t, sin_t, n_pos, s))
    return launched_or("rope_at");
  const int64_t units = rows * n_heads * (head_dim - rot_dim / 2), g = (units + 255) / 256;
  const unsigned grid = (unsigned)(g < 65536 ? g : 65536);
  if (dtype == ZOACT_BF16)
    rope_at_kernel<uint16_t><<<grid, 256, 0, s>>>((const uint16_t*)x, ldx, (uint16_t*)out, ldo, rows, n_heads, head_dim,
                                                  rot_dim, layout, pos, cos_t, sin_t, n_pos);
  else
    rope_at_kernel<float><<<grid, 256, 0, s>>>((const float*)x, ldx, (float*)out, ldo, rows, n_heads, head_dim, rot_dim,
                                               layout, pos, cos_t, sin_t, n_pos);
  return launched_or("rope_at");
}

extern "C" zoact_status zoact_attention_packed(const zoact_packed* s, const void* q, int64_t ldq, const void* k,
                                               int64_t ldk, const void* v, int64_t ldv, int32_t n_heads,
                                               int32_t n_kv_heads, int32_t head_dim, float scale, int32_t dtype,
                                               void* out, zoact_stream stream) {
  const zoact_status st = check_packed(s);
  if (st != ZOACT_OK) return st;
  ZP_CHECK(dtype == ZOACT_F32 || dtype == ZOACT_BF16, "attention_packed: dtype must be F32 or BF16");
  ZP_CHECK(n_heads >= 1 && n_heads <= 65535 && n_kv_heads >= 1 && n_heads % n_kv_heads == 0,
           "attention_packed: bad head grouping");
  ZP_CHECK(head_dim >= 1 && head_dim <= 256, "attention_packed: head_dim outside [1, 256]");
  ZP_CHECK(scale - scale == 0.f, "attention_packed: scale must be finite");
  ZP_CHECK((q && k && v && out) || s->rows == 0, "attention_packed: NULL pointer");
  const int64_t kvw = (int64_t)n_kv_heads * head_dim;
  ZP_CHECK(ldq >= (int64_t)n_heads * head_dim && ldk >= kvw && ldv >= kvw,
           "attention_packed: row strides smaller than the heads");
  const size_t esize = dtype == ZOACT_F32 ? 4 : 2;
  ZP_CHECK(aligned_to(q, esize) && aligned_to(k, esize) && aligned_to(v, esize) && aligned_to(out, esize),
           "attention_packed: tensors must be aligned to their type");
  if (s->rows == 0) return ZOACT_OK;
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  const hipError_t e = launch_attention_packed(*s, q, ldq, k, ldk, v, ldv, n_heads, n_kv_heads, head_dim, scale, dtype,
                                               out, hs);
  if (e == hipSuccess) return ZOACT_OK;
  if (e != hipErrorNotSupported) return set_error(ZOACT_E_HIP, hipGetErrorString(e));
  const int64_t waves = s->rows * n_heads, g = (waves + 3) / 4;
  const unsigned grid = (unsigned)(g < (1 << 20) ? g : (1 << 20));
  if (dtype == ZOACT_BF16)
    attention_packed_any<uint16_t><<<grid, 256, 0, hs>>>(*s, (const uint16_t*)q, ldq, (const uint16_t*)k, ldk,
                                                         (const uint16_t*)v, ldv, n_heads, n_kv_heads, head_dim, scale,
                                                         (uint16_t*)out);
  else
    attention_packed_any<float><<<grid, 256, 0, hs>>>(*s, (const float*)q, ldq, (const float*)k, ldk, (const float*)v,
                                                      ldv, n_heads, n_kv_heads, head_dim, scale, (float*)out);
  return launched_or("attention_packed");
}
