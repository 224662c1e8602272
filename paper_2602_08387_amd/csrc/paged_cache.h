// A paged cache of keys and values as the kernels see it, and e4m3 with a power of two for each vector.
#pragma once
#include "common.h"
#include "kernels.h"

namespace dl {

// k, v: [n_pages][heads][page tokens][dh], bf16 or e4m3; the vectors' exponents (e4m3 only) [n_pages][heads][page tokens], one byte with a bias of 127
struct PagedCache {
  char *x[2];                // k, v
  uint8_t *scale[2];         // null for bf16
  const int32_t* table;      // [batch][columns]: the page of every page_size tokens of a row
  int n_pages, heads, shift, columns, batch;   // page_size = 1 << shift
};

inline PagedCache paged_cache(const CacheCall& c) {
  PagedCache p{};
  p.x[0] = (char*)c.k; p.x[1] = (char*)c.v;
  p.scale[0] = (uint8_t*)c.k_scale; p.scale[1] = (uint8_t*)c.v_scale;
  p.table = c.table;
  p.n_pages = (int)c.n_pages; p.heads = (int)c.heads; p.columns = (int)c.columns; p.batch = (int)c.batch;
  while ((int64_t)1 << p.shift < c.page_size) ++p.shift;
  return p;
}

// The page that holds position p of batch row b, or -1 where there is none: behind the table, or a page that does not exist.
__device__ __forceinline__ int page_of(const PagedCache& c, int64_t b, int64_t p) {
  if (p < 0 || (p >> c.shift) >= c.columns) return -1;
  const int page = c.table[b * c.columns + (p >> c.shift)];
  return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}
// Vector number of a page's head and slot, in x and in scale.
__device__ __forceinline__ int64_t vector_of(const PagedCache& c, int page, int head, int64_t p) {
  return (((int64_t)page * c.heads + head) << c.shift) + (p & ((1 << c.shift) - 1));
}
// Position of a row's first new token, far enough from the ends of 64 bits that a sequence can be added, and its number of new tokens.
__device__ __forceinline__ int64_t row_start(const int64_t* start, int64_t b) {
  constexpr int64_t far = (int64_t)1 << 62;
  const int64_t p = start ? start[b] : 0;
  return p < -far ? -far : p > far ? far : p;
}
__device__ __forceinline__ int row_length(const int64_t* lengths, int64_t b, int seq) {
  const int64_t n = lengths ? lengths[b] : seq;
  return n < 0 ? 0 : n > seq ? seq : (int)n;
}

// e4m3 (4 bits of exponent, 3 of mantissa, up to 448, no infinities).  The exponent of a vector whose largest magnitude is amax: the smallest e with
// amax <= 448 * 2^e = 1.75 * 2^(e + 8), from the float's own bits; 0 for zeros.  Below 2^-110 the step of e4m3 would leave the range of bf16.
// A power of two, so that scaling back is exact: what is read is a bf16 value (4 significant bits), with e4m3's one rounding.
constexpr int kScaleBias = 127, kScaleLeast = -110, kScaleMost = 120;
__device__ __forceinline__ int e4m3_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return amax == 0.f ? 0 : e < kScaleLeast ? kScaleLeast : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Four floats, scaled already, as e4m3, to nearest and ties to even; values that are not finite become its NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint32_t u = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, (int)u, true);
}
// Eight e4m3 times a power of two as bf16, exact.
__device__ __forceinline__ bf16x8 unpack_e4m3(u32x2 u, float scale) {
  bf16x8 v;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[0], scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[0], scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[1], scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[1], scale, true);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
  v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
  return v;
}

}  // namespace dl
