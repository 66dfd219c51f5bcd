// Device helpers for rows in 8 bits: where a block's codes and exponents lie, and a row on its way into it.
#pragma once
#include "oxy_kv8.h"
#include "oxy_device.h"

namespace oxy {

// ------------------------------------------------------------------------------------------
// page layout (see oxy.h)
// ------------------------------------------------------------------------------------------
// K page: chunk (jj, g, key) holds K[key][64jj+16g .. +15]
__device__ __forceinline__ int k8_chunk_offset(int jj, int g, int key) { return ((jj * 4 + g) * 16 + key) * 16; }
// V page: chunk (w, g, n) holds four keys 4g..4g+3 of dim d = 64w+4n, then those of d+1, d+2 and d+3
__device__ __forceinline__ int v8_chunk_offset(int w, int g, int n) { return ((w * 4 + g) * 16 + n) * 16; }
// byte of (dim d, key)
__device__ __forceinline__ int v8_offset(int d, int key) {
  return v8_chunk_offset(d >> 6, key >> 2, (d >> 2) & 15) + (d & 3) * 4 + (key & 3);
}
// A block's exponent bytes: its K rows', then its V rows'.
__device__ __forceinline__ int k8_scale_offset(int key) { return key; }
__device__ __forceinline__ int v8_scale_offset(int key) { return kPage + key; }

// Rows and columns of a 4 x 4 square of bytes (a word per row) change places.
__device__ __forceinline__ u32x4 transposed4(const u32x4 r) {
  const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), d = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
  return (u32x4){__builtin_amdgcn_perm(c, a, 0x05040100u), __builtin_amdgcn_perm(c, a, 0x07060302u),
                 __builtin_amdgcn_perm(d, b, 0x05040100u), __builtin_amdgcn_perm(d, b, 0x07060302u)};
}

__device__ __forceinline__ float scale_of(uint32_t exponent_byte) { return __uint_as_float(exponent_byte << 23); }

// ------------------------------------------------------------------------------------------
// quantising
// ------------------------------------------------------------------------------------------
// magnitude of a bf16 as ordered bits; what is not finite has no say in a row's exponent
__device__ __forceinline__ uint32_t finite_magnitude(uint32_t bf16) {
  const uint32_t m = bf16 & 0x7fffu;
  return m < 0x7f80u ? m : 0u;
}
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
// exponent byte of a row whose largest magnitude has these bits: 448 = 1.75 * 2^8
__device__ __forceinline__ uint32_t exponent_byte(uint32_t largest) {
  const int b = (int)(largest >> 7) - 8 + ((largest & 0x7fu) > 0x60u ? 1 : 0);
  return (uint32_t)max(b, 1);
}
// four bf16 (two words) -> four codes
__device__ __forceinline__ uint32_t quantise4(uint32_t lo, uint32_t hi, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(lo << 16) * inv, __uint_as_float(lo & 0xffff0000u) * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(hi << 16) * inv, __uint_as_float(hi & 0xffff0000u) * inv, w, true);
}
// maximum over the 32 lanes of a half wavefront / over lanes n, n+16, n+32, n+48
__device__ __forceinline__ uint32_t swap16_max(uint32_t x) {
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return larger(a[0], a[1]);
}
template <int N>
__device__ __forceinline__ uint32_t dpp_ror_u32(const uint32_t x) {
  return __builtin_amdgcn_update_dpp(0, x, 0x120 + N, 0xf, 0xf, false);
}
__device__ __forceinline__ uint32_t lanes16_largest(uint32_t x) {
  x = larger(x, dpp_ror_u32<8>(x));
  x = larger(x, dpp_ror_u32<4>(x));
  x = larger(x, dpp_ror_u32<2>(x));
  return larger(x, dpp_ror_u32<1>(x));
}
__device__ __forceinline__ uint32_t lanes32_largest(uint32_t x) { return swap16_max(lanes16_largest(x)); }

// A row on its way into a page: a half wavefront, lane c of 32 has elements 8c..8c+7.
struct Row8 {
  uint32_t codes[2];
  uint32_t exponent;
};
__device__ __forceinline__ Row8 quantise_row(const u32x4 x) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = larger(top, larger(finite_magnitude(x[i]), finite_magnitude(x[i] >> 16)));
  Row8 r;
  r.exponent = exponent_byte(lanes32_largest(top));
  const float inv = __uint_as_float((254u - r.exponent) << 23);
  r.codes[0] = quantise4(x[0], x[1], inv);
  r.codes[1] = quantise4(x[2], x[3], inv);
  return r;
}
__device__ __forceinline__ void store_key(const Row8& r, int key, char* __restrict__ block, uint8_t* __restrict__ scales,
                                          int c) {
  *(u32x2*)(block + k8_chunk_offset(c >> 3, (c >> 1) & 3, key) + (c & 1) * 8) = (u32x2){r.codes[0], r.codes[1]};
  if (c == 0) scales[k8_scale_offset(key)] = (uint8_t)r.exponent;
}
// dims 8c..8c+7 of one key, byte by byte
__device__ __forceinline__ void store_value(const Row8& r, int key, char* __restrict__ block, uint8_t* __restrict__ scales,
                                            int c) {
  char* p = block + kPageBytes8;
#pragma unroll
  for (int e = 0; e < 8; ++e) p[v8_offset(8 * c + e, key)] = (char)(r.codes[e >> 2] >> (8 * (e & 3)));
  if (c == 0) scales[v8_scale_offset(key)] = (uint8_t)r.exponent;
}

}  // namespace oxy
