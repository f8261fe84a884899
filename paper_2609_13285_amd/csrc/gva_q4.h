// The 4-bit cache's layout and conversions, for the sources that read it.

#pragma once

#include "gva_common.h"

namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlockBytes = 1024;              // codes: a wave's load
constexpr int kScaleCols = 32;
constexpr int kScaleNaN = 255, kScaleLow = 127 - 119, kScaleHigh = 127 + 125;
__host__ __device__ constexpr int block_rows(int d_v) { return 2048 / d_v; }

// Byte offset, inside a stream, of piece p (d_v / 8 bytes) of row t, and of
// the scale byte of block c of row t.
__device__ __forceinline__ int64_t code_off(int t, int p, int d_v) {
  const int rows = block_rows(d_v);
  return (int64_t)(t / rows) * kBlockBytes + (p * 16 + t % 16) * 16 + (t % rows / 16) * 8;
}
__device__ __forceinline__ int64_t scale_off(int t, int c, int d_v) {
  return (int64_t)(t / 32) * d_v + (c * 16 + t % 16) * 2 + t / 16 % 2;
}

__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte << 23); }

// Eight codes of a word as bf16, times the scale of the byte.
__device__ __forceinline__ bf16x8 dequant8(unsigned w, unsigned byte) {
  const float s = scale_of(byte);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  bf16x8 out;
  out[0] = a[0]; out[1] = a[1]; out[2] = b[0]; out[3] = b[1];
  out[4] = c[0]; out[5] = c[1]; out[6] = d[0]; out[7] = d[1];
  return out;                                  // (byte 255 is an infinite scale here, and the converter gives NaN)
}

inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace
