// Device code of 4-bit rows: 32 neighbouring columns of a row (a block) are e2m1
// numbers times one power of two.  A lane of the scaled matrix instructions takes
// one block of one row: 16 bytes and a scale byte.
#pragma once

#include "row_device.h"

namespace saga {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A block whose largest magnitude A has the exponent field f (bits 30 to 23 of the
// float32 A) has the scale 2^(max(f - 2, 0) - 127): floor(log2 A) - 2 in a byte with
// the bias 127.  A is then below 8 scales.  A block that holds a NaN or an infinity has the
// byte 255, which stands for NaN, and zeros.
struct BlockScale {
  uint32_t byte;
  float s;   // the scale as a float32 (of a bad block: any)
  bool bad;
};
// amax: the largest magnitude as bits
__device__ __forceinline__ BlockScale block_scale(uint32_t amax) {
  BlockScale b;
  const uint32_t field = amax >> 23;
  b.byte = (field > 2u ? field : 2u) - 2u;
  b.bad = field == 255u;
  b.s = __uint_as_float(b.byte ? b.byte << 23 : 0x00400000u);  // (2^-127 is below the normal numbers)
  if (b.bad) b.byte = 255u;
  return b;
}

// 8 columns to 4 bytes: to the nearest number, ties to the even one, at most 6 scales
// (the instruction does all three)
__device__ __forceinline__ uint32_t round_mx4(const Raw<uint16_t>& x, const BlockScale& b) {
  uint32_t o = 0;
  bf16x2 p[4];
  __builtin_memcpy(p, &x.v, 16);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, p[0], b.s, 0);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, p[1], b.s, 1);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, p[2], b.s, 2);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, p[3], b.s, 3);
  return b.bad ? 0u : o;
}
__device__ __forceinline__ uint32_t round_mx4(const Raw<float>& r, const BlockScale& b) {
  float x[8];
  r.widen(x);
  uint32_t o = 0;
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[0], x[1], b.s, 0);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[2], x[3], b.s, 1);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[4], x[5], b.s, 2);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[6], x[7], b.s, 3);
  return b.bad ? 0u : o;
}

// a scale byte's value: 2^(byte - 127), 0 below the normal numbers, 255 a NaN (both by the
// bit that is set then: no branch)
__device__ __forceinline__ float scale_value(uint32_t byte) {
  const uint32_t ends = ((byte + 1u) & 255u) < 2u ? 0x00400000u : 0u;
  return __uint_as_float(byte << 23 | ends);
}

// bytes past `left` cleared (left below 16)
__device__ __forceinline__ u32x4 clear_bytes(u32x4 v, int left) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int n = left - 4 * d;
    if (n <= 0) v[d] = 0;
    else if (n < 4) v[d] &= (1u << (8 * n)) - 1u;
  }
  return v;
}

// A block as the matrix instructions take it.  Past a row's end: zeros of scale 1.
struct Mx4Block {
  u32x4 v;
  uint32_t scale;  // in the low byte
};

// Columns col.. of a row of K floats, 8 of them and without a branch: past the row's end its last
// 16 bytes are read again (each half by itself: rows are whole 16 bytes, not 32), to be cleared.
__device__ __forceinline__ void load_clamped(Raw<float>& r, const float* x, int col, int K) {
  const int most = (K - 1) / 4 * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) r.v[h] = *reinterpret_cast<const u32x4*>(x + min(col + 4 * h, most));
}
__device__ __forceinline__ void load_clamped(Raw<uint16_t>& r, const uint16_t* x, int col, int K) {
  r.v = *reinterpret_cast<const u32x4*>(x + min(col, (K - 1) / 8 * 8));
}

// What a row's source is: 4-bit rows with their scales, or floats.  Block b of the row of K
// columns; `take` apart from `load`, so that loads run ahead, and without a branch in it: past
// the row's end its last piece is read again, and `take` clears it (LAST: where that can be).
template <typename T>
struct RowSource {  // float or uint16_t
  const T* x;
  Raw<T> raw[4];
  __device__ __forceinline__ void at(const void* base, int64_t ld, const uint8_t*, int64_t, int64_t row) {
    x = static_cast<const T*>(base) + row * ld;
  }
  __device__ __forceinline__ void load(int b, int K) {
#pragma unroll
    for (int u = 0; u < 4; ++u) load_clamped(raw[u], x, b * 32 + u * 8, K);
  }
  __device__ __forceinline__ Mx4Block take(int b, int K, bool last) {
    if (last) {
#pragma unroll
      for (int u = 0; u < 4; ++u) raw[u].clear(K - b * 32 - u * 8);
    }
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) top = max(top, raw[u].top());
    const BlockScale s = block_scale(top);
    Mx4Block o;
#pragma unroll
    for (int u = 0; u < 4; ++u) o.v[u] = round_mx4(raw[u], s);
    o.scale = s.byte;
    return o;
  }
};
template <>
struct RowSource<uint8_t> {
  const uint8_t *q, *s;
  u32x4 v;
  uint32_t scale;
  __device__ __forceinline__ void at(const void* base, int64_t ld, const uint8_t* scales, int64_t lds, int64_t row) {
    q = static_cast<const uint8_t*>(base) + row * ld;
    s = scales + row * lds;
  }
  __device__ __forceinline__ void load(int b, int K) {
    b = min(b, (K - 1) / 32);
    v = *reinterpret_cast<const u32x4*>(q + b * 16);
    scale = s[b];
  }
  __device__ __forceinline__ Mx4Block take(int b, int K, bool last) {
    if (last) {
      const int left = (K + 1) / 2 - b * 16;
      if (left < 16) v = clear_bytes(v, left);
      if (left <= 0) scale = 127u;
    }
    return {v, scale};
  }
};

// 16 x 16 sums over 4 blocks, or 128 k: lane l holds row l % 16 and block l / 16 of each
// operand, and of the sums column l % 16 of b's rows by four of a's, 4 (l / 16)..
__device__ __forceinline__ f32x4 mma_mx4(const Mx4Block& a, const Mx4Block& b, f32x4 c) {
  const i32x8 x = {(int)a.v[0], (int)a.v[1], (int)a.v[2], (int)a.v[3], 0, 0, 0, 0};
  const i32x8 y = {(int)b.v[0], (int)b.v[1], (int)b.v[2], (int)b.v[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)a.scale, 0, (int)b.scale);
}

}  // namespace
}  // namespace saga
