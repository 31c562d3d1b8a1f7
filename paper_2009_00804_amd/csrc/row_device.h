// Device code of the kernels that work on whole rows (8-bit rows, block norms,
// label log probabilities): reductions over a row's lanes, 8-column units of a
// row, and the rounding to 8 bits.
#pragma once

#include "saga_device.h"

namespace saga {
namespace {

// --------------------------------------------------------------------------
// reductions over aligned groups of G lanes (8 to 64); every lane gets the
// result.  A step combines groups that are uniform already, so a mirror serves
// as well as an exchange, and up to 16 lanes stay in one DPP row.
// --------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_mov(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}

struct OpSum {
  __device__ __forceinline__ static uint32_t of(uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }
};
struct OpMax {  // floats; a NaN gives way to a number
  __device__ __forceinline__ static uint32_t of(uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }
};
struct OpMaxU {
  __device__ __forceinline__ static uint32_t of(uint32_t a, uint32_t b) { return max(a, b); }
};

template <typename OP, int G>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v) {
  static_assert(G == 8 || G == 16 || G == 32 || G == 64, "group size");
  v = OP::of(v, dpp_mov<0xB1>(v));   // quad_perm [1,0,3,2]
  v = OP::of(v, dpp_mov<0x4E>(v));   // quad_perm [2,3,0,1]
  v = OP::of(v, dpp_mov<0x141>(v));  // row_half_mirror
  if constexpr (G >= 16) v = OP::of(v, dpp_mov<0x140>(v));  // row_mirror
  if constexpr (G >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = OP::of(p[0], p[1]);
  }
  if constexpr (G == 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = OP::of(p[0], p[1]);
  }
  return v;
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  return __uint_as_float(group_reduce<OpSum, G>(__float_as_uint(v)));
}
template <int G>
__device__ __forceinline__ float group_max(float v) {
  return __uint_as_float(group_reduce<OpMax, G>(__float_as_uint(v)));
}
template <int G>
__device__ __forceinline__ uint32_t group_maxu(uint32_t v) {
  return group_reduce<OpMaxU, G>(v);
}

// A row on G lanes; G > 64: G / 64 waves, joined through LDS (red: 2 G / 64 words,
// turn: the reductions so far)
template <int G>
struct RowGroup {
  static constexpr int THREADS = G > 256 ? G : 256;
  static constexpr int ROWS = THREADS / G;

  template <typename OP>
  __device__ __forceinline__ static uint32_t reduce(uint32_t v, uint32_t* red, int& turn) {
    if constexpr (G <= 64) {
      return group_reduce<OP, G>(v);
    } else {
      constexpr int W = G / 64;
      v = group_reduce<OP, 64>(v);
      uint32_t* r = red + (turn++ & 1) * W;  // the other half may still be read
      if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
      __syncthreads();
      v = r[0];
#pragma unroll
      for (int i = 1; i < W; ++i) v = OP::of(v, r[i]);
      return v;
    }
  }
  __device__ __forceinline__ static float sum(float v, uint32_t* red, int& turn) {
    return __uint_as_float(reduce<OpSum>(__float_as_uint(v), red, turn));
  }
};

// --------------------------------------------------------------------------
// units: 8 columns of a row, columns past `left` read as 0.  A 16-byte piece
// is touched only if its first column is in the row: the rest of it is padding
// of the same 16 bytes.
// --------------------------------------------------------------------------
__device__ __forceinline__ void load_unit(const float* p, int64_t left, float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (left > 4 * h) x = *reinterpret_cast<const f32x4*>(p + 4 * h);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[4 * h + j] = left > 4 * h + j ? x[j] : 0.0f;
  }
}
__device__ __forceinline__ void load_unit(const uint16_t* p, int64_t left, float (&v)[8]) {
  u32x4 x = {0u, 0u, 0u, 0u};
  if (left > 0) x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = left > 2 * j ? __uint_as_float(x[j] << 16) : 0.0f;
    v[2 * j + 1] = left > 2 * j + 1 ? __uint_as_float(x[j] & 0xffff0000u) : 0.0f;
  }
}
__device__ __forceinline__ void store_unit(float* p, int64_t left, const float (&v)[8]) {
  if (left >= 8) {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = v[j];
  }
}
__device__ __forceinline__ void store_unit(uint16_t* p, int64_t left, const float (&v)[8]) {
  if (left >= 8) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = (uint32_t)f32_to_bf16(v[2 * j]) | ((uint32_t)f32_to_bf16(v[2 * j + 1]) << 16);
    *reinterpret_cast<u32x4*>(p) = w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = f32_to_bf16(v[j]);
  }
}
__device__ __forceinline__ void store_unit_i8(int8_t* p, int64_t left, uint2 q) {
  if (left >= 8) {
    *reinterpret_cast<uint2*>(p) = q;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = (int8_t)((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
  }
}

// --------------------------------------------------------------------------
// 8-bit rows
// --------------------------------------------------------------------------
// A row whose largest magnitude is A has the scale s = A / 127, rounded to
// float32 and 2^-126 at least, and holds rint(x / s) (ties to even), at most
// 127 in magnitude since A / s is below 127.5.  A row that holds a NaN or an
// infinity has the scale NaN and all zeros.
struct RowScale {
  float s, inv;
  bool bad;
};
// amax: the largest magnitude as bits (a NaN is above infinity, infinity above numbers)
__device__ __forceinline__ RowScale row_scale(uint32_t amax) {
  RowScale r;
  r.bad = amax >= 0x7f800000u;
  r.s = fmaxf(__uint_as_float(amax) / 127.0f, 0x1p-126f);
  r.inv = 1.0f / r.s;
  if (r.bad) r.s = __uint_as_float(0x7fc00000u), r.inv = 0.0f;
  return r;
}
// x * inv is within 2^-23 of x / s, so its rounding is right or one next to a
// half.  The remainder x - q s is then exact in float32 (a multiple of ulp(s),
// at most about s / 2), and says on which side of the half x / s lies.
__device__ __forceinline__ int round_q(float x, const RowScale& r) {
  const float q = rintf(x * r.inv);
  const float e = fmaf(-q, r.s, x), d = 2.0f * fabsf(e);
  int k = (int)q;
  if (d > r.s || (d == r.s && (k & 1))) k += e > 0.0f ? 1 : -1;
  return k;
}
__device__ __forceinline__ uint2 round_unit(const float (&x)[8], const RowScale& r) {
  uint2 o = make_uint2(0u, 0u);
  if (r.bad) return o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    o.x |= (uint32_t)(round_q(x[j], r) & 0xff) << (8 * j);
    o.y |= (uint32_t)(round_q(x[4 + j], r) & 0xff) << (8 * j);
  }
  return o;
}

}  // namespace
}  // namespace saga
