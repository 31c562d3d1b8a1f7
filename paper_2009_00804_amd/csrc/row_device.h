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
  static constexpr int THREADS = G > 64 ? G : 256;  // (a row of several waves has barriers: it owns its workgroup)
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
// units: 8 columns of a row.  A 16-byte piece is touched only if its first column
// is in the row (`left` columns of it are): the rest of it is padding of the same
// 16 bytes.
// --------------------------------------------------------------------------
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
// two values rounded to bfloat16 (to nearest, ties to even; one instruction)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 b = __builtin_convertvector((f32x2{lo, hi}), bf16x2);
  uint32_t u;
  __builtin_memcpy(&u, &b, 4);
  return u;
}
__device__ __forceinline__ void store_unit(uint16_t* p, int64_t left, const float (&v)[8]) {
  if (left >= 8) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
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
// x * inv is within 2^-24 of x / s, so its rounding q is right or one next to a
// half.  The remainder x - q s is then exact in float32 (a multiple of ulp(s), at
// most about s / 2), and says on which side of the half x / s lies.
__device__ __forceinline__ uint32_t round_exact(float x, const RowScale& r) {
  const float q = rintf(x * r.inv);
  const float e = fmaf(-q, r.s, x), d = 2.0f * fabsf(e);
  int k = (int)q;
  if (d > r.s || (d == r.s && (k & 1))) k += e > 0.0f ? 1 : -1;
  return (uint32_t)k & 0xffu;
}
// 8 values to 8 bytes.  Added to 1.5 * 2^23 the product x * inv is rounded to a
// whole number, ties to even, whose low byte is q; values further than 2e-5 from a
// half (x / s is below 127.5: x * inv is within 8e-6 of it) are right as they are.
__device__ __forceinline__ uint2 round_unit(const float (&x)[8], const RowScale& r) {
  constexpr float kWhole = 12582912.0f;
  uint32_t t[8];
  float far = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float m = fmaf(x[j], r.inv, kWhole);
    far = fmaxf(far, fabsf(fmaf(x[j], r.inv, kWhole - m)));
    t[j] = __float_as_uint(m);
  }
  if (far > 0.49998f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = round_exact(x[j], r);
  }
  uint32_t o[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(t[4 * h + 1], t[4 * h], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(t[4 * h + 3], t[4 * h + 2], 0x0c0c0400u);
    o[h] = r.bad ? 0u : __builtin_amdgcn_perm(hi, lo, 0x05040100u);
  }
  return make_uint2(o[0], o[1]);
}

// A unit as it lies in memory: half the registers of its float32 values where it is
// bfloat16.  `clear` zeroes the columns past `left` (apart from `load`, so that it
// does not wait for loads that are still under way).
template <typename T> struct Raw;
template <> struct Raw<float> {
  u32x4 v[2];
  __device__ __forceinline__ void load(const float* p, int left) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v[h] = u32x4{0u, 0u, 0u, 0u};
      if (left > 4 * h) v[h] = *reinterpret_cast<const u32x4*>(p + 4 * h);
    }
  }
  __device__ __forceinline__ void clear(int left) {
    if (left < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (left <= j) v[j / 4][j % 4] = 0u;
    }
  }
  __device__ __forceinline__ uint32_t top() const {  // largest magnitude, as float32 bits
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, v[j / 4][j % 4] & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(v[j / 4][j % 4]);
  }
};
template <> struct Raw<uint16_t> {
  u32x4 v;
  __device__ __forceinline__ void load(const uint16_t* p, int left) {
    v = u32x4{0u, 0u, 0u, 0u};
    if (left > 0) v = *reinterpret_cast<const u32x4*>(p);
  }
  __device__ __forceinline__ void clear(int left) {
    if (left < 8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (left <= 2 * j) v[j] = 0u;
        else if (left == 2 * j + 1) v[j] &= 0xffffu;
      }
    }
  }
  __device__ __forceinline__ uint32_t top() const {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = v[j] & 0x7fff7fffu;
      u16x2 b;
      __builtin_memcpy(&b, &a, 4);
      m = __builtin_elementwise_max(m, b);
    }
    return (uint32_t)max(m[0], m[1]) << 16;
  }
  __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(v[j] << 16);
      x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
    }
  }
};

}  // namespace
}  // namespace saga
