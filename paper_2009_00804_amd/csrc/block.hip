// The end of a block in a deep network: norm of the block's output, gate,
// channel and residual scales, residual sum, and the norm before the next block,
//     u = post(block), y = x + c ch * act(gate) * u, z = pre(y)
// in one pass over the rows.  rms: v / sqrt(mean v^2 + eps) * w + b; layer:
// (v - mean) / sqrt(mean (v - mean)^2 + eps) * w + b.  z takes y as summed, before
// y's own rounding to the stream's type.
//
// Memory bounds it: each row is read once into registers (8 columns a lane and
// unit), both norms reduce over the row's lanes, and y and z leave from there.  2^20
// x 128 in bfloat16 273 to 287 us, 4.7 to 4.9 TB/s; 100003 x 602 170 to 185 us, 4.6
// to 5.0 TB/s; 32768 x 4096 to 8-bit rows 335 us, 5.1 TB/s (a copy: 4.7).  The sums
// of both norms are float32, the layer norm's about its own mean; z is rounded once,
// from y's float32 values (a norm of the rounded y would add y's rounding).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "row_device.h"
#include "saga_internal.h"

namespace saga {
namespace {

constexpr int64_t kMostBlocks = 2048;  // groups keep their vectors over many rows

// A lane's share of a row: U units, unit u at column col0 + u * 8 * G.
template <int G, int U>
struct Share {
  typedef RowGroup<G> R;
  static constexpr int STEP = 8 * G;

  // v / sqrt(mean v^2 + eps), for LAYER of v less its mean.  Columns past F are 0
  // before and after.
  __device__ __forceinline__ static void normalise(int kind, float eps, float inv_f, int left, float (&v)[U][8],
                                                   uint32_t* red, int& turn) {
    if (kind == SAGA_NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[u][j];
      const float mean = R::sum(s, red, turn) * inv_f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = j < left - u * STEP ? v[u][j] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(v[u][j], v[u][j], s);
    const float r = 1.0f / sqrtf(R::sum(s, red, turn) * inv_f + eps);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] *= r;
  }
};

// Gate activations, with the card's own exponential and reciprocal: nothing beside a row's
// bytes.  In units of 2^-24 of their values sigmoid is good to 7 + 2.3 |x|, and 0 where it is
// below 2^-126; tanh to 32 (most near 0.3: its series stands where 1 - 2 / (e^2x + 1) would
// cancel, below 0.3, and the first term left out is 5e-8 x).
__device__ __forceinline__ float gate_value(int act, float x) {
  switch (act) {
    case SAGA_ACT_RELU: return x > 0.0f ? x : 0.0f;
    case SAGA_ACT_ELU: return x > 0.0f ? x : expm1f(x);
    case SAGA_ACT_SIGMOID: return __builtin_amdgcn_rcpf(1.0f + __expf(-x));
    case SAGA_ACT_TANH: {
      const float q = x * x;
      const float p = fmaf(q, fmaf(q, fmaf(q, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f);
      const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__expf(2.0f * x) + 1.0f);
      return q < 0.09f ? fmaf(x * q, p, x) : t;
    }
    default: return x;
  }
}

// a lane's vector values at its columns, `other` where there is no vector, 0 past F
template <int U, int STEP>
__device__ __forceinline__ void load_vector(const float* w, float other, int col0, int left, float (&v)[U][8]) {
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool in_row = j < left - u * STEP;
      v[u][j] = in_row ? (w ? w[col0 + u * STEP + j] : other) : 0.0f;
    }
}

template <typename XT, typename BT, int U>
struct Inputs {
  Raw<BT> block[U], gate[U];
  Raw<XT> x[U];
};

// The vectors of a lane's columns stay in its registers for all rows of its group,
// post's weights with the channel and residual scales taken in; a row's loads are
// issued while the row before it is computed.
template <typename XT, typename BT, int G, int U>
__global__ __launch_bounds__(RowGroup<G>::THREADS) void k_block_norm(BlockArgs a) {
  typedef RowGroup<G> R;
  typedef Share<G, U> H;
  __shared__ uint32_t red[2 * (G > 64 ? G / 64 : 1)];
  int turn = 0;
  const int col0 = (threadIdx.x % G) * 8, left = a.F - col0;
  const float inv_f = 1.0f / (float)a.F;
  float aw[U][8], ab[U][8], pw[U][8], pb[U][8];
  {
    float ch[U][8];
    load_vector<U, H::STEP>(a.channel, 1.0f, col0, left, ch);
    load_vector<U, H::STEP>(a.post_kind != SAGA_NORM_NONE ? a.post_w : nullptr, 1.0f, col0, left, aw);
    load_vector<U, H::STEP>(a.post_kind != SAGA_NORM_NONE ? a.post_b : nullptr, 0.0f, col0, left, ab);
    load_vector<U, H::STEP>(a.pre_kind != SAGA_NORM_NONE ? a.pre_w : nullptr, 1.0f, col0, left, pw);
    load_vector<U, H::STEP>(a.pre_kind != SAGA_NORM_NONE ? a.pre_b : nullptr, 0.0f, col0, left, pb);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        aw[u][j] *= ch[u][j] * a.res_scale;
        ab[u][j] *= ch[u][j] * a.res_scale;
      }
  }
  const int64_t stride = gridDim.x * (int64_t)R::ROWS;
  int64_t row = blockIdx.x * (int64_t)R::ROWS + threadIdx.x / G;
  Inputs<XT, BT, U> in;
  const auto load = [&](int64_t r) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = col0 + u * H::STEP, l = left - u * H::STEP;
      in.block[u].load(static_cast<const BT*>(a.block) + r * a.ld_block + col, l);
      if (a.gate) in.gate[u].load(static_cast<const BT*>(a.gate) + r * a.ld_gate + col, l);
      if (a.x) in.x[u].load(static_cast<const XT*>(a.x) + r * a.ld_x + col, l);
    }
  };
  if (row < a.M) load(row);
  // (a row's lanes stay together: rows of several waves own their workgroup)
  for (; row < a.M; row += stride) {
    Inputs<XT, BT, U> now = in;
    if (row + stride < a.M) load(row + stride);
    float v[U][8], y[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      now.block[u].clear(left - u * H::STEP);
      now.block[u].widen(v[u]);
    }
    if (a.post_kind != SAGA_NORM_NONE) H::normalise(a.post_kind, a.post_eps, inv_f, left, v, red, turn);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] = fmaf(v[u][j], aw[u][j], ab[u][j]);
    if (a.gate) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float g[8];
        now.gate[u].clear(left - u * H::STEP);
        now.gate[u].widen(g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] *= gate_value(a.gate_act, g[j]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (a.x) {
        now.x[u].clear(left - u * H::STEP);
        now.x[u].widen(y[u]);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[u][j] += v[u][j];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[u][j] = v[u][j];
      }
      if (a.y)
        store_unit(static_cast<XT*>(a.y) + row * a.ld_y + col0 + u * H::STEP, left - u * H::STEP, y[u]);
    }
    if (!a.z) continue;
    if (a.pre_kind != SAGA_NORM_NONE) {
      H::normalise(a.pre_kind, a.pre_eps, inv_f, left, y, red, turn);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[u][j] = fmaf(y[u][j], pw[u][j], pb[u][j]);
    }
    if (a.z_scale) {
      uint32_t top = 0;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(y[u][j]) & 0x7fffffffu);
      const RowScale s = row_scale(R::template reduce<OpMaxU>(top, red, turn));
#pragma unroll
      for (int u = 0; u < U; ++u)
        store_unit_i8(static_cast<int8_t*>(a.z) + row * a.ld_z + col0 + u * H::STEP, left - u * H::STEP,
                      round_unit(y[u], s));
      if (threadIdx.x % G == 0) a.z_scale[row] = s.s;
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        store_unit(static_cast<BT*>(a.z) + row * a.ld_z + col0 + u * H::STEP, left - u * H::STEP, y[u]);
    }
  }
}

template <typename XT, typename BT, int G, int U>
hipError_t launch(const BlockArgs& a, hipStream_t st) {
  typedef RowGroup<G> R;
  const int64_t blocks = std::min<int64_t>((a.M + R::ROWS - 1) / R::ROWS, kMostBlocks);
  hipLaunchKernelGGL((k_block_norm<XT, BT, G, U>), dim3((unsigned)blocks), dim3(R::THREADS), 0, st, a);
  return hipGetLastError();
}

template <typename XT, typename BT>
hipError_t dispatch(const BlockArgs& a, hipStream_t st) {
  // Lanes per row and units per lane (us, float32 stream, bfloat16 blocks): 200000 x
  // 300 64 x 1 204, 32 x 2 217; 400000 x 256 32 x 1 260, 16 x 2 262; 100003 x 602 128
  // x 1 185, 32 x 3 197, 64 x 2 218, 16 x 5 295; 131072 x 1024 128 x 1 340, 64 x 2
  // 336; 65536 x 2048 256 x 1 370, 128 x 2 393; 32768 x 4096 512 x 1 347, 256 x 2
  // 369, 1024 x 1 487; 16384 x 8192 1024 x 1 358, 512 x 2 379.
  // Past 4096 that is one workgroup a CU, of which a row of 5000 uses 625 lanes (15000 x 5000
  // 242 against 225 for its bytes, in bfloat16 throughout 274 against 161; 10000 x 8192 208
  // against 176).  Past 8192 two units do not fit the 128 registers of 1024 threads: 52 to
  // 95 spill, and a row takes 2.0 to 2.5 times its bytes' time (8000 x 12000 630 against 288, in
  // bfloat16 throughout 513 against 206).
  if (a.F <= 64) return launch<XT, BT, 8, 1>(a, st);
  if (a.F <= 128) return launch<XT, BT, 16, 1>(a, st);
  if (a.F <= 256) return launch<XT, BT, 32, 1>(a, st);
  if (a.F <= 512) return launch<XT, BT, 64, 1>(a, st);
  if (a.F <= 1024) return launch<XT, BT, 128, 1>(a, st);
  if (a.F <= 2048) return launch<XT, BT, 256, 1>(a, st);
  if (a.F <= 4096) return launch<XT, BT, 512, 1>(a, st);
  if (a.F <= 8192) return launch<XT, BT, 1024, 1>(a, st);
  return launch<XT, BT, 1024, 2>(a, st);
}

}  // namespace

hipError_t launch_block_norm(const BlockArgs& a, hipStream_t st) {
  if (a.M == 0) return hipSuccess;
  if (a.x_dtype == SAGA_BF16) return dispatch<uint16_t, uint16_t>(a, st);
  if (a.dtype == SAGA_BF16) return dispatch<float, uint16_t>(a, st);
  return dispatch<float, float>(a, st);
}

}  // namespace saga
