// The end of a block in a deep network: norm of the block's output, gate,
// channel and residual scales, residual sum, and the norm before the next block,
//     u = post(block), y = x + c ch * act(gate) * u, z = pre(y)
// in one pass over the rows.  rms: v / sqrt(mean v^2 + eps) * w + b; layer:
// (v - mean) / sqrt(mean (v - mean)^2 + eps) * w + b.  z takes y as summed, before
// y's own rounding to the stream's type.
//
// Memory bounds it: each row is read once into registers (8 columns a lane and
// unit), both norms reduce over the row's lanes, and y and z leave from there.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "row_device.h"
#include "saga_internal.h"

namespace saga {
namespace {

constexpr int64_t kMostBlocks = 1 << 20;  // (a grid holds less than 2^32 threads)

template <int G, int U>
__device__ __forceinline__ void normalise(int kind, float eps, float inv_f, int col0, int F, float (&v)[U][8],
                                          uint32_t* red, int& turn) {
  typedef RowGroup<G> R;
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
      for (int j = 0; j < 8; ++j) v[u][j] = col0 + u * 8 * G + j < F ? v[u][j] - mean : 0.0f;
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

// v = v * w + b on the unit's columns (w, b nullable)
__device__ __forceinline__ void affine(const float* w, const float* b, int col, int F, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (col + j < F) {
      if (w) v[j] *= w[col + j];
      if (b) v[j] += b[col + j];
    }
}

template <typename XT, typename BT, int G, int U>
__device__ __forceinline__ void block_row(const BlockArgs& a, int64_t row, uint32_t* red, int& turn) {
  typedef RowGroup<G> R;
  const int col0 = (threadIdx.x % G) * 8, F = a.F;
  const float inv_f = 1.0f / (float)F;
  float u[U][8], y[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = col0 + i * 8 * G;
    load_unit(static_cast<const BT*>(a.block) + row * a.ld_block + col, F - col, u[i]);
    if (a.x) {
      load_unit(static_cast<const XT*>(a.x) + row * a.ld_x + col, F - col, y[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) y[i][j] = 0.0f;
    }
  }
  if (a.post_kind != SAGA_NORM_NONE) normalise<G, U>(a.post_kind, a.post_eps, inv_f, col0, F, u, red, turn);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = col0 + i * 8 * G;
    if (a.post_kind != SAGA_NORM_NONE) affine(a.post_w, a.post_b, col, F, u[i]);
    affine(a.channel, nullptr, col, F, u[i]);
    if (a.gate) {
      float g[8];
      load_unit(static_cast<const BT*>(a.gate) + row * a.ld_gate + col, F - col, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[i][j] *= apply_act(a.gate_act, g[j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) y[i][j] = col + j < F ? fmaf(a.res_scale, u[i][j], y[i][j]) : 0.0f;
    if (a.y) store_unit(static_cast<XT*>(a.y) + row * a.ld_y + col, F - col, y[i]);
  }
  if (!a.z) return;
  if (a.pre_kind != SAGA_NORM_NONE) {
    normalise<G, U>(a.pre_kind, a.pre_eps, inv_f, col0, F, y, red, turn);
#pragma unroll
    for (int i = 0; i < U; ++i) affine(a.pre_w, a.pre_b, col0 + i * 8 * G, F, y[i]);
  }
  if (a.z_scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(y[i][j]) & 0x7fffffffu);
    const RowScale s = row_scale(R::template reduce<OpMaxU>(top, red, turn));
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = col0 + i * 8 * G;
      store_unit_i8(static_cast<int8_t*>(a.z) + row * a.ld_z + col, F - col, round_unit(y[i], s));
    }
    if (threadIdx.x % G == 0) a.z_scale[row] = s.s;
  } else {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = col0 + i * 8 * G;
      store_unit(static_cast<BT*>(a.z) + row * a.ld_z + col, F - col, y[i]);
    }
  }
}

template <typename XT, typename BT, int G, int U>
__global__ __launch_bounds__(RowGroup<G>::THREADS) void k_block_norm(BlockArgs a) {
  typedef RowGroup<G> R;
  __shared__ uint32_t red[2 * (G > 64 ? G / 64 : 1)];
  int turn = 0;
  // (a row's lanes stay together: rows of several waves own their workgroup)
  for (int64_t row = blockIdx.x * (int64_t)R::ROWS + threadIdx.x / G; row < a.M;
       row += gridDim.x * (int64_t)R::ROWS)
    block_row<XT, BT, G, U>(a, row, red, turn);
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
  if (a.F <= 64) return launch<XT, BT, 8, 1>(a, st);
  if (a.F <= 128) return launch<XT, BT, 16, 1>(a, st);
  if (a.F <= 256) return launch<XT, BT, 32, 1>(a, st);
  if (a.F <= 512) return launch<XT, BT, 64, 1>(a, st);
  if (a.F <= 1024) return launch<XT, BT, 64, 2>(a, st);
  if (a.F <= 2048) return launch<XT, BT, 256, 1>(a, st);
  if (a.F <= 4096) return launch<XT, BT, 256, 2>(a, st);
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
