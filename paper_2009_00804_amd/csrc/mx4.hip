// Rows in microscaled 4-bit floating point and products of them:
// out = act(rs * (sum_k a_ik w_jk) + bias_j).  Both operands are rows of k (w: one
// output channel a row).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gemm_device.h"
#include "mx4_device.h"

namespace saga {
namespace {

constexpr int64_t kMostBlocks = 1 << 20;  // (a grid holds less than 2^32 threads)

// --------------------------------------------------------------------------
// float rows to 4-bit rows and back: G lanes a row, 8 columns a lane; the four lanes
// of a block join their largest magnitudes.
// --------------------------------------------------------------------------
template <typename T, int G>
__global__ __launch_bounds__(256) void k_quantize_mx4(Mx4RowsArgs a) {
  const int64_t bytes = (a.K + 1) / 2, end = (a.K + 31) / 32 * 32;
  for (int64_t row = blockIdx.x * (int64_t)(256 / G) + threadIdx.x / G; row < a.M;
       row += gridDim.x * (int64_t)(256 / G)) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    uint8_t* q = a.q + row * a.ldq;
    for (int64_t col = (threadIdx.x % G) * 8; col < end; col += G * 8) {
      const int left = (int)min(a.K - col, (int64_t)8);
      Raw<T> v;
      v.load(x + col, left);
      v.clear(left);
      uint32_t top = v.top();
      top = max(top, dpp_mov<0xB1>(top));  // quad_perm [1,0,3,2]
      top = max(top, dpp_mov<0x4E>(top));  // quad_perm [2,3,0,1]
      const BlockScale s = block_scale(top);
      const uint32_t o = round_mx4(v, s);
      const int64_t at = col / 2;
      if (at + 4 <= bytes) {
        *reinterpret_cast<uint32_t*>(q + at) = o;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at + j < bytes) q[at + j] = (uint8_t)(o >> (8 * j));
      }
      if ((threadIdx.x & 3) == 0) a.scale[row * a.lds + col / 32] = (uint8_t)s.byte;
    }
  }
}

template <typename T, int G>
__global__ __launch_bounds__(256) void k_dequantize_mx4(Mx4RowsArgs a) {
  const int64_t bytes = (a.K + 1) / 2;
  for (int64_t row = blockIdx.x * (int64_t)(256 / G) + threadIdx.x / G; row < a.M;
       row += gridDim.x * (int64_t)(256 / G)) {
    T* x = static_cast<T*>(const_cast<void*>(a.x)) + row * a.ldx;
    const uint8_t* q = a.q + row * a.ldq;
    for (int64_t col = (threadIdx.x % G) * 8; col < a.K; col += G * 8) {
      uint32_t o = 0;
      if (col / 2 < bytes) o = *reinterpret_cast<const uint32_t*>(q + col / 2);  // (rows are whole 16 bytes)
      const uint32_t byte = a.scale[row * a.lds + col / 32];
      const float s = byte == 255u ? __uint_as_float(0x7fc00000u)
                                   : __uint_as_float(byte ? byte << 23 : 0x00400000u);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = o >> (4 * j), e = (c >> 1) & 3u, m = c & 1u;
        const float mag = e ? __uint_as_float((126u + e) << 23 | m << 22) : (m ? 0.5f : 0.0f);
        v[j] = ((c & 8u) ? -mag : mag) * s;
      }
      store_unit(x + col, a.K - col, v);
    }
  }
}

// --------------------------------------------------------------------------
// product: 16 rows and 16 channels a workgroup, k divided among its eight waves.  A
// lane takes its blocks of a and w straight from memory; float rows are rounded in
// its registers, since the 32 columns that a matrix instruction wants of a lane are
// a block.
// --------------------------------------------------------------------------
// four neighbouring channels n.. of row m: scale, bias, activation, rounding
__device__ __forceinline__ void store_quad(const Mx4GemmArgs& g, int64_t m, int64_t n, const f32x4& sum, float rs,
                                           const f32x4& tb) {
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = sum[j] * rs + tb[j];
  if (g.act == SAGA_ACT_RELU) {
    // (a NaN stays: it is all that is left of a row that held no number; -0 becomes +0)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_elementwise_maximum(v[j], 0.0f);
  } else if (g.act != SAGA_ACT_NONE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = apply_act(g.act, v[j]);
  }
  if (g.out_dtype == SAGA_BF16) {
    uint16_t* o = static_cast<uint16_t*>(g.out) + m * g.ldo + n;
    if (n + 4 <= g.N) {
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < g.N) o[j] = f32_to_bf16(v[j]);
    }
  } else {
    float* o = static_cast<float*>(g.out) + m * g.ldo + n;
    if (n + 4 <= g.N) {
      *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < g.N) o[j] = v[j];
    }
  }
}

__device__ __forceinline__ f32x4 bias_quad(const Mx4GemmArgs& g, int64_t n) {
  f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (g.bias && n + j < g.N) b[j] = g.bias[n + j];
  return b;
}

template <typename T>
__global__ __launch_bounds__(512) void k_mx4_few(Mx4GemmArgs g, int64_t tiles_m, int64_t tiles) {
  constexpr int NW = 8;
  __shared__ f32x4 part[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15, K = (int)g.K;
  const int steps = (K + 127) / 128, per = (steps + NW - 1) / NW, s0 = wave * per, s1 = min(steps, s0 + per);
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t m0 = t % tiles_m * 16, n0 = t / tiles_m * 16;
    RowSource<T> a;
    RowSource<uint8_t> w;
    a.at(g.a, g.lda, g.a_scale, g.lda_s, min(m0 + lr, g.M - 1));  // (rows past the last: not stored)
    w.at(g.w, g.ldw, g.w_scale, g.ldw_s, min(n0 + lr, g.N - 1));
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = s0; s < s1; ++s) {
      const int b = s * 4 + quarter;
      a.load(b, K);
      w.load(b, K);
      acc = mma_mx4(w.take(b, K), a.take(b, K), acc);
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int k = 1; k < NW; ++k) acc += part[k][lane];
      const int64_t m = m0 + lr, n = n0 + quarter * 4;
      if (m < g.M && n < g.N)
        store_quad(g, m, n, acc, g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[m]) : 1.0f, bias_quad(g, n));
    }
    __syncthreads();
  }
}

template <typename T>
hipError_t launch_few(const Mx4GemmArgs& g, hipStream_t st) {
  const int64_t tm = (g.M + 15) / 16, tiles = tm * ((g.N + 15) / 16);
  hipLaunchKernelGGL((k_mx4_few<T>), dim3((unsigned)std::min(tiles, kMostBlocks)), dim3(512), 0, st, g, tm, tiles);
  return hipGetLastError();
}

template <typename T>
hipError_t rows_mx4(const Mx4RowsArgs& a, bool back, hipStream_t st) {
  const auto go = [&](auto kernel, int rows) {
    const int64_t blocks = std::min<int64_t>((a.M + rows - 1) / rows, kMostBlocks);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, a);
    return hipGetLastError();
  };
  if (a.K <= 1024) return back ? go(k_dequantize_mx4<T, 16>, 16) : go(k_quantize_mx4<T, 16>, 16);
  return back ? go(k_dequantize_mx4<T, 256>, 1) : go(k_quantize_mx4<T, 256>, 1);
}

}  // namespace

hipError_t launch_rows_mx4(const Mx4RowsArgs& a, bool back, hipStream_t st) {
  if (a.M == 0) return hipSuccess;
  return a.dtype == SAGA_BF16 ? rows_mx4<uint16_t>(a, back, st) : rows_mx4<float>(a, back, st);
}

size_t mx4_workspace_bytes(int, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_gemm_mx4(const Mx4GemmArgs& g, hipStream_t st) {
  if (g.M == 0) return hipSuccess;
  if (g.a_dtype == SAGA_MX4) return launch_few<uint8_t>(g, st);
  return g.a_dtype == SAGA_BF16 ? launch_few<uint16_t>(g, st) : launch_few<float>(g, st);
}

}  // namespace saga
