// A layer of experts over a few rows: a router chooses top_k experts of each row, an
// expert is two products with an activation (or a gate) between them, and a row's
// results are summed by the router's weights.
//
// The rows' float values go through the matrix cores as sums of bfloat16 terms (one for
// bfloat16 rows, three for float32 ones, which is exact; the values between the products
// two and three), the experts' weights as bfloat16 values, which hold a 4-bit value times
// its scale exactly.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gemm_device.h"
#include "mx4_device.h"

namespace saga {
namespace {

// --------------------------------------------------------------------------
// router: a workgroup a row.  Logits are float64 sums: which expert a row takes hangs
// on which of two close values is larger, so the products' rounding must not decide.
// --------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// x as terms bfloat16 values, each the rest cut to 8 bits of its mantissa: three hold a float32
__device__ __forceinline__ uint32_t cut_term(float& rest) {
  const uint32_t hi = __float_as_uint(rest) & 0xffff0000u;
  rest -= __uint_as_float(hi);
  return hi;
}

template <typename T, typename TR>
__global__ __launch_bounds__(256) void k_route(ExpertArgs a) {
  __shared__ double logits[kExpertsMax];
  __shared__ int bad_row;
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, F = a.F;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  if (threadIdx.x == 0) bad_row = 0;
  __syncthreads();

  // the row's terms, and whether it holds numbers only
  bool bad = false;
  for (int c = threadIdx.x * 8; c < a.ld_xt; c += 2048) {
    Raw<T> v;
    v.load(x + c, F - c);
    v.clear(F - c);
    bad |= v.top() >= 0x7f800000u;
    float f[8];
    v.widen(f);
    for (int t = 0; t < a.x_terms; ++t) {
      u32x4 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = cut_term(f[2 * j]), hi = cut_term(f[2 * j + 1]);
        o[j] = lo >> 16 | hi;
      }
      *reinterpret_cast<u32x4*>(a.xt + (t * a.M + row) * a.ld_xt + c) = o;
    }
  }
  for (int e = wave; e < a.E; e += 4) {
    const TR* r = static_cast<const TR*>(a.router) + e * a.ld_router;
    double sum = 0.0;
    for (int c = lane * 8; c < F; c += 512) {
      Raw<T> v;
      Raw<TR> w;
      v.load(x + c, F - c);
      w.load(r + c, F - c);
      v.clear(F - c);
      w.clear(F - c);
      float f[8], g[8];
      v.widen(f);
      w.widen(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fma((double)f[j], (double)g[j], sum);
    }
    sum = wave_sum(sum);
    if (a.router_bias) sum += (double)a.router_bias[e];
    if (lane == 0) logits[e] = sum;
    bad |= !(sum < (double)INFINITY);
  }
  if (bad) bad_row = 1;
  __syncthreads();
  if (wave != 0) return;
  const double low = -(double)INFINITY;
  double total = 0.0, top = 0.0;
  float mine = 0.0f;      // lane j: of the j-th choice
  int chosen = -1;
  for (int k = 0; k < a.top_k; ++k) {
    double best = low;
    int at = -1;
    for (int e = lane; e < a.E; e += 64) {
      const double v = logits[e];
      if (v > best) best = v, at = e;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double v = __shfl_xor(best, d);
      const int e = __shfl_xor(at, d);
      if (v > best || (v == best && (uint32_t)e < (uint32_t)at)) best = v, at = e;
    }
    if (k == 0) {
      top = at >= 0 ? best : 0.0;
      if (!a.renormalise) {
        for (int e = lane; e < a.E; e += 64) total += (double)expf((float)(logits[e] - top));
        total = wave_sum(total);
      }
    }
    const float p = at >= 0 ? expf((float)(best - top)) : 0.0f;
    if (a.renormalise) total += (double)p;
    if (lane == k) chosen = at, mine = p;
    if (at >= 0 && lane == (at & 63)) logits[at] = low;
    __builtin_amdgcn_wave_barrier();
  }
  if (lane < a.top_k) {
    float p = chosen >= 0 ? (float)((double)mine / total) : 0.0f;
    if (bad_row) chosen = -1, p = __uint_as_float(0x7fc00000u);
    a.index[row * a.top_k + lane] = chosen;
    a.weight[row * a.top_k + lane] = p;
  }
}

// --------------------------------------------------------------------------
// an expert's product: 16 channels of one expert and the rows that take it, 16 at a
// time, k divided among four waves.
// --------------------------------------------------------------------------
// 32 k of a channel as four groups of 8 bfloat16 values
template <bool MX4>
struct WeightBlock;
template <>
struct WeightBlock<true> {
  RowSource<uint8_t> s;
  __device__ __forceinline__ void at(const void* w, int64_t ld, const uint8_t* scale, int64_t lds, int64_t row) {
    s.at(w, ld, scale, lds, row);
  }
  __device__ __forceinline__ void load(int b, int K) { s.load(b, K); }
  __device__ __forceinline__ void take(int b, int K, bf16x8 (&o)[4]) {
    const Mx4Block m = s.take(b, K);
    const float f = __uint_as_float(m.scale == 255u ? 0x7fc00000u : m.scale ? m.scale << 23 : 0x00400000u);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(m.v[t], f, 0),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(m.v[t], f, 1),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(m.v[t], f, 2),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(m.v[t], f, 3)};
      __builtin_memcpy(&o[t], p, 16);
    }
  }
};
template <>
struct WeightBlock<false> {
  const uint16_t* p;
  Raw<uint16_t> v[4];
  __device__ __forceinline__ void at(const void* w, int64_t ld, const uint8_t*, int64_t, int64_t row) {
    p = static_cast<const uint16_t*>(w) + row * ld;
  }
  __device__ __forceinline__ void load(int b, int K) {
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t].load(p + b * 32 + t * 8, K - b * 32 - t * 8);
  }
  __device__ __forceinline__ void take(int b, int K, bf16x8 (&o)[4]) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v[t].clear(K - b * 32 - t * 8);
      __builtin_memcpy(&o[t], &v[t].v, 16);
    }
  }
};

// This workgroup's expert (-1: none) and its pairs (row * top_k + place), in order.
// Up to E pairs a slot is a pair, which stands for its expert if no earlier pair does;
// otherwise a slot is an expert.
__device__ __forceinline__ int slot_expert(const ExpertArgs& a, int slot, int* list, int& count) {
  const int pairs = (int)(a.M * a.top_k);
  const bool by_pair = pairs <= a.E;
  const int e = by_pair ? a.index[slot] : slot;
  __shared__ int base, seen;
  if (threadIdx.x == 0) base = 0, seen = 0;
  __syncthreads();
  if (e < 0) return -1;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int p0 = 0; p0 < pairs; p0 += blockDim.x) {
    const int p = p0 + threadIdx.x;
    const bool mine = p < pairs && a.index[p] == e;
    if (by_pair && mine && p < slot) seen = 1;
    const uint64_t all = __ballot(mine);
    for (int w = 0; w < waves; ++w) {  // (in order, wave by wave)
      if (w == wave) {
        if (mine) list[base + __popcll(all & lanemask_lt())] = p;
      }
      __syncthreads();
      if (w == wave && lane == 0) base += __popcll(all);
      __syncthreads();
    }
  }
  count = base;
  return seen || count == 0 ? -1 : e;
}

template <bool MX4, int TERMS, bool UP, bool GATED>
__global__ __launch_bounds__(256) void k_expert_product(ExpertArgs a) {
  constexpr int NW = 4, NO = GATED ? 2 : 1;
  __shared__ int list[kExpertRows];
  __shared__ f32x4 part[NW][NO][64];
  int count;
  const int e = slot_expert(a, blockIdx.y, list, count);
  if (e < 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15;
  const int K = UP ? a.F : a.H, N = UP ? a.H : a.N, n0 = blockIdx.x * 16, steps = (K + 127) / 128;
  const int64_t ld = UP ? a.ld_xt : a.ld_ht, plane = (UP ? a.M : a.M * a.top_k) * ld;
  const uint16_t* const rows = UP ? a.xt : a.ht;
  WeightBlock<MX4> w[NO];
#pragma unroll
  for (int o = 0; o < NO; ++o) {
    const int64_t r = (int64_t)e * N * NO + (int64_t)o * N + min(n0 + lr, N - 1);
    if (UP) w[o].at(a.up, a.ld_up, a.up_scale, a.lds_up, r);
    else w[o].at(a.down, a.ld_down, a.down_scale, a.lds_down, r);
  }
  for (int i0 = 0; i0 < count; i0 += 16) {
    const int pair = list[min(i0 + lr, count - 1)];
    const uint16_t* const x = rows + (UP ? pair / a.top_k : pair) * ld;
    f32x4 acc[NO];
#pragma unroll
    for (int o = 0; o < NO; ++o) acc[o] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = wave; s < steps; s += NW) {
      const int b = s * 4 + quarter;
      bf16x8 wv[NO][4];
#pragma unroll
      for (int o = 0; o < NO; ++o) w[o].load(b, K);
#pragma unroll
      for (int o = 0; o < NO; ++o) w[o].take(b, K, wv[o]);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int k = b * 32 + t * 8;
#pragma unroll
        for (int p = 0; p < TERMS; ++p) {
          u32x4 v = {0u, 0u, 0u, 0u};
          if (k < ld) v = *reinterpret_cast<const u32x4*>(x + p * plane + k);
          bf16x8 xv;
          __builtin_memcpy(&xv, &v, 16);
#pragma unroll
          for (int o = 0; o < NO; ++o)
            acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[o][t], xv, acc[o], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int o = 0; o < NO; ++o) part[wave][o][lane] = acc[o];
    __syncthreads();
    if (wave == 0) {
      const int n = n0 + quarter * 4;
#pragma unroll
      for (int o = 0; o < NO; ++o)
#pragma unroll
        for (int k = 1; k < NW; ++k) acc[o] += part[k][o][lane];
      if (i0 + lr < count) {
        if constexpr (UP) {
          uint32_t term[3][4];
          const float* bias = a.up_bias ? a.up_bias + (int64_t)e * N * NO : nullptr;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float v = 0.0f;
            if (n + j < N) {
              v = apply_act(a.act, acc[0][j] + (bias ? bias[n + j] : 0.0f));
              if constexpr (GATED) v *= acc[NO - 1][j] + (bias ? bias[N + n + j] : 0.0f);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              // (the last term is rounded: of three it holds what is left)
              if (t + 1 == a.h_terms) term[t][j] = (uint32_t)f32_to_bf16(v) << 16;
              else term[t][j] = cut_term(v);
            }
            term[2][j] = (uint32_t)f32_to_bf16(v) << 16;
          }
          if (n < a.ld_ht)
            for (int t = 0; t < a.h_terms; ++t)
              *reinterpret_cast<uint2*>(a.ht + (t * a.M * a.top_k + pair) * a.ld_ht + n) =
                  make_uint2(term[t][0] >> 16 | term[t][1], term[t][2] >> 16 | term[t][3]);
        } else if (n < N) {
          *reinterpret_cast<f32x4*>(a.part + pair * a.ld_part + n) = acc[0];
        }
      }
    }
    __syncthreads();
  }
}

// out = sum of a row's choices by their weights, in the order of the choices
__global__ __launch_bounds__(256) void k_expert_sum(ExpertArgs a) {
  const int64_t quads = a.ld_part / 4, all = a.M * quads;
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < all; i += gridDim.x * (int64_t)256) {
    const int64_t row = i / quads;
    const int n = (int)(i % quads) * 4;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < a.top_k; ++k) {
      const int64_t pair = row * a.top_k + k;
      const int e = a.index[pair];
      const float p = a.weight[pair];
      f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
      if (e >= 0) d = *reinterpret_cast<const f32x4*>(a.part + pair * a.ld_part + n);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (e >= 0 && a.down_bias && n + j < a.N) d[j] += a.down_bias[(int64_t)e * a.N + n + j];
        v[j] = fmaf(p, d[j], v[j]);  // (a row without numbers: p is NaN)
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (n + j >= a.N) continue;
      if (a.dtype == SAGA_BF16) static_cast<uint16_t*>(a.out)[row * a.ldo + n + j] = f32_to_bf16(v[j]);
      else static_cast<float*>(a.out)[row * a.ldo + n + j] = v[j];
    }
  }
}

template <bool MX4>
hipError_t products(const ExpertArgs& a, hipStream_t st) {
  const unsigned slots = (unsigned)std::min<int64_t>(a.M * a.top_k, a.E);
  const dim3 up((unsigned)((a.H + 15) / 16), slots), down((unsigned)((a.N + 15) / 16), slots);
  const auto go = [&](auto kernel, dim3 grid) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
    return hipGetLastError();
  };
  hipError_t e;
  if (a.gated) e = a.x_terms == 1 ? go(k_expert_product<MX4, 1, true, true>, up) : go(k_expert_product<MX4, 3, true, true>, up);
  else e = a.x_terms == 1 ? go(k_expert_product<MX4, 1, true, false>, up) : go(k_expert_product<MX4, 3, true, false>, up);
  if (e != hipSuccess) return e;
  return a.h_terms == 2 ? go(k_expert_product<MX4, 2, false, false>, down) : go(k_expert_product<MX4, 3, false, false>, down);
}

size_t whole(size_t n) { return (n + 255) & ~(size_t)255; }

// the parts of the workspace, of up to kExpertRows rows
struct ExpertSpace {
  int64_t rows, ld_xt, ld_ht, ld_part;
  int x_terms, h_terms;
  size_t xt, ht, part, total;
};
ExpertSpace expert_space(int dtype, int64_t M, int64_t F, int64_t H, int64_t N, int top_k) {
  ExpertSpace s;
  s.rows = std::min<int64_t>(M, kExpertRows);
  s.x_terms = dtype == SAGA_BF16 ? 1 : 3;
  s.h_terms = dtype == SAGA_BF16 ? 2 : 3;
  s.ld_xt = (F + 15) / 16 * 16;
  s.ld_ht = (H + 15) / 16 * 16;
  s.ld_part = (N + 3) / 4 * 4;
  s.xt = 0;
  s.ht = s.xt + whole((size_t)s.x_terms * s.rows * s.ld_xt * 2);
  s.part = s.ht + whole((size_t)s.h_terms * s.rows * top_k * s.ld_ht * 2);
  s.total = s.part + whole((size_t)s.rows * top_k * s.ld_part * 4);
  return s;
}

}  // namespace

size_t experts_workspace_bytes(int dtype, int64_t M, int64_t F, int64_t H, int64_t N, int top_k) {
  return M == 0 ? 0 : expert_space(dtype, M, F, H, N, top_k).total;
}

hipError_t launch_experts(const ExpertArgs& a0, hipStream_t st) {
  if (a0.M == 0) return hipSuccess;
  const ExpertSpace s = expert_space(a0.dtype, a0.M, a0.F, a0.H, a0.N, a0.top_k);
  const size_t es = a0.dtype == SAGA_BF16 ? 2 : 4;
  for (int64_t m = 0; m < a0.M; m += s.rows) {
    ExpertArgs a = a0;
    a.M = std::min(s.rows, a0.M - m);
    a.x = static_cast<const char*>(a0.x) + m * a0.ldx * es;
    a.out = static_cast<char*>(a0.out) + m * a0.ldo * es;
    a.index += m * a0.top_k;
    a.weight += m * a0.top_k;
    char* const ws = static_cast<char*>(a0.ws);
    a.xt = reinterpret_cast<uint16_t*>(ws + s.xt);
    a.ht = reinterpret_cast<uint16_t*>(ws + s.ht);
    a.part = reinterpret_cast<float*>(ws + s.part);
    a.ld_xt = s.ld_xt;
    a.ld_ht = s.ld_ht;
    a.ld_part = s.ld_part;
    a.x_terms = s.x_terms;
    a.h_terms = s.h_terms;
    const auto route = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)a.M), dim3(256), 0, st, a);
      return hipGetLastError();
    };
    hipError_t e;
    if (a.dtype == SAGA_BF16)
      e = a.router_dtype == SAGA_BF16 ? route(k_route<uint16_t, uint16_t>) : route(k_route<uint16_t, float>);
    else
      e = a.router_dtype == SAGA_BF16 ? route(k_route<float, uint16_t>) : route(k_route<float, float>);
    if (e != hipSuccess) return e;
    e = a.weight_dtype == SAGA_MX4 ? products<true>(a, st) : products<false>(a, st);
    if (e != hipSuccess) return e;
    const int64_t quads = a.M * (a.ld_part / 4);
    hipLaunchKernelGGL(k_expert_sum, dim3((unsigned)std::min<int64_t>((quads + 255) / 256, 1 << 16)), dim3(256), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace saga
