// A layer of experts over a few rows: a router chooses top_k experts of each row, an
// expert is two products with an activation (or a gate) between them, and a row's
// results are summed by the router's weights.
//
// The rows' float values go through the matrix cores as sums of bfloat16 terms (one for
// bfloat16 rows, three for float32 ones, which is exact down to 2^-133; the values between the products
// two and three), the experts' weights as bfloat16 values, which hold a 4-bit value times
// its scale exactly.
//
// Two terms hold the values between the products of bfloat16 rows to 2^-16, a 256th of the half step that the
// result is rounded by.  With three the errors against float64 are the same to five digits (1.6623e-3 of the results' size,
// 512 rows of 32 experts of 2048 x 4096), 0.12 % of the results and not 0.47 % differ from those of a
// float32 product by a step, and the layer takes 267 us and not 221 (64 rows of 64 experts of 1024 x 4096 127
// and 119, a row 26.7 and 24.0).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gemm_device.h"
#include "mx4_device.h"

namespace saga {
namespace {

// x as terms bfloat16 values, each the rest cut to 8 bits of its mantissa: three hold a float32
__device__ __forceinline__ uint32_t cut_term(float& rest) {
  const uint32_t hi = __float_as_uint(rest) & 0xffff0000u;
  rest -= __uint_as_float(hi);
  return hi;
}

// the terms of 8 columns of a row
template <typename T>
__device__ __forceinline__ void store_terms(const ExpertArgs& a, int64_t row, int c, const Raw<T>& v) {
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

// --------------------------------------------------------------------------
// router: a workgroup a row.  Logits are float64 sums: which expert a row takes hangs
// on which of two close values is larger, so the products' rounding must not decide.
// A wave takes kTogether experts at a time, which share the row's values and whose loads
// are on their way together; the choice is a rank by counting, a thread an expert.  64 rows and
// experts of 1024 columns take 8.4 us (24 with an expert at a time), 512 rows and 32 experts of 2048 15.
// --------------------------------------------------------------------------
constexpr int kTogether = 4;

// 64 lanes' sums of C values; the steps of different values run side by side
template <int C>
__device__ __forceinline__ void wave_sums(double (&v)[C]) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] += __shfl_xor(v[i], d);
}

// logits[e] = x . router_e + bias_e for all experts; true: one that is NaN or +inf
template <typename T, typename TR, int NW, int C>
__device__ __forceinline__ bool route_logits(const ExpertArgs& a, const T* x, double* logits) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, F = a.F;
  bool bad = false;
  for (int e0 = wave * C; e0 < a.E; e0 += NW * C) {
    double sum[C] = {};
    for (int c = lane * 8; c < F; c += 512) {
      Raw<T> v;
      Raw<TR> w[C];
      v.load(x + c, F - c);
#pragma unroll
      for (int i = 0; i < C; ++i)
        w[i].load(static_cast<const TR*>(a.router) + min(e0 + i, a.E - 1) * a.ld_router + c, F - c);
      v.clear(F - c);
      float f[8];
      v.widen(f);
#pragma unroll
      for (int i = 0; i < C; ++i) {
        w[i].clear(F - c);
        float g[8];
        w[i].widen(g);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[i] = fma((double)f[j], (double)g[j], sum[i]);
      }
    }
    wave_sums(sum);
#pragma unroll
    for (int i = 0; i < C; ++i) {
      if (e0 + i >= a.E) break;
      if (a.router_bias) sum[i] += (double)a.router_bias[e0 + i];
      if (lane == 0) logits[e0 + i] = sum[i];
      bad |= !(sum[i] < (double)INFINITY);
    }
  }
  return bad;
}

// The choices of a row by its logits, with THREADS threads; the workgroup's own memory
struct RouteSpace {
  double logits[kExpertsMax];
  double top, share[16];
  double best[SAGA_MAX_CHOICES];
  int chosen[SAGA_MAX_CHOICES];
  int bad;
};
template <int THREADS>
__device__ __forceinline__ void route_choose(const ExpertArgs& a, RouteSpace& s, int32_t* index, float* weight) {
  const int tid = threadIdx.x;
  if (tid < SAGA_MAX_CHOICES) s.chosen[tid] = -1;
  __syncthreads();
  for (int e = tid; e < a.E; e += THREADS) {
    const double v = s.logits[e];
    if (!(v > -(double)INFINITY)) continue;
    int rank = 0;
    for (int i = 0; i < a.E; ++i) {
      const double o = s.logits[i];
      rank += o > v || (o == v && i < e);
    }
    if (rank < a.top_k) s.chosen[rank] = e, s.best[rank] = v;
  }
  __syncthreads();
  const bool any = s.chosen[0] >= 0;
  const double top = any ? s.best[0] : 0.0;
  if (!a.renormalise) {
    double part = 0.0;
    for (int e = tid; e < a.E; e += THREADS) part += (double)expf((float)(s.logits[e] - top));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) part += __shfl_xor(part, d);
    if ((tid & 63) == 0) s.share[tid >> 6] = part;
    __syncthreads();
  }
  if (tid < a.top_k) {
    double total = 0.0;
    if (a.renormalise) {
      for (int k = 0; k < a.top_k; ++k)
        if (s.chosen[k] >= 0) total += (double)expf((float)(s.best[k] - top));
    } else {
      for (int w = 0; w < THREADS / 64; ++w) total += s.share[w];
    }
    int chosen = s.chosen[tid];
    float p = chosen >= 0 ? (float)((double)expf((float)(s.best[tid] - top)) / total) : 0.0f;
    if (s.bad) chosen = -1, p = __uint_as_float(0x7fc00000u);
    index[tid] = chosen;
    weight[tid] = p;
  }
}

constexpr int kRouteThreads = 1024;
template <typename T, typename TR>
__global__ __launch_bounds__(kRouteThreads) void k_route(ExpertArgs a) {
  __shared__ RouteSpace s;
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  if (threadIdx.x == 0) s.bad = 0;
  if (row == 0 && threadIdx.x < 8) a.zeros[threadIdx.x] = 0;
  __syncthreads();
  // the row's terms, and whether it holds numbers only
  bool bad = false;
  for (int c = threadIdx.x * 8; c < a.ld_xt; c += kRouteThreads * 8) {
    Raw<T> v;
    v.load(x + c, a.F - c);
    v.clear(a.F - c);
    bad |= v.top() >= 0x7f800000u;
    store_terms(a, row, c, v);
  }
  bad |= route_logits<T, TR, kRouteThreads / 64, kTogether>(a, x, s.logits);
  if (bad) s.bad = 1;
  __syncthreads();
  route_choose<kRouteThreads>(a, s, a.index + row * a.top_k, a.weight + row * a.top_k);
}

// where a lane reads its channel's weights
template <bool MX4>
struct WeightRow {
  const uint8_t *q, *s;
  __device__ __forceinline__ void at(const void* w, int64_t ld, const uint8_t* scale, int64_t lds, int64_t row) {
    q = static_cast<const uint8_t*>(w) + row * ld * (MX4 ? 1 : 2);
    s = MX4 ? scale + row * lds : nullptr;
  }
};
template <bool MX4, bool UP>
__device__ __forceinline__ WeightRow<MX4> weight_row(const ExpertArgs& a, int64_t row) {
  WeightRow<MX4> r;
  if (UP) r.at(a.up, a.ld_up, a.up_scale, a.lds_up, row);
  else r.at(a.down, a.ld_down, a.down_scale, a.lds_down, row);
  return r;
}

// A lane's weights of one step: J blocks of 32 k of a channel (b.. of K columns), each four
// groups of 8 bfloat16 values.  `load` has no branch, so that many run ahead: past the
// row's end it reads the row's last piece again, and `clear` has to follow in the last step
// of a row.  Two blocks of 4-bit weights are 32 bytes: four lanes take a whole line, and
// half as many loads of scales are needed.
template <bool MX4, int J>
struct WeightBlocks;
template <int J>
struct WeightBlocks<true, J> {
  static_assert(J == 1 || J == 2, "one load for the scales");
  u32x4 v[J];
  uint32_t scale;  // a byte for each block
  __device__ __forceinline__ void load(const WeightRow<true>& r, int b, int K) {
    const int most = (K - 1) / 32;
#pragma unroll
    for (int j = 0; j < J; ++j) v[j] = *reinterpret_cast<const u32x4*>(r.q + min(b + j, most) * 16);
    if constexpr (J == 1) scale = r.s[min(b, most)];
    else scale = *reinterpret_cast<const uint16_t*>(r.s + min(b, most / 2 * 2));  // (rows are whole 4 bytes)
  }
  __device__ __forceinline__ void clear(int b, int K) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int left = (K + 1) / 2 - (b + j) * 16;
      if (left < 16) v[j] = clear_bytes(v[j], left);
      if (left <= 0) scale = (scale & ~(255u << (8 * j))) | 127u << (8 * j);
    }
  }
  __device__ __forceinline__ bf16x8 take(int j, int t) const {
    const float f = scale_value(J == 1 ? scale : (scale >> (8 * j)) & 255u);
    const uint32_t d = v[j][t];
    const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, f, 0),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, f, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, f, 2),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, f, 3)};
    bf16x8 o;
    __builtin_memcpy(&o, p, 16);
    return o;
  }
};
template <>
struct WeightBlocks<false, 1> {
  Raw<uint16_t> v[4];
  __device__ __forceinline__ void load(const WeightRow<false>& r, int b, int K) {
    const int most = (K - 1) / 8 * 8;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      v[t].load(reinterpret_cast<const uint16_t*>(r.q) + min(b * 32 + t * 8, most), 8);
  }
  __device__ __forceinline__ void clear(int b, int K) {
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t].clear(K - b * 32 - t * 8);
  }
  __device__ __forceinline__ bf16x8 take(int, int t) const {
    bf16x8 o;
    __builtin_memcpy(&o, &v[t].v, 16);
    return o;
  }
};

// What a workgroup works on: `runs` parts of the weights' rows and `parts` of k for each slot.  Workgroup
// w runs on XCD w % 8: all of a slot's go to one, whose L2 then has the rows of x that they share.
struct Share {
  int slot, run, part;
};
__device__ __forceinline__ Share share_of(int slots, int runs, int parts) {
  const int i = blockIdx.x / kXcds, each = runs * parts;
  return {i / each * kXcds + (int)(blockIdx.x % kXcds), i % each % runs, i % each / runs};
}
unsigned share_blocks(int64_t slots, int64_t runs, int64_t parts) {
  return (unsigned)((slots + kXcds - 1) / kXcds * kXcds * runs * parts);
}

// This workgroup's expert (-1: none) and its pairs (row * top_k + place), in some order (no
// result depends on it).  Up to E pairs a slot is a pair, which stands for its expert if no
// earlier pair does; otherwise a slot is an expert.
template <int NW>
__device__ __forceinline__ int slot_expert(const ExpertArgs& a, int slot, int* list, int& count) {
  __shared__ int found, seen;
  const int pairs = (int)(a.M * a.top_k);
  const bool by_pair = pairs <= a.E;
  const int e = by_pair ? a.index[slot] : slot;
  if (e < 0) return -1;
  if (threadIdx.x == 0) found = seen = 0;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  constexpr int TOGETHER = 4;  // (loads on their way)
  for (int p0 = threadIdx.x - lane; p0 < pairs; p0 += NW * 64 * TOGETHER) {
    int at[TOGETHER];
#pragma unroll
    for (int j = 0; j < TOGETHER; ++j) at[j] = a.index[min(p0 + j * NW * 64 + lane, pairs - 1)];
#pragma unroll
    for (int j = 0; j < TOGETHER; ++j) {
      const int p = p0 + j * NW * 64 + lane;
      const bool mine = p < pairs && at[j] == e;
      const uint64_t all = __ballot(mine);
      if (all == 0) continue;
      if (by_pair && mine && p < slot) seen = 1;
      int base = 0;
      if (lane == 0) base = atomicAdd(&found, __popcll(all));
      base = __builtin_amdgcn_readfirstlane(base);
      if (mine) list[base + __popcll(all & lanemask_lt())] = p;
    }
  }
  __syncthreads();
  count = found;
  return seen || count == 0 ? -1 : e;
}

// e^x to about 2 units of 2^-24, x from -87 to 87: the product with log2 e has a second part
__device__ __forceinline__ float exp_in_range(float x) {
  constexpr float kLog2e = 1.44269504f, kRest = 1.92596299e-8f, kLn2 = 0.693147181f;
  const float h = x * kLog2e, l = fmaf(x, kLog2e, -h) + x * kRest, e = __builtin_amdgcn_exp2f(h);
  return fmaf(e, l * kLn2, e);
}
template <int C>
__device__ __forceinline__ void activate(int act, float (&v)[C]) {
  if (act == SAGA_ACT_SIGMOID) {  // (the values between the products are many: no call, no division)
#pragma unroll
    for (int j = 0; j < C; ++j)
      v[j] = __builtin_amdgcn_rcpf(1.0f + exp_in_range(-__builtin_elementwise_maximum(
                                              -87.0f, __builtin_elementwise_minimum(v[j], 87.0f))));
  } else if (act == SAGA_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] = __builtin_elementwise_maximum(v[j], 0.0f);  // (a NaN stays)
  } else if (act != SAGA_ACT_NONE) {
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] = apply_act(act, v[j]);
  }
}

// h of C channels n.. of a pair (C neighbours), to its terms
template <int C>
__device__ __forceinline__ void store_hidden(const ExpertArgs& a, int e, int pair, int n, float (&v)[C],
                                             const float (&up)[C]) {
  if (n >= a.ld_ht) return;
  if (a.up_bias) {
    const float* bias = a.up_bias + (int64_t)e * a.H * (a.gated ? 2 : 1);
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] += bias[min(n + j, a.H - 1)];
  }
  activate(a.act, v);
  if (a.gated) {
    const float* bias = a.up_bias ? a.up_bias + ((int64_t)e * 2 + 1) * a.H : nullptr;
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] *= up[j] + (bias ? bias[min(n + j, a.H - 1)] : 0.0f);
  }
  if (n + C > a.H)
#pragma unroll
    for (int j = 0; j < C; ++j)
      if (n + j >= a.H) v[j] = 0.0f;
  for (int t = 0; t < a.h_terms; ++t) {
    uint32_t o[C / 2];
#pragma unroll
    for (int j = 0; j < C; j += 2) {
      // (the last term is rounded: of three it holds what is left)
      if (t + 1 == a.h_terms) {
        o[j / 2] = pack_bf16(v[j], v[j + 1]);
      } else {
        const uint32_t lo = cut_term(v[j]), hi = cut_term(v[j + 1]);
        o[j / 2] = lo >> 16 | hi;
      }
    }
    uint16_t* const to = a.ht + (t * a.M * a.top_k + pair) * a.ld_ht + n;
    if constexpr (C == 8) *reinterpret_cast<u32x4*>(to) = u32x4{o[0], o[1], o[2], o[3]};
    else *reinterpret_cast<uint2*>(to) = make_uint2(o[0], o[1]);
  }
}
__device__ __forceinline__ void store_hidden(const ExpertArgs& a, int e, int pair, int n, const f32x4& first,
                                             const f32x4& second) {
  float v[4] = {first[0], first[1], first[2], first[3]};
  const float up[4] = {second[0], second[1], second[2], second[3]};
  store_hidden(a, e, pair, n, v, up);
}

// --------------------------------------------------------------------------
// an expert's product: 16 channels of one expert and the rows that take it, 16 at a
// time, k divided among four waves.  A wave's loads, of the weights and of x, are AHEAD
// steps of 128 k at a time.  The weights' zeros past a row's end make what x has there not
// count.
// --------------------------------------------------------------------------
template <bool MX4, int TERMS, bool UP, bool GATED, int AHEAD>
__global__ __launch_bounds__(256) void k_expert_few(ExpertArgs a) {
  constexpr int NW = 4, NO = GATED ? 2 : 1;
  __shared__ int list[kExpertRows];
  __shared__ f32x4 part[NW][NO][64];
  int count;
  const int e = slot_expert<NW>(a, blockIdx.y, list, count);
  if (e < 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15;
  const int K = UP ? a.F : a.H, N = UP ? a.H : a.N, n0 = blockIdx.x * 16, all = (K + 127) / 128;
  const int steps = (all - wave + NW - 1) / NW;  // of this wave: wave, wave + NW, ..
  const int64_t ld = UP ? a.ld_xt : a.ld_ht, plane = (UP ? a.M : a.M * a.top_k) * ld;
  const uint16_t* const rows = UP ? a.xt : a.ht;
  WeightRow<MX4> from[NO];
#pragma unroll
  for (int o = 0; o < NO; ++o)
    from[o] = weight_row<MX4, UP>(a, (int64_t)e * N * NO + (int64_t)o * N + min(n0 + lr, N - 1));
  for (int i0 = 0; i0 < count; i0 += 16) {
    const int pair = list[min(i0 + lr, count - 1)];
    const uint16_t* const x = rows + (UP ? pair / a.top_k : pair) * ld;
    WeightBlocks<MX4, 1> w[AHEAD][NO];
    u32x4 xv[AHEAD][4][TERMS];
    const auto load = [&](int d, int i) {
      const int b = (wave + i * NW) * 4 + quarter;
#pragma unroll
      for (int o = 0; o < NO; ++o) w[d][o].load(from[o], b, K);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int p = 0; p < TERMS; ++p)
          xv[d][t][p] = *reinterpret_cast<const u32x4*>(x + p * plane + min(b * 32 + t * 8, (int)ld - 8));
    };
    f32x4 acc[NO];
#pragma unroll
    for (int o = 0; o < NO; ++o) acc[o] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int ib = 0; ib < steps; ib += AHEAD) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) load(d, ib + d);
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) {
        const int i = ib + d;
        if (i < steps) {
          const int b = (wave + i * NW) * 4 + quarter;
          if (wave + i * NW == all - 1)
#pragma unroll
            for (int o = 0; o < NO; ++o) w[d][o].clear(b, K);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            bf16x8 wv[NO];
#pragma unroll
            for (int o = 0; o < NO; ++o) wv[o] = w[d][o].take(0, t);
#pragma unroll
            for (int p = 0; p < TERMS; ++p) {
              bf16x8 v;
              __builtin_memcpy(&v, &xv[d][t][p], 16);
#pragma unroll
              for (int o = 0; o < NO; ++o) acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[o], v, acc[o], 0, 0, 0);
            }
          }
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
          store_hidden(a, e, pair, n, acc[0], acc[NO - 1]);
        } else if (n < N) {
          *reinterpret_cast<f32x4*>(a.part + pair * a.ld_part + n) = acc[0];
        }
      }
    }
    __syncthreads();
  }
}

// --------------------------------------------------------------------------
// a layer of few rows (at most 16, and 64 pairs) in two kernels: the latency of each counts (one row
// of 4 experts of 128 x 256: 7.3 and 5.4 us, 4 launches took 17 with the gaps between them; of 8 of
// 1024 x 4096 12 and 12).
// The first chooses the experts itself where that is little work (FUSED; every workgroup
// does, the first one's choice is the result), takes x as it is, and writes h.  The second
// has 16 channels of out for all rows a workgroup: its waves share the k of all experts
// that are taken, and sum by the choices' weights.
// --------------------------------------------------------------------------
constexpr int kFewRows = 16, kFewPairs = 64;

// 8 columns of x as terms
__device__ __forceinline__ void split_unit(const Raw<uint16_t>& x, bf16x8 (&o)[1]) { __builtin_memcpy(&o[0], &x.v, 16); }
__device__ __forceinline__ void split_unit(const Raw<float>& x, bf16x8 (&o)[3]) {
  float f[8];
  x.widen(f);
#pragma unroll
  for (int t = 0; t < 3; ++t) {
    u32x4 d;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = cut_term(f[2 * j]), hi = cut_term(f[2 * j + 1]);
      d[j] = lo >> 16 | hi;
    }
    __builtin_memcpy(&o[t], &d, 16);
  }
}

template <bool MX4, typename T, bool GATED, bool FUSED>
__global__ __launch_bounds__(512) void k_expert_up_few(ExpertArgs a) {
  constexpr int NW = 8, NO = GATED ? 2 : 1, TERMS = sizeof(T) == 2 ? 1 : 3, AHEAD = 2;
  __shared__ f32x4 part[NW][NO][64];
  __shared__ int index[kFewPairs], list[NW][kFewRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15, pairs = (int)a.M * a.top_k, slot = blockIdx.y;
  if constexpr (FUSED) {
    __shared__ RouteSpace s;
    __shared__ float weight[kFewPairs];
    for (int row = 0; row < (int)a.M; ++row) {
      const T* x = static_cast<const T*>(a.x) + row * a.ldx;
      if (threadIdx.x == 0) s.bad = 0;
      __syncthreads();
      bool bad = false;
      for (int c = threadIdx.x * 8; c < a.F; c += 512 * 8) {
        Raw<T> v;
        v.load(x + c, a.F - c);
        v.clear(a.F - c);
        bad |= v.top() >= 0x7f800000u;
      }
      bad |= a.router_dtype == SAGA_BF16 ? route_logits<T, uint16_t, NW, 1>(a, x, s.logits)
                                         : route_logits<T, float, NW, 1>(a, x, s.logits);
      if (bad) s.bad = 1;
      __syncthreads();
      route_choose<512>(a, s, index + row * a.top_k, weight + row * a.top_k);
      __syncthreads();
    }
    if (blockIdx.x == 0 && slot == 0 && (int)threadIdx.x < pairs) {
      a.index[threadIdx.x] = index[threadIdx.x];
      a.weight[threadIdx.x] = weight[threadIdx.x];
    }
  } else {
    if ((int)threadIdx.x < pairs) index[threadIdx.x] = a.index[threadIdx.x];
    __syncthreads();
  }
  const bool by_pair = pairs <= a.E;
  const int e = __builtin_amdgcn_readfirstlane(by_pair ? index[slot] : slot);
  if (e < 0) return;
  const bool mine = lane < pairs && index[lane] == e;
  const uint64_t all_mine = __ballot(mine);
  if (all_mine == 0 || (by_pair && __ffsll((unsigned long long)all_mine) - 1 < slot)) return;
  const int count = __popcll(all_mine);
  if (mine) list[wave][__popcll(all_mine & lanemask_lt())] = lane;
  asm volatile("" ::: "memory");
  const int pair = list[wave][min(lr, count - 1)];

  const int K = a.F, n0 = blockIdx.x * 16, all = (K + 127) / 128;
  const int steps = (all - wave + NW - 1) / NW;  // of this wave: wave, wave + NW, ..
  const T* const x = static_cast<const T*>(a.x) + pair / a.top_k * a.ldx;
  WeightRow<MX4> from[NO];
#pragma unroll
  for (int o = 0; o < NO; ++o)
    from[o] = weight_row<MX4, true>(a, (int64_t)e * a.H * NO + (int64_t)o * a.H + min(n0 + lr, a.H - 1));
  WeightBlocks<MX4, 1> w[AHEAD][NO];
  Raw<T> xv[AHEAD][4];
  const auto load = [&](int d, int i) {
    const int b = (wave + i * NW) * 4 + quarter;
#pragma unroll
    for (int o = 0; o < NO; ++o) w[d][o].load(from[o], b, K);
#pragma unroll
    for (int t = 0; t < 4; ++t) load_clamped(xv[d][t], x, b * 32 + t * 8, K);
  };
  f32x4 acc[NO];
#pragma unroll
  for (int o = 0; o < NO; ++o) acc[o] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int ib = 0; ib < steps; ib += AHEAD) {
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) load(d, ib + d);
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      const int i = ib + d;
      if (i >= steps) continue;
      const int b = (wave + i * NW) * 4 + quarter;
      if (wave + i * NW == all - 1) {
#pragma unroll
        for (int o = 0; o < NO; ++o) w[d][o].clear(b, K);
#pragma unroll
        for (int t = 0; t < 4; ++t) xv[d][t].clear(K - b * 32 - t * 8);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        bf16x8 term[TERMS];
        split_unit(xv[d][t], term);
#pragma unroll
        for (int o = 0; o < NO; ++o) {
          const bf16x8 wv = w[d][o].take(0, t);
#pragma unroll
          for (int p = 0; p < TERMS; ++p) acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, term[p], acc[o], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int o = 0; o < NO; ++o) part[wave][o][lane] = acc[o];
  __syncthreads();
  if (wave != 0 || lr >= count) return;
#pragma unroll
  for (int o = 0; o < NO; ++o)
#pragma unroll
    for (int k = 1; k < NW; ++k) acc[o] += part[k][o][lane];
  store_hidden(a, e, pair, n0 + quarter * 4, acc[0], acc[NO - 1]);
}

// four channels n.. of a row of out, from their sum without biases
__device__ __forceinline__ void store_out(const ExpertArgs& a, int64_t row, int n, const float (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (n + j >= a.N) continue;
    if (a.dtype == SAGA_BF16) static_cast<uint16_t*>(a.out)[row * a.ldo + n + j] = f32_to_bf16(v[j]);
    else static_cast<float*>(a.out)[row * a.ldo + n + j] = v[j];
  }
}

template <bool MX4, int TERMS>
__global__ __launch_bounds__(512) void k_expert_down_few(ExpertArgs a) {
  constexpr int NW = 8, AHEAD = 2;
  __shared__ f32x4 part[NW][64];
  __shared__ int index[kFewPairs], expert[kFewPairs], pair_of[kFewPairs][kFewRows];
  __shared__ float weight[kFewPairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15, pairs = (int)a.M * a.top_k;
  for (int i = threadIdx.x; i < kFewPairs * kFewRows; i += 512) pair_of[0][i] = -1;
  const int mine = lane < pairs ? a.index[lane] : -1;
  if ((int)threadIdx.x < pairs) index[threadIdx.x] = mine, weight[threadIdx.x] = a.weight[threadIdx.x];
  __syncthreads();
  // The experts that are taken, by number, and each row's pair of them.  (By number: a row's
  // results are then summed in an order that no other row has a say in.)
  int first = lane;
  for (int p = 0; p < pairs; ++p)
    if (p < first && index[p] == mine) first = p;
  const uint64_t firsts = __ballot(mine >= 0 && first == lane);
  const int taken = __popcll(firsts);
  if (wave == 0 && mine >= 0) {
    int place = 0;
    for (int p = 0; p < pairs; ++p) place += (firsts >> p & 1) && index[p] < mine;
    if (first == lane) expert[place] = mine;
    pair_of[place][lane / a.top_k] = lane;
  }
  __syncthreads();

  const int K = a.H, n0 = blockIdx.x * 16, all = (K + 127) / 128, ld = (int)a.ld_ht;
  const int64_t plane = a.M * a.top_k * a.ld_ht;
  const int steps = (all - wave + NW - 1) / NW, items = taken * steps;  // of this wave
  WeightBlocks<MX4, 1> w[AHEAD];
  u32x4 xv[AHEAD][4][TERMS];
  const auto load = [&](int d, int item) {
    item = min(item, items - 1);
    const int u = item / steps, b = (wave + item % steps * NW) * 4 + quarter;
    const WeightRow<MX4> from = weight_row<MX4, false>(a, (int64_t)expert[u] * a.N + min(n0 + lr, a.N - 1));
    w[d].load(from, b, K);
    const uint16_t* const x = a.ht + (int64_t)max(pair_of[u][lr], 0) * a.ld_ht;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int p = 0; p < TERMS; ++p)
        xv[d][t][p] = *reinterpret_cast<const u32x4*>(x + p * plane + min(b * 32 + t * 8, ld - 8));
  };
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (items > 0) {
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) load(d, d);
    for (int ib = 0; ib < items; ib += AHEAD) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) {
        const int item = ib + d, u = min(item, items - 1) / steps, s = wave + item % steps * NW;
        if (s == all - 1) w[d].clear(s * 4 + quarter, K);
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bf16x8 wv = w[d].take(0, t);
#pragma unroll
          for (int p = 0; p < TERMS; ++p) {
            bf16x8 v;
            __builtin_memcpy(&v, &xv[d][t][p], 16);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, v, acc, 0, 0, 0);
          }
        }
        load(d, item + AHEAD);
        // (a row that does not take the expert has another row's values here)
        const int pair = pair_of[u][lr];
        const bool has = pair >= 0 && item < items;
        const float p = has ? weight[max(pair, 0)] : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = has ? fmaf(p, acc[j], sum[j]) : sum[j];
      }
    }
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || lr >= (int)a.M) return;
#pragma unroll
  for (int k = 1; k < NW; ++k) sum += part[k][lane];
  const int n = n0 + quarter * 4;
  float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  for (int k = 0; k < a.top_k; ++k) {
    const int e = index[lr * a.top_k + k];
    const float p = weight[lr * a.top_k + k];
#pragma unroll
    for (int j = 0; j < 4; ++j)  // (a row without numbers: p is NaN)
      v[j] = fmaf(p, e >= 0 && a.down_bias && n + j < a.N ? a.down_bias[(int64_t)e * a.N + n + j] : 0.0f, v[j]);
  }
  store_out(a, lr, n, v);
}

// --------------------------------------------------------------------------
// the same where the experts' weights, of bfloat16, take most of the time and many rows take an
// expert: a workgroup of NW waves holds 32 NW rows of an expert's weights (32 a wave: gate and up of
// 16 channels, or 32 channels) and RT tiles of 16 rows of x.  A wave reads its weights from
// memory into registers, two steps of 128 k ahead; the rows of x go through
// LDS, a step at a time and two of them in turn, where all waves
// read them.  One barrier for each.  Loads are not inside a branch: where one path has
// loads and the other none, the compiler waits for all of them.  512 rows of 32 experts of 2048 x 4096 take
// 412 us for gates and ups and 241 for downs, where the layer's bytes take 341: all 256 registers are taken, and 18
// (bfloat16 rows' downs) to 67 (float32 rows' ups) more spill.
// --------------------------------------------------------------------------
template <int TERMS, bool UP, int RT, int NW>
__global__ __launch_bounds__(64 * NW) void k_expert_wide(ExpertArgs a) {
  constexpr int AHEAD = 2, ROWS = RT * 16;
  constexpr int PIECES = (ROWS * 16 * TERMS + 64 * NW - 1) / (64 * NW);  // 16-byte pieces a thread stages at a time
  static_assert(ROWS * 16 * TERMS % (64 * NW) == 0, "whole pieces");
  extern __shared__ uint4 space[];  // x: twice TERMS x ROWS x 16 pieces, then the list
  u32x4* const xs = reinterpret_cast<u32x4*>(space);
  constexpr int PART = TERMS * ROWS * 16;
  int* const list = reinterpret_cast<int*>(space + 2 * PART);
  int count;
  const int slots = min((int)a.M * a.top_k, a.E), width = NW * (UP && a.gated ? 16 : 32);
  const Share me = share_of(slots, ((UP ? a.H : a.N) + width - 1) / width, UP ? 1 : a.splits);
  if (me.slot >= slots) return;
  const int e = slot_expert<NW>(a, me.slot, list, count);
  if (e < 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15;
  const int K = UP ? a.F : a.H, N = UP ? a.H : a.N;
  const bool gated = UP && a.gated;
  const int all = (K + 127) / 128, per = UP ? all : (all + a.splits - 1) / a.splits;
  const int s0 = UP ? 0 : me.part * per, s1 = UP ? all : min(all, s0 + per);
  const int64_t ld = UP ? a.ld_xt : a.ld_ht, plane = (UP ? a.M : a.M * a.top_k) * ld;
  const uint16_t* const rows = UP ? a.xt : a.ht;
  const int n0 = me.run * width + wave * (gated ? 16 : 32);
  WeightBlocks<false, 1> w[AHEAD][2];
  WeightRow<false> weights[2];
#pragma unroll
  for (int o = 0; o < 2; ++o)
    weights[o] = weight_row<false, UP>(a, gated ? ((int64_t)e * 2 + o) * N + min(n0 + lr, N - 1)
                                                : (int64_t)e * N + min(n0 + o * 16 + lr, N - 1));
  const auto load = [&](int d, int s) {
    w[d][0].load(weights[0], s * 4 + quarter, K);
    w[d][1].load(weights[1], s * 4 + quarter, K);
  };
  for (int i0 = 0; i0 < count; i0 += ROWS) {
    const int here = min(count - i0, ROWS), tiles = (here + 15) / 16;
    // the pieces that this thread stages: term t, row r, piece p (4 quarter + group)
    const uint16_t* from[PIECES];
    u32x4 piece[PIECES];
    const int p = threadIdx.x & 15, col = (p >> 2) * 32 + (p & 3) * 8;
    int to[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const int i = j * 4 * NW + (threadIdx.x >> 4), r = i % ROWS, t = i / ROWS;
      const int pair = list[i0 + min(r, here - 1)];
      from[j] = rows + t * plane + (UP ? pair / a.top_k : pair) * ld;
      to[j] = (t * ROWS + r) * 16 + (p ^ (r & 15));
    }
    const auto fetch = [&](int s) {
      const int k = min(s * 128 + col, (int)ld - 8);
#pragma unroll
      for (int j = 0; j < PIECES; ++j) piece[j] = *reinterpret_cast<const u32x4*>(from[j] + k);
    };
    const auto put = [&](int s) {
#pragma unroll
      for (int j = 0; j < PIECES; ++j) xs[(s & 1) * PART + to[j]] = piece[j];
    };
    f32x4 acc[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r][0] = acc[r][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    fetch(s0);
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) load(d, s0 + d);
    put(s0);
    fetch(s0 + 1);
    for (int sb = s0; sb < s1; sb += AHEAD) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) {
        const int s = sb + d;
        if (s >= all - 1) {
          w[d][0].clear(s * 4 + quarter, K);
          w[d][1].clear(s * 4 + quarter, K);
        }
        ring_barrier();  // step s is in LDS, and nobody reads step s - 1 any more
        put(s + 1);
        fetch(s + 2);
        bf16x8 wv[2][4];
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int t = 0; t < 4; ++t) wv[o][t] = w[d][o].take(0, t);
        load(d, s + AHEAD);
        const u32x4* const x = xs + (s & 1) * PART + lr * 16;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          if (r < tiles && s < s1) {
#pragma unroll
            for (int p = 0; p < TERMS; ++p)
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                const u32x4 v = x[(p * ROWS + r * 16) * 16 + ((quarter * 4 + t) ^ lr)];
                bf16x8 xv;
                __builtin_memcpy(&xv, &v, 16);
#pragma unroll
                for (int o = 0; o < 2; ++o)
                  acc[r][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[o][t], xv, acc[r][o], 0, 0, 0);
              }
          }
        }
      }
    }
    ring_barrier();  // (the next rows' first step takes the place of one that may still be read)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if (r * 16 + lr >= here) continue;
      const int pair = list[i0 + r * 16 + lr], n = n0 + quarter * 4;
      if constexpr (UP) {
        store_hidden(a, e, pair, n, acc[r][0], acc[r][1]);
        if (!gated) store_hidden(a, e, pair, n + 16, acc[r][1], acc[r][1]);
      } else {
        float* const o = a.part + (me.part * a.M * a.top_k + pair) * a.ld_part + n;
        if (n < N) *reinterpret_cast<f32x4*>(o) = acc[r][0];
        if (n + 16 < N) *reinterpret_cast<f32x4*>(o + 16) = acc[r][1];
      }
    }
  }
}

// --------------------------------------------------------------------------
// 4-bit weights and many rows: 256 rows of an expert's weights and RT tiles of 16 rows of x
// a workgroup.  Both come through LDS by direct-to-LDS loads, weights by whole lines (half
// of them cost as much), each well ahead of its use.  A wave has 64 rows of weights (gate and up of 32 channels, or 64
// channels) and every second tile of x.  Past the rows' ends x is zeros and scales are 1,
// whatever the weights' bits are there.
//
// 512 rows and 32 experts of 2048 x 4096 (64 rows an expert): 112 to 134 us for gates and ups, 87 to 105 for downs
// (machines differ in the clock that their power leaves), where
// their weights alone would take 60 and 30 and the products 45 and 45.  The loads alone take 90: x comes
// from L2 (24 KB for each 17 KB of weights), and nothing runs beside a tile's first loads and its
// values' way out.  128 rows (16 an expert): 77 and 46, three quarters of the copy's rate.
// --------------------------------------------------------------------------
typedef __attribute__((address_space(3))) uint4 lds_uint4;

// LDS at `to` + the lane's place <- 16 bytes at the lane's offset from `base`, or 4 bytes of its address
__device__ __forceinline__ void lds_load16(uint32_t to, const void* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base)
               : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(uint32_t to, const void* from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
               : "memory", "m0");
}

template <int TERMS, int RT>
struct ExpertTile {
  static constexpr int NW = 8, WROWS = 256, ROWS = RT * 16;
  // weights: 256 k (whole lines) a slot, two slots; x: TC groups of 8 k of each lane's block, all
  // terms, a part, three parts.  A slot is SL parts.
  static constexpr int TC = TERMS == 1 || RT * TERMS <= 6 ? 4 : 2, SL = 8 / TC;
  static constexpr int PPR = 4 * TC;                        // pieces of a row and term in a part
  static constexpr int XL = TERMS * ROWS * PPR / 64 / NW;   // load instructions of a wave for a part
  static constexpr int WL = 4 + 1;                          // and for a slot: weights, scales
  static constexpr int W_BYTES = WROWS * 128, S_BYTES = WROWS * 8, SLOT = W_BYTES + S_BYTES;
  static constexpr int PART = TERMS * ROWS * PPR * 16;
  static constexpr int PITCH = WROWS + 4;                   // of the sums on their way out, in floats
  static constexpr int RING = 2 * SLOT + 3 * PART, LDS = RING + kExpertRows * 4;
  static_assert(TERMS * ROWS * PPR % (64 * NW) == 0 && RT % 2 == 0, "the same loads and tiles on every wave");
  static_assert(ROWS * PITCH * 4 <= RING && RT <= 6 && LDS <= 160 * 1024 - 64, "LDS");
  // where piece p of row r is among its row's: 16 rows of a fragment read fall on all banks
  __device__ __forceinline__ static int place(int r, int p) {
    return p ^ (PPR == 16 ? r & 15 : PPR == 8 ? r >> 1 & 7 : r >> 2 & 3);
  }
};

template <int TERMS, bool UP, int RT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_expert_tile(ExpertArgs a) {
  typedef ExpertTile<TERMS, RT> R;
  extern __shared__ uint4 space[];
  char* const base = reinterpret_cast<char*>(space);
  int* const list = reinterpret_cast<int*>(base + R::RING);
  int count;
  const int slots = min((int)a.M * a.top_k, a.E), width = UP && a.gated ? 128 : 256;
  const Share me = share_of(slots, ((UP ? a.H : a.N) + width - 1) / width, UP ? 1 : a.splits);
  if (me.slot >= slots) return;
  const int e = slot_expert<R::NW>(a, me.slot, list, count);
  if (e < 0) return;
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_uint4*)space;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15;
  const int wm = wave & 3, wx = wave >> 2;  // (waves w and w + 4 share a SIMD: one of each half of x)
  const int K = UP ? a.F : a.H, N = UP ? a.H : a.N, bytes = (K + 1) / 2, kmax = (bytes - 1) / 16 * 16;
  const int smax = (K - 1) / 128 * 4;  // the last scales' word
  const bool gated = UP && a.gated;
  const int all = (K + 255) / 256, per = UP ? all : (all + a.splits - 1) / a.splits;
  const int s0 = UP ? 0 : min(all, me.part * per), s1 = UP ? all : min(all, s0 + per);
  const int n0 = me.run * width;
  // row r of the stage's weights: 64 a wave; gated: gates of 32 channels, then ups
  const int64_t ld_w = UP ? a.ld_up : a.ld_down, ld_s = UP ? a.lds_up : a.lds_down;
  const auto row_of = [&](int r) {
    return gated ? ((int64_t)e * 2 + (r >> 5 & 1)) * N + min(n0 + (r >> 6) * 32 + (r & 31), N - 1)
                 : (int64_t)e * N + min(n0 + r, N - 1);
  };
  // a load of weights has 8 rows: of gates or of ups (from the first row of all of these)
  const int64_t first = gated ? ((int64_t)e * 2 + (wave >> 2)) * N + n0 : (int64_t)e * N + n0;
  const uint8_t* const w_base = static_cast<const uint8_t*>(UP ? a.up : a.down) + first * ld_w;
  const uint8_t* const s_base = UP ? a.up_scale : a.down_scale;
  uint32_t w_at[4];
  const int w_piece = ((lane & 7) ^ (lane >> 4 & 3 | (wave & 1) << 2)) * 16;  // (r >> 1 & 7 of row r = 8 i + lane / 8)
#pragma unroll
  for (int j = 0; j < 4; ++j) w_at[j] = (uint32_t)(row_of(8 * (wave + 8 * j) + lane / 8) - first) * (uint32_t)ld_w;
  const uint8_t* const s_at = s_base + row_of(wave * 32 + lane / 2) * ld_s;
  const char* const rows = reinterpret_cast<const char*>(UP ? a.xt : a.ht);
  const uint32_t ld = (uint32_t)(UP ? a.ld_xt : a.ld_ht) * 2, plane = (uint32_t)(UP ? a.M : a.M * a.top_k) * ld;
  const uint32_t zeros = (uint32_t)(reinterpret_cast<const char*>(a.zeros) - rows);
  // this lane's piece of a row in every load of x: quarter p / TC, group p % TC
  const int x_row = (wave * 64 + lane) / R::PPR % R::ROWS, p = R::place(x_row, lane % R::PPR);
  const uint32_t x_piece = p / R::TC * 128 + p % R::TC * 16;

  for (int i0 = 0; i0 < count; i0 += R::ROWS) {
    const int here = min(count - i0, R::ROWS), tiles = (here + 15) / 16;
    uint32_t x_at[R::XL];
#pragma unroll
    for (int j = 0; j < R::XL; ++j) {
      const int i = ((wave + 8 * j) * 64 + lane) / R::PPR, r = i % R::ROWS, t = i / R::ROWS;
      const int pair = list[i0 + min(r, here - 1)];
      x_at[j] = t * plane + (uint32_t)(UP ? pair / a.top_k : pair) * ld;
    }
    const auto issue_w = [&](int s) {
      const uint32_t to = lds + (s & 1) * R::SLOT, k = (uint32_t)min(s * 128 + w_piece, kmax);
#pragma unroll
      for (int j = 0; j < 4; ++j) lds_load16(to + (wave + 8 * j) * 1024, w_base, w_at[j] + k);
      lds_load4(to + R::W_BYTES + wave * 256, s_at + min(s * 8 + (lane & 1) * 4, smax));
    };
    const auto issue_x = [&](int v, int ring) {  // part v
      const uint32_t to = lds + 2 * R::SLOT + ring * R::PART;
      const int g = v % R::SL * R::TC;  // its first group: of block g / 4, groups g % 4..
      const uint32_t k = v / R::SL * 512 + (g >> 2) * 64 + (g & 3) * 16 + x_piece;
#pragma unroll
      for (int j = 0; j < R::XL; ++j) lds_load16(to + (wave + 8 * j) * 1024, rows, k < ld ? x_at[j] + k : zeros);
    };
    f32x4 acc[4][RT / 2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < RT / 2; ++r) acc[i][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (s0 < s1) {
      issue_w(s0);
      issue_x(s0 * R::SL, 0);
      issue_x(s0 * R::SL + 1, 1);
    }
    // (how many tiles the wave has is part of the code: a branch around each would keep the
    // reads of the next one behind the products of the last)
    const auto products = [&](auto count_tag) {
      constexpr int NT = decltype(count_tag)::value;
      int ring = 0;  // where part v is; v + 1 and v + 2 follow
      for (int s = s0; s < s1; ++s) {
        const bool more = s + 1 < s1;
        WeightBlocks<true, 2> w[4];
#pragma unroll
        for (int m = 0; m < R::SL; ++m) {
          // Part v = s SL + m has to be there, and with m = 0 slot s: of what was asked for later,
          // part v + 1 and (behind part s SL + 2) slot s + 1 may still be on their way.
          const int v = s * R::SL + m;
          if (m + 1 == R::SL && !more) wait_vm<0>();
          else if ((m == 1 || (m == 2 && R::SL > 2)) && more) wait_vm<R::XL + R::WL>();
          else wait_vm<R::XL>();
          ring_barrier();  // and nobody reads part v - 1, or with m = 0 slot s - 1, any more
          if (m + 2 < R::SL || more) issue_x(v + 2, ring == 0 ? 2 : ring - 1);
          if (m == 0 && more) issue_w(s + 1);
          const char* const slot = base + (s & 1) * R::SLOT;
          const char* const part = base + 2 * R::SLOT + ring * R::PART;
          ring = ring == 2 ? 0 : ring + 1;
          const int j = m * R::TC / 4, t0 = m * R::TC % 4;
          if (t0 == 0) {  // the lane's block 2 quarter + j of the slot
            const int r0 = wm * 64 + lr;
            const char* const wl = slot + r0 * 128 + ((quarter * 2 + j) ^ (r0 >> 1 & 7)) * 16;
            const bool past = (s * 8 + quarter * 2 + j) * 32 >= K;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i].v[j] = *reinterpret_cast<const u32x4*>(wl + i * 16 * 128);
              const uint32_t b = *reinterpret_cast<const uint8_t*>(slot + R::W_BYTES + r0 * 8 + i * 128 + quarter * 2 + j);
              w[i].scale = (past ? 127u : b) << (8 * j);
            }
          }
#pragma unroll
          for (int t = 0; t < R::TC; ++t) {
            bf16x8 wv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) wv[i] = w[i].take(j, t0 + t);
            const char* const xl = part + ((wx * 16 + lr) * R::PPR + R::place(lr, quarter * R::TC + t)) * 16;
#pragma unroll
            for (int r = 0; r < NT; ++r) {
#pragma unroll
              for (int p = 0; p < TERMS; ++p) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(xl + (p * R::ROWS + r * 32) * R::PPR * 16);
                bf16x8 xv;
                __builtin_memcpy(&xv, &x, 16);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  acc[i][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], xv, acc[i][r], 0, 0, 0);
              }
            }
          }
        }
      }
    };
    switch ((tiles - wx + 1) / 2) {
      case 0: products(std::integral_constant<int, 0>{}); break;
      case 1: products(std::integral_constant<int, 1>{}); break;
      case 2: products(std::integral_constant<int, RT / 2 < 2 ? RT / 2 : 2>{}); break;
      default: products(std::integral_constant<int, RT / 2>{}); break;
    }
    ring_barrier();  // the stages are free: the sums go through them, to leave by whole rows
    float* const sums = reinterpret_cast<float*>(base);
#pragma unroll
    for (int r = 0; r < RT / 2; ++r)
      if (2 * r + wx < tiles)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(sums + ((2 * r + wx) * 16 + lr) * R::PITCH + quarter * 4 +
                                    (gated ? (i >> 1) * 128 + wm * 32 + (i & 1) * 16 : wm * 64 + i * 16)) = acc[i][r];
    __syncthreads();
    if constexpr (UP) {
      const int octs = gated ? 16 : 32;
      for (int i = threadIdx.x; i < here * octs; i += 512) {
        const int row = i / octs, q = i % octs;
        const float* const from = sums + row * R::PITCH + q * 8;  // (gated: gates, then ups)
        float v[8], up[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = from[j], up[j] = from[j + (gated ? 128 : 0)];
        store_hidden(a, e, list[i0 + row], n0 + q * 8, v, up);
      }
    } else {
      for (int i = threadIdx.x; i < here * 64; i += 512) {
        const int row = i / 64, q = i % 64;
        if (n0 + q * 4 < N)
          *reinterpret_cast<f32x4*>(a.part + (me.part * a.M * a.top_k + list[i0 + row]) * a.ld_part + n0 + q * 4) =
              *reinterpret_cast<const f32x4*>(sums + row * R::PITCH + q * 4);
      }
    }
    __syncthreads();
  }
}

// --------------------------------------------------------------------------
// the same where the experts' weights take most of the time and few rows take an expert:
// reading the weights is all that counts.  The rows of x (16 at a time) lie in LDS,
// all of k if it fits, so that nothing but weights is loaded in the loop: loads come back in
// their order, and a wait for x would be one for the weights that were asked for before.  A
// workgroup takes `per` runs of 32 NW rows of weights one after the other, and a wave's
// loads run AHEAD steps ahead across them.  64 rows and 64 experts of 1024 x 4096 in 4 bits (two rows
// an expert): 64 us for gates and ups (3.8 TB/s of weights), 38 for downs; with half lines a load
// 84 and 48, with loads in branches 106 and 53.  In bfloat16 4.2 TB/s.
// --------------------------------------------------------------------------
constexpr int kStreamPieces = 48 * 64;  // 48 KB (three workgroups a CU)

template <bool MX4, int TERMS, bool UP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void k_expert_stream(ExpertArgs a, int runs,
                                                                                              int per) {
  constexpr int NW = 4, J = MX4 ? 2 : 1, AHEAD = 2;
  static_assert(AHEAD * TERMS * 16 * 16 * J <= kStreamPieces, "a round of steps fits LDS");
  __shared__ u32x4 xs[kStreamPieces];
  __shared__ int list[kExpertRows];
  int count;
  const int slots = min((int)a.M * a.top_k, a.E);
  const Share me = share_of(slots, (runs + per - 1) / per, UP ? 1 : a.splits);
  if (me.slot >= slots) return;
  const int e = slot_expert<NW>(a, me.slot, list, count);
  if (e < 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15;
  const int K = UP ? a.F : a.H, N = UP ? a.H : a.N;
  const bool gated = UP && a.gated;
  const int all = (K + 128 * J - 1) / (128 * J), part = UP ? all : (all + a.splits - 1) / a.splits;
  const int k0 = UP ? 0 : min(all, me.part * part), steps = UP ? all : min(part, all - k0);  // from step k0 on
  const int64_t ld = UP ? a.ld_xt : a.ld_ht, plane = (UP ? a.M : a.M * a.top_k) * ld;
  const uint16_t* const rows = UP ? a.xt : a.ht;
  const int run0 = me.run * per, run1 = min(runs, run0 + per);
  const auto channel = [&](int run) { return (run * NW + wave) * (gated ? 16 : 32); };
  WeightRow<MX4> from[2];
  const auto rows_of = [&](int run) {
    const int n = channel(run) + lr;
    from[0] = weight_row<MX4, UP>(a, (int64_t)e * N * (gated ? 2 : 1) + min(n, N - 1));
    from[1] = weight_row<MX4, UP>(a, gated ? ((int64_t)e * 2 + 1) * N + min(n, N - 1) : (int64_t)e * N + min(n + 16, N - 1));
  };
  WeightBlocks<MX4, J> w[AHEAD][2];
  const auto load = [&](int d, int s) {
    w[d][0].load(from[0], ((k0 + s) * 4 + quarter) * J, K);
    w[d][1].load(from[1], ((k0 + s) * 4 + quarter) * J, K);
  };
  for (int i0 = 0; i0 < count; i0 += 16) {
    const int here = min(count - i0, 16), a_step = here * TERMS * 16 * J;
    const int fit = kStreamPieces / a_step, chunk = fit >= steps ? steps : fit / AHEAD * AHEAD;
    const auto stage = [&](int first) {  // (what lies past a row's end does not count: weights are zeros there)
      const int n = min(chunk, steps - first) * a_step;
      for (int i = threadIdx.x; i < n; i += 4 * 256) {
        u32x4 v[4];
        int to[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int at = min(i + j * 256, n - 1), p = at % (16 * J), q = at / (16 * J), r = q % here, st = q / here;
          const int t = st % TERMS, k = ((k0 + first + st / TERMS) * 16 * J + p) * 8, pair = list[i0 + r];
          v[j] = *reinterpret_cast<const u32x4*>(rows + t * plane + (UP ? pair / a.top_k : pair) * ld +
                                                 min(k, (int)ld - 8));
          to[j] = q * 16 * J + (p ^ r);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) xs[to[j]] = v[j];
      }
    };
    rows_of(run0);
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) load(d, d);
    const bool whole = chunk >= steps;
    if (whole) {
      stage(0);
      __syncthreads();
    }
    const int row = min(lr, here - 1);  // (rows past the last: not stored)
    for (int run = run0; run < run1; ++run) {
      f32x4 acc[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
      for (int sb = 0; sb < steps; sb += AHEAD) {
        if (!whole && sb % chunk == 0) {
          __syncthreads();
          stage(sb);
          __syncthreads();
        }
        // What the places of the ring hold next: of this run, or of the next one (of the
        // last run again, unused).  Steps past a run's last have its last piece for weights,
        // cleared: there is no branch around what is loaded, which would end in waits for it.
        int next = sb + AHEAD;
        if (next >= steps) {
          next = 0;
          rows_of(min(run + 1, run1 - 1));
        }
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
          const int s = sb + d;
          if (s >= steps || k0 + s == all - 1) {
            const int b = s >= steps ? all * 4 * J : ((k0 + s) * 4 + quarter) * J;
            w[d][0].clear(b, K);
            w[d][1].clear(b, K);
          }
          const int at = min(s, steps - 1);
          const u32x4* const x = xs + (whole ? at : at % chunk) * a_step + row * 16 * J;
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const bf16x8 wv[2] = {w[d][0].take(j, t), w[d][1].take(j, t)};
#pragma unroll
              for (int p = 0; p < TERMS; ++p) {
                const u32x4 v = x[p * here * 16 * J + (((quarter * J + j) * 4 + t) ^ row)];
                bf16x8 xv;
                __builtin_memcpy(&xv, &v, 16);
                acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[0], xv, acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[1], xv, acc[1], 0, 0, 0);
              }
            }
          load(d, next + d);
        }
      }
      if (lr < here) {
        const int pair = list[i0 + lr], n = channel(run) + quarter * 4;
        if constexpr (UP) {
          store_hidden(a, e, pair, n, acc[0], acc[1]);
          if (!gated) store_hidden(a, e, pair, n + 16, acc[1], acc[1]);
        } else {
          float* const o = a.part + (me.part * a.M * a.top_k + pair) * a.ld_part + n;
          if (n < N) *reinterpret_cast<f32x4*>(o) = acc[0];
          if (n + 16 < N) *reinterpret_cast<f32x4*>(o + 16) = acc[1];
        }
      }
    }
    __syncthreads();  // (the next rows take x's place)
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
      if (e >= 0)
        for (int z = 0; z < a.splits; ++z)
          d += *reinterpret_cast<const f32x4*>(a.part + (z * a.M * a.top_k + pair) * a.ld_part + n);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (e >= 0 && a.down_bias && n + j < a.N) d[j] += a.down_bias[(int64_t)e * a.N + n + j];
        v[j] = fmaf(p, d[j], v[j]);  // (a row without numbers: p is NaN)
      }
    }
    store_out(a, row, n, v);
  }
}

// Whether the wide kernels take the products: their workgroups fill the CUs (us of the layer, wide / k_expert_few: 32
// rows of 8 experts of 1024 x 4096 in 4 bits 32 / 44; 64 of 16 of 256 x 1024, where they just do, 26 / 26; 42 of 5 of
// 3872 x 1757, gated, 140 workgroups, 51 / 44).  k_expert_few reads an expert's weights again for every 16 rows: many
// rows of 4-bit weights gain by fewer workgroups (all of 3 experts of 1761 x 3362, gated, 530 rows, 159 workgroups,
// 336 / 709; both of 2 of 1656 x 5333, gated, 304, 168, 323 / 373; two of 6 of 1124 x 2530, 163, 120, 49 / 79; below the
// rule: three of 22 of 2938 x 223, gated, 672, 88, 117 / 134; three of 11 of 279 x 591, 688, 55, 101 / 82; one of
// 3043 x 4902, gated, 132, 77, 244 / 159).  bfloat16 ones do not always: four of 11 of 2621 x 1147, gated, 196 rows, 198
// workgroups, 212 / 289, but four of 17 of 74 x 850, gated, 722, 238, 138 / 92; four of 7 of 1061 x 1005, gated, 153,
// 112, 113 / 80; four of 4 of 3726 x 1697, 260, 56, 712 / 500.
bool experts_wide(int64_t M, int64_t H, int E, int top_k, bool gated, bool mx4) {
  const int64_t slots = std::min<int64_t>(M * top_k, E), mean = M * top_k / E;
  return slots * ((H * (gated ? 2 : 1) + 127) / 128) >= (mx4 && mean >= 48 ? 96 : 256);
}
// parts of k of the second product, so that it has workgroups enough (us of the layer, with / without: 512
// rows of 8 experts of 1024 x 4096 in 4 bits 82 / 176, 128 of 32 80 / 91, 64 of 64, where there is one part, 114)
int expert_splits(int64_t M, int64_t H, int64_t N, int E, int top_k) {
  const int64_t slots = std::min<int64_t>(M * top_k, E), wgs = slots * ((N + 127) / 128), steps = (H + 127) / 128;
  return (int)std::max<int64_t>(1, std::min<int64_t>({8, 512 / wgs, steps / 4}));
}

// Whether the two kernels of few rows take the layer: the second one's workgroups, 16 channels
// of out each, read their channels of all experts that are taken one after the other (us, two kernels /
// four; 4 bits: a row, two of 8 experts of 1024 x 2048 20 / 26, of 1024 x 4096 24 / 26, two rows of these
// 43 / 35; 16 rows of 8 of 128 x 256 22 / 25, of 4 of 256 x 1024 25 / 23, of 32 of 128 x 256 27 / 25.
// bfloat16, twice the cost: a row, two of 8 of 1024 x 1024 20 / 24, of 1024 x 2048 23 / 24, of 1024 x 4096 33 / 28.)
bool experts_few(int64_t M, int64_t H, int top_k, int E, bool mx4) {
  return M <= kFewRows && M * top_k <= kFewPairs &&
         std::min<int64_t>(M * top_k, E) * H * (mx4 ? 1 : 2) <= (M <= 2 ? 8192 : 2048);
}
// and whether the first one chooses: a float64 product by the waves of every workgroup (us, chosen
// there / by k_route before: a row and 16 experts of 1024 columns 20 / 23, two rows of 512 19 / 22, of 8 of 602
// 21 / 23, four rows of 4 of 128 18 / 21, of 16 of 256 23 / 22, 16 rows of 8 of 128 51 / 22)
bool experts_fused(int64_t M, int64_t F, int E) { return M <= 4 && M * E * F <= (M <= 2 ? 16384 : 4096); }

template <bool MX4, typename T>
hipError_t few_rows(const ExpertArgs& a, hipStream_t st) {
  const dim3 up((unsigned)((a.H + 15) / 16), (unsigned)std::min<int64_t>(a.M * a.top_k, a.E));
  const auto go = [&](auto kernel, dim3 grid) {
    hipLaunchKernelGGL(kernel, grid, dim3(512), 0, st, a);
    return hipGetLastError();
  };
  hipError_t e;
  if (experts_fused(a.M, a.F, a.E))
    e = a.gated ? go(k_expert_up_few<MX4, T, true, true>, up) : go(k_expert_up_few<MX4, T, false, true>, up);
  else
    e = a.gated ? go(k_expert_up_few<MX4, T, true, false>, up) : go(k_expert_up_few<MX4, T, false, false>, up);
  if (e != hipSuccess) return e;
  return go(k_expert_down_few<MX4, sizeof(T) == 2 ? 2 : 3>, dim3((unsigned)((a.N + 15) / 16)));
}

template <int TERMS, bool UP, int RT, int NW>
hipError_t launch_wide(const ExpertArgs& a, hipStream_t st) {
  const unsigned slots = (unsigned)std::min<int64_t>(a.M * a.top_k, a.E);
  const int per = NW * (UP && a.gated ? 16 : 32), n = UP ? a.H : a.N;
  const size_t lds = (size_t)2 * TERMS * RT * 16 * 16 * 16 + (size_t)a.M * 4;
  hipLaunchKernelGGL((k_expert_wide<TERMS, UP, RT, NW>),
                     dim3(share_blocks(slots, (n + per - 1) / per, UP ? 1 : a.splits)), dim3(64 * NW), lds, st, a);
  return hipGetLastError();
}
template <int TERMS, bool UP, int RT>
hipError_t launch_expert_tile(const ExpertArgs& a, hipStream_t st) {
  const unsigned slots = (unsigned)std::min<int64_t>(a.M * a.top_k, a.E);
  const int per = UP && a.gated ? 128 : 256, n = UP ? a.H : a.N;
  constexpr size_t lds = ExpertTile<TERMS, RT>::LDS;
  hipLaunchKernelGGL((k_expert_tile<TERMS, UP, RT>), dim3(share_blocks(slots, (n + per - 1) / per, UP ? 1 : a.splits)),
                     dim3(512), lds, st, a);
  return hipGetLastError();
}
template <bool MX4, int TERMS, bool UP>
hipError_t dispatch_wide(const ExpertArgs& a, hipStream_t st) {
  // Rows an expert has on average (us of both products, 4-bit weights, k_expert_stream / k_expert_tile: two,
  // 64 rows of 64 experts of 1024 x 4096, 102 / 116; eight, 128 rows of 32, 82 / 69.  Of the layer, bfloat16
  // weights, k_expert_stream / k_expert_wide: four, 64 rows of 32 experts, 193 / 238; eight 219 / 244.)
  const int64_t mean = a.M * a.top_k / a.E;
  if (mean <= (MX4 ? 4 : 8)) {
    const int64_t slots = std::min<int64_t>(a.M * a.top_k, a.E), rows = UP ? (int64_t)a.H * (a.gated ? 2 : 1) : a.N;
    const int64_t z = UP ? 1 : a.splits, runs = (rows + 127) / 128, per = std::max<int64_t>(1, runs * slots * z / 640);
    hipLaunchKernelGGL((k_expert_stream<MX4, TERMS, UP>),
                       dim3(share_blocks(slots, (runs + per - 1) / per, z)), dim3(256), 0, st, a, (int)runs, (int)per);
    return hipGetLastError();
  }
  // (us of the layer by tiles of 32, 64 and 96 rows, 32 experts of 2048 x 4096: 16 rows an expert 136, 144,
  // 150; 32: 194, 159, 167; 64: 306, 255, 214.  Three terms of 96 rows do not fit LDS.)
  if constexpr (MX4) {
    if (mean <= 20) return launch_expert_tile<TERMS, UP, 2>(a, st);
    if (mean <= 40 || TERMS == 3) return launch_expert_tile<TERMS, UP, 4>(a, st);
    if constexpr (TERMS < 3) return launch_expert_tile<TERMS, UP, 6>(a, st);
  } else {
    return launch_wide<TERMS, UP, 4, 8>(a, st);
  }
}

template <bool MX4>
hipError_t products(const ExpertArgs& a, hipStream_t st) {
  hipError_t e;
  if (experts_wide(a.M, a.H, a.E, a.top_k, a.gated, MX4)) {
    e = a.x_terms == 1 ? dispatch_wide<MX4, 1, true>(a, st) : dispatch_wide<MX4, 3, true>(a, st);
    if (e != hipSuccess) return e;
    return a.h_terms == 2 ? dispatch_wide<MX4, 2, false>(a, st) : dispatch_wide<MX4, 3, false>(a, st);
  }
  const unsigned slots = (unsigned)std::min<int64_t>(a.M * a.top_k, a.E);
  const dim3 up((unsigned)((a.H + 15) / 16), slots), down((unsigned)((a.N + 15) / 16), slots);
  const auto go = [&](auto kernel, auto deep, dim3 grid, int k) {  // (deep: two steps at a time)
    if (k > 512) hipLaunchKernelGGL(deep, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
    return hipGetLastError();
  };
  if (a.gated)
    e = a.x_terms == 1 ? go(k_expert_few<MX4, 1, true, true, 1>, k_expert_few<MX4, 1, true, true, 2>, up, a.F)
                       : go(k_expert_few<MX4, 3, true, true, 1>, k_expert_few<MX4, 3, true, true, 2>, up, a.F);
  else
    e = a.x_terms == 1 ? go(k_expert_few<MX4, 1, true, false, 1>, k_expert_few<MX4, 1, true, false, 2>, up, a.F)
                       : go(k_expert_few<MX4, 3, true, false, 1>, k_expert_few<MX4, 3, true, false, 2>, up, a.F);
  if (e != hipSuccess) return e;
  return a.h_terms == 2 ? go(k_expert_few<MX4, 2, false, false, 1>, k_expert_few<MX4, 2, false, false, 2>, down, a.H)
                        : go(k_expert_few<MX4, 3, false, false, 1>, k_expert_few<MX4, 3, false, false, 2>, down, a.H);
}

size_t whole(size_t n) { return (n + 255) & ~(size_t)255; }

// the parts of the workspace, of up to kExpertRows rows
struct ExpertSpace {
  int64_t rows, ld_xt, ld_ht, ld_part;
  int x_terms, h_terms, splits;
  size_t xt, ht, zeros, part, total;
};
ExpertSpace expert_space(int dtype, bool mx4, int64_t M, int64_t F, int64_t H, int64_t N, int E, int top_k, bool gated) {
  ExpertSpace s;
  s.x_terms = dtype == SAGA_BF16 ? 1 : 3;
  s.h_terms = dtype == SAGA_BF16 ? 2 : 3;
  s.ld_xt = (F + 15) / 16 * 16;
  s.ld_ht = (H + 15) / 16 * 16;
  // (xt, ht and zeros lie within 32-bit offsets of each other)
  const int64_t row_bytes = 2 * (s.x_terms * s.ld_xt + s.h_terms * top_k * s.ld_ht);
  s.rows = std::min<int64_t>({M, kExpertRows, ((int64_t)1 << 31) / row_bytes});
  s.ld_part = (N + 3) / 4 * 4;
  s.xt = 0;
  s.ht = s.xt + whole((size_t)s.x_terms * s.rows * s.ld_xt * 2);
  s.zeros = s.ht + whole((size_t)s.h_terms * s.rows * top_k * s.ld_ht * 2);
  s.part = s.zeros + 256;
  s.splits = experts_wide(s.rows, H, E, top_k, gated, mx4) ? expert_splits(s.rows, H, N, E, top_k) : 1;
  s.total = s.part + whole((size_t)s.splits * s.rows * top_k * s.ld_part * 4);
  return s;
}

}  // namespace

size_t experts_workspace_bytes(int dtype, int weight_dtype, int64_t M, int64_t F, int64_t H, int64_t N, int E, int top_k,
                               bool gated) {
  return M == 0 ? 0 : expert_space(dtype, weight_dtype == SAGA_MX4, M, F, H, N, E, top_k, gated).total;
}

hipError_t launch_experts(const ExpertArgs& a0, hipStream_t st) {
  if (a0.M == 0) return hipSuccess;
  const bool mx4 = a0.weight_dtype == SAGA_MX4;
  const ExpertSpace s = expert_space(a0.dtype, mx4, a0.M, a0.F, a0.H, a0.N, a0.E, a0.top_k, a0.gated);
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
    a.zeros = reinterpret_cast<uint16_t*>(ws + s.zeros);
    a.part = reinterpret_cast<float*>(ws + s.part);
    a.ld_xt = s.ld_xt;
    a.ld_ht = s.ld_ht;
    a.ld_part = s.ld_part;
    a.x_terms = s.x_terms;
    a.h_terms = s.h_terms;
    a.splits = s.splits;
    if (a.M < s.rows)  // (the rest of many rows: never more parts than there is room for)
      a.splits = std::min(s.splits, experts_wide(a.M, a.H, a.E, a.top_k, a.gated, mx4)
                                        ? expert_splits(a.M, a.H, a.N, a.E, a.top_k) : 1);
    const bool few = experts_few(a.M, a.H, a.top_k, a.E, mx4);
    const auto route = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)a.M), dim3(kRouteThreads), 0, st, a);
      return hipGetLastError();
    };
    hipError_t e = hipSuccess;
    if (!few || !experts_fused(a.M, a.F, a.E)) {
      if (a.dtype == SAGA_BF16)
        e = a.router_dtype == SAGA_BF16 ? route(k_route<uint16_t, uint16_t>) : route(k_route<uint16_t, float>);
      else
        e = a.router_dtype == SAGA_BF16 ? route(k_route<float, uint16_t>) : route(k_route<float, float>);
      if (e != hipSuccess) return e;
    }
    if (few) {
      if (a.dtype == SAGA_BF16) e = mx4 ? few_rows<true, uint16_t>(a, st) : few_rows<false, uint16_t>(a, st);
      else e = mx4 ? few_rows<true, float>(a, st) : few_rows<false, float>(a, st);
      if (e != hipSuccess) return e;
      continue;
    }
    e = mx4 ? products<true>(a, st) : products<false>(a, st);
    if (e != hipSuccess) return e;
    const int64_t quads = a.M * (a.ld_part / 4);
    hipLaunchKernelGGL(k_expert_sum, dim3((unsigned)std::min<int64_t>((quads + 255) / 256, 1 << 16)), dim3(256), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace saga
