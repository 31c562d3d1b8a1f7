// 8-bit rows (largest magnitude 127, a float32 scale per row) and products of
// them:  out = act(rs * (a_scale_i w_scale_j sum_k a_ik w_jk) + bias_j).  Both
// operands are rows of k (w: one output channel a row), the sums whole numbers
// in 32 bits, so their order does not matter.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gemm_device.h"
#include "row_device.h"

namespace saga {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) uint4 lds_uint4;

constexpr int64_t kMostBlocks = 1 << 20;  // (a grid holds less than 2^32 threads)

// --------------------------------------------------------------------------
// float rows to 8-bit rows; memory bounds it: a row is read once into registers
// --------------------------------------------------------------------------
template <int U>
__device__ __forceinline__ uint32_t top_bits(const float (&v)[U][8]) {
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[u][j]) & 0x7fffffffu);
  return top;
}

template <typename T, int G, int U>
__global__ __launch_bounds__(RowGroup<G>::THREADS) void k_quantize_rows(QuantRowsArgs a) {
  typedef RowGroup<G> R;
  __shared__ uint32_t red[2 * (G > 64 ? G / 64 : 1)];
  int turn = 0;
  const int col0 = (threadIdx.x % G) * 8, K = (int)a.K;
  for (int64_t row = blockIdx.x * (int64_t)R::ROWS + threadIdx.x / G; row < a.M;
       row += gridDim.x * (int64_t)R::ROWS) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) load_unit(x + col0 + u * 8 * G, K - col0 - u * 8 * G, v[u]);
    const RowScale s = row_scale(R::template reduce<OpMaxU>(top_bits(v), red, turn));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = col0 + u * 8 * G;
      store_unit_i8(a.q + row * a.ldq + col, K - col, round_unit(v[u], s));
    }
    if (threadIdx.x % G == 0) a.scale[row] = s.s;
  }
}

// rows past the registers: read twice
template <typename T>
__global__ __launch_bounds__(1024) void k_quantize_long(QuantRowsArgs a) {
  typedef RowGroup<1024> R;
  __shared__ uint32_t red[2 * 16];
  int turn = 0;
  const int K = (int)a.K;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    float v[1][8];
    uint32_t top = 0;
    for (int col = threadIdx.x * 8; col < K; col += 8192) {
      load_unit(x + col, K - col, v[0]);
      top = max(top, top_bits(v));
    }
    const RowScale s = row_scale(R::reduce<OpMaxU>(top, red, turn));
    for (int col = threadIdx.x * 8; col < K; col += 8192) {
      load_unit(x + col, K - col, v[0]);
      store_unit_i8(a.q + row * a.ldq + col, K - col, round_unit(v[0], s));
    }
    if (threadIdx.x == 0) a.scale[row] = s.s;
  }
}

template <typename T, int G, int U>
hipError_t launch_rows(const QuantRowsArgs& a, hipStream_t st) {
  typedef RowGroup<G> R;
  const int64_t blocks = std::min<int64_t>((a.M + R::ROWS - 1) / R::ROWS, kMostBlocks);
  hipLaunchKernelGGL((k_quantize_rows<T, G, U>), dim3((unsigned)blocks), dim3(R::THREADS), 0, st, a);
  return hipGetLastError();
}
template <typename T>
hipError_t dispatch_rows(const QuantRowsArgs& a, hipStream_t st) {
  if (a.K <= 64) return launch_rows<T, 8, 1>(a, st);
  if (a.K <= 128) return launch_rows<T, 16, 1>(a, st);
  if (a.K <= 256) return launch_rows<T, 32, 1>(a, st);
  if (a.K <= 512) return launch_rows<T, 64, 1>(a, st);
  if (a.K <= 1024) return launch_rows<T, 64, 2>(a, st);
  if (a.K <= 2048) return launch_rows<T, 256, 1>(a, st);
  if (a.K <= 4096) return launch_rows<T, 256, 2>(a, st);
  if (a.K <= 8192) return launch_rows<T, 1024, 1>(a, st);
  hipLaunchKernelGGL((k_quantize_long<T>), dim3((unsigned)std::min<int64_t>(a.M, kMostBlocks)), dim3(1024), 0, st,
                     a);
  return hipGetLastError();
}

// --------------------------------------------------------------------------
// product: a workgroup of WM x WN waves holds BM rows of a and BN rows of w, a
// wave MI x NI tiles of 32 x 32 sums.  128 bytes of k a step, both operands
// through two LDS stages filled by direct-to-LDS loads.  The 16-byte piece p of
// row r lies at piece p ^ ((r >> 1) & 7), so that the 32 rows a fragment read
// touches fall on all banks.  The matrix instruction takes w as its first
// operand: a lane then holds four neighbouring channels of one row.
// --------------------------------------------------------------------------
template <int WM, int WN, int MI, int NI>
struct Tile {
  static constexpr int NW = WM * WN, THREADS = 64 * NW;
  static constexpr int BM = 32 * MI * WM, BN = 32 * NI * WN;
  static constexpr int STAGE = (BM + BN) * 8;  // 16-byte slots
  static constexpr int LB = (BM + BN) / 8 / NW;  // loads a wave issues per stage, 8 rows each
  static_assert((BM + BN) / 8 % NW == 0, "loads divide among the waves");
};

// bytes past `left` cleared
__device__ __forceinline__ i32x4 mask_bytes(i32x4 v, int left) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int n = left - 4 * d;
    if (n <= 0) v[d] = 0;
    else if (n < 4) v[d] &= (int)((1u << (8 * n)) - 1u);
  }
  return v;
}

// four neighbouring channels n.. of row m: scales, bias, activation, rounding
__device__ __forceinline__ void store_quad(const QuantGemmArgs& g, int64_t m, int64_t n, i32x4 sum, float sa,
                                           const float (&tw)[4], const float (&tb)[4]) {
  float v[4];
  const float rs = g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[m]) : 1.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = (float)sum[j] * sa * tw[j] * rs;
    if (g.bias) v[j] += tb[j];
    v[j] = apply_act(g.act, v[j]);
  }
  if (g.out_dtype == SAGA_BF16) {
    uint16_t* o = static_cast<uint16_t*>(g.out) + m * g.ldo + n;
    if (n + 4 <= g.N) {
      *reinterpret_cast<uint2*>(o) = make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                                                (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
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

template <int WM, int WN, int MI, int NI>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm_quant(QuantGemmArgs g, int tiles_m,
                                                                            int tiles_n) {
  typedef Tile<WM, WN, MI, NI> R;
  __shared__ uint4 ring[2 * R::STAGE];
  // Workgroup w runs on XCD w % 8: every XCD gets a run of tiles, and in it eight
  // row tiles share each column tile.
  const int total = tiles_m * tiles_n, per = (total + kXcds - 1) / kXcds;
  const int t = (int)(blockIdx.x % kXcds) * per + (int)(blockIdx.x / kXcds);
  if (t >= total || (int)(blockIdx.x / kXcds) >= per) return;
  const int band = t / (8 * tiles_n), in = t % (8 * tiles_n), bm = min(8, tiles_m - band * 8);
  const int64_t m0 = (int64_t)(band * 8 + in % bm) * R::BM, n0 = (int64_t)(in / bm) * R::BN;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  lds_uint4* lds = (lds_uint4*)ring;

  // this lane's share of the loads: row 8 (wave + j NW) + lane / 8 of the stage
  // (rows past the last read the last one; their sums are not stored)
  const int8_t* const A = g.a + m0 * g.lda;
  const int8_t* const W = g.w + n0 * g.ldw;
  const int K = (int)g.K, kmax = (K - 1) / 16 * 16, last = (K - 1) / 128;
  uint32_t off[R::LB];
  int piece[R::LB];
#pragma unroll
  for (int j = 0; j < R::LB; ++j) {
    const int r = 8 * (wave + j * R::NW) + (lane >> 3);
    const bool is_a = r < R::BM;
    const int rr = is_a ? (int)min((int64_t)r, g.M - 1 - m0) : (int)min((int64_t)(r - R::BM), g.N - 1 - n0);
    off[j] = (uint32_t)rr * (uint32_t)(is_a ? g.lda : g.ldw);
    piece[j] = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
  }
  const auto issue = [&](int c) {
    const uint32_t dst = (uint32_t)(uintptr_t)(lds + (c & 1) * R::STAGE);
#pragma unroll
    for (int j = 0; j < R::LB; ++j) {
      const int grp = wave + j * R::NW;
      const int8_t* base = grp * 8 < R::BM ? A : W;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :
                   : "s"(__builtin_amdgcn_readfirstlane(dst + grp * 1024)),
                     "v"(off[j] + (uint32_t)min(c * 128 + piece[j], kmax)), "s"(base)
                   : "memory", "m0");
    }
  };

  i32x16 acc[MI][NI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[mi][ni][r] = 0;

  const int half = lane >> 5, lr = lane & 31;
  uint32_t at[4];  // this lane's piece of each 32 k, in the row lr of a 32-row tile
#pragma unroll
  for (int s = 0; s < 4; ++s) at[s] = lr * 8 + ((2 * s + half) ^ ((lr >> 1) & 7));
  const auto frag = [&](const lds_uint4* st, int row0, int s) {
    return *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(st + row0 * 8 + at[s]);
  };
  const auto chunk = [&](int c, auto whole) {
    const lds_uint4* st = lds + (c & 1) * R::STAGE;
    const lds_uint4* sa = st + wm * MI * 256;
    const lds_uint4* sw = st + R::BM * 8 + wn * NI * 256;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      i32x4 a[MI], w[NI];
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        w[ni] = frag(sw, ni * 32, s);
        if constexpr (!decltype(whole)::value) w[ni] = mask_bytes(w[ni], K - c * 128 - (2 * s + half) * 16);
      }
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) a[mi] = frag(sa, mi * 32, s);
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
          acc[mi][ni] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[ni], a[mi], acc[mi][ni], 0, 0, 0);
    }
  };

  issue(0);
  for (int c = 0; c < last; ++c) {
    wait_vm<0>();    // chunk c has landed
    ring_barrier();  // for every wave, and all are done with the other stage
    issue(c + 1);
    chunk(c, std::true_type{});
  }
  wait_vm<0>();
  ring_barrier();
  chunk(last, std::false_type{});
  ring_barrier();  // the stages are free

  // Each 32 x 32 tile goes through 4 KB of LDS of this wave's own: a lane holds
  // channels 8 q + 4 half + (0..3) of row lr, and takes back four channels of the
  // rows lane / 8 + 8 i, so that stores cover whole pieces of rows.
  lds_uint4* const mine = lds + wave * 256;
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const i32x16& v = acc[mi][ni];
        *reinterpret_cast<__attribute__((address_space(3))) i32x4*>(mine + at[q]) =
            i32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
      }
      asm volatile("" ::: "memory");
      const int p = lane & 7;
      const int64_t n = n0 + (wn * NI + ni) * 32 + 4 * p;
      float tw[4], tb[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        tw[j] = n + j < g.N ? g.w_scale[n + j] : 0.0f;
        tb[j] = g.bias && n + j < g.N ? g.bias[n + j] : 0.0f;
      }
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 3);
        const int64_t m = m0 + (wm * MI + mi) * 32 + r;
        const i32x4 v =
            *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(mine + r * 8 + (p ^ ((r >> 1) & 7)));
        if (m >= g.M || n >= g.N) continue;
        store_quad(g, m, n, v, g.a_scale[m], tw, tb);
      }
    }
}

template <int WM, int WN, int MI, int NI>
hipError_t launch_tile(const QuantGemmArgs& g0, hipStream_t st) {
  typedef Tile<WM, WN, MI, NI> R;
  const int64_t tn = (g0.N + R::BN - 1) / R::BN;
  const int64_t slice = std::max<int64_t>(1, kMostBlocks / tn) * R::BM;  // rows per launch
  for (int64_t m = 0; m < g0.M; m += slice) {
    QuantGemmArgs g = g0;
    g.M = std::min(slice, g0.M - m);
    g.a += m * g.lda;
    g.a_scale += m;
    if (g.row_scale_deg) g.row_scale_deg += m;
    g.out = static_cast<char*>(g.out) + m * g.ldo * (g.out_dtype == SAGA_BF16 ? 2 : 4);
    const int64_t tm = (g.M + R::BM - 1) / R::BM, blocks = (tm * tn + kXcds - 1) / kXcds * kXcds;
    hipLaunchKernelGGL((k_gemm_quant<WM, WN, MI, NI>), dim3((unsigned)blocks), dim3(R::THREADS), 0, st, g,
                       (int)tm, (int)tn);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_quantize_rows(const QuantRowsArgs& a, hipStream_t st) {
  if (a.M == 0) return hipSuccess;
  return a.dtype == SAGA_BF16 ? dispatch_rows<uint16_t>(a, st) : dispatch_rows<float>(a, st);
}

hipError_t launch_gemm_quant(const QuantGemmArgs& g, hipStream_t st) {
  if (g.M == 0) return hipSuccess;
  if (g.N <= 32) return launch_tile<4, 1, 1, 1>(g, st);
  if (g.N <= 64) return launch_tile<4, 1, 1, 2>(g, st);
  const int64_t large = ((g.M + 255) / 256) * ((g.N + 255) / 256);
  if (large >= 256) return launch_tile<2, 4, 4, 2>(g, st);
  return launch_tile<2, 2, 2, 2>(g, st);
}

}  // namespace saga
