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
typedef __attribute__((address_space(3))) uint4 lds_uint4;

constexpr int64_t kMostBlocks = 1 << 20;  // (a grid holds less than 2^32 threads)

// --------------------------------------------------------------------------
// float rows to 8-bit rows: a row is read once into registers, its largest
// magnitude taken over its lanes, and rounded from there.  Memory bounds it (2^20 x 602
// in bfloat16 391 us, 4.9 TB/s, in float32 675 us, 4.7 TB/s; 100000 x 602 34 and 67 us).
// Past 8192 columns a row is read twice (8000 x 12000 in bfloat16 75 us, 3.8 TB/s).
// --------------------------------------------------------------------------
template <typename T, int G, int U>
__global__ __launch_bounds__(RowGroup<G>::THREADS) void k_quantize_rows(QuantRowsArgs a) {
  typedef RowGroup<G> R;
  __shared__ uint32_t red[2 * (G > 64 ? G / 64 : 1)];
  int turn = 0;
  const int col0 = (threadIdx.x % G) * 8, K = (int)a.K;
  for (int64_t row = blockIdx.x * (int64_t)R::ROWS + threadIdx.x / G; row < a.M;
       row += gridDim.x * (int64_t)R::ROWS) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    Raw<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u].load(x + col0 + u * 8 * G, K - col0 - u * 8 * G);
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[u].clear(K - col0 - u * 8 * G);
      top = max(top, v[u].top());
    }
    const RowScale s = row_scale(R::template reduce<OpMaxU>(top, red, turn));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = col0 + u * 8 * G;
      float f[8];
      v[u].widen(f);
      store_unit_i8(a.q + row * a.ldq + col, K - col, round_unit(f, s));
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
    Raw<T> v;
    uint32_t top = 0;
    for (int64_t col = threadIdx.x * 8; col < K; col += 8192) {
      v.load(x + col, (int)(K - col));
      v.clear((int)(K - col));
      top = max(top, v.top());
    }
    const RowScale s = row_scale(R::reduce<OpMaxU>(top, red, turn));
    for (int64_t col = threadIdx.x * 8; col < K; col += 8192) {
      v.load(x + col, (int)(K - col));
      v.clear((int)(K - col));
      float f[8];
      v.widen(f);
      store_unit_i8(a.q + row * a.ldq + col, K - col, round_unit(f, s));
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
// 16 lanes a row where there are many rows: less of a row's last unit is idle.  Over
// few rows a wave or workgroup a row: more lanes work at all.
template <typename T>
hipError_t dispatch_rows(const QuantRowsArgs& a, hipStream_t st) {
  if (a.M <= 4096) {
    if (a.K <= 512) return launch_rows<T, 64, 1>(a, st);
    if (a.K <= 2048) return launch_rows<T, 256, 1>(a, st);
    if (a.K <= 8192) return launch_rows<T, 1024, 1>(a, st);
  }
  if (a.K <= 128) return launch_rows<T, 16, 1>(a, st);
  if (a.K <= 256) return launch_rows<T, 16, 2>(a, st);
  if (a.K <= 384) return launch_rows<T, 16, 3>(a, st);
  if (a.K <= 512) return launch_rows<T, 16, 4>(a, st);
  if (a.K <= 640) return launch_rows<T, 16, 5>(a, st);
  if (a.K <= 768) return launch_rows<T, 16, 6>(a, st);
  if (a.K <= 1024) return launch_rows<T, 16, 8>(a, st);
  if (a.K <= 1536) return launch_rows<T, 64, 3>(a, st);
  if (a.K <= 2048) return launch_rows<T, 64, 4>(a, st);
  if (a.K <= 4096) return launch_rows<T, 64, 8>(a, st);
  if (a.K <= 8192) return launch_rows<T, 256, 4>(a, st);
  hipLaunchKernelGGL((k_quantize_long<T>), dim3((unsigned)std::min<int64_t>(a.M, kMostBlocks)), dim3(1024), 0, st,
                     a);
  return hipGetLastError();
}

// --------------------------------------------------------------------------
// product: a workgroup of WM x WN waves holds BM rows of a and BN rows of w, a
// wave MI x NI tiles of 16 x 16 sums.  KB bytes of k a stage, ST stages in LDS
// filled by direct-to-LDS loads, which run between the products of a stage rather
// than ahead of them.  The matrix instruction takes w as its first operand: a lane
// then holds four neighbouring channels of one row.  16 x 16 x 64 and not 32 x 32 x
// 32: by itself it reaches 3225 against 2860 TOPS on random bytes, where power
// bounds both.
//
// 32768 x 4096 x 4096 takes 510 us, 2150 TOPS: two thirds of what the instruction
// reaches alone.  The products' units are busy half of the time; the barrier of
// each stage and the two thirds of the CU's LDS bandwidth that fragments and loads
// take stand against it.  Short k (40001 x 1024 x 1024 68 to 75 us, 1.2 POPS) is
// bounded by the first loads and the epilogue of every tile, which nothing hides
// with one workgroup a CU, and by 628 tiles in 2.5 rounds of 256.  The 256 x 256 tiles spill
// two of 128 registers, reloaded after the main loop.
// --------------------------------------------------------------------------
template <int WM, int WN, int MI, int NI, int KB, int ST>
struct Tile {
  static constexpr int NW = WM * WN, THREADS = 64 * NW;
  static constexpr int BM = 16 * MI * WM, BN = 16 * NI * WN;
  static constexpr int PR = KB / 16;                            // 16-byte pieces of a row
  static constexpr int STAGE = (BM + BN) * PR;                  // 16-byte slots
  static constexpr int RL = 64 / PR;                            // rows a load instruction covers
  static constexpr int GROUPS = (BM + BN) / RL;                 // load instructions per stage
  static constexpr int LB = (GROUPS + NW - 1) / NW;             // of one wave
  static constexpr int PH = KB / 64;                            // products' steps of 64 k
  static constexpr int NP = 4 * NI;                             // 16-byte pieces of a wave's row of sums
  static constexpr int SLOTS = ST * STAGE > NW * 16 * NP ? ST * STAGE : NW * 16 * NP;
  static_assert(ST == 2 || GROUPS % NW == 0, "a wait counts the same loads on every wave");
  static constexpr int LDS = SLOTS * 16 + (BM + 2 * BN) * 4;
  static constexpr int WPE = 160 * 1024 / LDS * NW / 4;         // waves a SIMD that LDS has room for
  // slot of piece p of row r: the 16 rows of a fragment read fall on all banks
  __device__ __forceinline__ static int slot(int r, int p) {
    return r * PR + (p ^ (PR == 8 ? (r >> 1) & 7 : (r >> 2) & 3));
  }
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

constexpr float kLargeScale = 0x1p64f;

// four neighbouring channels n.. of row m: scales, bias, activation, rounding
__device__ __forceinline__ void store_quad(const QuantGemmArgs& g, int64_t m, int64_t n, i32x4 sum, float sa,
                                           const f32x4& tw, const f32x4& tb) {
  float v[4];
  // A sum is below 2^31, so its product with a row scale of up to kLargeScale is finite.
  // A larger one comes last: a result that is finite has no infinite step.
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = (float)sum[j] * sa;
  if (__builtin_expect(__ballot(fabsf(sa) > kLargeScale) != 0, 0)) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = fabsf(sa) > kLargeScale ? (float)sum[j] * tw[j] * sa + tb[j] : v[j] * tw[j] + tb[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = v[j] * tw[j] + tb[j];
  }
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

template <int WM, int WN, int MI, int NI, int KB, int ST>
__global__ __launch_bounds__(64 * WM * WN)
__attribute__((amdgpu_waves_per_eu(Tile<WM, WN, MI, NI, KB, ST>::WPE))) void k_gemm_quant(QuantGemmArgs g,
                                                                                         int tiles_m,
                                                                                         int tiles_n) {
  typedef Tile<WM, WN, MI, NI, KB, ST> R;
  __shared__ uint4 ring[R::SLOTS];
  __shared__ f32x4 scales[(R::BM + 2 * R::BN) / 4];  // of the rows, of the channels, and the bias
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

  // this lane's share of the loads: row RL (wave + j NW) + lane / PR of the stage
  // (rows past the last read the last one; their sums are not stored)
  const int8_t* const A = g.a + m0 * g.lda;
  const int8_t* const W = g.w + n0 * g.ldw;
  const int K = (int)g.K, kmax = (K - 1) / 16 * 16, last = (K - 1) / KB;
  uint32_t off[R::LB];
  int piece[R::LB];
#pragma unroll
  for (int j = 0; j < R::LB; ++j) {
    const int r = R::RL * (wave + j * R::NW) + lane / R::PR;
    const bool is_a = r < R::BM;
    const int rr = is_a ? (int)min((int64_t)r, g.M - 1 - m0) : (int)min((int64_t)(r - R::BM), g.N - 1 - n0);
    piece[j] = (R::slot(r, lane % R::PR) % R::PR) * 16;
    off[j] = (uint32_t)rr * (uint32_t)(is_a ? g.lda : g.ldw);
  }
  // load j of chunk c; only the last chunk can reach past the rows' ends, where it
  // reads their last piece again (masked before use)
  const auto issue = [&](int c, int j) {
    const int grp = wave + j * R::NW;
    if (R::GROUPS % R::NW != 0 && grp >= R::GROUPS) return;
    const int8_t* base = grp * R::RL < R::BM ? A : W;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds + (c % ST) * R::STAGE) + grp * 1024)),
                   "v"(off[j] + (uint32_t)min(c * KB + piece[j], kmax)), "s"(base)
                 : "memory", "m0");
  };
#pragma unroll
  for (int c = 0; c < ST; ++c)
    if (c <= last)
#pragma unroll
      for (int j = 0; j < R::LB; ++j) issue(c, j);
  {
    float* sc = reinterpret_cast<float*>(scales);
    for (int i = threadIdx.x; i < R::BM; i += R::THREADS) {
      const int64_t m = min(m0 + i, g.M - 1);
      sc[i] = g.a_scale[m] * (g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[m]) : 1.0f);
    }
    for (int i = threadIdx.x; i < R::BN; i += R::THREADS) {
      const int64_t n = min(n0 + i, g.N - 1);
      sc[R::BM + i] = g.w_scale[n];
      sc[R::BM + R::BN + i] = g.bias ? g.bias[n] : 0.0f;
    }
  }

  i32x4 acc[MI][NI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = i32x4{0, 0, 0, 0};

  const int quarter = lane >> 4, lr = lane & 15;
  uint32_t at[R::PH];  // this lane's piece of each 64 k, in the row lr of a 16-row tile
#pragma unroll
  for (int s = 0; s < R::PH; ++s) at[s] = R::slot(lr, 4 * s + quarter);

  // Fragments of 64 k are read into one half of a and w while those in the other
  // half are multiplied.
  i32x4 a[2][MI], w[2][NI];
  const auto read_w = [&](int c, int s, int b, int ni) {
    w[b][ni] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(
        lds + (c % ST) * R::STAGE + at[s] + (R::BM + (wn * NI + ni) * 16) * R::PR);
  };
  const auto read_a = [&](int c, int s, int b, int mi) {
    a[b][mi] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(
        lds + (c % ST) * R::STAGE + at[s] + (wm * MI + mi) * 16 * R::PR);
  };
  // Multiplies half b row tile by row tile; between the row tiles go the reads of
  // the next fragments (chunk c, step s) and, where FILL, the loads of chunk `fill`:
  // in one run either would hold up the products behind it.
  const auto step = [&](auto fill_tag, int b, int c, int s, int fill) {
    constexpr bool FILL = decltype(fill_tag)::value;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      constexpr int WR = (NI + MI - 1) / MI;
#pragma unroll
      for (int k = 0; k < WR; ++k)
        if (mi * WR + k < NI) read_w(c, s, b ^ 1, mi * WR + k);
      read_a(c, s, b ^ 1, mi);
      if constexpr (FILL) {
#pragma unroll
        for (int j = 0; j < R::LB; ++j)
          if (j * MI / R::LB == mi) issue(fill, j);
      }
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
        acc[mi][ni] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[b][ni], a[b][mi], acc[mi][ni], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Chunk c, its first fragments in half b0.  Before its last step chunk c + 1 has
  // to have landed, for every wave; every wave then has chunk c's fragments in
  // registers, and chunk c + ST takes its stage.
  const auto chunk = [&](auto fill_tag, int c, int b0) {
#pragma unroll
    for (int s = 0; s < R::PH; ++s) {
      const int b = (b0 + s) & 1;
      if (s < R::PH - 1) {
        step(std::false_type{}, b, c, s + 1, 0);
      } else {
        if constexpr (decltype(fill_tag)::value) wait_vm<(ST - 2) * R::LB>();
        else wait_vm<0>();
        ring_barrier();
        step(fill_tag, b, c + 1, 0, c + ST);
      }
    }
  };

  wait_vm<0>();
  ring_barrier();
#pragma unroll
  for (int ni = 0; ni < NI; ++ni) read_w(0, 0, 0, ni);
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) read_a(0, 0, 0, mi);
  constexpr int FLIP = R::PH & 1;  // a chunk of one step leaves the fragments in the other half
  int c = 0;
  for (; c + 1 + ST <= last; c += 2) {
    chunk(std::true_type{}, c, 0);
    chunk(std::true_type{}, c + 1, FLIP);
  }
  if (c + ST <= last) {
    chunk(std::true_type{}, c, 0);
    ++c;
    if constexpr (FLIP) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) w[0][ni] = w[1][ni];
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) a[0][mi] = a[1][mi];
    }
  }
  for (; c < last; ++c) {
    chunk(std::false_type{}, c, 0);
    if constexpr (FLIP) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) w[0][ni] = w[1][ni];
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) a[0][mi] = a[1][mi];
    }
  }
#pragma unroll
  for (int s = 0; s < R::PH; ++s) {
    const int b = s & 1;
    if (s + 1 < R::PH) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) read_w(last, s + 1, b ^ 1, ni);
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) read_a(last, s + 1, b ^ 1, mi);
    }
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) w[b][ni] = mask_bytes(w[b][ni], K - last * KB - (4 * s + quarter) * 16);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
        acc[mi][ni] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[b][ni], a[b][mi], acc[mi][ni], 0, 0, 0);
  }
  ring_barrier();  // the stages are free

  // 16 rows at a time go through LDS of this wave's own: a lane holds channels
  // 4 quarter + (0..3) of row lr, and takes back four channels of a row, so that
  // a store covers whole rows of the wave's columns.
  constexpr int NP = R::NP, ROWS = 64 / (NP < 64 ? NP : 64);
  lds_uint4* const mine = lds + wave * 16 * NP;
  const int p = lane % NP;
  const int64_t n = n0 + (int64_t)wn * NI * 16 + 4 * p;
  const f32x4 tw = scales[(R::BM + wn * NI * 16) / 4 + p], tb = scales[(R::BM + R::BN + wn * NI * 16) / 4 + p];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
      *reinterpret_cast<__attribute__((address_space(3))) i32x4*>(mine + lr * NP + ((ni * 4 + quarter) ^ (lr & (NP - 1)))) =
          acc[mi][ni];
    asm volatile("" ::: "memory");
#pragma unroll 2
    for (int i = 0; i < 16 / ROWS; ++i) {
      const int r = i * ROWS + lane / NP, rr = (wm * MI + mi) * 16 + r;
      const i32x4 v =
          *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(mine + r * NP + (p ^ (r & (NP - 1))));
      const float sa = reinterpret_cast<const float*>(scales)[rr];
      if (m0 + rr < g.M && n < g.N) store_quad(g, m0 + rr, n, v, sa, tw, tb);
    }
  }
}

template <int WM, int WN, int MI, int NI, int KB, int ST>
hipError_t launch_tile(const QuantGemmArgs& g0, hipStream_t st) {
  typedef Tile<WM, WN, MI, NI, KB, ST> R;
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
    hipLaunchKernelGGL((k_gemm_quant<WM, WN, MI, NI, KB, ST>), dim3((unsigned)blocks), dim3(R::THREADS), 0, st, g,
                       (int)tm, (int)tn);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// --------------------------------------------------------------------------
// float rows of up to kFusedK columns: a workgroup quantises BM rows into LDS and
// multiplies them by all of w from there, so that the rows are read once and their
// 8-bit form never leaves the CU.  2^20 x 602 x 128 in bfloat16 takes 405 to 425 us, 3.6
// to 3.8 TB/s of the bytes it cannot do without (a copy: 4.7).  Vector instructions bound
// it, about 25 a value with the epilogue's: counters show them issued in all of its
// cycles, and where the card has just been idle and its clock is lower (1.7 GHz) it
// takes 550 us, as kernels that memory bounds do not.  float32 rows of that size are
// bound by memory (617 us, 4.7 TB/s).
//
// Quantising: 16 lanes a row, four rows a wave and pass, U units a lane.  Rows lie
// an odd number of 16-byte pieces apart, so that the 16 rows a fragment read
// touches fall on all banks.  w's fragments come straight from memory (the second
// level cache), kAhead steps ahead of their products.
// --------------------------------------------------------------------------
constexpr int kFusedK = 1248, kAhead = 4;

__device__ __forceinline__ int fused_pitch(int K) { return ((K + 15) / 16) | 1; }  // in pieces

template <typename T, int BM, int U, int WM, int WN, int NI>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(4))) void k_quant_fused(
    QuantFloatArgs f) {
  constexpr int MI = BM / 16 / WM, RW = BM / (WM * WN);  // RW: rows a wave quantises
  static_assert(MI * 16 * WM == BM && RW % 4 == 0, "whole tiles and passes");
  extern __shared__ uint4 rows[];  // BM rows of `pitch` pieces, and four pieces that a last step may read
  __shared__ float scales[BM];
  const QuantGemmArgs& g = f.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = (int)g.K, pitch = fused_pitch(K), steps = (K + 63) / 64;
  const int64_t m0 = blockIdx.x * (int64_t)BM;
  char* const lds = reinterpret_cast<char*>(rows);

  // four rows a pass, the next pass's on their way while these are rounded (where
  // their registers have room for both)
  constexpr int PASSES = RW / 4, NB = sizeof(T) * U <= 20 ? 2 : 1;
  Raw<T> v[NB][U];
  const auto load_pass = [&](int p) {
    const int64_t m = min(m0 + wave * RW + p * 4 + (lane >> 4), g.M - 1);
    const int col0 = (lane & 15) * 8;
    const T* x = static_cast<const T*>(f.x) + m * f.ldx + col0;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * 128 < K) v[p % NB][u].load(x + u * 128, K - col0 - u * 128);
  };
  load_pass(0);
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (p + 1 < PASSES && NB == 2) load_pass(p + 1);
    const int r = wave * RW + p * 4 + (lane >> 4), col0 = (lane & 15) * 8;
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * 128 < K) {
        v[p % NB][u].clear(K - col0 - u * 128);
        top = max(top, v[p % NB][u].top());
      }
    const RowScale s = row_scale(group_maxu<16>(top));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * 128 < K) {
        const int col = col0 + u * 128;
        float x8[8];
        v[p % NB][u].widen(x8);
        if (col < pitch * 16) *reinterpret_cast<uint2*>(lds + r * pitch * 16 + col) = round_unit(x8, s);
      }
    }
    if ((lane & 15) == 0)
      scales[r] = s.s * (g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[min(m0 + r, g.M - 1)]) : 1.0f);
    if (p + 1 < PASSES && NB == 1) load_pass(p + 1);
  }
  __syncthreads();

  const int wm = wave / WN, wn = wave % WN, quarter = lane >> 4, lr = lane & 15;
  const uint4* const ar = rows + (wm * MI * 16 + lr) * pitch + quarter;
  for (int64_t n0 = wn * NI * 16; n0 < g.N; n0 += WN * NI * 16) {
    const int8_t* wr[NI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) wr[ni] = g.w + min(n0 + ni * 16 + lr, g.N - 1) * g.ldw + quarter * 16;
    i32x4 w[kAhead][NI];
    // (pieces past the rows' end read as 0: what lies behind a row in LDS then does not count)
    const auto load_w = [&](int s, i32x4 (&o)[NI]) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        o[ni] = i32x4{0, 0, 0, 0};
        if (s * 64 + quarter * 16 < K) o[ni] = *reinterpret_cast<const i32x4*>(wr[ni] + s * 64);
      }
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k) load_w(k, w[k]);
    i32x4 acc[MI][NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = i32x4{0, 0, 0, 0};
    for (int s0 = 0; s0 < steps; s0 += kAhead) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (s0 + k < steps) {
          i32x4 a[MI];
#pragma unroll
          for (int mi = 0; mi < MI; ++mi) a[mi] = *reinterpret_cast<const i32x4*>(ar + mi * 16 * pitch + (s0 + k) * 4);
#pragma unroll
          for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
              acc[mi][ni] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[k][ni], a[mi], acc[mi][ni], 0, 0, 0);
        }
        load_w(s0 + k + kAhead, w[k]);
      }
    }
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      const int64_t n = n0 + ni * 16 + quarter * 4;
      if (n >= g.N) continue;
      f32x4 tw, tb;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        tw[j] = n + j < g.N ? g.w_scale[n + j] : 0.0f;
        tb[j] = g.bias && n + j < g.N ? g.bias[n + j] : 0.0f;
      }
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        const int r = (wm * MI + mi) * 16 + lr;
        if (m0 + r < g.M) store_quad(g, m0 + r, n, acc[mi][ni], scales[r], tw, tb);
      }
    }
  }
}

template <typename T, int BM, int U, int WM, int WN, int NI>
hipError_t launch_fused(const QuantFloatArgs& f0, hipStream_t st) {
  const int64_t slice = kMostBlocks * BM;  // rows per launch
  for (int64_t m = 0; m < f0.g.M; m += slice) {
    QuantFloatArgs f = f0;
    QuantGemmArgs& g = f.g;
    g.M = std::min(slice, f0.g.M - m);
    f.x = static_cast<const T*>(f.x) + m * f.ldx;
    if (g.row_scale_deg) g.row_scale_deg += m;
    g.out = static_cast<char*>(g.out) + m * g.ldo * (g.out_dtype == SAGA_BF16 ? 2 : 4);
    const size_t lds = ((size_t)BM * (((g.K + 15) / 16) | 1) + 4) * 16;
    hipLaunchKernelGGL((k_quant_fused<T, BM, U, WM, WN, NI>), dim3((unsigned)((g.M + BM - 1) / BM)),
                       dim3(64 * WM * WN), lds, st, f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// 64 rows by eight waves, each of all rows and 16 columns: w's fragments are loaded
// once a workgroup (2^20 x 602 x 128 in bfloat16, us: 392; 128 rows 442; 128 rows by
// 2 x 4 waves, which load them twice, 523; 64 rows by four waves of 32 columns 434;
// w's first fragments loaded before the rows 423: their registers cost a workgroup a
// CU).
template <typename T, int U>
hipError_t dispatch_fused(const QuantFloatArgs& f, hipStream_t st) {
  if (f.g.N <= 32) return launch_fused<T, 64, U, 4, 2, 1>(f, st);
  if (f.g.N <= 64) return launch_fused<T, 64, U, 2, 4, 1>(f, st);
  return launch_fused<T, 64, U, 1, 8, 1>(f, st);
}

// --------------------------------------------------------------------------
// many short float rows (up to kShortK columns) by a w of up to 128 rows: w's
// fragments fit a wave's registers, so a workgroup keeps them and takes tile after
// tile of 64 rows, the next tile's rows on their way while this one is multiplied and
// stored.  Two LDS buffers in turn: one barrier a tile.  2^20 x 128 x 128 in bfloat16
// takes 137 us, 3.9 TB/s; the rounding and the stores of few bytes a row bound it
// (x 40 channels 101 us, 3.5 TB/s).  Consecutive tiles for a workgroup, instead of every
// 1024th: 142.
// --------------------------------------------------------------------------
constexpr int kShortK = 256;

template <typename T, int U, int WM, int WN>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(4))) void k_quant_short(QuantFloatArgs f,
                                                                                           int64_t tiles) {
  constexpr int BM = 64, MI = BM / 16 / WM, STEPS = U * 2, PITCH = (U * 8) | 1;
  static_assert(WM * WN == 8 && MI * 16 * WM == BM, "eight waves");
  __shared__ uint4 rows[2][BM * PITCH + 4];
  __shared__ float scales[2][BM];
  const QuantGemmArgs& g = f.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = (int)g.K, quarter = lane >> 4, lr = lane & 15, wm = wave / WN, wn = wave % WN;

  // (pieces past the rows' end are 0: what lies there in LDS then does not count)
  const int64_t n = wn * 16 + quarter * 4;
  const int8_t* const wr = g.w + min((int64_t)wn * 16 + lr, g.N - 1) * g.ldw + quarter * 16;
  i32x4 w[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    w[k] = i32x4{0, 0, 0, 0};
    if (k * 64 + quarter * 16 < K) w[k] = *reinterpret_cast<const i32x4*>(wr + k * 64);
  }
  f32x4 tw, tb;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    tw[j] = n + j < g.N ? g.w_scale[n + j] : 0.0f;
    tb[j] = g.bias && n + j < g.N ? g.bias[n + j] : 0.0f;
  }

  Raw<T> v[2][U];  // two passes of four rows
  const int col0 = (lane & 15) * 8;
  const auto load = [&](int64_t t) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int64_t m = min(t * BM + wave * 8 + p * 4 + quarter, g.M - 1);
      const T* x = static_cast<const T*>(f.x) + m * f.ldx + col0;
#pragma unroll
      for (int u = 0; u < U; ++u) v[p][u].load(x + u * 128, K - col0 - u * 128);
    }
  };
  int buf = 0;
  load(blockIdx.x);
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x, buf ^= 1) {
    char* const lds = reinterpret_cast<char*>(rows[buf]);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int r = wave * 8 + p * 4 + quarter;
      uint32_t top = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[p][u].clear(K - col0 - u * 128);
        top = max(top, v[p][u].top());
      }
      const RowScale s = row_scale(group_maxu<16>(top));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x8[8];
        v[p][u].widen(x8);
        *reinterpret_cast<uint2*>(lds + r * PITCH * 16 + col0 + u * 128) = round_unit(x8, s);
      }
      if (lr == 0)
        scales[buf][r] =
            s.s * (g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[min(t * BM + r, g.M - 1)]) : 1.0f);
    }
    if (t + gridDim.x < tiles) load(t + gridDim.x);
    ring_barrier();  // (leaves the loads under way; the other buffer's readers are past the last one)
    const uint4* const ar = rows[buf] + (wm * MI * 16 + lr) * PITCH + quarter;
    i32x4 acc[MI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) acc[mi] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      if (k * 64 < K) {
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
          const i32x4 a = *reinterpret_cast<const i32x4*>(ar + mi * 16 * PITCH + k * 4);
          acc[mi] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[k], a, acc[mi], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int r = (wm * MI + mi) * 16 + lr;
      if (t * BM + r < g.M && n < g.N) store_quad(g, t * BM + r, n, acc[mi], scales[buf][r], tw, tb);
    }
  }
}

template <typename T, int U>
hipError_t launch_short(const QuantFloatArgs& f, hipStream_t st) {
  const int64_t tiles = (f.g.M + 63) / 64;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(tiles, 1024)), dim3(512), 0, st, f, tiles);
    return hipGetLastError();
  };
  if (f.g.N <= 32) return go(k_quant_short<T, U, 4, 2>);
  if (f.g.N <= 64) return go(k_quant_short<T, U, 2, 4>);
  return go(k_quant_short<T, U, 1, 8>);
}

// --------------------------------------------------------------------------
// few rows: 16 of them and 16 channels a workgroup, k divided among its eight
// waves.  Every workgroup quantises the rows for itself (8-bit rows come straight
// from memory): reading w over many CUs at once is what counts, and one launch.
// 1 x 1024 x 1024 of float32 takes 4.8 us, most of it the latency of three loads
// one after another (the row twice, w beside it).
// --------------------------------------------------------------------------
constexpr int kFewK = 4096;

template <typename T>
__global__ __launch_bounds__(512) void k_quant_few(QuantFloatArgs f) {
  constexpr int NW = 8;
  constexpr bool I8 = sizeof(T) == 1;
  extern __shared__ uint4 rows[];  // 16 rows of `pitch` pieces, and four pieces that a last step may read
  __shared__ float scales[16];
  __shared__ i32x4 part[NW][64];
  const QuantGemmArgs& g = f.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15;
  const int K = (int)g.K, pitch = fused_pitch(K), steps = (K + 63) / 64, per = (steps + NW - 1) / NW;
  const int64_t m0 = blockIdx.y * (int64_t)16, n0 = blockIdx.x * (int64_t)16;
  const int here = (int)min((int64_t)16, g.M - m0);
  const int s0 = wave * per, s1 = min(steps, s0 + per);

  const int8_t* const wr = g.w + min(n0 + lr, g.N - 1) * g.ldw + quarter * 16;
  const auto load_w = [&](int s) {
    i32x4 o = {0, 0, 0, 0};
    if (s < s1 && s * 64 + quarter * 16 < K) o = *reinterpret_cast<const i32x4*>(wr + s * 64);
    return o;
  };
  i32x4 w[kAhead], acc = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < kAhead; ++k) w[k] = load_w(s0 + k);

  if constexpr (!I8) {
    char* const lds = reinterpret_cast<char*>(rows);
    for (int r = wave; r < here; r += NW) {
      const T* x = static_cast<const T*>(f.x) + (m0 + r) * f.ldx;
      uint32_t top = 0;
      Raw<T> v;
#pragma unroll 2
      for (int col = lane * 8; col < K; col += 512) {
        v.load(x + col, K - col);
        v.clear(K - col);
        top = max(top, v.top());
      }
      const RowScale s = row_scale(group_maxu<64>(top));
#pragma unroll 2
      for (int col = lane * 8; col < pitch * 16; col += 512) {
        v.load(x + col, K - col);
        v.clear(K - col);
        float x8[8];
        v.widen(x8);
        *reinterpret_cast<uint2*>(lds + r * pitch * 16 + col) = round_unit(x8, s);
      }
      if (lane == 0) scales[r] = s.s;
    }
    __syncthreads();
  }
  // (rows past the last: another row's values, not stored)
  const uint4* const al = rows + min(lr, here - 1) * pitch + quarter;
  const int8_t* const ag = I8 ? g.a + (m0 + min(lr, here - 1)) * g.lda + quarter * 16 : nullptr;
  for (int s = s0; s < s1; s += kAhead) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (s + k < s1) {
        i32x4 a;
        if constexpr (I8) {
          // (a piece that reaches past K holds padding: cleared)
          a = i32x4{0, 0, 0, 0};
          const int left = K - (s + k) * 64 - quarter * 16;
          if (left > 0) a = mask_bytes(*reinterpret_cast<const i32x4*>(ag + (s + k) * 64), left);
        } else {
          a = *reinterpret_cast<const i32x4*>(al + (s + k) * 4);
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[k], a, acc, 0, 0, 0);
      }
      w[k] = load_w(s + k + kAhead);
    }
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int k = 1; k < NW; ++k) acc += part[k][lane];
  const int64_t m = m0 + lr, n = n0 + quarter * 4;
  if (lr >= here || n >= g.N) return;
  f32x4 tw, tb;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    tw[j] = n + j < g.N ? g.w_scale[n + j] : 0.0f;
    tb[j] = g.bias && n + j < g.N ? g.bias[n + j] : 0.0f;
  }
  const float sa = I8 ? g.a_scale[m] : scales[lr];
  store_quad(g, m, n, acc, sa * (g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[m]) : 1.0f), tw, tb);
}

template <typename T>
hipError_t launch_few(const QuantFloatArgs& f, hipStream_t st) {
  const size_t lds = sizeof(T) == 1 ? 0 : ((size_t)16 * (((f.g.K + 15) / 16) | 1) + 4) * 16;
  hipLaunchKernelGGL((k_quant_few<T>), dim3((unsigned)((f.g.N + 15) / 16), (unsigned)((f.g.M + 15) / 16)), dim3(512),
                     lds, st, f);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const QuantRowsArgs& a, hipStream_t st) {
  if (a.M == 0) return hipSuccess;
  return a.dtype == SAGA_BF16 ? dispatch_rows<uint16_t>(a, st) : dispatch_rows<float>(a, st);
}

// Which kernel takes a product (us, measured on bfloat16 or 8-bit rows).
// k_quant_few while its workgroups and their steps are few: 8-bit rows against 64 x
// 64 tiles 16 x 1024 x 1024 3.5 / 5.2, 1000 x 600 x 100 4.2 / 5.1, 16 x 4096 x 4096
// 6.9 / 9.1, 64 x 1024 x 1024 6.0 / 5.5, 64 x 4096 x 4096 18 / 10, 2000 x 130 x 300 5.8 /
// 4.2; float rows, which every workgroup quantises again, against two launches 64 x
// 1024 x 1024 7.0 / 9.5, 128 x 1024 x 1024 8.1 / 9.1, 256 x 1024 x 1024 13 / 9, 16 x 4096 x
// 4096 16 / 13.
bool quant_few(int64_t M, int64_t N, int64_t K, int64_t workgroups, int64_t steps) {
  const int64_t wgs = ((M + 15) / 16) * ((N + 15) / 16);
  return M <= 16384 && N <= 16384 && wgs <= workgroups && wgs * ((K + 63) / 64) <= steps;
}
bool quant_few_float(int64_t M, int64_t N, int64_t K) { return K <= kFewK && quant_few(M, N, K, 512, 8192); }
// k_quant_fused while w is narrow, against two launches: 10000 x 602 x 128 14 / 17,
// 40000 x 602 x 128 24 / 33, 2^18 x 602 x 128 107 / 175, 5000 x 128 x 128 5.5 / 7.4, 16384
// x 602 x 256 18 / 26, 60000 x 1000 x 512 83 / 87, 100000 x 602 x 1024 182 / 163; over
// few rows its sweeps of 128 columns, and of long rows the first, take too long
// (2000 x 1000 x 512 31 / 24, 2000 x 602 x 128 12.5 / 10.4).  (Kernels alone, bfloat16 out.)
// Two launches write and read the 8-bit rows and are 2 to 3 times as long as their bytes:
// 100000 x 602 x 1024 180, 34 for the rows and 147 for the product of short k, against 70;
// 100000 x 1500 x 64 130 against 67.
// Its units for 640 columns serve 257 to 512 too, in bfloat16 at 1.2 to 1.4 times the
// bytes' time like 602 itself (2^20 x 257 x 128 248 / 173, 300 262 / 193, 400 313 / 238, 512
// 354 / 288, 602 409 / 329), in float32 at 1.0 to 1.1.
// k_quant_short from a tile for each of its 1024 workgroups on, against k_quant_fused: in
// bfloat16 2^20 x 128 x 128 137 / 159, 2^20 x 100 x 32 93 / 106, 2^20 x 64 x 64 100 / 101,
// 2^20 x 256 x 128 204 / 219, 65536 x 256 x 128 18.9 / 21.2; in float32 151 / 177, 95 / 98,
// 89 / 98, 249 / 294, 19.7 / 22.9; 40000 x 256 x 128 15.6 / 14.9 in bfloat16, 14.1 / 16.3 in
// float32.  Not where float32 rows of up to 128 columns go into output rows with gaps
// between them, which make their lines' writes partial (2^20 x 128 x 41 153 / 132, x 44
// 160 / 129, x 9 111 / 104; without gaps x 40 118 / 122; 400000 x 128 x 41 39 / 42, 2^20 x
// 200 x 41 198 / 227; in bfloat16 2^20 x 128 x 41 108 / 118, x 44 104 / 118).
bool quant_short(int dtype, const QuantGemmArgs& g) {
  return g.K <= kShortK && g.N <= 128 && g.M >= 65536 && (dtype == SAGA_BF16 || g.K > 128 || g.ldo == g.N);
}
bool quant_fuses(int64_t M, int64_t N, int64_t K) {
  if (quant_few_float(M, N, K)) return true;
  return K <= kFusedK && (N <= 128 ? M >= 4096 || K <= 128 : N <= 512 && M >= 16384);
}

hipError_t launch_quant_fused(int dtype, const QuantFloatArgs& f, hipStream_t st) {
  if (f.g.M == 0) return hipSuccess;
  const bool bf = dtype == SAGA_BF16;
  if (quant_few_float(f.g.M, f.g.N, f.g.K)) return bf ? launch_few<uint16_t>(f, st) : launch_few<float>(f, st);
  if (quant_short(dtype, f.g)) {
    if (f.g.K <= 128) return bf ? launch_short<uint16_t, 1>(f, st) : launch_short<float, 1>(f, st);
    return bf ? launch_short<uint16_t, 2>(f, st) : launch_short<float, 2>(f, st);
  }
  if (f.g.K <= 128) return bf ? dispatch_fused<uint16_t, 1>(f, st) : dispatch_fused<float, 1>(f, st);
  if (f.g.K <= 640) return bf ? dispatch_fused<uint16_t, 5>(f, st) : dispatch_fused<float, 5>(f, st);
  return bf ? dispatch_fused<uint16_t, 10>(f, st) : dispatch_fused<float, 10>(f, st);
}

hipError_t launch_gemm_quant(const QuantGemmArgs& g, hipStream_t st) {
  if (g.M == 0) return hipSuccess;
  if (quant_few(g.M, g.N, g.K, 448, 16384)) return launch_few<int8_t>(QuantFloatArgs{g, nullptr, 0}, st);
  const int64_t cols = (g.N + 127) / 128, rows = (g.M + 127) / 128;
  // Too few 128 x 128 tiles for all CUs: 64 x 64, and seven stages on their way
  // instead of two, as a workgroup's time is its loads' latency (4000 x 4000 x 300 15 /
  // 31).
  if (cols * rows <= 256) return launch_tile<2, 2, 2, 2, 64, 8>(g, st);
  // 256 x 256 by 16 waves, one workgroup a CU, where its tiles fill whole rounds of
  // the CUs to four fifths (us, against 128 x 128 by four waves, three workgroups a
  // CU: 32768 x 4096 x 4096 510 / 670, 16384 x 2048 x 1024, one round, 39 / 50, 16384
  // x 1024 x 4096 96 / 107, 300000 x 128 x 512 117 / 132, 60000 x 600 x 2000 157 / 165,
  // 40001 x 1024 x 1024, 0.82 of three rounds, 72 / 68 to 75; 5000 x 1024 x 4096, 0.63
  // of two, 41 / 36; 20000 x 512 x 512, 0.62 of one, 18 / 17).
  const int64_t large = ((g.M + 255) / 256) * ((g.N + 255) / 256), rounds = (large + 255) / 256;
  // (not where 128-wide tiles leave out a tenth or more of its columns: 2^20 x 602 x
  // 128 to bfloat16 263 / 361.  That is 1.36 times its bytes' time: the ten chunks of a
  // tile's k do not hide its first loads and its epilogue.  Vector units are busy a quarter of
  // the cycles, matrix units 14 %, and rows 608 bytes apart are fetched in 1.17 times their
  // bytes, as 64-byte chunks do not begin on lines.)
  if (large * 5 >= rounds * 256 * 4 && (g.N + 255) / 256 * 20 <= cols * 11) return launch_tile<4, 4, 4, 4, 64, 4>(g, st);
  if (g.N <= 16) return launch_tile<4, 1, 2, 1, 128, 2>(g, st);
  if (g.N <= 32) return launch_tile<4, 1, 2, 2, 128, 2>(g, st);
  if (g.N <= 64) return launch_tile<4, 1, 2, 4, 128, 2>(g, st);
  return launch_tile<2, 2, 4, 4, 64, 3>(g, st);
}

}  // namespace saga
