// Rows in microscaled 4-bit floating point and products of them:
// out = act(rs * (sum_k a_ik w_jk) + bias_j).  Both operands are rows of k (w: one
// output channel a row).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gemm_device.h"
#include "mx4_device.h"

namespace saga {
namespace {

constexpr int64_t kMostBlocks = 1 << 20;  // (a grid holds less than 2^32 threads)

// --------------------------------------------------------------------------
// float rows to 4-bit rows and back: G lanes a row, U units of 8 columns a lane at a time;
// the four lanes of a block join their largest magnitudes.  Blocks know nothing of each
// other, so a long row is divided among workgroups.  Memory bounds both: 2^20 x 602 of bfloat16
// take 343 us to 4 bits (4.7 TB/s) and 363 back (4.4 TB/s), 4099 x 4096 of float32 15 and 17.
// --------------------------------------------------------------------------
template <typename T, int G, int U>
__global__ __launch_bounds__(256) void k_quantize_mx4(Mx4RowsArgs a) {
  const int64_t bytes = (a.K + 1) / 2;
  for (int64_t row = blockIdx.x * (int64_t)(256 / G) + threadIdx.x / G; row < a.M;
       row += gridDim.x * (int64_t)(256 / G)) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    uint8_t* q = a.q + row * a.ldq;
    uint8_t* scale = a.scale + row * a.lds;
    for (int64_t col0 = blockIdx.y * (int64_t)(G * 8 * U) + (threadIdx.x % G) * 8; col0 < a.K + 24;
         col0 += gridDim.y * (int64_t)(G * 8 * U)) {  // (+ 24: all four lanes of the last block)
      Raw<T> v[U];
      int left[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        left[u] = (int)min(a.K - col0 - u * 8 * G, (int64_t)8);
        v[u].load(x + col0 + u * 8 * G, left[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u].clear(left[u]);
        uint32_t top = v[u].top();
        top = max(top, dpp_mov<0xB1>(top));  // quad_perm [1,0,3,2]
        top = max(top, dpp_mov<0x4E>(top));  // quad_perm [2,3,0,1]
        const BlockScale s = block_scale(top);
        const uint32_t o = round_mx4(v[u], s);
        const int64_t at = (col0 + u * 8 * G) / 2;
        if (at + 4 <= bytes) {
          *reinterpret_cast<uint32_t*>(q + at) = o;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (at + j < bytes) q[at + j] = (uint8_t)(o >> (8 * j));
        }
        if ((threadIdx.x & 3) == 0 && left[u] > 0) scale[(col0 + u * 8 * G) / 32] = (uint8_t)s.byte;
      }
    }
  }
}

// 8 values, not to be read again here
__device__ __forceinline__ void store_whole(float* p, const float (&v)[8]) {
  __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4*>(p + 4));
}
__device__ __forceinline__ void store_whole(uint16_t* p, const float (&v)[8]) {
  __builtin_nontemporal_store(u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                    pack_bf16(v[6], v[7])}, reinterpret_cast<u32x4*>(p));
}

template <typename T, int G, int U, bool PAST>
__global__ __launch_bounds__(256) void k_dequantize_mx4(Mx4RowsArgs a) {
  for (int64_t row = blockIdx.x * (int64_t)(256 / G) + threadIdx.x / G; row < a.M;
       row += gridDim.x * (int64_t)(256 / G)) {
    T* x = static_cast<T*>(const_cast<void*>(a.x)) + row * a.ldx;
    const uint8_t* q = a.q + row * a.ldq;
    const uint8_t* scale = a.scale + row * a.lds;
    for (int64_t col0 = blockIdx.y * (int64_t)(G * 8 * U) + (threadIdx.x % G) * 8; col0 < a.K;
         col0 += gridDim.y * (int64_t)(G * 8 * U)) {
      uint32_t o[U], byte[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t col = col0 + u * 8 * G;
        o[u] = byte[u] = 0;
        if (col < a.K) {  // (4 bytes of the last 16 of a row at most)
          o[u] = *reinterpret_cast<const uint32_t*>(q + col / 2);
          byte[u] = scale[col / 32];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t col = col0 + u * 8 * G;
        if (col >= a.K) break;
        const float s = scale_value(byte[u]);
        float v[8];
        const auto pair = [&](auto p, float& lo, float& hi) { lo = p[0], hi = p[1]; };
        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(o[u], s, 0), v[0], v[1]);
        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(o[u], s, 1), v[2], v[3]);
        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(o[u], s, 2), v[4], v[5]);
        pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(o[u], s, 3), v[6], v[7]);
        if (PAST && a.K - col >= 8) store_whole(x + col, v);
        else store_unit(x + col, a.K - col, v);
      }
    }
  }
}

// 16 lanes a row where a row fits them: less of its last unit is idle
template <typename T, int G, int U>
hipError_t launch_rows(const Mx4RowsArgs& a, bool back, hipStream_t st) {
  const int64_t blocks = std::min<int64_t>((a.M + 256 / G - 1) / (256 / G), kMostBlocks / 4);
  const int64_t parts = (a.K + G * 8 * U - 1) / (G * 8 * U);
  const dim3 grid((unsigned)blocks, (unsigned)std::min(parts, std::max<int64_t>(1, 32768 / blocks)));
  // Values that the last cache (256 MiB) does not hold go past it: 2^20 x 602 of bfloat16 363 us
  // against 407, but 4099 x 4096 of float32 28 against 17.
  if (back && a.M * a.K > (int64_t)((256 << 20) / sizeof(T)))
    hipLaunchKernelGGL((k_dequantize_mx4<T, G, U, true>), grid, dim3(256), 0, st, a);
  else if (back) hipLaunchKernelGGL((k_dequantize_mx4<T, G, U, false>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_quantize_mx4<T, G, U>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename T>
hipError_t rows_mx4(const Mx4RowsArgs& a, bool back, hipStream_t st) {
  if (a.K <= 128) return launch_rows<T, 16, 1>(a, back, st);
  if (a.K <= 256) return launch_rows<T, 16, 2>(a, back, st);
  if (a.K <= 384) return launch_rows<T, 16, 3>(a, back, st);
  if (a.K <= 512) return launch_rows<T, 16, 4>(a, back, st);
  if (a.K <= 640) return launch_rows<T, 16, 5>(a, back, st);
  if (a.K <= 768) return launch_rows<T, 16, 6>(a, back, st);
  return launch_rows<T, 64, 2>(a, back, st);
}

// --------------------------------------------------------------------------
// few rows: up to 64 of them and 16 channels a workgroup, k divided among its eight waves.
// Latency bounds it: 1 x 1024 x 1024 takes 3.6 to 4.2 us, 16 x 4096 x 4096 of 4-bit rows 6.7.  A
// lane takes its blocks of a and w straight from memory; float rows are rounded in
// its registers, since the 32 columns that a matrix instruction wants of a lane are
// a block.
// --------------------------------------------------------------------------
template <int C>
__device__ __forceinline__ void finish(int act, float (&v)[C]) {
  if (act == SAGA_ACT_RELU) {
    // (a NaN stays: it is all that is left of a row that held no number; -0 becomes +0)
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] = __builtin_elementwise_maximum(v[j], 0.0f);
  } else if (act != SAGA_ACT_NONE) {
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] = apply_act(act, v[j]);
  }
}

// four neighbouring channels n.. of row m: scale, bias, activation, rounding
__device__ __forceinline__ void store_quad(const Mx4GemmArgs& g, int64_t m, int64_t n, const f32x4& sum, float rs,
                                           const f32x4& tb) {
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = sum[j] * rs + tb[j];
  finish(g.act, v);
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

// (AHEAD steps' loads at a time: what registers hold, and not more than a wave has)
template <typename T, int MI, int AHEAD>
__global__ __launch_bounds__(512) void k_mx4_few(Mx4GemmArgs g, int64_t tiles_n, int64_t tiles) {
  constexpr int NW = 8;
  __shared__ f32x4 part[NW][MI][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15, K = (int)g.K;
  const int all = (K + 127) / 128, steps = (all - wave + NW - 1) / NW;  // of this wave: wave, wave + NW, ..
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t m0 = tile / tiles_n * (16 * MI), n0 = tile % tiles_n * 16;
    RowSource<T> a[AHEAD][MI];
    RowSource<uint8_t> w[AHEAD];
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)  // (rows past the last: not stored)
        a[d][mi].at(g.a, g.lda, g.a_scale, g.lda_s, min(m0 + mi * 16 + lr, g.M - 1));
      w[d].at(g.w, g.ldw, g.w_scale, g.ldw_s, min(n0 + lr, g.N - 1));
    }
    const auto load = [&](int d, int i) {
      const int b = (wave + i * NW) * 4 + quarter;
      w[d].load(b, K);
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) a[d][mi].load(b, K);
    };
    f32x4 acc[MI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) acc[mi] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int ib = 0; ib < steps; ib += AHEAD) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) load(d, ib + d);
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) {
        const int i = ib + d, s = wave + i * NW, b = s * 4 + quarter;
        if (i >= steps) continue;
        const bool last = s == all - 1;
        const Mx4Block wb = w[d].take(b, K, last);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) acc[mi] = mma_mx4(wb, a[d][mi].take(b, K, last), acc[mi]);
      }
    }
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) part[wave][mi][lane] = acc[mi];
    __syncthreads();
    if (wave < MI) {
      f32x4 sum = part[0][wave][lane];
#pragma unroll
      for (int k = 1; k < NW; ++k) sum += part[k][wave][lane];
      const int64_t m = m0 + wave * 16 + lr, n = n0 + quarter * 4;
      if (m < g.M && n < g.N)
        store_quad(g, m, n, sum, g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[m]) : 1.0f, bias_quad(g, n));
    }
    __syncthreads();
  }
}

template <typename T, int MI, int AHEAD>
hipError_t launch_few_steps(const Mx4GemmArgs& g, hipStream_t st) {
  const int64_t tn = (g.N + 15) / 16, tiles = tn * ((g.M + 16 * MI - 1) / (16 * MI));
  hipLaunchKernelGGL((k_mx4_few<T, MI, AHEAD>), dim3((unsigned)std::min(tiles, kMostBlocks)), dim3(512), 0, st, g, tn,
                     tiles);
  return hipGetLastError();
}
template <typename T, int MI>
hipError_t launch_few_rows(const Mx4GemmArgs& g, hipStream_t st) {
  constexpr int MOST = sizeof(T) == 1 ? 4 : std::min(4, 8 / (MI * (int)sizeof(T) / 2));
  const int64_t steps = (g.K + 1023) / 1024;  // of a wave
  if constexpr (MOST >= 4)
    if (steps > 2) return launch_few_steps<T, MI, 4>(g, st);
  if constexpr (MOST >= 2)
    if (steps > 1) return launch_few_steps<T, MI, 2>(g, st);
  return launch_few_steps<T, MI, 1>(g, st);
}
template <typename T>
hipError_t launch_few(const Mx4GemmArgs& g, hipStream_t st) {
  if (g.M <= 16) return launch_few_rows<T, 1>(g, st);
  if (g.M <= 32) return launch_few_rows<T, 2>(g, st);
  return launch_few_rows<T, 4>(g, st);
}

// --------------------------------------------------------------------------
// large products of 4-bit rows: a workgroup of WM x WN waves holds BM rows of a and BN
// rows of w, a wave MI x NI tiles of 32 x 32 sums.  64 bytes (128 k) of every row a stage,
// ST stages in LDS filled by direct-to-LDS loads, which run between
// the products of a stage rather than ahead of them.  The matrix instruction takes w as
// its first operand: a lane then holds groups of four neighbouring channels of one row.
// 32 x 32 x 64 and not 16 x 16 x 128: by itself it reaches 6.5 against 5.5 PFLOP/s on random
// bytes, where power bounds both.
//
// 16384 x 4096 x 4096 takes 156 to 180 us, 3.1 to 3.5 PFLOP/s: half of what the instruction reaches alone.
// Nothing runs beside a tile's first loads (about 2 us) and its results' way out (128 KB, 7 us at
// the copy's rate while all CUs write), and a stage's 32 KB take longer than its products.
// 256 x 256 by 16 waves of 64 x 64 sums: 1028 us (spills); 8 waves of 64 x 128 the same as 128 x 64
// (within 3 %); 128 x 128 by 4 waves 219, by 128 x 256 221.
//
// A lane takes the pieces (16 bytes, a block) 2 (l / 32) and 2 (l / 32) + 1 of a stage in
// its two steps, so that both scales are one 16-bit read.
// --------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) uint4 lds_uint4;
typedef const __attribute__((address_space(3))) u32x4 lds_cu32x4;

template <int WM, int WN, int MI, int NI, int ST>
struct Tile {
  static constexpr int NW = WM * WN, THREADS = 64 * NW;
  static constexpr int BM = 32 * MI * WM, BN = 32 * NI * WN, ROWS = BM + BN;
  static constexpr int PR = 4;                                  // 16-byte pieces of a row
  static constexpr int STAGE = ROWS * PR;                       // 16-byte slots
  static constexpr int GROUPS = ROWS / 16;                      // load instructions per stage
  static constexpr int LB = (GROUPS + NW - 1) / NW;             // of one wave
  // Scales are loaded for four stages at a time, 16 bytes a row, a quarter of a wave's SR rows
  // with each stage: a word a row for every stage asked for as many lines as the rows do.
  // The four stages AHEAD of the present four are on their way.
  static constexpr int SR = (ROWS + NW - 1) / NW / 4 * 4, AHEAD = (ST + 7) / 4, SETS = AHEAD + 1;
  static constexpr int LOADS = LB + 1;
  static constexpr int NP = 8 * NI;                             // 16-byte pieces of a wave's row of sums
  static constexpr int SLOTS = ST * STAGE > NW * 32 * NP ? ST * STAGE : NW * 32 * NP;
  static_assert(SR <= 64 && SR * NW == ROWS, "one load instruction for a quarter of a wave's scales");
  static_assert(ST == 2 || (GROUPS % NW == 0 && ROWS % NW == 0), "a wait counts the same loads on every wave");
  static constexpr int LDS = SLOTS * 16 + SETS * ROWS * 16 + ROWS * 4;
  static constexpr int WAVES = 160 * 1024 / LDS * NW / 4;       // waves a SIMD that LDS has room for
  static constexpr int WPE = WAVES < 4 ? WAVES : 4;             // (more would spill registers)
  // slot of piece p of row r: the 16 rows of a fragment read fall on all banks
  __device__ __forceinline__ static int slot(int r, int p) { return r * PR + (p ^ ((r >> 2) & 3)); }
};

template <int OPSEL>
__device__ __forceinline__ f32x16 mma_tile(const u32x4& w, const u32x4& a, const f32x16& c, uint32_t sw, uint32_t sa) {
  const i32x8 x = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
  const i32x8 y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, OPSEL, (int)sw, OPSEL, (int)sa);
}

template <int WM, int WN, int MI, int NI, int ST>
__global__ __launch_bounds__(64 * WM * WN)
__attribute__((amdgpu_waves_per_eu(Tile<WM, WN, MI, NI, ST>::WPE))) void k_gemm_mx4(Mx4GemmArgs g, int tiles_m,
                                                                                    int tiles_n) {
  typedef Tile<WM, WN, MI, NI, ST> R;
  __shared__ uint4 ring[R::SLOTS];
  __shared__ uint32_t scales[R::SETS][R::ROWS * 4];
  __shared__ f32x4 ends[R::ROWS / 4];  // the rows' degrees, the channels' bias
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

  // this lane's share of the loads: row 16 (wave + j NW) + lane / 4 of the stage
  // (rows past the last read the last one; their sums are not stored)
  const uint8_t* const A = static_cast<const uint8_t*>(g.a) + m0 * g.lda;
  const uint8_t* const W = g.w + n0 * g.ldw;
  const int K = (int)g.K, bytes = (K + 1) / 2, kmax = (bytes - 1) / 16 * 16, last = (bytes - 1) / 64;
  const auto row_of = [&](int r) {
    return r < R::BM ? (int)min((int64_t)r, g.M - 1 - m0) : (int)min((int64_t)(r - R::BM), g.N - 1 - n0);
  };
  uint32_t off[R::LB];
  int piece[R::LB];
#pragma unroll
  for (int j = 0; j < R::LB; ++j) {
    const int r = 16 * (wave + j * R::NW) + lane / 4;
    piece[j] = (R::slot(r, lane % 4) % 4) * 16;
    off[j] = (uint32_t)row_of(r) * (uint32_t)(r < R::BM ? g.lda : g.ldw);
  }
  const int smax = (K - 1) / 128;  // the last scales' word
  // a quarter of this wave's scales of the chunks 4 t.. : lane / 4 a row, lane % 4 a chunk
  const auto issue_scales = [&](int t, int q) {
    const int r = wave * R::SR + q * (R::SR / 4) + lane / 4;
    const bool is_a = r < R::BM;
    const uint32_t at = (uint32_t)row_of(r) * (uint32_t)(is_a ? g.lda_s : g.ldw_s) + min(t * 4 + (lane & 3), smax) * 4;
    const uint8_t* const from = (is_a ? g.a_scale + m0 * g.lda_s : g.w_scale + n0 * g.ldw_s) + at;
    if (R::SR == 64 || lane < R::SR)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                   :
                   : "s"(__builtin_amdgcn_readfirstlane(
                         (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t*)scales[t % R::SETS] +
                         (wave * R::SR + q * (R::SR / 4)) * 16)),
                     "v"(from)
                   : "memory", "m0");
  };
  // load j of chunk c; only the last chunk can reach past the rows' ends, where it
  // reads their last piece again (masked before use).  Load LB: scales, of a quarter of
  // the rows for four chunks; the first ones come before all chunks.
  const auto issue = [&](int c, int j) {
    if (j == R::LB) {
      const int i = 4 * R::AHEAD - ST + c;
      issue_scales(i >> 2, i & 3);
      return;
    }
    const int grp = wave + j * R::NW;
    if (R::GROUPS % R::NW != 0 && grp >= R::GROUPS) return;
    const uint8_t* base = grp * 16 < R::BM ? A : W;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds + (c % ST) * R::STAGE) + grp * 1024)),
                   "v"(off[j] + (uint32_t)min(c * 64 + piece[j], kmax)), "s"(base)
                 : "memory", "m0");
  };
  // (degrees and bias go first, straight to LDS too: a load into registers would be waited for
  // with all that are under way)
  const auto issue_ends = [&](const void* from, int64_t i0, int64_t count, int at, int n) {
    for (int i = wave * 64; i < n; i += R::THREADS)
      if (n % 64 == 0 || i + lane < n)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                     :
                     : "s"(__builtin_amdgcn_readfirstlane(
                           (uint32_t)(uintptr_t)(__attribute__((address_space(3))) f32x4*)ends + (at + i) * 4)),
                       "v"(static_cast<const char*>(from) + min(i0 + i + lane, count - 1) * 4)
                     : "memory", "m0");
  };
  if (g.row_scale_deg) issue_ends(g.row_scale_deg, m0, g.M, 0, R::BM);
  if (g.bias) issue_ends(g.bias, n0, g.N, R::BM, R::BN);
  else
    for (int i = threadIdx.x; i < R::BN; i += R::THREADS) reinterpret_cast<float*>(ends)[R::BM + i] = 0.0f;
#pragma unroll
  for (int i = 0; i < 4 * R::AHEAD - ST; ++i) issue_scales(i >> 2, i & 3);
#pragma unroll
  for (int c = 0; c < ST; ++c)
    if (c <= last)
#pragma unroll
      for (int j = 0; j < R::LOADS; ++j) issue(c, j);
  f32x16 acc[MI][NI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[mi][ni][i] = 0.0f;

  const int half = lane >> 5, lr = lane & 31;
  uint32_t at[2];  // this lane's piece of each step, in the row lr of a 32-row tile
#pragma unroll
  for (int s = 0; s < 2; ++s) at[s] = R::slot(lr, 2 * half + s);

  // Fragments of a step are read into one half of a and w while those in the other
  // half are multiplied.
  u32x4 a[2][MI], w[2][NI];
  uint32_t sa[MI], sw[NI], sa_next[MI], sw_next[NI];
  const auto read_w = [&](int c, int s, int ni) {
    w[s][ni] = *(lds_cu32x4*)(lds + (c % ST) * R::STAGE + at[s] + (R::BM + (wn * NI + ni) * 32) * R::PR);
  };
  const auto read_a = [&](int c, int s, int mi) {
    a[s][mi] = *(lds_cu32x4*)(lds + (c % ST) * R::STAGE + at[s] + (wm * MI + mi) * 32 * R::PR);
  };
  const auto read_scales = [&](int c) {
    const uint16_t* const sc =
        reinterpret_cast<const uint16_t*>(scales[c / 4 % R::SETS]) + lr * 8 + (c & 3) * 2 + half;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) sa_next[mi] = sc[(wm * MI + mi) * 256];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) sw_next[ni] = sc[(R::BM + (wn * NI + ni) * 32) * 8];
  };
  const auto turn = [&] {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) sa[mi] = sa_next[mi];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) sw[ni] = sw_next[ni];
  };
  // Chunk c, its first fragments and scales read.  Before its last step chunk
  // c + 1 has to have landed, for every wave; every wave then has chunk c's fragments in
  // registers, and chunk c + ST takes its stage.  The reads of the next fragments and, where
  // FILL, the loads go between the row tiles: in one run either would hold up the products
  // behind it.
  const auto chunk = [&](auto fill_tag, int c) {
    constexpr bool FILL = decltype(fill_tag)::value;
    constexpr int WR = (NI + MI - 1) / MI;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
      for (int k = 0; k < WR; ++k)
        if (mi * WR + k < NI) read_w(c, 1, mi * WR + k);
      read_a(c, 1, mi);
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = mma_tile<0>(w[0][ni], a[0][mi], acc[mi][ni], sw[ni], sa[mi]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (FILL) wait_vm<(ST - 2) * R::LOADS>();
    else wait_vm<0>();
    ring_barrier();
    read_scales(c + 1);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
      for (int k = 0; k < WR; ++k)
        if (mi * WR + k < NI) read_w(c + 1, 0, mi * WR + k);
      read_a(c + 1, 0, mi);
      if constexpr (FILL) {
#pragma unroll
        for (int j = 0; j < R::LOADS; ++j)
          if (j * MI / R::LOADS == mi) issue(c + ST, j);
      }
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = mma_tile<1>(w[1][ni], a[1][mi], acc[mi][ni], sw[ni], sa[mi]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (last >= ST - 1 && R::GROUPS % R::NW == 0) wait_vm<(ST - 1) * R::LOADS>();
  else wait_vm<0>();
  ring_barrier();
  read_scales(0);
  turn();
#pragma unroll
  for (int ni = 0; ni < NI; ++ni) read_w(0, 0, ni);
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) read_a(0, 0, mi);
  int c = 0;
  for (; c + ST <= last; ++c) {
    chunk(std::true_type{}, c);
    turn();
  }
  for (; c < last; ++c) {
    chunk(std::false_type{}, c);
    turn();
  }
  // the last chunk: w's bytes past the rows' ends are zeros, scales past them 1 (they
  // might stand for NaN)
#pragma unroll
  for (int ni = 0; ni < NI; ++ni) read_w(last, 1, ni);
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) read_a(last, 1, mi);
  const int left = bytes - last * 64 - half * 32;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (left < 16 * (s + 1)) {
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) w[s][ni] = clear_bytes(w[s][ni], left - 16 * s);
    }
    if (left <= 16 * s) {
      const uint32_t keep = s ? 0x00ffu : 0xff00u, one = s ? 0x7f00u : 0x007fu;
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) sw[ni] = (sw[ni] & keep) | one;
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) sa[mi] = (sa[mi] & keep) | one;
    }
  }
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      acc[mi][ni] = mma_tile<0>(w[0][ni], a[0][mi], acc[mi][ni], sw[ni], sa[mi]);
      acc[mi][ni] = mma_tile<1>(w[1][ni], a[1][mi], acc[mi][ni], sw[ni], sa[mi]);
    }
  ring_barrier();  // the stages are free

  // 32 rows at a time go through LDS of this wave's own: a lane holds channels
  // 8 i + 4 half + (0..3) of row lr, and takes back eight channels of a row (four of
  // float32 ones), so that a store covers whole rows of the wave's columns.
  const auto row_scale = [&](int r) {
    return g.row_scale_deg ? rsqrt_deg(reinterpret_cast<const int*>(ends)[r]) : 1.0f;
  };
  const f32x4* const bias = ends + (R::BM + wn * NI * 32) / 4;
  // bfloat16 and no activation but ReLU: rounded before they go through LDS.  (Others after it,
  // from a loop: their code for every value here would be longer than the rest.)
  if (g.out_dtype == SAGA_BF16 && g.act <= SAGA_ACT_RELU) {
    const float floor = g.act == SAGA_ACT_RELU ? 0.0f : -INFINITY;  // (a NaN stays; -0 becomes +0)
    constexpr int NP = 4 * NI, RS = 64 / NP;
    lds_uint4* const mine = lds + wave * 32 * NP;
    const int p = lane % NP;
    const int64_t n = n0 + (int64_t)wn * NI * 32 + 8 * p;
    const auto turned = [](int r) { return (r * NP / 16) & (NP - 1); };  // (16 rows fall on all banks)
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const float rs = row_scale((wm * MI + mi) * 32 + lr);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 b = bias[ni * 8 + i * 2 + half];
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = __builtin_elementwise_maximum(acc[mi][ni][4 * i + j] * rs + b[j], floor);
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          *(__attribute__((address_space(3))) u32x2*)(
              (__attribute__((address_space(3))) char*)(mine + lr * NP + ((ni * 4 + i) ^ turned(lr))) + half * 8) =
              u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 32 / RS; ++i) {
        const int r = i * RS + lane / NP, rr = (wm * MI + mi) * 32 + r;
        const u32x4 v = *(lds_cu32x4*)(mine + r * NP + (p ^ turned(r)));
        if (m0 + rr >= g.M || n >= g.N) continue;
        uint16_t* const o = static_cast<uint16_t*>(g.out) + (m0 + rr) * g.ldo + n;
        if (n + 8 <= g.N) {
          *reinterpret_cast<u32x4*>(o) = v;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (n + j < g.N) o[j] = (uint16_t)(v[j / 2] >> (16 * (j & 1)));
        }
      }
    }
    return;
  }
  constexpr int NP = R::NP, RS = 64 / NP;
  lds_uint4* const mine = lds + wave * 32 * NP;
  const int p = lane % NP;
  const int64_t n = n0 + (int64_t)wn * NI * 32 + 4 * p;
  const f32x4 tb = bias[p];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<__attribute__((address_space(3))) f32x4*>(
            mine + lr * NP + ((ni * 8 + i * 2 + half) ^ (lr & (NP - 1)))) =
            f32x4{acc[mi][ni][4 * i], acc[mi][ni][4 * i + 1], acc[mi][ni][4 * i + 2], acc[mi][ni][4 * i + 3]};
    asm volatile("" ::: "memory");
#pragma unroll 2
    for (int i = 0; i < 32 / RS; ++i) {
      const int r = i * RS + lane / NP, rr = (wm * MI + mi) * 32 + r;
      const f32x4 v =
          *reinterpret_cast<const __attribute__((address_space(3))) f32x4*>(mine + r * NP + (p ^ (r & (NP - 1))));
      const float rs = row_scale(rr);
      if (m0 + rr < g.M && n < g.N) store_quad(g, m0 + rr, n, v, rs, tb);
    }
  }
}

template <int WM, int WN, int MI, int NI, int ST>
hipError_t launch_tile(const Mx4GemmArgs& g0, hipStream_t st) {
  typedef Tile<WM, WN, MI, NI, ST> R;
  const int64_t tn = (g0.N + R::BN - 1) / R::BN;
  const int64_t slice = std::max<int64_t>(1, kMostBlocks / tn) * R::BM;  // rows per launch
  for (int64_t m = 0; m < g0.M; m += slice) {
    Mx4GemmArgs g = g0;
    g.M = std::min(slice, g0.M - m);
    g.a = static_cast<const uint8_t*>(g.a) + m * g.lda;
    g.a_scale += m * g.lda_s;
    if (g.row_scale_deg) g.row_scale_deg += m;
    g.out = static_cast<char*>(g.out) + m * g.ldo * (g.out_dtype == SAGA_BF16 ? 2 : 4);
    const int64_t tm = (g.M + R::BM - 1) / R::BM, blocks = (tm * tn + kXcds - 1) / kXcds * kXcds;
    hipLaunchKernelGGL((k_gemm_mx4<WM, WN, MI, NI, ST>), dim3((unsigned)blocks), dim3(R::THREADS), 0, st, g, (int)tm,
                       (int)tn);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// --------------------------------------------------------------------------
// many float rows by a narrow w (2^20 x 602 x 128 of bfloat16 315 us, 4.9 TB/s of the bytes it cannot do
// without; of float32 720, 4.3; rounding and product in two launches 516): w stays in LDS in the
// order of its fragments, and a
// wave takes 16 rows after 16 rows past it, 128 k at a time, with the next 128 on their
// way.  Rows are loaded 16 lanes a row and rounded there; a piece of LDS of the wave's
// own turns the four bytes that a lane then has into the block that the matrix
// instruction wants of it.  The rows' 4-bit form never leaves the CU.
//
// A lane's channels of all NT column tiles are neighbours (tile t takes the channels
// 4 NT q + 4 t + (0..3), q = 0..3), so that a store holds 16 bytes.
// --------------------------------------------------------------------------
// channels n.. of row m, 8 of them
__device__ __forceinline__ void store_oct(const Mx4GemmArgs& g, int64_t m, int64_t n, const f32x4& lo, const f32x4& hi,
                                          float rs, const f32x4& blo, const f32x4& bhi) {
  if (g.out_dtype != SAGA_BF16 || n + 8 > g.N) {
    if (n < g.N) store_quad(g, m, n, lo, rs, blo);
    if (n + 4 < g.N) store_quad(g, m, n + 4, hi, rs, bhi);
    return;
  }
  float v[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = lo[j] * rs + blo[j], v[4 + j] = hi[j] * rs + bhi[j];
  finish(g.act, v);
  store_unit(static_cast<uint16_t*>(g.out) + m * g.ldo + n, 8, v);
}

constexpr int kStreamWaves = 8;
// LDS: w's fragments, their scales (a byte for each of four steps), the bias, the waves' pieces
struct StreamSpace {
  int steps, w_scales, bias, turn, total;  // (bytes)
  __host__ __device__ StreamSpace(int64_t K, int NT) {
    steps = (int)((K + 127) / 128);
    w_scales = steps * NT * 1024;
    bias = w_scales + (steps + 3) / 4 * NT * 256;
    turn = bias + NT * 64;
    total = turn + kStreamWaves * (1024 + 64);
  }
};

// waves a SIMD: eight column tiles spill at four (us, two / four: 2^20 x 602 x 128 of float32 720 / 973, of bfloat16,
// which spill 18 registers, 315 / 329, 2^20 x 128 x 128 127 / 140, 65536 x 1024 x 128 32 / 38)
template <int NT>
constexpr int kStreamPerSimd = NT == 8 ? 2 : 4;

template <typename T, int NT>
__global__ __launch_bounds__(64 * kStreamWaves)
__attribute__((amdgpu_waves_per_eu(kStreamPerSimd<NT>))) void k_mx4_stream(
    Mx4GemmArgs g, int64_t tiles) {
  extern __shared__ uint4 space[];
  const int K = (int)g.K;
  const StreamSpace at(K, NT);
  char* const base = reinterpret_cast<char*>(space);
  u32x4* const lw = reinterpret_cast<u32x4*>(base);
  uint32_t* const lws = reinterpret_cast<uint32_t*>(base + at.w_scales);
  f32x4* const lb = reinterpret_cast<f32x4*>(base + at.bias);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quarter = lane >> 4, lr = lane & 15;
  uint32_t* const turn = reinterpret_cast<uint32_t*>(base + at.turn + wave * 1088);
  uint8_t* const turn_scale = reinterpret_cast<uint8_t*>(turn) + 1024;
  const int steps = at.steps;

  for (int f = wave; f < steps * NT; f += kStreamWaves) {
    const int s = f / NT, t = f % NT;
    RowSource<uint8_t> w;
    w.at(g.w, g.ldw, g.w_scale, g.ldw_s, min((int64_t)((lr >> 2) * 4 * NT + t * 4 + (lr & 3)), g.N - 1));
    w.load(s * 4 + quarter, K);
    const Mx4Block b = w.take(s * 4 + quarter, K, s == steps - 1);
    lw[f * 64 + lane] = b.v;
    reinterpret_cast<uint8_t*>(lws + ((s / 4) * NT + t) * 64 + lane)[s % 4] = (uint8_t)b.scale;
  }
  for (int i = threadIdx.x; i < NT * 4; i += 64 * kStreamWaves) lb[i] = bias_quad(g, i * 4);
  __syncthreads();

  const int64_t stride = (int64_t)gridDim.x * kStreamWaves;
  int64_t tile = (int64_t)blockIdx.x * kStreamWaves + wave;
  if (tile >= tiles) return;
  // four rows a load: this lane's columns col.. of rows 4 j + lane / 16
  Raw<T> v[4];
  const T* x;
  uint32_t off[4];
  const auto rows_at = [&](int64_t t) {
    x = static_cast<const T*>(g.a) + t * 16 * g.lda;
    const int here = (int)min((int64_t)16, g.M - t * 16) - 1;  // (rows past the last: not stored)
#pragma unroll
    for (int j = 0; j < 4; ++j) off[j] = (uint32_t)min(4 * j + quarter, here) * (uint32_t)g.lda + lr * 8;
  };
  const auto load = [&](int s) {
    if (s * 128 + 128 <= K) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j].load(x + (off[j] + s * 128), 8);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j].load(x + (off[j] + s * 128), K - s * 128 - lr * 8);
    }
  };
  rows_at(tile);
  load(0);
  for (; tile < tiles; tile += stride) {
    const int64_t m = tile * 16 + lr;
    const float rs = g.row_scale_deg ? rsqrt_deg(g.row_scale_deg[min(m, g.M - 1)]) : 1.0f;
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < steps; s0 += 4) {
      const auto step = [&](auto opsel) {
        constexpr int J = decltype(opsel)::value;
        const int s = s0 + J;
        if (s >= steps) return;
        if (s * 128 + 128 > K) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j].clear(K - s * 128 - lr * 8);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t top = v[j].top();
          top = max(top, dpp_mov<0xB1>(top));
          top = max(top, dpp_mov<0x4E>(top));
          const BlockScale b = block_scale(top);
          turn[((4 * j + quarter) * 4 + ((lr >> 2) ^ j)) * 4 + (lr & 3)] = round_mx4(v[j], b);
          if ((lr & 3) == 0) turn_scale[(lr >> 2) * 16 + 4 * j + quarter] = (uint8_t)b.byte;
        }
        if (s + 1 < steps) {
          load(s + 1);
        } else if (tile + stride < tiles) {
          rows_at(tile + stride);
          load(0);
        }
        asm volatile("" ::: "memory");
        Mx4Block a;
        a.v = *reinterpret_cast<const u32x4*>(turn + (lr * 4 + (quarter ^ (lr >> 2))) * 4);
        a.scale = turn_scale[quarter * 16 + lr];
        asm volatile("" ::: "memory");
        const u32x4* const f = lw + s * NT * 64 + lane;
        const uint32_t* const fs = lws + (s0 / 4) * NT * 64 + lane;
        const i32x8 y = {(int)a.v[0], (int)a.v[1], (int)a.v[2], (int)a.v[3], 0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const u32x4 w = f[t * 64];
          const i32x8 z = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
          acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(z, y, acc[t], 4, 4, J, (int)fs[t * 64], 0, (int)a.scale);
        }
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
    }
    if (m < g.M) {
      if constexpr (NT == 1) {
        if (quarter * 4 < g.N) store_quad(g, m, quarter * 4, acc[0], rs, lb[quarter]);
      } else {
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
          __builtin_amdgcn_sched_barrier(0);  // (two tiles' values at a time: registers)
          store_oct(g, m, quarter * 4 * NT + t * 4, acc[t], acc[t + 1], rs, lb[quarter * NT + t], lb[quarter * NT + t + 1]);
        }
      }
    }
  }
}

template <typename T, int NT>
hipError_t launch_stream(const Mx4GemmArgs& g, hipStream_t st) {
  const int64_t tiles = (g.M + 15) / 16;
  const int lds = StreamSpace(g.K, NT).total, per = std::max(1, std::min(kStreamPerSimd<NT> / 2, 160 * 1024 / lds));
  const int64_t blocks = std::min<int64_t>((tiles + kStreamWaves - 1) / kStreamWaves, 256 * per);
  hipLaunchKernelGGL((k_mx4_stream<T, NT>), dim3((unsigned)blocks), dim3(64 * kStreamWaves), lds, st, g, tiles);
  return hipGetLastError();
}
template <typename T>
hipError_t dispatch_stream(const Mx4GemmArgs& g, hipStream_t st) {
  if (g.N <= 16) return launch_stream<T, 1>(g, st);
  if (g.N <= 32) return launch_stream<T, 2>(g, st);
  if (g.N <= 64) return launch_stream<T, 4>(g, st);
  return launch_stream<T, 8>(g, st);
}

}  // namespace

hipError_t launch_rows_mx4(const Mx4RowsArgs& a, bool back, hipStream_t st) {
  if (a.M == 0) return hipSuccess;
  return a.dtype == SAGA_BF16 ? rows_mx4<uint16_t>(a, back, st) : rows_mx4<float>(a, back, st);
}

// Which kernel takes a product (us of kernels alone, bfloat16 out).
// k_mx4_few, whose workgroups each round the rows, while that is little, against 64 x 64 tiles: 4-bit
// rows 1 x 1024 x 1024 3.6 / 5.4, 16 x 4096 x 4096 6.7 / 10.9, 32 8.8 / 11.0, 48 11.0 / 11.0, 64 12.3 / 11.1;
// against a launch more for the rows' 4-bit form (about 4): bfloat16 1 x 1024 x 1024 4.0 / 7.8, 16 x 4096
// x 4096 8.6 / 14.1, 32 13.5 / 14.7, 48 18.5 / 14.7, float32 16 12.6 / 14.1, 32 19.7 / 14.7.
bool mx4_few(int a_dtype, int64_t M, int64_t N, int64_t K) {
  const int64_t work = ((M + 15) / 16) * ((N + 15) / 16) * ((K + 127) / 128);
  return M < 4096 && N <= 1 << 20 && work <= (a_dtype == SAGA_F32 ? 8192 : 16384);
}

// k_mx4_stream while w fits LDS, against rounding and product in two launches (us, bfloat16: 4096 x 602 x 128 11
// / 13, 65536 x 1024 x 64 27 / 45, 2^20 x 128 x 128 127 / 178, 2^20 x 602 x 128 315 / 516)
bool mx4_streams(int64_t M, int64_t N, int64_t K) {
  return M >= 4096 && N <= 128 && StreamSpace(K, N <= 16 ? 1 : N <= 32 ? 2 : N <= 64 ? 4 : 8).total <= 150 * 1024;
}

// float rows for the tiles are quantised into the workspace: q, then their scales
struct Mx4Space {
  int64_t ldq, lds;
  size_t scale, total;
};
Mx4Space mx4_space(int64_t M, int64_t K) {
  Mx4Space s;
  s.ldq = ((K + 1) / 2 + 15) / 16 * 16;
  s.lds = ((K + 31) / 32 + 3) / 4 * 4;
  s.scale = ((size_t)M * s.ldq + 255) & ~(size_t)255;
  s.total = s.scale + (((size_t)M * s.lds + 255) & ~(size_t)255);
  return s;
}

size_t mx4_workspace_bytes(int a_dtype, int64_t M, int64_t N, int64_t K) {
  if (a_dtype == SAGA_MX4 || M == 0 || mx4_few(a_dtype, M, N, K) || mx4_streams(M, N, K)) return 0;
  return mx4_space(M, K).total;
}

hipError_t launch_gemm_mx4(const Mx4GemmArgs& g0, hipStream_t st) {
  if (g0.M == 0) return hipSuccess;
  Mx4GemmArgs g = g0;
  if (mx4_few(g.a_dtype, g.M, g.N, g.K)) {
    if (g.a_dtype == SAGA_MX4) return launch_few<uint8_t>(g, st);
    return g.a_dtype == SAGA_BF16 ? launch_few<uint16_t>(g, st) : launch_few<float>(g, st);
  }
  if (g.a_dtype != SAGA_MX4 && mx4_streams(g.M, g.N, g.K))
    return g.a_dtype == SAGA_BF16 ? dispatch_stream<uint16_t>(g, st) : dispatch_stream<float>(g, st);
  if (g.a_dtype != SAGA_MX4) {
    const Mx4Space s = mx4_space(g.M, g.K);
    uint8_t* const q = static_cast<uint8_t*>(g.ws);
    const Mx4RowsArgs r = {g.a_dtype, g.M, g.K, g.a, g.lda, q, s.ldq, q + s.scale, s.lds};
    const hipError_t e = launch_rows_mx4(r, false, st);
    if (e != hipSuccess) return e;
    g.a = q;
    g.lda = s.ldq;
    g.a_scale = q + s.scale;
    g.lda_s = s.lds;
  }
  // Too few 128 x 128 tiles for all CUs: 64 x 64, and eight stages on their way (256 x 4096 x 4096 11 us).
  const int64_t cols = (g.N + 127) / 128, rows = (g.M + 127) / 128;
  if (cols * rows <= 256) return launch_tile<2, 2, 1, 1, 8>(g, st);
  // 256 x 256, one workgroup a CU, where its tiles fill whole rounds of the CUs to four fifths and
  // 128-wide ones do not leave out a tenth of its columns (us, against 128 x 128, two workgroups a
  // CU: 16384 x 4096 x 4096 166 / 221, 16384 x 2048 x 2048 51 / 60, 16384 x 4096 x 1024 42 / 57, 16384 x 1024
  // x 4096 67 / 71, 40001 x 1024 x 1024, four fifths, 42 / 44, 200000 x 602 x 300 to float32 129 / 118).
  const int64_t large = ((g.M + 255) / 256) * ((g.N + 255) / 256), rounds = (large + 255) / 256;
  if (large * 5 >= rounds * 256 * 4 && (g.N + 255) / 256 * 20 <= cols * 11) return launch_tile<2, 4, 4, 2, 4>(g, st);
  if (g.N <= 32) return launch_tile<4, 1, 1, 1, 2>(g, st);
  if (g.N <= 64) return launch_tile<4, 1, 1, 2, 2>(g, st);
  return launch_tile<2, 2, 2, 2, 3>(g, st);
}

}  // namespace saga
