// Answers of a network: for every row of logits the log probability of its
// label, the entropy, and the top_k classes with their log probabilities, in one
// pass over the logits.  With m the row's largest logit, S = sum e^(x - m) and
// T = sum e^(x - m) (x - m):
//     log p_j = x_j - m - log S,   H = log S - T / S
// Every lane keeps m, S and T of its own columns and rescales them as m grows.
// The classes come by value, equal ones by index.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "row_device.h"
#include "saga_internal.h"

namespace saga {
namespace {

constexpr int64_t kMostBlocks = 1 << 20;  // (a grid holds less than 2^32 threads)
constexpr float kNegInf = -__builtin_huge_valf();

// 16-byte piece of a row, columns past `left` read as -inf
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  __device__ __forceinline__ static void load(const float* p, int left, float* v) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (left > 0) x = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = left > j ? x[j] : kNegInf;
  }
  __device__ __forceinline__ static float one(const float* p) { return *p; }
};
template <> struct Piece<uint16_t> {
  static constexpr int N = 8;
  __device__ __forceinline__ static void load(const uint16_t* p, int left, float* v) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (left > 0) x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = left > 2 * j ? __uint_as_float(x[j] << 16) : kNegInf;
      v[2 * j + 1] = left > 2 * j + 1 ? __uint_as_float(x[j] & 0xffff0000u) : kNegInf;
    }
  }
  __device__ __forceinline__ static float one(const uint16_t* p) { return bf16_to_f32(*p); }
};

// m, S and T of some columns.  Nothing but -inf: m = -inf, S = T = 0.  A NaN or
// +inf among them makes S a NaN.
struct Stats {
  float m, s, t;
};
constexpr float kFar = -1e4f;  // (e^-10000 is 0: keeps 0 * inf out of T)

// the same sums about another largest value mm (finite)
__device__ __forceinline__ Stats about(const Stats& a, float mm) {
  const float d = a.m - mm, c = __expf(d);
  return Stats{mm, a.s * c, c * fmaf(fmaxf(d, kFar), a.s, a.t)};
}
__device__ __forceinline__ float finite_top(float m) { return m == kNegInf ? 0.0f : m; }

template <int NV>
__device__ __forceinline__ void add_values(Stats& a, float top, const float (&v)[NV]) {
  const float m = fmaxf(a.m, top), mm = finite_top(m);
  Stats b = about(a, mm);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const float d = v[i] - mm, e = __expf(d);
    b.s += e;
    b.t = fmaf(e, fmaxf(d, kFar), b.t);
  }
  a.s = b.s;
  a.t = b.t;
  a.m = m;
}
template <int G>
__device__ __forceinline__ Stats join_lanes(const Stats& a) {
  const float m = group_max<G>(a.m);
  const Stats b = about(a, finite_top(m));
  return Stats{m, group_sum<G>(b.s), group_sum<G>(b.t)};
}

// what a row's sums give; bad: NaN or +inf among the logits
struct Row {
  float m, log_s, entropy;
  bool bad, empty;
};
__device__ __forceinline__ Row row_of(const Stats& a) {
  Row r;
  r.bad = !(a.s < __builtin_huge_valf());
  r.empty = !r.bad && a.m == kNegInf;
  r.m = finite_top(a.m);
  r.log_s = logf(a.s);
  r.entropy = r.bad ? __uint_as_float(0x7fc00000u) : r.empty ? 0.0f : r.log_s - a.t / a.s;
  return r;
}
// log probability of a logit; an empty row has -inf for every class
__device__ __forceinline__ float log_prob(const Row& r, float x) {
  return r.bad ? __uint_as_float(0x7fc00000u) : r.empty ? kNegInf : x - r.m - r.log_s;
}
// logp and entropy of a row (one lane)
template <typename T>
__device__ __forceinline__ void write_row(const LabelArgs& a, int64_t row, const Row& r) {
  if (a.logp) {
    const int32_t c = a.labels[row];
    float lp = 0.0f;  // no label
    if (c >= a.C) lp = __uint_as_float(0x7fc00000u);
    else if (c >= 0) lp = log_prob(r, Piece<T>::one(static_cast<const T*>(a.logits) + row * a.ld + c));
    a.logp[row] = lp;
  }
  if (a.entropy) a.entropy[row] = r.entropy;
}
__device__ __forceinline__ void write_top(const LabelArgs& a, int64_t row, int k, const Row& r, float v, int c) {
  const bool none = r.bad || v == kNegInf;
  a.top_index[row * a.top_k + k] = none ? -1 : c;
  a.top_logp[row * a.top_k + k] = r.bad ? __uint_as_float(0x7fc00000u) : none ? kNegInf : log_prob(r, v);
}

// --------------------------------------------------------------------------
// one piece a lane: G lanes hold a row.  The top classes come one after another,
// each the largest of what is left.
// --------------------------------------------------------------------------
template <typename T, int G>
__global__ __launch_bounds__(256) void k_labels_narrow(LabelArgs a) {
  typedef Piece<T> P;
  constexpr int ROWS = 256 / G;
  const int g = threadIdx.x % G, col = g * P::N;
  for (int64_t row = blockIdx.x * (int64_t)ROWS + threadIdx.x / G; row < a.M; row += gridDim.x * (int64_t)ROWS) {
    float v[P::N];
    P::load(static_cast<const T*>(a.logits) + row * a.ld + col, (int)(a.C - col), v);
    float top = v[0];
#pragma unroll
    for (int j = 1; j < P::N; ++j) top = fmaxf(top, v[j]);
    Stats s{kNegInf, 0.0f, 0.0f};
    const float m = group_max<G>(top);
    add_values(s, m, v);
    s = Stats{m, group_sum<G>(s.s), group_sum<G>(s.t)};
    const Row r = row_of(s);
    if (g == 0) write_row<T>(a, row, r);
    for (int k = 0; k < a.top_k; ++k) {
      float best = v[0];
      int at = 0;
#pragma unroll
      for (int j = 1; j < P::N; ++j)
        if (v[j] > best) best = v[j], at = j;
      const float most = group_max<G>(best);
      // the lowest column that has it (columns are below 2^31: the largest complement)
      const uint32_t mine = best == most ? ~(uint32_t)(col + at) : 0u;
      const int c = (int)~group_maxu<G>(mine);
      if (g == k % G) write_top(a, row, k, r, most, c);
#pragma unroll
      for (int j = 0; j < P::N; ++j)
        if (col + j == c) v[j] = kNegInf;
    }
  }
}

// --------------------------------------------------------------------------
// longer rows: a wave streams a range of columns and keeps the best 64 so far
// one a lane, in order
// --------------------------------------------------------------------------
struct Best {
  float v;     // this lane's entry
  int c;
  float last;  // entry top_k - 1: what a value has to exceed
  int k;

  __device__ __forceinline__ void clear(int top_k) {
    v = last = top_k > 0 ? kNegInf : __builtin_huge_valf();
    c = -1;
    k = top_k;
  }
  // x (uniform) > last; equal values are put behind those that are there, so
  // they have to come in the order of their columns
  __device__ __forceinline__ void put(float x, int col) {
    const int lane = threadIdx.x & 63;
    const int pos = __popcll(__ballot(v >= x));
    const float uv = __shfl_up(v, 1, 64);
    const int uc = __shfl_up(c, 1, 64);
    v = lane < pos ? v : lane == pos ? x : uv;
    c = lane < pos ? c : lane == pos ? col : uc;
    last = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), k - 1));
  }
  // one value a lane, columns in the order of the lanes
  __device__ __forceinline__ void offer(float x, int col) {
    uint64_t hits = __ballot(x > last);
    while (hits) {
      const int l = __ffsll((unsigned long long)hits) - 1;
      hits &= hits - 1;
      const float y = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), l));
      if (y > last) put(y, __builtin_amdgcn_readlane(col, l));
    }
  }
  // N values a lane, in consecutive columns
  template <int N>
  __device__ __forceinline__ void offer(const float* x, int col) {
    float top = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) top = fmaxf(top, x[j]);
    uint64_t hits = __ballot(top > last);
    while (hits) {
      const int l = __ffsll((unsigned long long)hits) - 1;
      hits &= hits - 1;
      const int c0 = __builtin_amdgcn_readlane(col, l);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float y = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x[j]), l));
        if (y > last) put(y, c0 + j);
      }
    }
  }
};

// columns [c0, c1) of a row; c0 a multiple of a piece
template <typename T>
__device__ __forceinline__ void stream_range(const T* x, int64_t c0, int64_t c1, Stats& s, Best& best) {
  typedef Piece<T> P;
  constexpr int R = 16 / P::N * 2;  // 32 columns a lane at a time
  const int lane = threadIdx.x & 63;
  for (int64_t at = c0; at < c1; at += R * 64 * P::N) {
    float v[R * P::N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t col = at + (r * 64 + lane) * P::N;
      P::load(x + col, (int)max((int64_t)0, min(c1 - col, (int64_t)P::N)), v + r * P::N);
    }
    float top = v[0];
#pragma unroll
    for (int i = 1; i < R * P::N; ++i) top = fmaxf(top, v[i]);
    add_values(s, top, v);
    if (__ballot(top > best.last)) {
#pragma unroll
      for (int r = 0; r < R; ++r) best.offer<P::N>(v + r * P::N, (int)(at + (r * 64 + lane) * P::N));
    }
  }
}

// Workgroup: 4 waves.  parts == 1: four rows, one a wave.  parts == 4: one row,
// its four ranges joined through LDS.  parts > 4 (a multiple of 4): every wave
// leaves its range's sums and best to k_labels_join.
template <typename T>
__global__ __launch_bounds__(256) void k_labels_wide(LabelArgs a) {
  __shared__ float ls[3][4], lv[4][64];
  __shared__ int lc[4][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t units = a.M * a.parts;
  for (int64_t u0 = blockIdx.x * (int64_t)4; u0 < units; u0 += gridDim.x * (int64_t)4) {
    const int64_t unit = u0 + wave;
    const bool have = unit < units;  // (parts == 1: the last rows)
    const int64_t row = have ? unit / a.parts : 0;
    const int part = (int)(unit % a.parts);
    Stats s{kNegInf, 0.0f, 0.0f};
    Best best;
    best.clear(a.top_k);
    if (have) {
      const int64_t c0 = part * a.range;
      stream_range<T>(static_cast<const T*>(a.logits) + row * a.ld, c0, min((int64_t)a.C, c0 + a.range), s, best);
      s = join_lanes<64>(s);
    }
    if (a.parts > 4) {
      float* p = a.part_stats + unit * 3;
      if (lane == 0) p[0] = s.m, p[1] = s.s, p[2] = s.t;
      if (lane < a.top_k) {
        a.part_value[unit * a.top_k + lane] = best.v;
        a.part_index[unit * a.top_k + lane] = best.c;
      }
      continue;
    }
    if (a.parts == 4) {
      if (lane == 0) ls[0][wave] = s.m, ls[1][wave] = s.s, ls[2][wave] = s.t;
      lv[wave][lane] = best.v;
      lc[wave][lane] = best.c;
      __syncthreads();
      if (wave == 0) {
        s = lane < 4 ? Stats{ls[0][lane], ls[1][lane], ls[2][lane]} : Stats{kNegInf, 0.0f, 0.0f};
        s = join_lanes<64>(s);
        for (int w = 1; w < 4; ++w) best.offer(lane < a.top_k ? lv[w][lane] : kNegInf, lc[w][lane]);
      }
    }
    if (have && (a.parts == 1 || wave == 0)) {
      const Row r = row_of(s);
      if (lane == 0) write_row<T>(a, row, r);
      if (lane < a.top_k) write_top(a, row, lane, r, best.v, best.c);
    }
    if (a.parts == 4) __syncthreads();  // the next row's waves write ls, lv and lc
  }
}

// a wave joins a row's parts: their columns ascend, and equal values of one part
// lie in the order of their columns
template <typename T>
__global__ __launch_bounds__(64) void k_labels_join(LabelArgs a) {
  const int lane = threadIdx.x;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    Stats s{kNegInf, 0.0f, 0.0f};
    for (int p = lane; p < a.parts; p += 64) {
      const float* q = a.part_stats + (row * a.parts + p) * 3;
      const Stats b{q[0], q[1], q[2]};
      const float m = fmaxf(s.m, b.m);
      const Stats x = about(s, finite_top(m)), y = about(b, finite_top(m));
      s = Stats{m, x.s + y.s, x.t + y.t};
    }
    s = join_lanes<64>(s);
    Best best;
    best.clear(a.top_k);
    const int n = a.parts * a.top_k;
    for (int i = 0; i < n; i += 64) {
      const int64_t at = row * n + i + lane;
      best.offer(i + lane < n ? a.part_value[at] : kNegInf, i + lane < n ? a.part_index[at] : -1);
    }
    const Row r = row_of(s);
    if (lane == 0) write_row<T>(a, row, r);
    if (lane < a.top_k) write_top(a, row, lane, r, best.v, best.c);
  }
}

// Waves per row: one where rows alone fill the card, a workgroup's four where
// they do not, and so many workgroups that all CUs have some where there are few.
struct Split {
  int parts;
  int64_t range;
};
template <typename T>
Split split_of(int64_t M, int64_t C) {
  constexpr int64_t tile = 64 * 32;  // columns a wave takes at a time
  const int64_t tiles = (C + tile - 1) / tile;
  int64_t parts = tiles < 4 ? 1 : 4;
  if (M < 1024 && tiles > 4) parts = std::min<int64_t>((tiles + 3) / 4, std::max<int64_t>(1, 1024 / M)) * 4;
  const int64_t per = (tiles + parts - 1) / parts;
  return Split{(int)parts, per * tile};
}

template <typename T>
hipError_t launch(LabelArgs a, hipStream_t st) {
  typedef Piece<T> P;
  const auto rows = [&](int g) {
    return dim3((unsigned)std::min<int64_t>((a.M + 256 / g - 1) / (256 / g), kMostBlocks));
  };
  if (a.C <= 8 * P::N) {
    hipLaunchKernelGGL((k_labels_narrow<T, 8>), rows(8), dim3(256), 0, st, a);
  } else if (a.C <= 16 * P::N) {
    hipLaunchKernelGGL((k_labels_narrow<T, 16>), rows(16), dim3(256), 0, st, a);
  } else if (a.C <= 32 * P::N) {
    hipLaunchKernelGGL((k_labels_narrow<T, 32>), rows(32), dim3(256), 0, st, a);
  } else if (a.C <= 64 * P::N) {
    hipLaunchKernelGGL((k_labels_narrow<T, 64>), rows(64), dim3(256), 0, st, a);
  } else {
    const Split sp = split_of<T>(a.M, a.C);
    a.parts = sp.parts;
    a.range = sp.range;
    const int64_t units = a.M * a.parts;
    if (a.parts > 4) {
      char* ws = static_cast<char*>(a.ws);
      a.part_stats = reinterpret_cast<float*>(ws);
      a.part_value = a.part_stats + units * 3;
      a.part_index = reinterpret_cast<int32_t*>(a.part_value + units * a.top_k);
    }
    hipLaunchKernelGGL((k_labels_wide<T>), dim3((unsigned)std::min<int64_t>((units + 3) / 4, kMostBlocks)),
                       dim3(256), 0, st, a);
    if (a.parts > 4) {
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL((k_labels_join<T>), dim3((unsigned)a.M), dim3(64), 0, st, a);
    }
  }
  return hipGetLastError();
}

}  // namespace

size_t labels_workspace_bytes(int dtype, int64_t M, int64_t C, int top_k) {
  if (M <= 0 || C <= 64 * (dtype == SAGA_BF16 ? 8 : 4)) return 0;
  const Split sp = dtype == SAGA_BF16 ? split_of<uint16_t>(M, C) : split_of<float>(M, C);
  return sp.parts > 4 ? (size_t)M * sp.parts * (3 + 2 * (size_t)top_k) * 4 : 0;
}

hipError_t launch_label_log_probs(const LabelArgs& a, hipStream_t st) {
  if (a.M == 0) return hipSuccess;
  return a.dtype == SAGA_BF16 ? launch<uint16_t>(a, st) : launch<float>(a, st);
}

}  // namespace saga
