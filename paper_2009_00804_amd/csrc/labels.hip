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
typedef volatile __attribute__((address_space(3))) float* lds_floats;

// 16-byte piece of a row as it lies in memory, and its values; of those past
// `left` -inf
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  __device__ __forceinline__ static void widen(const u32x4& x, float* v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(x[j]);
  }
  __device__ __forceinline__ static float one(const float* p) { return *p; }
};
template <> struct Piece<uint16_t> {
  static constexpr int N = 8;
  __device__ __forceinline__ static void widen(const u32x4& x, float* v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(x[j] << 16);
      v[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static float one(const uint16_t* p) { return bf16_to_f32(*p); }
};
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T* p, int64_t left) {
  u32x4 x = {0u, 0u, 0u, 0u};
  if (left > 0) x = *reinterpret_cast<const u32x4*>(p);
  return x;
}
template <typename T>
__device__ __forceinline__ void widen_piece(const u32x4& x, int64_t left, float* v) {
  Piece<T>::widen(x, v);
  if (left < Piece<T>::N) {
#pragma unroll
    for (int j = 0; j < Piece<T>::N; ++j)
      if (left <= j) v[j] = kNegInf;
  }
}

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
// a row's label and the label's logit (0 if there is none), loaded ahead
struct Label {
  int32_t c;
  float x;
};
template <typename T>
__device__ __forceinline__ Label load_label(const LabelArgs& a, int64_t row) {
  Label l{-1, 0.0f};
  if (a.logp) {
    l.c = a.labels[row];
    if (l.c >= 0 && l.c < a.C) l.x = Piece<T>::one(static_cast<const T*>(a.logits) + row * a.ld + l.c);
  }
  return l;
}
// logp and entropy of a row (one lane)
__device__ __forceinline__ void write_row(const LabelArgs& a, int64_t row, const Row& r, const Label& l) {
  if (a.logp) a.logp[row] = l.c < 0 ? 0.0f : l.c >= a.C ? __uint_as_float(0x7fc00000u) : log_prob(r, l.x);
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
    const u32x4 raw = load_piece(static_cast<const T*>(a.logits) + row * a.ld + col, a.C - col);
    const Label l = load_label<T>(a, row);
    widen_piece<T>(raw, a.C - col, v);
    float top = v[0];
#pragma unroll
    for (int j = 1; j < P::N; ++j) top = fmaxf(top, v[j]);
    Stats s{kNegInf, 0.0f, 0.0f};
    const float m = group_max<G>(top);
    add_values(s, m, v);
    s = Stats{m, group_sum<G>(s.s), group_sum<G>(s.t)};
    const Row r = row_of(s);
    if (g == 0) write_row(a, row, r, l);
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
// many rows of up to 64 columns: a lane a row, so that nothing is reduced between
// lanes.  The top classes are kept in order by insertion, two instructions a value
// and place for bfloat16: value and column make one whole number there.
// --------------------------------------------------------------------------
constexpr int kLaneC = 64;

template <typename T, int K> struct TopList;
template <int K> struct TopList<uint16_t, K> {
  uint32_t t[K > 0 ? K : 1];
  __device__ __forceinline__ TopList() {
#pragma unroll
    for (int k = 0; k < K; ++k) t[k] = 0x007fffffu;  // -inf
  }
  __device__ __forceinline__ void offer(float x, int col) {
    const uint32_t u = __float_as_uint(x + 0.0f);  // (-0 counts as 0)
    uint32_t key = ((u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) & 0xffff0000u) | (0xffffu - (uint32_t)col);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t m = max(t[k], key);
      key = min(t[k], key);
      t[k] = m;
    }
  }
  __device__ __forceinline__ float value(int k) const {
    const uint32_t h = t[k] & 0xffff0000u;
    return __uint_as_float(h & 0x80000000u ? h ^ 0x80000000u : ~h & 0xffff0000u);
  }
  __device__ __forceinline__ int column(int k) const { return (int)(0xffffu - (t[k] & 0xffffu)); }
};
template <int K> struct TopList<float, K> {
  float v[K > 0 ? K : 1];
  int c[K > 0 ? K : 1];
  __device__ __forceinline__ TopList() {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = kNegInf, c[k] = -1;
  }
  __device__ __forceinline__ void offer(float x, int col) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool up = x > v[k];  // equal values stay behind those of lower columns
      const float ov = v[k];
      const int oc = c[k];
      v[k] = up ? x : ov;
      c[k] = up ? col : oc;
      x = up ? ov : x;
      col = up ? oc : col;
    }
  }
  __device__ __forceinline__ float value(int k) const { return v[k]; }
  __device__ __forceinline__ int column(int k) const { return c[k]; }
};

template <typename T, int K>
__global__ __launch_bounds__(256) void k_labels_lane(LabelArgs a) {
  typedef Piece<T> P;
  constexpr int NP = kLaneC / P::N;
  const int C = (int)a.C;
  for (int64_t row = blockIdx.x * (int64_t)256 + threadIdx.x; row < a.M; row += gridDim.x * (int64_t)256) {
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    u32x4 raw[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (p * P::N < C) raw[p] = load_piece(x + p * P::N, C - p * P::N);
    const Label l = load_label<T>(a, row);
    TopList<T, K> best;
    float m = kNegInf;
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (p * P::N < C) {
        float v[P::N];
        widen_piece<T>(raw[p], C - p * P::N, v);
#pragma unroll
        for (int j = 0; j < P::N; ++j) {
          m = fmaxf(m, v[j]);
          best.offer(v[j], p * P::N + j);
        }
      }
    Stats s{m, 0.0f, 0.0f};
    const float mm = finite_top(m);
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (p * P::N < C) {
        float v[P::N];
        widen_piece<T>(raw[p], C - p * P::N, v);
#pragma unroll
        for (int j = 0; j < P::N; ++j) {
          const float d = v[j] - mm, e = __expf(d);
          s.s += e;
          s.t = fmaf(e, fmaxf(d, kFar), s.t);
        }
      }
    const Row r = row_of(s);
    write_row(a, row, r, l);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (k < a.top_k) write_top(a, row, k, r, best.value(k), best.column(k));
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
    last = fmaxf(last, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), k - 1)));
  }
  // k or more values are at least x (uniform): smaller ones need not be looked at
  __device__ __forceinline__ void at_least(float x) { last = fmaxf(last, below(x)); }
  // the largest x that k or more lanes reach with `top`
  __device__ __forceinline__ float reached(float top) const {
    int n = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i)
      n += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(top), i)) >= top ? 1 : 0;
    return group_max<64>(n >= k ? top : kNegInf);
  }
  // the next smaller number
  __device__ __forceinline__ static float below(float x) {
    const uint32_t u = __float_as_uint(x);
    if (x == 0.0f) return __uint_as_float(0x80000001u);
    return x == kNegInf ? x : __uint_as_float(x > 0.0f ? u - 1u : u + 1u);
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

// Columns [c0, c1) of a row; c0 a multiple of a piece.  The next 32 columns a lane
// are on their way while these are summed.  share: the waves of one row tell each
// other (in shared) what they have reached (which only spares work: a value below what some
// wave has top_k values of is none of the row's best).
template <typename T>
__device__ __forceinline__ void stream_range(const T* x, int64_t c0, int64_t c1, Stats& s, Best& best,
                                             bool share, lds_floats shared) {
  typedef Piece<T> P;
  constexpr int R = 32 / P::N, TILE = 64 * 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u32x4 next[R];
  const auto load = [&](int64_t at) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t col = at + (r * 64 + lane) * P::N;
      next[r] = load_piece(x + col, c1 - col);
    }
  };
  if (c0 < c1) load(c0);
  for (int64_t at = c0; at < c1; at += TILE) {
    float v[32];
    if (at + TILE <= c1) {
#pragma unroll
      for (int r = 0; r < R; ++r) P::widen(next[r], v + r * P::N);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) widen_piece<T>(next[r], c1 - at - (r * 64 + lane) * P::N, v + r * P::N);
    }
    if (at + TILE < c1) load(at + TILE);
    float top = v[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, v[i]);
    add_values(s, top, v);
    if (best.k > 0) {
      if (at == c0) best.at_least(best.reached(top));
      if (share) {
        float far = shared[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) far = fmaxf(far, shared[w]);
        best.last = fmaxf(best.last, far);
      }
      if (__ballot(top > best.last)) {
#pragma unroll
        for (int r = 0; r < R; ++r) best.offer<P::N>(v + r * P::N, (int)(at + (r * 64 + lane) * P::N));
        if (share && lane == 0) shared[wave] = Best::below(best.last);
      }
    }
  }
}

// Workgroup: 4 waves.  parts == 1: four rows, one a wave.  parts == 4: one row,
// its four ranges joined through LDS.  parts > 4 (a multiple of 4): every wave
// leaves its range's sums and best to k_labels_join.
template <typename T>
__global__ __launch_bounds__(256) void k_labels_wide(LabelArgs a) {
  __shared__ float ls[3][4], lv[4][64], reached[4];
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
    if (a.parts == 4) {
      if (lane == 0) reached[wave] = kNegInf;
      __syncthreads();
    }
    const Label l = a.parts <= 4 && have ? load_label<T>(a, row) : Label{-1, 0.0f};
    if (have) {
      const int64_t c0 = part * a.range;
      stream_range<T>(static_cast<const T*>(a.logits) + row * a.ld, c0, min(a.C, c0 + a.range), s, best,
                      a.parts == 4, (lds_floats)reached);
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
      if (lane == 0) write_row(a, row, r, l);
      if (lane < a.top_k) write_top(a, row, lane, r, best.v, best.c);
    }
    if (a.parts == 4) __syncthreads();  // the next row's waves write to the same places
  }
}

// a wave joins a row's parts: their columns ascend, and equal values of one part
// lie in the order of their columns
template <typename T>
__global__ __launch_bounds__(64) void k_labels_join(LabelArgs a) {
  const int lane = threadIdx.x;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const Label l = load_label<T>(a, row);
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
    if (n > 0) {
      // every part's best comes first in it
      float top = kNegInf;
      for (int p = lane; p < a.parts; p += 64) top = fmaxf(top, a.part_value[(row * a.parts + p) * a.top_k]);
      best.at_least(best.reached(top));
      for (int i = 0; i < n; i += 256) {
        float x[4];
        int c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int e = i + k * 64 + lane;
          x[k] = e < n ? a.part_value[row * n + e] : kNegInf;
          c[k] = e < n ? a.part_index[row * n + e] : -1;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) best.offer(x[k], c[k]);
      }
    }
    const Row r = row_of(s);
    if (lane == 0) write_row(a, row, r, l);
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
  // a lane a row from 16384 rows on: fewer do not fill the card
  if (a.C <= kLaneC && a.M >= 16384 && a.top_k <= 8) {
    const dim3 grid((unsigned)std::min<int64_t>((a.M + 255) / 256, kMostBlocks));
    const auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
      return hipGetLastError();
    };
    switch (a.top_k) {
      case 0: return go(k_labels_lane<T, 0>);
      case 1: return go(k_labels_lane<T, 1>);
      case 2: return go(k_labels_lane<T, 2>);
      case 3: return go(k_labels_lane<T, 3>);
      case 4: return go(k_labels_lane<T, 4>);
      case 5:
      case 6: return go(k_labels_lane<T, 6>);
      default: return go(k_labels_lane<T, 8>);
    }
  }
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
