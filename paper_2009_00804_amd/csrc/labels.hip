// Answers of a network: for every row of logits the log probability of its
// label, the entropy, and the top_k classes with their log probabilities, in one
// pass over the logits.  With m the row's largest logit, S = sum e^(x - m) and
// T = sum e^(x - m) (x - m):
//     log p_j = x_j - m - log S,   H = log S - T / S
// Every lane keeps m, S and T of its own columns (terms in float32, sums over many of
// them in float64) and rescales them as m grows.  The classes come by value, equal ones
// by index.
//
// Memory bounds the sums (4099 x 100003 in bfloat16 147 to 158 us without alternatives, 5.2
// to 5.6 TB/s), vector instructions what the alternatives add: top 3 15 us, top 10 40, top 20 85,
// where they are issued in four fifths of the cycles.  2^21 x 41 with top 3 takes 68 to 73
// us (40 us without, 4.3 TB/s), as much of it vector instructions.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "row_device.h"
#include "saga_internal.h"

namespace saga {
namespace {

constexpr int64_t kMostBlocks = 1 << 20;  // (a grid holds less than 2^32 threads)
constexpr float kNegInf = -__builtin_huge_valf();

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

// S and T of a few values about mm, in N chains of additions
template <int N>
struct Chains {
  float s[N] = {}, t[N] = {};
  // FIRST: nothing has been added yet
  template <bool FIRST, int NV>
  __device__ __forceinline__ void add(float mm, const float (&v)[NV]) {
    static_assert(NV >= N, "a value for each chain");
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float d = v[i] - mm, e = __expf(d), far = fmaxf(d, kFar);
      const bool first = FIRST && i < N;
      s[i % N] = first ? e : s[i % N] + e;
      t[i % N] = first ? e * far : fmaf(e, far, t[i % N]);
    }
  }
  __device__ __forceinline__ static float total(const float (&x)[N]) {
    if constexpr (N == 2) return x[0] + x[1];
    else return (x[0] + x[1]) + (x[2] + x[3]);
  }
};

// m, S and T of a lane's columns, tile after tile.  A tile's terms are added in float32.
// A is what the tiles' sums are held in: float where a row is one tile, else float64
// (1 to 3 % of the time).  Added one by one to a float32 sum, terms of few distinct values round
// to one side: rows of 2^18 classes and two values had log S off by 9e-6, of 2^22 by 2e-4.
template <typename A>
struct Sums {
  float m = kNegInf;    // the largest value
  float ref = kNegInf;  // what s and t are about
  A s = 0, t = 0;

  template <int NV>
  __device__ __forceinline__ void add(float top, const float (&v)[NV]) {
    m = fmaxf(m, top);
    // Only a clearly larger value moves the sums: one that grows a little in every tile
    // would round them every time.
    if (m > ref + 2.0f) {
      const float d = ref - m, c = __expf(d);
      t = (A)c * (t + (A)fmaxf(d, kFar) * s);
      s *= (A)c;
      ref = m;
    }
    Chains<2> f;  // (of at most 8 additions)
    f.template add<true>(finite_top(ref), v);
    s += (A)f.total(f.s);
    t += (A)f.total(f.t);
  }
  // over the wave's lanes
  __device__ __forceinline__ Stats join() const {
    const float most = group_max<64>(m);
    const Stats b = about(Stats{ref, (float)s, (float)t}, finite_top(most));
    return Stats{most, group_sum<64>(b.s), group_sum<64>(b.t)};
  }
};
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
    const float m = group_max<G>(top);
    Chains<2> f;
    f.template add<true>(finite_top(m), v);
    const Row r = row_of(Stats{m, group_sum<G>(f.total(f.s)), group_sum<G>(f.total(f.t))});
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
    // behind equal values, whose columns are lower; from there on all move by one,
    // equal ones too
    bool up = false;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      up = up || x > v[k];
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
    Chains<4> f;
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (p * P::N < C) {
        float v[P::N];
        widen_piece<T>(raw[p], C - p * P::N, v);
        f.template add<false>(finite_top(m), v);
      }
    const Row r = row_of(Stats{m, f.total(f.s), f.total(f.t)});
    write_row(a, row, r, l);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (k < a.top_k) write_top(a, row, k, r, best.value(k), best.column(k));
  }
}

// --------------------------------------------------------------------------
// longer rows: a wave streams a range of columns and gathers in LDS what may be
// among the best.  Every now and then the gathered values are ranked against each
// other (by value, then column) and the best top_k kept in order; a value has to
// exceed the last of them from then on.
// --------------------------------------------------------------------------
typedef volatile __attribute__((address_space(3))) float* lds_floats;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) u32x2 lds_pair;
constexpr int kGather = 128;  // values a wave's list holds: SAGA_MAX_TOP kept ones of four waves

// the next smaller number
__device__ __forceinline__ float below(float x) {
  const uint32_t u = __float_as_uint(x);
  if (x == 0.0f) return __uint_as_float(0x80000001u);
  return x == kNegInf ? x : __uint_as_float(x > 0.0f ? u - 1u : u + 1u);
}
// The largest x that k or more lanes reach with `top`: the largest of the lanes
// left, again and again, while that is fewer steps than counting for every lane.
__device__ __forceinline__ float reached_by(int k, float top) {
  if (k <= 16) {
    for (int n = 0;;) {
      const float m = group_max<64>(top);
      const uint64_t have = __ballot(top == m);
      n += __popcll(have);
      if (n >= k || m == kNegInf || have == 0) return m;
      top = top == m ? kNegInf : top;
    }
  }
  int n = 0;
#pragma unroll
  for (int i = 0; i < 64; ++i)
    n += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(top), i)) >= top ? 1 : 0;
  return group_max<64>(n >= k ? top : kNegInf);
}

struct Best {
  lds_pair* list;  // (value, column): kGather + 4 places of this wave's own
  int n, k;         // values gathered
  float last;       // what a value has to exceed

  __device__ __forceinline__ void clear(lds_pair* at, int top_k) {
    list = at;
    n = 0;
    k = top_k;
    last = top_k > 0 ? kNegInf : __builtin_huge_valf();
  }
  // Keeps the best k, in order.  Up to E values a lane; a value's place is the
  // number of those before it.
  template <int E>
  __device__ __forceinline__ void rank() {
    const int lane = threadIdx.x & 63;
    float v[E];
    int c[E], place[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u32x2 x = {0u, 0u};
      if (e * 64 + lane < n) x = list[e * 64 + lane];
      v[e] = __uint_as_float(x.x);
      c[e] = (int)x.y;
      place[e] = 0;
    }
    if (lane < 4) list[n + lane] = u32x2{__float_as_uint(kNegInf), 0x7fffffffu};  // before nothing
    asm volatile("" ::: "memory");
    for (int i = 0; i < n; i += 4) {
      u32x2 x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = list[i + q];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float w = __uint_as_float(x[q].x);
#pragma unroll
        for (int e = 0; e < E; ++e) place[e] += w > v[e] || (w == v[e] && (int)x[q].y < c[e]) ? 1 : 0;
      }
    }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e * 64 + lane < n && place[e] < k) list[place[e]] = u32x2{__float_as_uint(v[e]), (uint32_t)c[e]};
    asm volatile("" ::: "memory");
  }
  // keeps the best k; later columns are higher, so a value has to exceed the k-th
  __device__ __forceinline__ void settle() {
    if (n <= 64) rank<1>();
    else rank<kGather / 64>();
    n = min(n, k);
    if (n == k) last = fmaxf(last, __uint_as_float(__builtin_amdgcn_readfirstlane(list[k - 1].x)));
  }
  // a value a lane, where there is room for all that count
  __device__ __forceinline__ void add(float x, int col) {
    const uint64_t m = __ballot(x > last);
    if (m == 0) return;
    const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
    if (x > last) list[at] = u32x2{__float_as_uint(x), (uint32_t)col};
    n += __popcll(m);
  }
  // The k best of N values a lane (value i in column col_of(i), ascending with i),
  // one after another: for tiles of which more count than there is room for, as
  // where many are equal.
  template <int N, typename F>
  __device__ __forceinline__ void add_best(float (&x)[N], F col_of) {
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int r = 0; r < k; ++r) {
      float best = x[0];
      int at = 0;
#pragma unroll
      for (int i = 1; i < N; ++i)
        if (x[i] > best) best = x[i], at = i;
      const float most = group_max<64>(best);
      if (!(most > last)) break;
      const uint32_t col = ~group_maxu<64>(best == most ? ~(uint32_t)col_of(at) : 0u);
      if (lane == 0) list[n] = u32x2{__float_as_uint(most), col};
      ++n;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if ((uint32_t)col_of(i) == col) x[i] = kNegInf;
    }
  }
};

// Columns [c0, c1) of a row, NV values a lane at a time; c0 a multiple of a piece.
// The next columns are on their way while these are summed.  share: the waves of
// one row tell each other (in shared) what they have reached (which only spares
// work: a value below what some wave has top_k values of is none of the row's best).
// Short rows (NV 8) are loaded 4 bytes a lane, so that all lanes hold some of them.
template <typename T, int NV, typename A>
__device__ __forceinline__ void stream_range(const T* x, int64_t c0, int64_t c1, Sums<A>& s, Best& best, bool share,
                                             lds_floats shared) {
  typedef Piece<T> P;
  constexpr int W = NV > 8 ? P::N : 4 / (int)sizeof(T);  // values a load brings a lane
  constexpr int R = NV / W, TILE = 64 * NV;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  typedef uint32_t words __attribute__((ext_vector_type(W * sizeof(T) / 4)));
  words next[R];
  const auto load = [&](int64_t at) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t col = at + (r * 64 + lane) * W;
      next[r] = words(0u);
      if (col < c1) next[r] = *reinterpret_cast<const words*>(x + col);
    }
  };
  bool changed = false;
  if (c0 < c1) load(c0);
  for (int64_t at = c0; at < c1; at += TILE) {
    float v[NV];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      u32x4 piece = {0u, 0u, 0u, 0u};
      if constexpr (W == P::N) piece = next[r];
      else piece[0] = next[r][0];
      float p[P::N];
      P::widen(piece, p);
#pragma unroll
      for (int j = 0; j < W; ++j) v[r * W + j] = p[j];
    }
    if (at + TILE > c1) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (at + (i / W * 64 + lane) * W + i % W >= c1) v[i] = kNegInf;
    }
    if (at + TILE < c1) load(at + TILE);
    float top = v[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) top = fmaxf(top, v[i]);
    s.add(top, v);
    if (best.k > 0) {
      // k lanes reach x: what is smaller need not be gathered
      if (at == c0) best.last = fmaxf(best.last, below(reached_by(best.k, top)));
      if (share) {
        float far = shared[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) far = fmaxf(far, shared[w]);
        best.last = fmaxf(best.last, far);
      }
      if (const uint64_t hits = __ballot(top > best.last)) {
        const auto col_of = [&](int i) { return (int)(at + (i / W * 64 + lane) * W + i % W); };
        int count = __popcll(hits) * NV;  // at most
        if (best.n + count > kGather) {
          count = 0;
#pragma unroll
          for (int i = 0; i < NV; ++i) count += __popcll(__ballot(v[i] > best.last));
        }
        if (best.n + count <= kGather) {
#pragma unroll
          for (int i = 0; i < NV; ++i) best.add(v[i], col_of(i));
        } else {
          best.add_best(v, col_of);
        }
        asm volatile("" ::: "memory");
        changed = true;
      }
      // ranked after the first columns and the last, and when there are many
      if (changed && (at == c0 || at + TILE >= c1 || best.n >= min(64, best.k + 24))) {
        best.settle();
        changed = false;
        if (share && lane == 0) shared[wave] = below(best.last);
      }
    }
  }
}

// Workgroup: 4 waves.  parts == 1: four rows, one a wave.  parts == 4: one row,
// its four ranges joined through LDS.  parts > 4 (a multiple of 4): every wave
// leaves its range's sums and best to k_labels_join.
template <typename T, int NV>
__global__ __launch_bounds__(256, 4) void k_labels_wide(LabelArgs a) {
  __shared__ float ls[3][4], reached[4];
  __shared__ u32x2 lists[4][kGather + 4];
  __shared__ int ln[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  lds_pair* const list = (lds_pair*)lists[wave];
  const int64_t units = a.M * a.parts;
  for (int64_t u0 = blockIdx.x * (int64_t)4; u0 < units; u0 += gridDim.x * (int64_t)4) {
    const int64_t unit = u0 + wave;
    const bool have = unit < units;  // (parts == 1: the last rows)
    const int64_t row = have ? unit / a.parts : 0;
    const int part = (int)(unit % a.parts);
    Stats s{kNegInf, 0.0f, 0.0f};
    Best best;
    best.clear(list, a.top_k);
    if (a.parts == 4) {
      if (lane == 0) reached[wave] = kNegInf;
      __syncthreads();
    }
    const Label l = a.parts <= 4 && have ? load_label<T>(a, row) : Label{-1, 0.0f};
    if (have) {
      const int64_t c0 = part * a.range;
      Sums<std::conditional_t<(NV > 8), double, float>> sums;  // (8: rows of one tile)
      stream_range<T, NV>(static_cast<const T*>(a.logits) + row * a.ld, c0, min(a.C, c0 + a.range), sums, best,
                          a.parts == 4, (lds_floats)reached);
      s = sums.join();
    }
    if (a.parts > 4) {
      float* p = a.part_stats + unit * 3;
      if (lane == 0) p[0] = s.m, p[1] = s.s, p[2] = s.t;
      if (lane < a.top_k) {
        const u32x2 x = lane < best.n ? list[lane] : u32x2{__float_as_uint(kNegInf), 0u};
        a.part_value[unit * a.top_k + lane] = __uint_as_float(x.x);
        a.part_index[unit * a.top_k + lane] = (int)x.y;
      }
      continue;
    }
    if (a.parts == 4) {
      if (lane == 0) ls[0][wave] = s.m, ls[1][wave] = s.s, ls[2][wave] = s.t, ln[wave] = best.n;
      __syncthreads();
      if (wave == 0) {
        s = lane < 4 ? Stats{ls[0][lane], ls[1][lane], ls[2][lane]} : Stats{kNegInf, 0.0f, 0.0f};
        s = join_lanes<64>(s);
        if (a.top_k > 0) {
          for (int w = 1; w < 4; ++w) {
            const int n = __builtin_amdgcn_readfirstlane(ln[w]);
            if (lane < n) list[best.n + lane] = ((lds_pair*)lists[w])[lane];
            best.n += n;
          }
          asm volatile("" ::: "memory");
          best.settle();
        }
      }
    }
    if (have && (a.parts == 1 || wave == 0)) {
      const Row r = row_of(s);
      if (lane == 0) write_row(a, row, r, l);
      if (lane < a.top_k) {
        const u32x2 x = lane < best.n ? list[lane] : u32x2{__float_as_uint(kNegInf), 0u};
        write_top(a, row, lane, r, __uint_as_float(x.x), (int)x.y);
      }
    }
    if (a.parts == 4) __syncthreads();  // the next row's waves write to the same places
  }
}

// a wave joins a row's parts: their columns ascend
template <typename T>
__global__ __launch_bounds__(64) void k_labels_join(LabelArgs a) {
  __shared__ u32x2 lists[kGather + 4];
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
    best.clear((lds_pair*)lists, a.top_k);
    const int n = a.parts * a.top_k;
    if (n > 0) {
      // every part's best comes first in it
      float top = kNegInf;
      for (int p = lane; p < a.parts; p += 64) top = fmaxf(top, a.part_value[(row * a.parts + p) * a.top_k]);
      best.last = fmaxf(best.last, below(reached_by(a.top_k, top)));
      for (int i = 0; i < n; i += 256) {
        float x[4];
        int c[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int e = i + q * 64 + lane;
          x[q] = e < n ? a.part_value[row * n + e] : kNegInf;
          c[q] = e < n ? a.part_index[row * n + e] : -1;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          best.add(x[q], c[q]);
          asm volatile("" ::: "memory");
          if (best.n > kGather - 64) best.settle();
        }
      }
      best.settle();
    }
    const Row r = row_of(s);
    if (lane == 0) write_row(a, row, r, l);
    if (lane < a.top_k) {
      const u32x2 x = lane < best.n ? ((lds_pair*)lists)[lane] : u32x2{__float_as_uint(kNegInf), 0u};
      write_top(a, row, lane, r, __uint_as_float(x.x), (int)x.y);
    }
  }
}

// Values a lane takes at a time: 16, 8 where a row has no more than 512.  Waves per row:
// one where a row is less than four tiles, else a workgroup's four, and so many workgroups
// that all CUs have some where there are few rows.
struct Split {
  int parts;
  int64_t range;
};
inline int values_of(int64_t C) { return C <= 512 ? 8 : 16; }
Split split_of(int64_t M, int64_t C) {
  const int64_t tile = 64 * values_of(C);  // columns a wave takes at a time
  const int64_t tiles = (C + tile - 1) / tile;
  // four waves a row, more where those are few in all (up to 128, all of whose best
  // k_labels_join reads: 8 x 262147, top 20: 27 us, with 264 waves a row 39)
  const int64_t want = tiles < 4 ? 1 : std::min<int64_t>(128, std::max<int64_t>(4, 2048 / M));
  const int64_t per = (tiles + want - 1) / want, parts = (tiles + per - 1) / per;
  return Split{(int)(parts > 1 ? (parts + 3) / 4 * 4 : 1), per * tile};
}
// Rows a wave or less holds at once, whose top classes come one after another:
// while that are few
inline bool is_narrow(int64_t C, int top_k, int piece) {
  return C <= 8 * piece || (C <= 64 * piece && top_k <= 8);
}

template <typename T>
hipError_t launch(LabelArgs a, hipStream_t st) {
  typedef Piece<T> P;
  const auto go = [&](auto kernel, int64_t rows_per_wg) {
    const int64_t blocks = std::min<int64_t>((a.M * a.parts + rows_per_wg - 1) / rows_per_wg, kMostBlocks);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, a);
    return hipGetLastError();
  };
  a.parts = 1;
  // a lane a row from 16384 rows on: fewer do not fill the card
  static_assert(SAGA_MAX_TOP == 32, "the last list holds them");
  if (a.C <= kLaneC && a.M >= 16384) {
    const int k = a.top_k;
    if (k == 0) return go(k_labels_lane<T, 0>, 256);
    if (k == 1) return go(k_labels_lane<T, 1>, 256);
    if (k == 2) return go(k_labels_lane<T, 2>, 256);
    if (k == 3) return go(k_labels_lane<T, 3>, 256);
    if (k <= 5) return go(k_labels_lane<T, 5>, 256);
    if (k <= 8) return go(k_labels_lane<T, 8>, 256);
    if (k <= 12) return go(k_labels_lane<T, 12>, 256);
    if (k <= 20) return go(k_labels_lane<T, 20>, 256);
    return go(k_labels_lane<T, 32>, 256);
  }
  if (is_narrow(a.C, a.top_k, P::N)) {
    if (a.C <= 8 * P::N) return go(k_labels_narrow<T, 8>, 32);
    if (a.C <= 16 * P::N) return go(k_labels_narrow<T, 16>, 16);
    if (a.C <= 32 * P::N) return go(k_labels_narrow<T, 32>, 8);
    return go(k_labels_narrow<T, 64>, 4);
  }
  const Split sp = split_of(a.M, a.C);
  a.parts = sp.parts;
  a.range = sp.range;
  if (a.parts > 4) {
    const int64_t units = a.M * a.parts;
    a.part_stats = static_cast<float*>(a.ws);
    a.part_value = a.part_stats + units * 3;
    a.part_index = reinterpret_cast<int32_t*>(a.part_value + units * a.top_k);
  }
  const hipError_t e = values_of(a.C) == 8 ? go(k_labels_wide<T, 8>, 4) : go(k_labels_wide<T, 16>, 4);
  if (e != hipSuccess || a.parts <= 4) return e;
  hipLaunchKernelGGL((k_labels_join<T>), dim3((unsigned)a.M), dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t labels_workspace_bytes(int dtype, int64_t M, int64_t C, int top_k) {
  if (M <= 0 || is_narrow(C, top_k, dtype == SAGA_BF16 ? 8 : 4)) return 0;
  const Split sp = split_of(M, C);
  return sp.parts > 4 ? (size_t)M * sp.parts * (3 + 2 * (size_t)top_k) * 4 : 0;
}

hipError_t launch_label_log_probs(const LabelArgs& a, hipStream_t st) {
  if (a.M == 0) return hipSuccess;
  return a.dtype == SAGA_BF16 ? launch<uint16_t>(a, st) : launch<float>(a, st);
}

}  // namespace saga
