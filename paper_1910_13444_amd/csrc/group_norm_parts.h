// Parts of group norm's kernels, forward and backward (group_norm_fwd.hip,
// group_norm_bwd.hip).
//
// A sample is P points of C channels; each of its n channel groups (C / n channels,
// all points) has one mean and variance.  Blocks take slabs of neighbouring channel
// groups, so that the pieces of a point lie side by side; a thread holds one column of
// 16-byte pieces and walks the points.
//
// Sums of x - k and (x - k)^2, k the group's first value, are held in fp64: one pass
// over the data without cancellation, partial sums of any order add up, and a constant
// group normalises to beta exactly.
//
// Results in 16 bits are as much bound by the vector units as by memory (a copy's rate
// leaves 31 lane operations for an element that is read and written): an activation's
// kernels are its own, whole numbers are divided by reciprocals, blocks are long.
#pragma once
#include <algorithm>
#include <type_traits>
#include <utility>

#include "act.h"
#include "group_norm.h"
#include "piece.h"

namespace pigan {
namespace {

// points that a thread has under way where blocks take ranges of points
constexpr int SUM_TURN = 4, APPLY_TURN = 2, BWD_TURN = 2;

// n / d for 0 <= n < 2^21: n + 1/2 is half a unit of 1 / d away from the whole quotients,
// the product's error is 2^-22 of it
struct Div {
  float inv;
  __device__ __forceinline__ explicit Div(int d) : inv(__builtin_amdgcn_rcpf((float)d)) {}
  __device__ __forceinline__ int operator()(int n) const { return (int)(((float)n + 0.5f) * inv); }
};

// valid > 0 columns of a piece; WHOLE: pieces are all there
// `stream`: past the caches, as GnPlan::stream says
template <bool WHOLE, class T>
__device__ __forceinline__ piece_t load_piece(const T* p, int valid, bool stream = false) {
  if constexpr (WHOLE) {
    piece_t v;
    if (stream) {
      asm volatile("; streamed");
      v = __builtin_nontemporal_load((const piece_u*)p);
      asm volatile("; streamed");
    } else {
      v = *(const piece_u*)p;
    }
    return v;
  } else {
    return piece_load(p, valid);
  }
}
template <bool WHOLE, class T>
__device__ __forceinline__ void store_piece(T* p, int valid, const float* f, bool stream) {
  if (WHOLE && stream) {
    T e[EPP<T>];
#pragma unroll
    for (int i = 0; i < EPP<T>; ++i) e[i] = Elem<T>::from_f(f[i]);
    piece_t v;
    __builtin_memcpy(&v, e, 16);
    asm volatile("; streamed");   // else the compiler joins both stores to a plain one
    __builtin_nontemporal_store(v, (piece_u*)p);
    asm volatile("; streamed");
  } else {
    piece_store(p, WHOLE ? EPP<T> : valid, f);
  }
}

// A slab's place: its first channel, width, first channel group and number of them
struct Slab { int64_t c0; int width; int64_t j0; int ng; };

template <class T>
__device__ __forceinline__ Slab slab_at(const GnArgs<T>& a, uint32_t k) {
  Slab s;
  if (a.pl.chan_parts > 1) {
    const uint32_t parts = (uint32_t)a.pl.chan_parts, j = k / parts, part = k - j * parts;
    s.c0 = j * a.pl.cg + part * a.pl.W;
    s.width = (int)min(a.pl.W, a.pl.cg - part * a.pl.W);
    s.j0 = j;
    s.ng = 1;
  } else {
    s.c0 = k * a.pl.W;
    s.width = (int)min(a.pl.W, a.C - s.c0);
    s.j0 = k * a.pl.ng;
    s.ng = (int)min(a.pl.ng, a.n - s.j0);
  }
  return s;
}

// the channel group, among a slab's, of element e of a thread's column.  A group has
// pl.span slots: pieces where a piece's channels are of one group (SL = 1), else channels.
template <class T, int SL>
__device__ __forceinline__ int group_of(const Slab& b, const Div& by_span, int col, int e) {
  return SL > 1 ? by_span(min(col * EPP<T> + e, b.width - 1)) : min(by_span(col), b.ng - 1);
}

// f(group, sums) of the sums over `lanes` (a power of two) lanes in a fixed order, called by
// one thread for each of `all`; add(group, lane) gives a lane's share
template <class A, class F>
__device__ __forceinline__ void lane_sums(int all, int lanes, A&& add, F&& f) {
  const int sh = 31 - __builtin_clz(lanes), l = threadIdx.x & (lanes - 1), each = blockDim.x >> sh;
  for (int k0 = 0; k0 < all; k0 += each) {   // the same number of turns for every thread
    const int k = k0 + (threadIdx.x >> sh);
    Pair t = {0.0, 0.0};
    if (k < all) t = add(k, l);
    for (int o = 1; o < lanes; o *= 2) {
      t.s += __shfl_xor(t.s, o);
      t.q += __shfl_xor(t.q, o);
    }
    if (k < all && l == 0) f(k, t);
  }
}

// Sums in LDS lie in rows of an odd number of entries, so that a slot's are in banks of their
// own; a block of N threads has N (slots + 1) entries at most.
__device__ __forceinline__ int row_of(int slots) { return slots | 1; }
struct PairF { float s, q; };

// sm[row][slot] of each of `ns` samples of `rows` rows: f(sample, group, sums) of each of its
// `ng` groups of `span` neighbouring slots
template <class P, class F>
__device__ __forceinline__ void group_sums(const P* sm, int ns, int rows, int per_row, int ng, int span, int lanes, F&& f) {
  const Div by_ng(ng), by_span(span);
  const int n = rows * span;
  lane_sums(ns * ng, lanes, [&](int k, int l) {
    const int i = ns > 1 ? by_ng(k) : 0, j = k - i * ng;
    const P* p = sm + i * rows * per_row + j * span;
    Pair t = {0.0, 0.0};
#pragma unroll 4
    for (int q = l; q < n; q += lanes) {
      const int r = by_span(q);
      const P v = p[r * per_row + (q - r * span)];
      t.s += v.s;
      t.q += v.q;
    }
    return t;
  }, [&](int k, const Pair& t) {
    const int i = ns > 1 ? by_ng(k) : 0;
    f(i, k - i * ng, t);
  });
}

// f(group, sums) of `ng` groups' `parts` sums of ranges in global memory
template <class F>
__device__ __forceinline__ void range_sums(const Pair* __restrict__ part, int ng, int parts, int lanes, F&& f) {
  lane_sums(ng, lanes, [&](int k, int l) {
    Pair t = {0.0, 0.0};
#pragma unroll 4
    for (int q = l; q < parts; q += lanes) {
      const Pair v = part[(int64_t)k * parts + q];
      t.s += v.s;
      t.q += v.q;
    }
    return t;
  }, f);
}

// a place for k: finite, else the sums would lose an infinity's sign
__device__ __forceinline__ float shift_of(float x) { return __builtin_isfinite(x) ? x : 0.0f; }

// 1 / sqrt(v) for v > 0: the hardware's fp64 reciprocal root (off by up to 2^-24.2 on 4 M values
// of [1, 4)) and two Newton steps
__device__ __forceinline__ double rsqrt64(double v) {
  double r = __builtin_amdgcn_rsq(v);
  r = r * (1.5 - 0.5 * v * r * r);
  return r * (1.5 - 0.5 * v * r * r);
}

struct Stat { float mean, rstd; };
// of the sums of n values from k on; a NaN stays one
__device__ __forceinline__ Stat stat_of(const Pair& t, float k, double inv_n, float eps) {
  const double m = t.s * inv_n, var = t.q * inv_n - m * m;
  return {(float)(k + m), (float)rsqrt64((var < 0.0 ? 0.0 : var) + eps)};
}

// NV pieces of a column, `step` elements apart from q on, of the `left` rows that are
// there, each `rows` behind the one before; for the others the first again
template <bool WHOLE, int NV, class T>
__device__ __forceinline__ void load_rows(piece_t (&raw)[NV], const T* q, int64_t step, int left, int rows, int valid) {
#pragma unroll
  for (int v = 0; v < NV; ++v) raw[v] = load_piece<WHOLE>(v == 0 || v * rows < left ? q + v * step : q, valid);
}

// Where a sample is shared by blocks, a block's turns of U rows of threads come in order
// with the others', `by` points apart, so that all blocks together read a window that moves
// over the sample: blocks that begin at strides of a power of two of their own meet in the
// same memory channels.  The results are formed from the last turn to the first and
// begin with the last samples: of a field that is larger than the last-level cache what the
// sums read last is still there.
struct Turns {
  int64_t first;   // a thread's first point
  int left, by;    // points from there on
  __host__ __device__ __forceinline__ Turns(const GnPlan& pl, int64_t P, int U, uint32_t split, int splits, int row)
      : first((int64_t)split * U * pl.rows + row), left((int)(P - first)), by(splits * U * pl.rows) {}
  // from the first turn's begin to the last one's; 0 without any
  __host__ __device__ __forceinline__ int last() const { return left > by ? (left - 1) / by * by : 0; }
  // whether a turn lies before the one with `at` points from its begin on.  A sample has up to
  // 2^31 - 1 points: at + by may pass that, the difference does not
  __host__ __device__ __forceinline__ bool before(int at) const { return left - at >= by; }
};
// of eight neighbours each stays on its XCD
__device__ __forceinline__ uint32_t from_last(uint32_t i, uint32_t n) {
  const uint32_t whole = n & ~7u;
  return i < whole ? whole - 8 - (i & ~7u) + (i & 7u) : i;
}

// ---------------------------------------------------------------------------
// Activations of 16-bit results in fewer operations than act.h's, with its errors: the
// exponential's argument and the tail's come from one product, the value's polynomial is
// shorter, and
//   a Phi(a) = max(a, 0) - |a| tail(|a|),   a s(a) = a / (1 + exp(-a))
// Sizes are bounded where the factors beside them have become 0.
// ---------------------------------------------------------------------------
// Phi(-|a|) and exp(-a^2 / 2); the polynomial of act.h's normal_cdf, halved
__device__ __forceinline__ float normal_tail(float a, float& gauss) {
  const float b = a * 0.84932180028801904f;                        // sqrt(1 / (2 ln 2))
  gauss = __builtin_amdgcn_exp2f(-b * b);
  const float t = __builtin_amdgcn_rcpf(1.0f + fabsf(b) * 0.33302184446307909f);   // 0.4 sqrt(ln 2)
  float q = 0.5f * 0.05027513951063156f;
  q = q * t - 0.5f * 0.18294988572597504f;
  q = q * t + 0.5f * 0.16915729641914368f;
  q = q * t - 0.5f * 0.0056617371737957f;
  q = q * t + 0.5f * 0.14145344495773315f;
  q = q * t + 0.5f * 0.1685371994972229f;
  q = q * t + 0.5f * 0.20784327387809753f;
  q = q * t + 0.5f * 0.22566954791545868f;
  q = q * t + 0.5f * 0.22567586600780487f;
  return q * t * gauss;
}

// |a| Phi(-|a|), 0 at infinity.  Phi(-z) = t Q(t) exp(-z^2 / 2), t = 1 / (1 + 0.28 z), Q the
// polynomial of degree 6 that is nearest in relative terms (3.7e-6, with the roundings and
// the exponential's 5e-6 for z < 6; 7e-7 of the result's unit): two operations of 24 less,
// a hundredth of an fp16 rounding
__device__ __forceinline__ float gelu_tail(float a) {
  const float b = a * 0.84932180028801904f;
  const float t = __builtin_amdgcn_rcpf(1.0f + fabsf(b) * 0.3296748101711273f);   // 0.28 sqrt(2 ln 2)
  float q = -0.050230927765369415f;
  q = q * t + 0.1054425984621048f;
  q = q * t + 0.024950530380010605f;
  q = q * t + 0.09445563703775406f;
  q = q * t + 0.10193581879138947f;
  q = q * t + 0.11174066364765167f;
  q = q * t + 0.11170384287834167f;
  return __builtin_amdgcn_fmed3f(fabsf(a), 0.0f, 64.0f) * t * q * __builtin_amdgcn_exp2f(-b * b);
}

template <int ACT, class T>
__device__ __forceinline__ float value_of(float a) {
  if constexpr (sizeof(T) == 2 && ACT == PIGAN_ACT_GELU) {
    return fmaxf(a, 0.0f) - gelu_tail(a);   // a NaN comes back by the tail
  } else if constexpr (sizeof(T) == 2 && ACT == PIGAN_ACT_SILU) {
    return a * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a * -1.4426950408889634f));
  } else {
    return act_value<ACT, T>(a);
  }
}

template <int ACT, class T>
__device__ __forceinline__ float slope_of(float a) {
  if constexpr (sizeof(T) == 2 && ACT == PIGAN_ACT_GELU) {
    float g;
    const float tail = normal_tail(a, g);
    return (a > 0.0f ? 1.0f - tail : tail) + __builtin_amdgcn_fmed3f(a, -64.0f, 64.0f) * 0.3989422804014327f * g;
  } else if constexpr (sizeof(T) == 2 && ACT == PIGAN_ACT_SILU) {
    // below -60 the slope is less than 2^-80; a NaN stays one
    const float b = a < -60.0f ? -60.0f : a;
    const float e = __builtin_amdgcn_exp2f(b * -1.4426950408889634f), s = __builtin_amdgcn_rcpf(1.0f + e);
    return s + fminf(b, 200.0f) * (s * (e * s));
  } else {
    return act_slope<ACT, T>(a);
  }
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
// f(ACT): the registers that all activations need at once would be too many
template <class F> void by_act(int act, F&& f) {
  PIGAN_ACT_SWITCH(act, { f(std::integral_constant<int, ACT>{}); })
}

// f(SL, WHOLE) of a call's widths
template <class T, class F> void by_width(const GnArgs<T>& a, F&& f) {
  constexpr int E = EPP<T>;
  const bool aligned = a.pl.cg % E == 0, one = a.pl.ng == 1 || aligned;
  const bool whole = aligned || (a.pl.ng > 1 && a.pl.W % E == 0 && a.C % E == 0);
  if (one && whole) f(std::integral_constant<int, 1>{}, std::true_type{});
  else if (one) f(std::integral_constant<int, 1>{}, std::false_type{});
  else if (whole) f(std::integral_constant<int, E>{}, std::true_type{});
  else f(std::integral_constant<int, E>{}, std::false_type{});
}

// f(NTH, NV) of a forward plan; the lists' shapes
template <bool ALIGNED, class F> void by_shape(const GnPlan& pl, F&& f) {
  constexpr const auto& list = [] () -> const auto& {
    if constexpr (ALIGNED) return FWD_SHAPES;
    else return FWD_ODD;
  }();
  constexpr int N = (int)(sizeof(list) / sizeof(Shape));
  [&]<int... I>(std::integer_sequence<int, I...>) {
    (void)((pl.nth == list[I].nth && pl.nv == list[I].nv &&
            (f(std::integral_constant<int, list[I].nth>{}, std::integral_constant<int, list[I].nv>{}), true)) || ...);
  }(std::make_integer_sequence<int, N>{});
}

}  // namespace
}  // namespace pigan
