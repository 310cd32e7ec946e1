// Group norm with an activation, channels last, forward and backward, for gfx950.
//
// A sample is P points of C channels; each of its n channel groups (C / n channels,
// all points) has one mean and variance.  Blocks take slabs of neighbouring channel
// groups, so that the pieces of a point lie side by side; a thread holds one column of
// 16-byte pieces and walks the points.
//
// Sums of x - k and (x - k)^2, k the group's first value, are held in fp64: one pass
// over the data without cancellation, partial sums of any order add up, and a constant
// group normalises to beta exactly.
#include "group_norm.h"

#include <algorithm>

#include "act.h"
#include "norm.h"
#include "piece.h"

namespace pigan {
namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int SPLIT_NTH = 256;   // threads of a block that takes a range of points

// valid > 0 columns of a piece; WHOLE: pieces are all there
template <bool WHOLE, class T>
__device__ __forceinline__ piece_t load_piece(const T* p, int valid) {
  if constexpr (WHOLE) return *(const piece_u*)p;
  else return piece_load(p, valid);
}
template <bool WHOLE, class T>
__device__ __forceinline__ void store_piece(T* p, int valid, const float* f) {
  piece_store(p, WHOLE ? EPP<T> : valid, f);
}

// A slab's place: its first channel, width, first channel group and number of them, and
// the slots of one group (a slot: a piece where its channels are of one group, SL = 1,
// else a channel)
struct Slab { int64_t c0; int width; int64_t j0; int ng; int slots; };

template <class T, int SL>
__device__ __forceinline__ Slab slab_at(const GnArgs<T>& a, int64_t k) {
  const int64_t cg = a.C / a.n;
  Slab s;
  if (a.pl.chan_parts > 1) {
    const int64_t j = k / a.pl.chan_parts, part = k - j * a.pl.chan_parts;
    s.c0 = j * cg + part * a.pl.W;
    s.width = (int)min(a.pl.W, cg - part * a.pl.W);
    s.j0 = j;
    s.ng = 1;
  } else {
    s.c0 = k * a.pl.W;
    s.width = (int)min(a.pl.W, a.C - s.c0);
    s.j0 = k * a.pl.ng;
    s.ng = (int)min(a.pl.ng, a.n - s.j0);
  }
  s.slots = SL > 1 ? (int)min(cg, a.pl.W) : a.pl.ng == 1 ? a.pl.pw : (int)(cg / EPP<T>);
  return s;
}

// the channel group, among a slab's, of element e of a thread's column
template <class T, int SL>
__device__ __forceinline__ int group_of(const Slab& b, int col, int e) {
  return SL > 1 ? min(col * EPP<T> + e, b.width - 1) / b.slots : min(col / b.slots, b.ng - 1);
}

struct Pair { double s, q; };

// sm[row][slot] of `rows` rows of `per_row` slots: the sums of `ng` groups of `slots`
// neighbouring slots, each by `lanes` lanes in a fixed order; f(group, sums) is called
// by one thread per group.
template <class F>
__device__ __forceinline__ void group_sums(const Pair* sm, int rows, int per_row, int ng, int slots, int lanes, F&& f) {
  const int l = threadIdx.x % lanes, each = blockDim.x / lanes, n = rows * slots;
  for (int j0 = 0; j0 < ng; j0 += each) {   // the same number of turns for every thread
    const int j = j0 + threadIdx.x / lanes;
    Pair t = {0.0, 0.0};
    if (j < ng) {
      const Pair* p = sm + j * slots;
      for (int i = l; i < n; i += lanes) {
        const int r = i / slots;
        const Pair v = p[r * per_row + (i - r * slots)];
        t.s += v.s;
        t.q += v.q;
      }
    }
    for (int o = 1; o < lanes; o *= 2) {
      t.s += __shfl_xor(t.s, o);
      t.q += __shfl_xor(t.q, o);
    }
    if (j < ng && l == 0) f(j, t);
  }
}

// a place for k: finite, else the sums would lose an infinity's sign
__device__ __forceinline__ float shift_of(float x) { return __builtin_isfinite(x) ? x : 0.0f; }

// ---------------------------------------------------------------------------
// Samples of more points than a block's registers hold, forward: sums of ranges of
// points, then the results.
// ---------------------------------------------------------------------------
// ws: Pair [G][S][n][chan_parts * splits]
template <class T, int SL, bool WHOLE>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_sums(const GnArgs<T> a, int64_t items) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  const int64_t cg = a.C / a.n;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t split = it % pl.splits, slab = it / pl.splits % pl.slabs, gs = it / (pl.splits * pl.slabs);
    const int64_t g = gs / a.S, s = gs - g * a.S;
    const Slab b = slab_at<T, SL>(a, slab);
    const int valid = b.width - col * E;
    const T* first = a.x.p + g * a.x.gs + s * a.x.ss;
    Pair acc[SL];
    float k[SL];
#pragma unroll
    for (int e = 0; e < SL; ++e) {
      acc[e] = {0.0, 0.0};
      const int64_t j = b.j0 + group_of<T, SL>(b, col, e);
      k[e] = shift_of(Elem<T>::to_f(first[j * cg]));
    }
    if (valid > 0 && row < pl.rows) {
      const int64_t end = min(a.P, (split + 1) * pl.split_rows);
      const T* base = first + b.c0 + col * E;
      for (int64_t p = split * pl.split_rows + row; p < end; p += pl.rows) {
        float f[E];
        piece_floats<T>(load_piece<WHOLE>(base + p * a.x.ld, valid), f);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const double d = (double)f[e] - k[SL > 1 ? e : 0];
          if (WHOLE || e < valid) {
            acc[SL > 1 ? e : 0].s += d;
            acc[SL > 1 ? e : 0].q += d * d;
          }
        }
      }
    }
    if (row < pl.rows)
#pragma unroll
      for (int e = 0; e < SL; ++e) sm[(row * pl.pw + col) * SL + e] = acc[e];
    __syncthreads();
    Pair* part = (Pair*)a.ws;
    const int64_t parts = pl.chan_parts * pl.splits, at = pl.chan_parts > 1 ? slab % pl.chan_parts * pl.splits + split : split;
    group_sums(sm, pl.rows, pl.pw * SL, b.ng, b.slots, pl.lanes,
               [&](int j, const Pair& t) { part[((g * a.S + s) * a.n + b.j0 + j) * parts + at] = t; });
    __syncthreads();
  }
}

struct Stat { float mean, rstd; };
__device__ __forceinline__ Stat stat_of(const Pair& t, float k, double n, float eps) {
  const double m = t.s / n, var = fmax(t.q / n - m * m, 0.0);
  // fmax drops a NaN
  return {(float)(k + m), (float)(1.0 / sqrt((t.q - t.q == 0.0 ? var : t.q / n - m * m) + eps))};
}

template <class T, int SL, bool WHOLE>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_apply(const GnArgs<T> a, int64_t items) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];   // of Stat
  Stat* stat = (Stat*)sm;
  const GnPlan& pl = a.pl;
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  const int64_t cg = a.C / a.n;
  const double n = (double)cg * (double)a.P;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t split = it % pl.splits, slab = it / pl.splits % pl.slabs, gs = it / (pl.splits * pl.slabs);
    const int64_t g = gs / a.S, s = gs - g * a.S;
    const Slab b = slab_at<T, SL>(a, slab);
    const int valid = b.width - col * E;
    const T* first = a.x.p + g * a.x.gs + s * a.x.ss;
    const int64_t parts = pl.chan_parts * pl.splits;
    const Pair* part = (const Pair*)a.ws + ((g * a.S + s) * a.n + b.j0) * parts;
    const bool tells = split == 0 && (pl.chan_parts == 1 || slab % pl.chan_parts == 0);
    group_sums(part, 1, 0, b.ng, (int)parts, pl.lanes, [&](int j, const Pair& t) {
      const Stat st = stat_of(t, shift_of(Elem<T>::to_f(first[(b.j0 + j) * cg])), n, a.eps);
      stat[j] = st;
      const int64_t at = (g * a.S + s) * a.n + b.j0 + j;
      if (tells && a.mean) a.mean[at] = st.mean;
      if (tells && a.rstd) a.rstd[at] = st.rstd;
    });
    __syncthreads();
    if (valid > 0 && row < pl.rows) {
      float mean[E], sc[E], be[E];
      vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 1.0f, sc);
      vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 0.0f, be);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const Stat st = stat[group_of<T, SL>(b, col, e)];
        mean[e] = st.mean;
        sc[e] *= st.rstd;
      }
      const int64_t end = min(a.P, (split + 1) * pl.split_rows);
      const T* base = first + b.c0 + col * E;
      T* out = a.out.p + g * a.out.gs + s * a.out.ss + b.c0 + col * E;
      PIGAN_ACT_SWITCH(a.act, {
        for (int64_t p = split * pl.split_rows + row; p < end; p += pl.rows) {
          float f[E];
          piece_floats<T>(load_piece<WHOLE>(base + p * a.x.ld, valid), f);
          for (int e = 0; e < E; ++e) f[e] = act_value<ACT, T>((f[e] - mean[e]) * sc[e] + be[e]);
          store_piece<WHOLE>(out + p * a.out.ld, valid, f);
        }
      })
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// The same, backward: a channel's sums of da and da xhat over ranges of points give
// dgamma and dbeta (summed over samples) and, with gamma, a group's sums of h and
// h xhat; then dx.
// ---------------------------------------------------------------------------
// the columns' coefficients of a thread
template <class T, int SL>
struct Column {
  float mean[SL], rstd[SL], ga[EPP<T>], be[EPP<T>];
  __device__ __forceinline__ void load(const GnArgs<T>& a, const Slab& b, int64_t g, int64_t s, int col) {
    constexpr int E = EPP<T>;
    vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 1.0f, ga);
    vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 0.0f, be);
#pragma unroll
    for (int e = 0; e < SL; ++e) {
      const int64_t at = (g * a.S + s) * a.n + b.j0 + group_of<T, SL>(b, col, e);
      mean[e] = a.mean[at];
      rstd[e] = a.rstd[at];
    }
  }
};

// xh and da of a piece; zeros past `valid`
template <int ACT, bool WHOLE, class T, int SL>
__device__ __forceinline__ void slope_piece(const Column<T, SL>& c, int valid, float (&xh)[EPP<T>], float (&da)[EPP<T>]) {
#pragma unroll
  for (int e = 0; e < EPP<T>; ++e) {
    xh[e] = (xh[e] - c.mean[SL > 1 ? e : 0]) * c.rstd[SL > 1 ? e : 0];
    if constexpr (ACT != PIGAN_ACT_NONE) da[e] *= act_slope<ACT, T>(xh[e] * c.ga[e] + c.be[e]);
    if (!WHOLE && e >= valid) xh[e] = da[e] = 0.0f;
  }
}

// ws: float [G][S * splits][2][C]
template <class T, int SL, bool WHOLE>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_bwd_sums(const GnArgs<T> a, int64_t items) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  float* fm = (float*)sm;   // [rows][2][pw * E]
  const GnPlan& pl = a.pl;
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw, wide = pl.pw * E;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t split = it % pl.splits, slab = it / pl.splits % pl.slabs, gs = it / (pl.splits * pl.slabs);
    const int64_t g = gs / a.S, s = gs - g * a.S;
    const Slab b = slab_at<T, SL>(a, slab);
    const int valid = b.width - col * E;
    float sg[E], sb[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sg[e] = sb[e] = 0.0f;
    if (valid > 0 && row < pl.rows) {
      Column<T, SL> c;
      c.load(a, b, g, s, col);
      const int64_t end = min(a.P, (split + 1) * pl.split_rows);
      const T* x = a.x.p + g * a.x.gs + s * a.x.ss + b.c0 + col * E;
      const T* dy = a.dy.p + g * a.dy.gs + s * a.dy.ss + b.c0 + col * E;
      PIGAN_ACT_SWITCH(a.act, {
        for (int64_t p = split * pl.split_rows + row; p < end; p += pl.rows) {
          float xh[E];
          float da[E];
          piece_floats<T>(load_piece<WHOLE>(x + p * a.x.ld, valid), xh);
          piece_floats<T>(load_piece<WHOLE>(dy + p * a.dy.ld, valid), da);
          slope_piece<ACT, WHOLE>(c, valid, xh, da);
          for (int e = 0; e < E; ++e) {
            sg[e] += da[e] * xh[e];
            sb[e] += da[e];
          }
        }
      })
    }
    if (row < pl.rows)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        fm[row * 2 * wide + col * E + e] = sg[e];
        fm[row * 2 * wide + wide + col * E + e] = sb[e];
      }
    __syncthreads();
    float* part = (float*)a.ws + (gs * pl.splits + split) * 2 * a.C + b.c0;
    for (int i = threadIdx.x; i < 2 * wide; i += SPLIT_NTH) {
      const int c = i < wide ? i : i - wide;
      double t = 0.0;
      for (int r = 0; r < pl.rows; ++r) t += fm[r * 2 * wide + i];
      if (c < b.width) part[(i < wide ? 0 : a.C) + c] = (float)t;
    }
    __syncthreads();
  }
}

// means of h and h xhat: Stat-like pairs [G][S][n] behind the partial sums, a wave each
template <class T>
__global__ void __launch_bounds__(256) k_gn_bwd_join(const GnArgs<T> a, float2* __restrict__ means, int64_t total) {
  const GnPlan& pl = a.pl;
  const int64_t cg = a.C / a.n;
  const int l = threadIdx.x & 63;
  const double n = (double)cg * (double)a.P;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < total; i += (int64_t)gridDim.x * 4) {
    const int64_t gs = i / a.n, j = i - gs * a.n, g = gs / a.S;
    const float* part = (const float*)a.ws + gs * pl.splits * 2 * a.C + j * cg;
    Pair t = {0.0, 0.0};
    for (int64_t k = l; k < pl.splits * cg; k += 64) {
      const int64_t sp = k / cg, c = k - sp * cg;
      const double ga = a.gamma ? a.gamma[g * a.C + j * cg + c] : 1.0f;
      t.q += ga * part[sp * 2 * a.C + c];
      t.s += ga * part[sp * 2 * a.C + a.C + c];
    }
    for (int o = 1; o < 64; o *= 2) {
      t.s += __shfl_xor(t.s, o);
      t.q += __shfl_xor(t.q, o);
    }
    if (l == 0) means[i] = {(float)(t.s / n), (float)(t.q / n)};
  }
}

template <class T, int SL, bool WHOLE>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_bwd_apply(const GnArgs<T> a, const float2* __restrict__ means, int64_t items) {
  constexpr int E = EPP<T>;
  const GnPlan& pl = a.pl;
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t split = it % pl.splits, slab = it / pl.splits % pl.slabs, gs = it / (pl.splits * pl.slabs);
    const int64_t g = gs / a.S, s = gs - g * a.S;
    const Slab b = slab_at<T, SL>(a, slab);
    const int valid = b.width - col * E;
    if (valid <= 0 || row >= pl.rows) continue;
    Column<T, SL> c;
    c.load(a, b, g, s, col);
    float2 m[SL];
#pragma unroll
    for (int e = 0; e < SL; ++e)
      m[e] = means[gs * a.n + b.j0 + group_of<T, SL>(b, col, e)];
    const int64_t end = min(a.P, (split + 1) * pl.split_rows);
    const T* x = a.x.p + g * a.x.gs + s * a.x.ss + b.c0 + col * E;
    const T* dy = a.dy.p + g * a.dy.gs + s * a.dy.ss + b.c0 + col * E;
    const T* add = a.add.p ? a.add.p + g * a.add.gs + s * a.add.ss + b.c0 + col * E : nullptr;
    T* out = a.out.p + g * a.out.gs + s * a.out.ss + b.c0 + col * E;
    PIGAN_ACT_SWITCH(a.act, {
      for (int64_t p = split * pl.split_rows + row; p < end; p += pl.rows) {
        float xh[E];
        float da[E];
        float r[E];
        piece_floats<T>(load_piece<WHOLE>(x + p * a.x.ld, valid), xh);
        piece_floats<T>(load_piece<WHOLE>(dy + p * a.dy.ld, valid), da);
        if (add) piece_floats<T>(load_piece<WHOLE>(add + p * a.add.ld, valid), r);
        slope_piece<ACT, WHOLE>(c, valid, xh, da);
        for (int e = 0; e < E; ++e) {
          const int k = SL > 1 ? e : 0;
          da[e] = c.rstd[k] * (da[e] * c.ga[e] - m[k].x - xh[e] * m[k].y);
          if (add) da[e] += r[e];
        }
        store_piece<WHOLE>(out + p * a.out.ld, valid, da);
      }
    })
  }
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
// f(SL, WHOLE) of a call's widths
template <class T, class F> void by_width(const GnArgs<T>& a, F&& f) {
  constexpr int E = EPP<T>;
  const int64_t cg = a.C / a.n;
  const bool one = a.pl.ng == 1 || cg % E == 0;
  const bool whole = cg % E == 0 || (a.pl.ng > 1 && a.pl.W % E == 0 && a.C % E == 0);
  if (one && whole) f(std::integral_constant<int, 1>{}, std::true_type{});
  else if (one) f(std::integral_constant<int, 1>{}, std::false_type{});
  else if (whole) f(std::integral_constant<int, E>{}, std::true_type{});
  else f(std::integral_constant<int, E>{}, std::false_type{});
}

unsigned grid_of(int64_t items) { return (unsigned)std::min<int64_t>(items, 1 << 20); }

}  // namespace

GnPlan gn_plan(bool backward, int elem_bytes, int64_t G, int64_t S, int64_t P, int64_t C, int64_t n) {
  GnPlan pl{};
  const int64_t E = 16 / elem_bytes, cg = C / n, most = SPLIT_NTH * E;
  pl.nth = SPLIT_NTH;
  if (cg > most) {
    pl.W = most;
    pl.ng = 1;
    pl.chan_parts = cdiv(cg, most);
    pl.slabs = n * pl.chan_parts;
  } else {
    // 512 bytes of a point: long runs, and rows enough for the threads
    pl.ng = std::min(n, std::max<int64_t>(1, 32 * E / cg));
    pl.W = pl.ng * cg;
    pl.chan_parts = 1;
    pl.slabs = cdiv(n, pl.ng);
  }
  pl.pw = (int32_t)cdiv(pl.W, E);
  pl.rows = SPLIT_NTH / pl.pw;
  pl.ns = 1;
  pl.lanes = 64;
  while (pl.lanes > 1 && pl.lanes * pl.ng > SPLIT_NTH) pl.lanes /= 2;
  const int64_t base = G * std::max<int64_t>(S, 1) * pl.slabs, least = cdiv(P, 4 * pl.rows);
  pl.splits = std::max<int64_t>(1, std::min<int64_t>({cdiv(2048, base), least, 64}));
  pl.split_rows = cdiv(cdiv(P, pl.splits), pl.rows) * pl.rows;
  pl.splits = cdiv(P, pl.split_rows);
  pl.slots = S * pl.splits;
  return pl;
}

size_t gn_forward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t n) {
  return (size_t)(G * S * n * pl.chan_parts * pl.splits) * sizeof(Pair);
}
static size_t sums_bytes(const GnPlan& pl, int64_t G, int64_t C) {
  return ((size_t)(G * pl.slots * 2 * C) * 4 + 15) / 16 * 16;
}
size_t gn_backward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t C, int64_t n, bool cols) {
  return sums_bytes(pl, G, C) + (size_t)(G * S * n) * sizeof(float2);
}

template <class T> hipError_t launch_gn_fwd(const GnArgs<T>& a, int G, hipStream_t st) {
  if (a.S <= 0) return hipSuccess;
  const int64_t items = (int64_t)G * a.S * a.pl.slabs * a.pl.splits;
  by_width(a, [&](auto sl, auto whole) {
    k_gn_sums<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, SPLIT_NTH * sl.value * sizeof(Pair), st>>>(a, items);
    k_gn_apply<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, (size_t)a.pl.ng * sizeof(Stat), st>>>(a, items);
  });
  return hipGetLastError();
}

template <class T> hipError_t launch_gn_bwd(const GnArgs<T>& a, int G, hipStream_t st) {
  const bool cols = a.dgamma || a.dbeta;
  if (a.S <= 0) {
    // sums over no samples
    for (float* sum : {a.dgamma, a.dbeta})
      if (sum)
        if (const hipError_t e = launch_zeros(sum, G * a.C, st); e != hipSuccess) return e;
    return hipSuccess;
  }
  const int64_t items = (int64_t)G * a.S * a.pl.slabs * a.pl.splits, total = (int64_t)G * a.S * a.n;
  float2* means = (float2*)(a.ws + sums_bytes(a.pl, G, a.C));
  by_width(a, [&](auto sl, auto whole) {
    k_gn_bwd_sums<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, SPLIT_NTH * EPP<T> * 8, st>>>(a, items);
    // dx may overwrite dy
    if (a.out.p) {
      k_gn_bwd_join<T><<<grid_of(cdiv(total, 4)), 256, 0, st>>>(a, means, total);
      k_gn_bwd_apply<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, 0, st>>>(a, means, items);
    }
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !cols) return e;
  return launch_slot_sum((const float*)a.ws, a.pl.slots * 2 * a.C, (int)a.pl.slots, 2 * a.C, a.dgamma, a.C, a.dbeta, G, st);
}

#define PIGAN_GN_INST(T)                                              \
  template hipError_t launch_gn_fwd<T>(const GnArgs<T>&, int, hipStream_t); \
  template hipError_t launch_gn_bwd<T>(const GnArgs<T>&, int, hipStream_t);
PIGAN_GN_INST(float)
PIGAN_GN_INST(bf16)
PIGAN_GN_INST(f16)

}  // namespace pigan
