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

// sm[row][slot]: of each of `ns` samples of `rows` rows, and of each of its `ng` groups of
// `slots` neighbouring slots, the sums, each by `lanes` lanes in a fixed order; f(sample,
// group, sums) is called by one thread per group.
template <class F>
__device__ __forceinline__ void group_sums(const Pair* sm, int ns, int rows, int per_row, int ng, int slots, int lanes, F&& f) {
  const int l = threadIdx.x % lanes, each = blockDim.x / lanes, n = rows * slots, all = ns * ng;
  for (int k0 = 0; k0 < all; k0 += each) {   // the same number of turns for every thread
    const int k = k0 + threadIdx.x / lanes, i = k / ng, j = k - i * ng;
    Pair t = {0.0, 0.0};
    if (k < all) {
      const Pair* p = sm + i * rows * per_row + j * slots;
      for (int q = l; q < n; q += lanes) {
        const int r = q / slots;
        const Pair v = p[r * per_row + (q - r * slots)];
        t.s += v.s;
        t.q += v.q;
      }
    }
    for (int o = 1; o < lanes; o *= 2) {
      t.s += __shfl_xor(t.s, o);
      t.q += __shfl_xor(t.q, o);
    }
    if (k < all && l == 0) f(i, j, t);
  }
}

// a place for k: finite, else the sums would lose an infinity's sign
__device__ __forceinline__ float shift_of(float x) { return __builtin_isfinite(x) ? x : 0.0f; }

// 1 / sqrt(v) for v > 0: the fp64 reciprocal root (2^-28 or better) and two Newton steps
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

// ---------------------------------------------------------------------------
// Rows: samples of one point, forward.  A group is 2^i <= 64 neighbouring lanes with a
// piece each, the sums are theirs by shuffles; a thread keeps its column over NV rows at
// a time.
// ---------------------------------------------------------------------------
template <class T, int NV>
__global__ void __launch_bounds__(256) k_gn_rows(const GnArgs<T> a) {
  constexpr int E = EPP<T>;
  const GnPlan& pl = a.pl;
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  const Slab b = slab_at<T, 1>(a, blockIdx.y);
  const int64_t g = blockIdx.z;
  const int lanes = b.slots, j = min(col / lanes, b.ng - 1);
  const bool head = threadIdx.x % lanes == 0;
  if (row >= pl.rows || col * E >= b.width) return;   // whole groups of lanes
  const double inv_n = 1.0 / (double)(a.C / a.n);
  float ga[E], be[E];
  vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, a.C, 1.0f, ga);
  vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, a.C, 0.0f, be);
  const T* x = a.x.p + g * a.x.gs + b.c0 + col * E;
  T* y = a.out.p + g * a.out.gs + b.c0 + col * E;
  const int64_t step = (int64_t)gridDim.x * pl.rows;
  PIGAN_ACT_SWITCH(a.act, {
    for (int64_t s0 = (int64_t)blockIdx.x * pl.rows + row; s0 < a.S; s0 += NV * step) {
      piece_t raw[NV];
      for (int v = 0; v < NV; ++v) {
        const int64_t s = s0 + v * step;
        raw[v] = *(const piece_u*)(x + (s < a.S ? s : s0) * a.x.ss);
      }
      for (int v = 0; v < NV; ++v) {
        const int64_t s = s0 + v * step;
        float f[E];
        piece_floats<T>(raw[v], f);
        const float k = shift_of(__shfl(f[0], (threadIdx.x & 63) & ~(lanes - 1)));
        Pair t = {0.0, 0.0};
        for (int e = 0; e < E; ++e) {
          const double d = (double)f[e] - k;
          t.s += d;
          t.q += d * d;
        }
        for (int o = 1; o < lanes; o *= 2) {
          t.s += __shfl_xor(t.s, o);
          t.q += __shfl_xor(t.q, o);
        }
        const Stat st = stat_of(t, k, inv_n, a.eps);
        if (s < a.S) {
          for (int e = 0; e < E; ++e) f[e] = act_value<ACT, T>((f[e] - st.mean) * (st.rstd * ga[e]) + be[e]);
          piece_store(y + s * a.out.ss, E, f);
          const int64_t at = (g * a.S + s) * a.n + b.j0 + j;
          if (head && a.mean) a.mean[at] = st.mean;
          if (head && a.rstd) a.rstd[at] = st.rstd;
        }
      }
    }
  })
}

// NV pieces of a column, `step` rows apart from row p0 on; past the last row, that one again
template <bool WHOLE, int NV, class T>
__device__ __forceinline__ void load_rows(piece_t (&raw)[NV], const T* base, int64_t ld, int64_t p0, int64_t step, int64_t P,
                                          int valid) {
#pragma unroll
  for (int v = 0; v < NV; ++v) raw[v] = load_piece<WHOLE>(base + min(p0 + v * step, P - 1) * ld, valid);
}

// ---------------------------------------------------------------------------
// Samples whose slabs fit a block's registers, forward: read once, written once.  Short
// samples share a block, NV = 1 then.
// ---------------------------------------------------------------------------
template <class T, int NTH, int NV, int SL, bool WHOLE>
__global__ void __launch_bounds__(NTH, NV >= 8 ? 4 : 1) k_gn_one(const GnArgs<T> a, int64_t items) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  Stat* stat = (Stat*)(sm + NTH * SL);
  float* shift = (float*)(stat + pl.ns * pl.ng);
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  const int si = NV == 1 && pl.ns > 1 ? row / (int)a.P : 0, pr = row - si * (int)a.P * (NV == 1 && pl.ns > 1);
  const int64_t cg = a.C / a.n, batches = (a.S + pl.ns - 1) / pl.ns;
  const double inv_n = 1.0 / ((double)cg * (double)a.P);
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t slab = it % pl.slabs, gb = it / pl.slabs, g = gb / batches, s0 = (gb - g * batches) * pl.ns, s = s0 + si;
    const Slab b = slab_at<T, SL>(a, slab);
    const int valid = b.width - col * E;
    const bool on = row < pl.rows && s < a.S && valid > 0;
    const T* first = a.x.p + g * a.x.gs + (on ? s : s0) * a.x.ss;
    piece_t raw[NV];
    load_rows<WHOLE>(raw, first + (on ? b.c0 + col * E : b.c0), a.x.ld, on ? pr : 0, pl.rows, a.P, on ? valid : b.width);
    float k[SL];
    Pair acc[SL];
#pragma unroll
    for (int e = 0; e < SL; ++e) {
      const int j = group_of<T, SL>(b, col, e);
      k[e] = shift_of(Elem<T>::to_f(first[(b.j0 + j) * cg]));
      acc[e] = {0.0, 0.0};
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (on && pr + (int64_t)v * pl.rows < a.P) {
        float f[E];
        piece_floats<T>(raw[v], f);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const double d = (double)f[e] - k[SL > 1 ? e : 0];
          if (WHOLE || e < valid) {
            acc[SL > 1 ? e : 0].s += d;
            acc[SL > 1 ? e : 0].q += d * d;
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (row < pl.rows)
#pragma unroll
      for (int e = 0; e < SL; ++e) {
        const int slot = col * SL + e;
        sm[row * pl.pw * SL + slot] = acc[e];
        if (on && pr == 0 && slot < b.ng * b.slots && slot % b.slots == 0) shift[si * b.ng + slot / b.slots] = k[e];
      }
    __syncthreads();
    group_sums(sm, pl.ns, pl.ns > 1 ? (int)a.P : pl.rows, pl.pw * SL, b.ng, b.slots, pl.lanes, [&](int i, int j, const Pair& t) {
      const Stat st = stat_of(t, shift[i * b.ng + j], inv_n, a.eps);
      stat[i * b.ng + j] = st;
      const int64_t at = (g * a.S + s0 + i) * a.n + b.j0 + j;
      if (s0 + i < a.S) {
        if (a.mean) a.mean[at] = st.mean;
        if (a.rstd) a.rstd[at] = st.rstd;
      }
    });
    __syncthreads();
    if (!on) continue;
    float mean[SL], sc[E], be[E];
    vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 1.0f, sc);
    vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 0.0f, be);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const Stat st = stat[si * b.ng + group_of<T, SL>(b, col, SL > 1 ? e : 0)];
      if (e < SL) mean[e] = st.mean;
      sc[e] *= st.rstd;
    }
    T* out = a.out.p + g * a.out.gs + s * a.out.ss + b.c0 + col * E;
    PIGAN_ACT_SWITCH(a.act, {
      _Pragma("unroll") for (int v = 0; v < NV; ++v) {
        const int64_t p = pr + (int64_t)v * pl.rows;
        if (p < a.P) {
          float f[E];
          piece_floats<T>(raw[v], f);
          _Pragma("unroll") for (int e = 0; e < E; ++e) f[e] = act_value<ACT, T>((f[e] - mean[SL > 1 ? e : 0]) * sc[e] + be[e]);
          store_piece<WHOLE>(out + p * a.out.ld, valid, f);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    })
  }
}

// ---------------------------------------------------------------------------
// Samples of more points than a block's registers hold, forward: sums of ranges of
// points, then the results.
// ---------------------------------------------------------------------------
// ws: Pair [G][S][n][chan_parts * splits], and float [G][S][n] behind them: the values that
// the sums begin at (y may overwrite x while other blocks still apply)
template <class T, int SL, bool WHOLE>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_sums(const GnArgs<T> a, int64_t items, int64_t all_groups) {
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
    float* shifts = (float*)(part + all_groups * pl.chan_parts * pl.splits);
    const int64_t parts = pl.chan_parts * pl.splits, at = pl.chan_parts > 1 ? slab % pl.chan_parts * pl.splits + split : split;
    group_sums(sm, 1, pl.rows, pl.pw * SL, b.ng, b.slots, pl.lanes,
               [&](int, int j, const Pair& t) {
      const int64_t i = gs * a.n + b.j0 + j;
      part[i * parts + at] = t;
      if (at == 0) shifts[i] = shift_of(Elem<T>::to_f(first[(b.j0 + j) * cg]));
    });
    __syncthreads();
  }
}

template <class T, int SL, bool WHOLE>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_apply(const GnArgs<T> a, int64_t items, int64_t all_groups) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];   // of Stat
  Stat* stat = (Stat*)sm;
  const GnPlan& pl = a.pl;
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  const int64_t cg = a.C / a.n;
  const double inv_n = 1.0 / ((double)cg * (double)a.P);
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t split = it % pl.splits, slab = it / pl.splits % pl.slabs, gs = it / (pl.splits * pl.slabs);
    const int64_t g = gs / a.S, s = gs - g * a.S;
    const Slab b = slab_at<T, SL>(a, slab);
    const int valid = b.width - col * E;
    const T* first = a.x.p + g * a.x.gs + s * a.x.ss;
    const int64_t parts = pl.chan_parts * pl.splits;
    const Pair* part = (const Pair*)a.ws + (gs * a.n + b.j0) * parts;
    const float* shifts = (const float*)((const Pair*)a.ws + all_groups * parts) + gs * a.n + b.j0;
    const bool tells = split == 0 && (pl.chan_parts == 1 || slab % pl.chan_parts == 0);
    group_sums(part, 1, 1, 0, b.ng, (int)parts, pl.lanes, [&](int, int j, const Pair& t) {
      const Stat st = stat_of(t, shifts[j], inv_n, a.eps);
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

// the columns' coefficients of a thread
template <class T, int SL>
struct Column {
  float mean[SL], rstd[SL], ga[EPP<T>], be[EPP<T>];
  __device__ __forceinline__ void load(const GnArgs<T>& a, const Slab& b, int64_t g, int64_t s, int col) {
    constexpr int E = EPP<T>;
    vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 1.0f, ga);
    vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 0.0f, be);
    load_stats(a, b, g, s, col);
  }
  // from LDS, [2][wide], again for every piece
  __device__ __forceinline__ void load_scales(const float* gab, int wide, int col) {
    constexpr int E = EPP<T>;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const f32x4 u = *(const f32x4*)(gab + col * E + i), w = *(const f32x4*)(gab + wide + col * E + i);
#pragma unroll
      for (int q = 0; q < 4; ++q) { ga[i + q] = u[q]; be[i + q] = w[q]; }
    }
  }
  __device__ __forceinline__ void load_stats(const GnArgs<T>& a, const Slab& b, int64_t g, int64_t s, int col) {
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

// ---------------------------------------------------------------------------
// Backward, rows and samples whose slabs fit a block's registers.  Blocks walk samples; a
// thread keeps its columns' sums of da xhat and da over all of them, a block writes one
// partial row of [dgamma, dbeta] (the final ones, where one block takes all samples).
// ---------------------------------------------------------------------------
// bytes of LDS that a group's sums, or half the columns' sums, take
constexpr size_t bwd_sums_lds(int nth, int sl, int e) {
  return (size_t)nth * (sl * sizeof(Pair) > (size_t)e * 4 ? sl * sizeof(Pair) : (size_t)e * 4);
}

// a block's rows of sums, added in order; fm: float [rows][pw * E]
template <class T>
__device__ __forceinline__ void store_columns(const GnArgs<T>& a, float* fm, const float (&sg)[EPP<T>], const float (&sb)[EPP<T>],
                                              const Slab& b, int64_t g, int col, int row) {
  constexpr int E = EPP<T>;
  const GnPlan& pl = a.pl;
  const int wide = pl.pw * E;
  const bool last = pl.slots == 1;
  float* d0 = last ? (a.dgamma ? a.dgamma + g * a.C : nullptr) : (float*)a.ws + (g * pl.slots + blockIdx.x) * 2 * a.C;
  float* d1 = last ? (a.dbeta ? a.dbeta + g * a.C : nullptr) : d0 + a.C;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    __syncthreads();
    if (row < pl.rows)
#pragma unroll
      for (int e = 0; e < E; ++e) fm[row * wide + col * E + e] = half ? sb[e] : sg[e];
    __syncthreads();
    float* d = half ? d1 : d0;
    for (int c = threadIdx.x; c < b.width; c += blockDim.x) {
      double t = 0.0;
      for (int r = 0; r < pl.rows; ++r) t += fm[r * wide + c];
      if (d) d[b.c0 + c] = (float)t;
    }
  }
  __syncthreads();
}

template <class T, int NV>
__global__ void __launch_bounds__(256) k_gn_rows_bwd(const GnArgs<T> a) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  const Slab b = slab_at<T, 1>(a, blockIdx.y);
  const int64_t g = blockIdx.z;
  const int lanes = b.slots;
  const float inv_n = 1.0f / (float)(a.C / a.n);
  const bool on = row < pl.rows && col * E < b.width;   // whole groups of lanes
  float sg[E], sb[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sg[e] = sb[e] = 0.0f;
  if (on) {
    Column<T, 1> c;
    c.load(a, b, g, 0, col);
    const T* x = a.x.p + g * a.x.gs + b.c0 + col * E;
    const T* dy = a.dy.p + g * a.dy.gs + b.c0 + col * E;
    const T* add = a.add.p ? a.add.p + g * a.add.gs + b.c0 + col * E : nullptr;
    T* out = a.out.p ? a.out.p + g * a.out.gs + b.c0 + col * E : nullptr;
    const int64_t stats = g * a.S * a.n + b.j0 + col / lanes;
    const int64_t step = (int64_t)gridDim.x * pl.rows;
    PIGAN_ACT_SWITCH(a.act, {
      for (int64_t s0 = (int64_t)blockIdx.x * pl.rows + row; s0 < a.S; s0 += NV * step) {
        piece_t rx[NV];
        piece_t rd[NV];
        piece_t ra[NV];
        float mean[NV];
        float rstd[NV];
        _Pragma("unroll") for (int v = 0; v < NV; ++v) {
          const int64_t s = s0 + v * step < a.S ? s0 + v * step : s0;
          rx[v] = *(const piece_u*)(x + s * a.x.ss);
          rd[v] = *(const piece_u*)(dy + s * a.dy.ss);
          if (add) ra[v] = *(const piece_u*)(add + s * a.add.ss);
          mean[v] = a.mean[stats + s * a.n];
          rstd[v] = a.rstd[stats + s * a.n];
        }
        _Pragma("unroll") for (int v = 0; v < NV; ++v) {
          const int64_t s = s0 + v * step;
          if (s >= a.S) break;
          float xh[E];
          float da[E];
          float h0 = 0.0f;
          float h1 = 0.0f;
          piece_floats<T>(rx[v], xh);
          piece_floats<T>(rd[v], da);
          c.mean[0] = mean[v];
          c.rstd[0] = rstd[v];
          slope_piece<ACT, true>(c, E, xh, da);
          _Pragma("unroll") for (int e = 0; e < E; ++e) {
            sg[e] += da[e] * xh[e];
            sb[e] += da[e];
            da[e] *= c.ga[e];
            h0 += da[e];
            h1 += da[e] * xh[e];
          }
          if (out) {
            for (int o = 1; o < lanes; o *= 2) {
              h0 += __shfl_xor(h0, o);
              h1 += __shfl_xor(h1, o);
            }
            h0 *= inv_n;
            h1 *= inv_n;
            float r[E];
            if (add) piece_floats<T>(ra[v], r);
            _Pragma("unroll") for (int e = 0; e < E; ++e) {
              da[e] = c.rstd[0] * (da[e] - h0 - xh[e] * h1);
              if (add) da[e] += r[e];
            }
            piece_store(out + s * a.out.ss, E, da);
          }
        }
      }
    })
  }
  if (a.dgamma || a.dbeta) store_columns(a, (float*)sm, sg, sb, b, g, col, row);
}

template <class T, int NTH, int NV, int SL, bool WHOLE>
__global__ void __launch_bounds__(NTH, NV >= 4 ? 4 : 1) k_gn_one_bwd(const GnArgs<T> a) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  float* gab = (float*)((char*)sm + bwd_sums_lds(NTH, SL, E));   // gamma and beta of the slab: beside the pieces they would not fit the registers
  float2* means = (float2*)(gab + 2 * pl.pw * E);
  const int col = threadIdx.x % pl.pw, row = threadIdx.x / pl.pw;
  const int si = NV == 1 && pl.ns > 1 ? row / (int)a.P : 0, pr = row - si * (int)a.P * (NV == 1 && pl.ns > 1);
  const int64_t cg = a.C / a.n, batches = (a.S + pl.ns - 1) / pl.ns, g = blockIdx.z;
  const double inv_n = 1.0 / ((double)cg * (double)a.P);
  for (int64_t slab = blockIdx.y; slab < pl.slabs; slab += gridDim.y) {
    const Slab b = slab_at<T, SL>(a, slab);
    const int valid = b.width - col * E;
    float sg[E], sb[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sg[e] = sb[e] = 0.0f;
    __syncthreads();   // the slab before may still be read
    for (int i = threadIdx.x; i < pl.pw * E; i += NTH) {
      gab[i] = a.gamma && i < b.width ? a.gamma[g * a.C + b.c0 + i] : 1.0f;
      gab[pl.pw * E + i] = a.beta && i < b.width ? a.beta[g * a.C + b.c0 + i] : 0.0f;
    }
    __syncthreads();
    for (int64_t bt = blockIdx.x; bt < batches; bt += gridDim.x) {
      const int64_t s = bt * pl.ns + si;
      const bool on = row < pl.rows && pr < a.P && s < a.S && valid > 0;
      const T* x = a.x.p + g * a.x.gs + s * a.x.ss + b.c0 + col * E;
      const T* dy = a.dy.p + g * a.dy.gs + s * a.dy.ss + b.c0 + col * E;
      piece_t rx[NV], rd[NV];
      Column<T, SL> c;
      float h0[SL], h1[SL];
#pragma unroll
      for (int e = 0; e < SL; ++e) h0[e] = h1[e] = 0.0f;
      if (on) {
        load_rows<WHOLE>(rx, x, a.x.ld, pr, pl.rows, a.P, valid);
        load_rows<WHOLE>(rd, dy, a.dy.ld, pr, pl.rows, a.P, valid);
        c.load_stats(a, b, g, s, col);
        PIGAN_ACT_SWITCH(a.act, {
          _Pragma("unroll") for (int v = 0; v < NV; ++v) {
            if (v > 0 && pr + (int64_t)v * pl.rows >= a.P) break;
            float xh[E];
            float da[E];
            piece_floats<T>(rx[v], xh);
            piece_floats<T>(rd[v], da);
            c.load_scales(gab, pl.pw * E, col);
            slope_piece<ACT, WHOLE>(c, valid, xh, da);
            _Pragma("unroll") for (int e = 0; e < E; ++e) {
              const int k = SL > 1 ? e : 0;
              const float t = da[e] * xh[e];
              sg[e] += t;
              sb[e] += da[e];
              h0[k] += da[e] * c.ga[e];
              h1[k] += t * c.ga[e];
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        })
      }
      if (!a.out.p) continue;   // the same for every thread
      if (row < pl.rows)
#pragma unroll
        for (int e = 0; e < SL; ++e) sm[row * pl.pw * SL + col * SL + e] = {h0[e], h1[e]};
      __syncthreads();
      group_sums(sm, pl.ns, pl.ns > 1 ? (int)a.P : pl.rows, pl.pw * SL, b.ng, b.slots, pl.lanes, [&](int i, int j, const Pair& t) {
        means[i * b.ng + j] = {(float)(t.s * inv_n), (float)(t.q * inv_n)};
      });
      __syncthreads();
      if (!on) continue;
      float2 m[SL];
#pragma unroll
      for (int e = 0; e < SL; ++e) m[e] = means[si * b.ng + group_of<T, SL>(b, col, e)];
      const T* add = a.add.p ? a.add.p + g * a.add.gs + s * a.add.ss + b.c0 + col * E : nullptr;
      T* out = a.out.p + g * a.out.gs + s * a.out.ss + b.c0 + col * E;
      PIGAN_ACT_SWITCH(a.act, {
        _Pragma("unroll") for (int v = 0; v < NV; ++v) {
          const int64_t p = pr + (int64_t)v * pl.rows;
          if (p < a.P) {
            float xh[E];
            float da[E];
            float r[E];
            if (add) piece_floats<T>(load_piece<WHOLE>(add + p * a.add.ld, valid), r);
            piece_floats<T>(rx[v], xh);
            piece_floats<T>(rd[v], da);
            c.load_scales(gab, pl.pw * E, col);
            slope_piece<ACT, WHOLE>(c, valid, xh, da);
            _Pragma("unroll") for (int e = 0; e < E; ++e) {
              const int k = SL > 1 ? e : 0;
              da[e] = c.rstd[k] * (da[e] * c.ga[e] - m[k].x - xh[e] * m[k].y);
              if (add) da[e] += r[e];
            }
            store_piece<WHOLE>(out + p * a.out.ld, valid, da);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      })
    }
    if (a.dgamma || a.dbeta) store_columns(a, (float*)sm, sg, sb, b, g, col, row);
  }
}

// ---------------------------------------------------------------------------
// Longer samples, backward: a channel's sums of da and da xhat over ranges of points give
// dgamma and dbeta (summed over samples) and, with gamma, a group's sums of h and
// h xhat; then dx.
// ---------------------------------------------------------------------------
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
template <class T> bool aligned(const GnArgs<T>& a) { return a.C / a.n % EPP<T> == 0; }

// f(SL, WHOLE) of a call's widths
template <class T, class F> void by_width(const GnArgs<T>& a, F&& f) {
  constexpr int E = EPP<T>;
  const bool one = a.pl.ng == 1 || aligned(a);
  const bool whole = aligned(a) || (a.pl.ng > 1 && a.pl.W % E == 0 && a.C % E == 0);
  if (one && whole) f(std::integral_constant<int, 1>{}, std::true_type{});
  else if (one) f(std::integral_constant<int, 1>{}, std::false_type{});
  else if (whole) f(std::integral_constant<int, E>{}, std::true_type{});
  else f(std::integral_constant<int, E>{}, std::false_type{});
}

unsigned grid_of(int64_t items) { return (unsigned)std::min<int64_t>(items, 1 << 20); }

// Threads and pieces of a thread of the one-pass kernels, by what they hold.
struct Shape { int nth, nv; };
constexpr Shape FWD_ONE[] = {{256, 1}, {256, 4}, {1024, 2}, {256, 16}, {512, 16}, {1024, 16}};
constexpr Shape FWD_MIXED[] = {{256, 1}, {256, 4}, {256, 8}};   // SL > 1
constexpr Shape BWD_ONE[] = {{256, 1}};
constexpr Shape BWD_MIXED[] = {{256, 1}};

// f(NTH, NV) of a plan; the lists' shapes
template <bool BACKWARD, int SL, class F> void by_shape(const GnPlan& pl, F&& f) {
  constexpr const auto& list = [] () -> const auto& {
    if constexpr (BACKWARD && SL == 1) return BWD_ONE;
    else if constexpr (BACKWARD) return BWD_MIXED;
    else if constexpr (SL == 1) return FWD_ONE;
    else return FWD_MIXED;
  }();
  constexpr int N = (int)(sizeof(list) / sizeof(Shape));
  [&]<int... I>(std::integer_sequence<int, I...>) {
    (void)((pl.nth == list[I].nth && pl.nv == list[I].nv &&
            (f(std::integral_constant<int, list[I].nth>{}, std::integral_constant<int, list[I].nv>{}), true)) || ...);
  }(std::make_integer_sequence<int, N>{});
}

}  // namespace

GnPlan gn_plan(bool backward, int elem_bytes, int64_t G, int64_t S, int64_t P, int64_t C, int64_t n) {
  GnPlan pl{};
  S = std::max<int64_t>(S, 1);
  const int64_t E = 16 / elem_bytes, cg = C / n;
  const bool whole_pieces = cg % E == 0;
  auto slab = [&](int64_t ng) {
    pl.ng = ng;
    pl.W = ng * cg;
    pl.chan_parts = 1;
    pl.slabs = cdiv(n, ng);
    pl.pw = (int32_t)std::min<int64_t>(cdiv(pl.W, E), 1 << 30);
  };
  auto finish = [&](int nth, int nv) {
    pl.nth = nth;
    pl.nv = nv;
    pl.rows = nth / pl.pw;
    pl.ns = 1;
    pl.lanes = 64;
  };
  auto fit_lanes = [&](int64_t entries) {
    // as many lanes as entries, and no more groups in turns than need be
    while (pl.lanes > 1 && (pl.lanes / 2 >= entries || pl.lanes * pl.ng * pl.ns > pl.nth)) pl.lanes /= 2;
  };
  const int64_t lanes = cg / E;
  if (P == 1 && whole_pieces && lanes <= 64 && (lanes & (lanes - 1)) == 0 && cdiv(n, 256 / lanes) <= 65535) {
    slab(std::min<int64_t>(n, 256 / lanes));
    finish(256, 4);
    pl.mode = GN_ROWS;
    const int64_t blocks = cdiv(S, pl.rows), most = std::max<int64_t>(1, 2048 / std::min<int64_t>(2048, G * pl.slabs));
    pl.slots = std::min(blocks, most);
    return pl;
  }
  // one pass: slabs of 128 bytes of a point, 64 where those do not fit
  for (int64_t bytes : {128, 64}) {
    slab(std::min<int64_t>(n, std::max<int64_t>(1, cdiv(bytes, cg * elem_bytes))));
    const bool mixed = !whole_pieces && pl.ng > 1;
    const Shape* list = backward ? (mixed ? BWD_MIXED : BWD_ONE) : mixed ? FWD_MIXED : FWD_ONE;
    const int count = backward ? 1 : mixed ? 3 : 6;
    for (int i = 0; i < count; ++i) {
      const Shape f = list[i];
      // backward: gamma and beta in LDS
      if (f.nth < pl.pw || (int64_t)(f.nth / pl.pw) * f.nv < P || (backward && pl.pw * E > 2048)) continue;
      const int64_t items = G * S * pl.slabs;
      if (items < 256 && (int64_t)f.nth * f.nv > 4096) break;   // few blocks with much to do: ranges of points
      finish(f.nth, f.nv);
      if (f.nv == 1 && P <= 256) {
        // short samples: wider slabs, then several samples of a block
        int64_t ng = pl.ng;
        while (ng < n && cdiv(std::min(n, 2 * ng) * cg, E) * P <= f.nth && (whole_pieces || mixed)) ng = std::min(n, 2 * ng);
        slab(ng);
        finish(f.nth, 1);
        pl.ns = (int32_t)std::max<int64_t>(1, std::min<int64_t>(pl.rows / P, S));
        if (pl.ns > 1) pl.rows = (int32_t)(pl.ns * P);
      }
      fit_lanes((pl.ns > 1 ? P : pl.rows) * (mixed ? cg : std::max<int64_t>(1, pl.pw / pl.ng)));
      pl.mode = GN_ONE;
      const int64_t batches = cdiv(S, pl.ns), most = std::max<int64_t>(1, 2048 * 256 / f.nth / std::min<int64_t>(2048 * 256 / f.nth, G * pl.slabs));
      pl.slots = std::min(batches, most);
      return pl;
    }
  }
  // ranges of points: 512 bytes of a point, for long runs
  const int64_t most = SPLIT_NTH * E;
  pl.mode = GN_SPLIT;
  if (cg > most) {
    pl.W = most;
    pl.ng = 1;
    pl.chan_parts = cdiv(cg, most);
    pl.slabs = n * pl.chan_parts;
    pl.pw = SPLIT_NTH;
  } else {
    slab(std::min<int64_t>(n, std::max<int64_t>(1, 32 * E / cg)));
  }
  finish(SPLIT_NTH, 1);
  while (pl.lanes > 1 && pl.lanes * pl.ng > SPLIT_NTH) pl.lanes /= 2;
  const int64_t base = G * S * pl.slabs, least = cdiv(P, 4 * pl.rows);
  pl.splits = std::max<int64_t>(1, std::min<int64_t>({cdiv(2048, base), least, 64}));
  pl.split_rows = cdiv(cdiv(P, pl.splits), pl.rows) * pl.rows;
  pl.splits = cdiv(P, pl.split_rows);
  pl.slots = S * pl.splits;
  return pl;
}

size_t gn_forward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t n) {
  return pl.mode == GN_SPLIT ? (size_t)(G * S * n) * ((size_t)(pl.chan_parts * pl.splits) * sizeof(Pair) + 4) : 0;
}
static size_t sums_bytes(const GnPlan& pl, int64_t G, int64_t C) {
  return ((size_t)(G * pl.slots * 2 * C) * 4 + 15) / 16 * 16;
}
size_t gn_backward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t C, int64_t n, bool cols) {
  if (pl.mode != GN_SPLIT) return cols && pl.slots > 1 ? sums_bytes(pl, G, C) : 0;
  return sums_bytes(pl, G, C) + (size_t)(G * S * n) * sizeof(float2);
}

template <class T> hipError_t launch_gn_fwd(const GnArgs<T>& a, int G, hipStream_t st) {
  if (a.S <= 0) return hipSuccess;
  const GnPlan& pl = a.pl;
  if (pl.mode == GN_ROWS) {
    const int64_t turns = cdiv(a.S, (int64_t)pl.rows * 4), most = std::max<int64_t>(1, 4096 / std::min<int64_t>(4096, G * pl.slabs));
    k_gn_rows<T, 4><<<dim3((unsigned)std::min(turns, most), (unsigned)pl.slabs, G), 256, 0, st>>>(a);
  } else if (pl.mode == GN_ONE) {
    const int64_t items = (int64_t)G * cdiv(a.S, pl.ns) * pl.slabs;
    by_width(a, [&](auto sl, auto whole) {
      by_shape<false, sl.value>(pl, [&](auto nth, auto nv) {
        const size_t lds = nth.value * sl.value * sizeof(Pair) + (size_t)pl.ns * pl.ng * (sizeof(Stat) + 4);
        k_gn_one<T, nth.value, nv.value, sl.value, whole.value><<<grid_of(items), nth.value, lds, st>>>(a, items);
      });
    });
  } else {
    const int64_t groups = (int64_t)G * a.S * a.n, items = (int64_t)G * a.S * pl.slabs * pl.splits;
    by_width(a, [&](auto sl, auto whole) {
      k_gn_sums<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, SPLIT_NTH * sl.value * sizeof(Pair), st>>>(a, items, groups);
      k_gn_apply<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, (size_t)pl.ng * sizeof(Stat), st>>>(a, items, groups);
    });
  }
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
  const GnPlan& pl = a.pl;
  if (pl.mode == GN_ROWS) {
    k_gn_rows_bwd<T, 2><<<dim3((unsigned)pl.slots, (unsigned)pl.slabs, G), 256, bwd_sums_lds(256, 1, EPP<T>), st>>>(a);
  } else if (pl.mode == GN_ONE) {
    const dim3 grid((unsigned)pl.slots, (unsigned)std::min<int64_t>(pl.slabs, 65535), G);
    by_width(a, [&](auto sl, auto whole) {
      by_shape<true, sl.value>(pl, [&](auto nth, auto nv) {
        const size_t lds = bwd_sums_lds(nth.value, sl.value, EPP<T>) + (size_t)pl.ns * pl.ng * sizeof(float2) +
                           (size_t)pl.pw * EPP<T> * 8;
        k_gn_one_bwd<T, nth.value, nv.value, sl.value, whole.value><<<grid, nth.value, lds, st>>>(a);
      });
    });
  } else {
    const int64_t items = (int64_t)G * a.S * pl.slabs * pl.splits, total = (int64_t)G * a.S * a.n;
    float2* means = (float2*)(a.ws + sums_bytes(pl, G, a.C));
    by_width(a, [&](auto sl, auto whole) {
      k_gn_bwd_sums<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, SPLIT_NTH * EPP<T> * 8, st>>>(a, items);
      // dx may overwrite dy
      if (a.out.p) {
        k_gn_bwd_join<T><<<grid_of(cdiv(total, 4)), 256, 0, st>>>(a, means, total);
        k_gn_bwd_apply<T, sl.value, whole.value><<<grid_of(items), SPLIT_NTH, 0, st>>>(a, means, items);
      }
    });
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !cols || (pl.mode != GN_SPLIT && pl.slots == 1)) return e;
  return launch_slot_sum((const float*)a.ws, pl.slots * 2 * a.C, (int)pl.slots, 2 * a.C, a.dgamma, a.C, a.dbeta, G, st);
}

#define PIGAN_GN_INST(T)                                              \
  template hipError_t launch_gn_fwd<T>(const GnArgs<T>&, int, hipStream_t); \
  template hipError_t launch_gn_bwd<T>(const GnArgs<T>&, int, hipStream_t);
PIGAN_GN_INST(float)
PIGAN_GN_INST(bf16)
PIGAN_GN_INST(f16)

}  // namespace pigan
