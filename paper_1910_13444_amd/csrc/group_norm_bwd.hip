// Group norm with an activation, channels last, backward, for gfx950.
#include "group_norm_parts.h"
#include "norm.h"

namespace pigan {
namespace {

// the columns' coefficients of a thread
template <class T, int SL>
struct Column {
  float mean[SL], rstd[SL], ga[EPP<T>], be[EPP<T>];
  __device__ __forceinline__ void load(const GnArgs<T>& a, const Slab& b, const Div& by_span, int64_t g, int64_t s, int col) {
    load_scales(a, b, g, col);
    load_stats(a, b, by_span, g, s, col);
  }
  __device__ __forceinline__ void load_scales(const GnArgs<T>& a, const Slab& b, int64_t g, int col) {
    constexpr int E = EPP<T>;
    vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 1.0f, ga);
    vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 0.0f, be);
  }
  __device__ __forceinline__ void load_stats(const GnArgs<T>& a, const Slab& b, const Div& by_span, int64_t g, int64_t s, int col) {
#pragma unroll
    for (int e = 0; e < SL; ++e) {
      const int64_t at = (g * a.S + s) * a.n + b.j0 + group_of<T, SL>(b, by_span, col, e);
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
    if constexpr (ACT != PIGAN_ACT_NONE) da[e] *= slope_of<ACT, T>(xh[e] * c.ga[e] + c.be[e]);
    if (!WHOLE && e >= valid) xh[e] = da[e] = 0.0f;
  }
}

// ---------------------------------------------------------------------------
// Backward, rows and short samples.  Blocks walk samples; a thread keeps its columns' sums
// of da xhat and da over all of them, a block writes one partial row of [dgamma, dbeta] (the
// final ones, where one block takes all samples).  Rows as forward: 47,020 x 176 bf16, 22
// groups, tanh, 16 us and 5 for the sum of the blocks' rows.
// ---------------------------------------------------------------------------
// bytes of LDS that a group's sums, or half the columns' sums, take
constexpr size_t bwd_sums_lds(int nth, int sl, int e) {
  return (size_t)nth * ((sl + 1) * sizeof(PairF) > (size_t)e * 4 ? (sl + 1) * sizeof(PairF) : (size_t)e * 4);
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
#pragma unroll 8
      for (int r = 0; r < pl.rows; ++r) t += fm[r * wide + c];
      if (d) d[b.c0 + c] = (float)t;
    }
  }
  __syncthreads();
}

template <class T, int NV, int ACT>
__global__ void __launch_bounds__(256) k_gn_rows_bwd(const GnArgs<T> a) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw;
  const Slab b = slab_at(a, blockIdx.y);
  const int64_t g = blockIdx.z;
  const int lanes = pl.span;
  const Div by_span(lanes);
  const float inv_n = (float)pl.inv_n;
  const bool on = row < pl.rows && col * E < b.width;   // whole groups of lanes
  float sg[E], sb[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sg[e] = sb[e] = 0.0f;
  if (on) {
    Column<T, 1> c;
    c.load(a, b, by_span, g, 0, col);
    const T* x = a.x.p + g * a.x.gs + b.c0 + col * E;
    const T* dy = a.dy.p + g * a.dy.gs + b.c0 + col * E;
    const T* add = a.add.p ? a.add.p + g * a.add.gs + b.c0 + col * E : nullptr;
    T* out = a.out.p ? a.out.p + g * a.out.gs + b.c0 + col * E : nullptr;
    const int64_t stats = g * a.S * a.n + b.j0 + by_span(col);
    const int64_t step = (int64_t)gridDim.x * pl.rows;
    for (int64_t s0 = (int64_t)blockIdx.x * pl.rows + row; s0 < a.S; s0 += NV * step) {
      piece_t rx[NV];
      piece_t rd[NV];
      piece_t ra[NV];
      float mean[NV];
      float rstd[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int64_t s = s0 + v * step < a.S ? s0 + v * step : s0;
        rx[v] = load_piece<true>(x + s * a.x.ss, E, pl.stream);
        rd[v] = load_piece<true>(dy + s * a.dy.ss, E, pl.stream);
        if (add) ra[v] = load_piece<true>(add + s * a.add.ss, E, pl.stream);
        mean[v] = a.mean[stats + s * a.n];
        rstd[v] = a.rstd[stats + s * a.n];
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
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
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sg[e] += da[e] * xh[e];
          sb[e] += da[e];
          da[e] *= c.ga[e];
          h0 += da[e];
          h1 += da[e] * xh[e];
        }
        if (out) {
          // fp32: 512 values at most, and fp64 shuffles cost 65,536 x 2048 fp16, eight groups, 5 us of 152
          for (int o = 1; o < lanes; o *= 2) {
            h0 += __shfl_xor(h0, o);
            h1 += __shfl_xor(h1, o);
          }
          h0 *= inv_n;
          h1 *= inv_n;
          float r[E];
          if (add) piece_floats<T>(ra[v], r);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            da[e] = c.rstd[0] * (da[e] - h0 - xh[e] * h1);
            if (add) da[e] += r[e];
          }
          store_piece<true>(out + s * a.out.ss, E, da, pl.stream);
        }
      }
    }
  }
  if (a.dgamma || a.dbeta) store_columns(a, (float*)sm, sg, sb, b, g, col, row);
}

// Short samples: a thread has one point's piece of a batch of samples, and the next batch's on
// its way; xhat and da stay in registers from the sums to dx.  Bound by the two barriers of a
// batch at four blocks to a CU (two where pieces are of several groups): 30,078 x 9 x 144 fp16,
// two groups, gelu, 112 us (2.1 TB/s).  With more pieces a thread the compiler spills (128 x
// 1024 x 256 bf16: 217 us where two passes take 76).
template <class T, int NTH, int SL, bool WHOLE, int ACT>
__global__ void __launch_bounds__(NTH) k_gn_one_bwd(const GnArgs<T> a) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  PairF* hs = (PairF*)sm;
  float2* means = (float2*)((char*)sm + bwd_sums_lds(NTH, SL, E));
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw, per = row_of(pl.pw * SL);
  const int si = pl.ns > 1 ? Div((int)a.P)(row) : 0, p = row - si * (int)a.P;
  const Div by_span(pl.span);
  const int64_t batches = (a.S + pl.ns - 1) / pl.ns, g = blockIdx.z;
  for (uint32_t slab = blockIdx.y; slab < pl.slabs; slab += gridDim.y) {
    const Slab b = slab_at(a, slab);
    const int valid = b.width - col * E;
    const bool here = row < pl.rows && p < a.P && valid > 0;
    const int64_t at = b.c0 + col * E;
    const T* x = a.x.p + g * a.x.gs + p * a.x.ld + at;
    const T* dy = a.dy.p + g * a.dy.gs + p * a.dy.ld + at;
    float sg[E], sb[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sg[e] = sb[e] = 0.0f;
    Column<T, SL> c;
    c.load_scales(a, b, g, col);
    piece_t rx, rd;
    auto load = [&](int64_t s) {
      if (here && s < a.S) {
        rx = load_piece<WHOLE>(x + s * a.x.ss, valid, pl.stream);
        rd = load_piece<WHOLE>(dy + s * a.dy.ss, valid, pl.stream);
      }
    };
    load(blockIdx.x * (int64_t)pl.ns + si);
    for (int64_t bt = blockIdx.x; bt < batches; bt += gridDim.x) {
      const int64_t s = bt * pl.ns + si;
      const bool on = here && s < a.S;
      float xh[E], da[E], h0[SL], h1[SL];
#pragma unroll
      for (int e = 0; e < SL; ++e) h0[e] = h1[e] = 0.0f;
      if (on) {
        c.load_stats(a, b, by_span, g, s, col);
        piece_floats<T>(rx, xh);
        piece_floats<T>(rd, da);
        slope_piece<ACT, WHOLE>(c, valid, xh, da);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int k = SL > 1 ? e : 0;
          const float t = da[e] * xh[e];
          sg[e] += t;
          sb[e] += da[e];
          h0[k] += da[e] * c.ga[e];
          h1[k] += t * c.ga[e];
        }
      }
      load(s + (int64_t)gridDim.x * pl.ns);
      if (!a.out.p) continue;   // the same for every thread
      if (row < pl.rows)
#pragma unroll
        for (int e = 0; e < SL; ++e) hs[row * per + col * SL + e] = {h0[e], h1[e]};
      __syncthreads();
      group_sums(hs, pl.ns, pl.ns > 1 ? (int)a.P : pl.rows, per, b.ng, pl.span, pl.lanes, [&](int i, int j, const Pair& t) {
        means[i * b.ng + j] = {(float)(t.s * pl.inv_n), (float)(t.q * pl.inv_n)};
      });
      __syncthreads();
      if (!on) continue;
      float r[E];
      if (a.add.p) piece_floats<T>(load_piece<WHOLE>(a.add.p + g * a.add.gs + s * a.add.ss + p * a.add.ld + at, valid, pl.stream), r);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 m = means[si * b.ng + group_of<T, SL>(b, by_span, col, SL > 1 ? e : 0)];
        da[e] = c.rstd[SL > 1 ? e : 0] * (da[e] * c.ga[e] - m.x - xh[e] * m.y);
        if (a.add.p) da[e] += r[e];
      }
      store_piece<WHOLE>(a.out.p + g * a.out.gs + s * a.out.ss + p * a.out.ld + at, valid, da, pl.stream);
    }
    __syncthreads();   // the sums' place is the columns', and the next slab's
    if (a.dgamma || a.dbeta) store_columns(a, (float*)sm, sg, sb, b, g, col, row);
  }
}

// ---------------------------------------------------------------------------
// Longer samples, backward: a channel's sums of da and da xhat over ranges of points give
// dgamma and dbeta (summed over samples) and, with gamma, a group's sums of h and
// h xhat; then dx, whose blocks join the ranges' sums themselves (a launch between cost 5 us)
// while others sum the columns (9 us).  128 x 1024 x 256 bf16, silu, with `add`: sums 32 us
// (4.2 TB/s), dx 45 us (5.9 TB/s); 4 x 21 x 1000 x 120 fp32, groups of five, tanh in fp64:
// 20 + 25 us, vector units 75 % busy.
// ---------------------------------------------------------------------------
// ws: Pair [G][S][n][chan_parts * splits], a group's sums of h and h xhat, and behind them
// float [G][slots][2][C], a block's sums of da xhat and da over all of its ranges.
// Blocks: [G][slabs][slots].
template <class T, int SL, bool WHOLE, int ACT>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_bwd_sums(const GnArgs<T> a, float* __restrict__ cols, uint32_t ranges) {
  constexpr int E = EPP<T>, U = BWD_TURN;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw, wide = pl.pw * E, parts = pl.chan_parts * pl.splits;
  const Div by_span(pl.span);
  double* all = (double*)sm;               // [2][wide]: of the block
  double* sums = all + 2 * wide;           // [2][wide]: of the range
  float* fm = (float*)(sums + 2 * wide);   // [rows][2][wide]
  const int64_t g = blockIdx.z;
  for (uint32_t slab = blockIdx.y; slab < pl.slabs; slab += gridDim.y) {
    const Slab b = slab_at(a, slab);
    const int valid = b.width - col * E;
    for (int i = threadIdx.x; i < 2 * wide; i += SPLIT_NTH) all[i] = 0.0;
    for (uint32_t it = blockIdx.x; it < ranges; it += gridDim.x) {
      const uint32_t s = it / (uint32_t)pl.splits, split = it - s * (uint32_t)pl.splits;
      float sg[E], sb[E];
#pragma unroll
      for (int e = 0; e < E; ++e) sg[e] = sb[e] = 0.0f;
      if (valid > 0 && row < pl.rows) {
        const Turns tn(pl, a.P, U, split, pl.splits, row);
        const int64_t xs = pl.rows * a.x.ld, ds = pl.rows * a.dy.ld;
        const T* x = a.x.p + g * a.x.gs + s * a.x.ss + b.c0 + col * E + tn.first * a.x.ld;
        const T* dy = a.dy.p + g * a.dy.gs + s * a.dy.ss + b.c0 + col * E + tn.first * a.dy.ld;
        Column<T, SL> c;
        c.load(a, b, by_span, g, s, col);
        for (int left = tn.left; left > 0; left -= tn.by) {
          piece_t rx[U], rd[U];
          load_rows<WHOLE>(rx, x, xs, left, pl.rows, valid);
          load_rows<WHOLE>(rd, dy, ds, left, pl.rows, valid);
          x += tn.by * a.x.ld;
          dy += tn.by * a.dy.ld;
#pragma unroll
          for (int v = 0; v < U; ++v) {
            if (v == 0 || v * pl.rows < left) {
              float xh[E], da[E];
              piece_floats<T>(rx[v], xh);
              piece_floats<T>(rd[v], da);
              slope_piece<ACT, WHOLE>(c, valid, xh, da);
#pragma unroll
              for (int e = 0; e < E; ++e) {
                sg[e] += da[e] * xh[e];
                sb[e] += da[e];
              }
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      if (row < pl.rows)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          fm[row * 2 * wide + col * E + e] = sg[e];
          fm[row * 2 * wide + wide + col * E + e] = sb[e];
        }
      __syncthreads();
      for (int i = threadIdx.x; i < 2 * wide; i += SPLIT_NTH) {
        double t = 0.0;
#pragma unroll 8
        for (int r = 0; r < pl.rows; ++r) t += fm[r * 2 * wide + i];
        sums[i] = t;
        all[i] += t;   // always by this thread
      }
      __syncthreads();
      if (a.out.p) {
        // gamma times a channel's sums, over a group's channels
        const int per = b.width / b.ng;
        const int at = pl.chan_parts > 1 ? slab % (uint32_t)pl.chan_parts * pl.splits + split : split;
        Pair* part = (Pair*)a.ws + ((g * a.S + s) * a.n + b.j0) * parts + at;
        lane_sums(b.ng, pl.lanes, [&](int j, int l) {
          Pair t = {0.0, 0.0};
          for (int i = j * per + l; i < (j + 1) * per; i += pl.lanes) {
            const double ga = a.gamma ? a.gamma[g * a.C + b.c0 + i] : 1.0f;
            t.s += ga * sums[wide + i];
            t.q += ga * sums[i];
          }
          return t;
        }, [&](int j, const Pair& t) { part[(int64_t)j * parts] = t; });
      }
    }
    if (cols) {
      float* d = cols + (g * pl.slots + blockIdx.x) * 2 * a.C + b.c0;
      for (int i = threadIdx.x; i < 2 * wide; i += SPLIT_NTH) {
        const int c = i < wide ? i : i - wide;
        if (c < b.width) d[(i < wide ? 0 : a.C) + c] = (float)all[i];
      }
    }
    __syncthreads();
  }
}

// dgamma and dbeta of a slab: 16 columns of a block, 16 threads to a column, added in order
constexpr int COLS = 16;
inline unsigned col_blocks_of(const GnPlan& pl) { return 2 * (unsigned)((pl.W + COLS - 1) / COLS); }
template <class T>
__device__ __forceinline__ void sum_columns(const GnArgs<T>& a, const Slab& b, const float* __restrict__ cols, double* sm) {
  const int cl = threadIdx.x % COLS, r = threadIdx.x / COLS;
  const unsigned half = (unsigned)((a.pl.W + COLS - 1) / COLS), second = blockIdx.x >= half;
  const int c = (int)(blockIdx.x - second * half) * COLS + cl;
  const int64_t g = blockIdx.z, ld = 2 * a.C, at = b.c0 + c;
  double t = 0.0;
  if (c < b.width) {
    const float* q = cols + g * a.pl.slots * ld + second * a.C + at;
#pragma unroll 8
    for (int k = r; k < a.pl.slots; k += SPLIT_NTH / COLS) t += (double)q[k * ld];
  }
  sm[r * COLS + cl] = t;
  __syncthreads();
  if (r == 0 && c < b.width) {
    for (int k = 1; k < SPLIT_NTH / COLS; ++k) t += sm[k * COLS + cl];
    float* d = second ? a.dbeta : a.dgamma;
    if (d) d[g * a.C + at] = (float)t;
  }
  __syncthreads();
}

// dx, and in the first `col_blocks` blocks of a slab, which are done before the others, the
// sums of `cols`.  Blocks: [G][slabs][col_blocks + S * splits].
template <class T, int SL, bool WHOLE, int ACT>
__global__ void __launch_bounds__(SPLIT_NTH, SL == 1 ? 3 : 2) k_gn_bwd_apply(const GnArgs<T> a, uint32_t ranges, const float* __restrict__ cols,
                                                            unsigned col_blocks) {
  constexpr int E = EPP<T>, U = BWD_TURN;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  if (blockIdx.x < col_blocks) {
    for (uint32_t slab = blockIdx.y; slab < pl.slabs; slab += gridDim.y) sum_columns(a, slab_at(a, slab), cols, (double*)sm);
    return;
  }
  float2* means = (float2*)sm;
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw, parts = pl.chan_parts * pl.splits;
  const Div by_span(pl.span);
  const int64_t g = blockIdx.z;
  for (uint32_t slab = blockIdx.y; slab < pl.slabs; slab += gridDim.y) {
    const Slab b = slab_at(a, slab);
    const int valid = b.width - col * E;
    for (uint32_t at = blockIdx.x - col_blocks; at < ranges; at += gridDim.x - col_blocks) {
      const uint32_t it = from_last(at, ranges), s = it / (uint32_t)pl.splits, split = it - s * (uint32_t)pl.splits;
      const Turns tn(pl, a.P, U, split, pl.splits, row);
      const int64_t p0 = tn.first + tn.last(), xs = pl.rows * a.x.ld, ds = pl.rows * a.dy.ld, as = pl.rows * a.add.ld;
      int left = valid > 0 && row < pl.rows ? tn.left - tn.last() : 0;
      const T* x = a.x.p + g * a.x.gs + s * a.x.ss + b.c0 + col * E + p0 * a.x.ld;
      const T* dy = a.dy.p + g * a.dy.gs + s * a.dy.ss + b.c0 + col * E + p0 * a.dy.ld;
      const T* add = a.add.p ? a.add.p + g * a.add.gs + s * a.add.ss + b.c0 + col * E + p0 * a.add.ld : nullptr;
      piece_t rx[U], rd[U], ra[U];
      auto load = [&](int n) {
        load_rows<WHOLE>(rx, x, xs, n, pl.rows, valid);
        load_rows<WHOLE>(rd, dy, ds, n, pl.rows, valid);
        if (add) load_rows<WHOLE>(ra, add, as, n, pl.rows, valid);
      };
      if (left > 0) load(left);
      range_sums((const Pair*)a.ws + ((g * a.S + s) * a.n + b.j0) * parts, b.ng, parts, pl.lanes,
                 [&](int j, const Pair& t) { means[j] = {(float)(t.s * pl.inv_n), (float)(t.q * pl.inv_n)}; });
      __syncthreads();
      if (left > 0) {
        Column<T, SL> c;
        c.load(a, b, by_span, g, s, col);
        float2 m[SL];
#pragma unroll
        for (int e = 0; e < SL; ++e) m[e] = means[group_of<T, SL>(b, by_span, col, e)];
        T* out = a.out.p + g * a.out.gs + s * a.out.ss + b.c0 + col * E + p0 * a.out.ld;
        const int64_t os = pl.rows * a.out.ld;
        for (;;) {
#pragma unroll
          for (int v = 0; v < U; ++v) {
            if (v == 0 || v * pl.rows < left) {
              float xh[E], da[E], r[E];
              piece_floats<T>(rx[v], xh);
              piece_floats<T>(rd[v], da);
              if (add) piece_floats<T>(ra[v], r);
              slope_piece<ACT, WHOLE>(c, valid, xh, da);
#pragma unroll
              for (int e = 0; e < E; ++e) {
                const int k = SL > 1 ? e : 0;
                da[e] = c.rstd[k] * (da[e] * c.ga[e] - m[k].x - xh[e] * m[k].y);
                if (add) da[e] += r[e];
              }
              store_piece<WHOLE>(out + v * os, valid, da, pl.stream);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          if (!tn.before(left)) break;
          left += tn.by;
          x -= tn.by * a.x.ld;
          dy -= tn.by * a.dy.ld;
          if (add) add -= tn.by * a.add.ld;
          out -= tn.by * a.out.ld;
          load(left);
        }
      }
      __syncthreads();
    }
  }
}

template <class T> __global__ void __launch_bounds__(SPLIT_NTH) k_gn_cols(const GnArgs<T> a, const float* __restrict__ cols) {
  __shared__ double sm[SPLIT_NTH];
  for (uint32_t slab = blockIdx.y; slab < a.pl.slabs; slab += gridDim.y) sum_columns(a, slab_at(a, slab), cols, sm);
}

}  // namespace

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
  by_act(a.act, [&](auto act) {
    constexpr int ACT = act.value;
    if (pl.mode == GN_ROWS) {
      k_gn_rows_bwd<T, 2, ACT><<<dim3((unsigned)pl.slots, (unsigned)pl.slabs, G), 256, bwd_sums_lds(256, 1, EPP<T>), st>>>(a);
    } else if (pl.mode == GN_ONE) {
      const dim3 grid((unsigned)pl.slots, (unsigned)std::min<int64_t>(pl.slabs, 65535), G);
      by_width(a, [&](auto sl, auto whole) {
        auto launch = [&](auto nth) {
          const size_t lds = bwd_sums_lds(nth.value, sl.value, EPP<T>) + (size_t)pl.ns * pl.ng * sizeof(float2);
          k_gn_one_bwd<T, nth.value, sl.value, whole.value, ACT><<<grid, nth.value, lds, st>>>(a);
        };
        if (pl.nth == 512) launch(std::integral_constant<int, 512>{});
        else launch(std::integral_constant<int, 256>{});
      });
    } else {
      const int64_t ranges = a.S * pl.splits;
      float* sums = cols ? (float*)(a.ws + gn_pairs_bytes(pl, G, a.S, a.n)) : nullptr;
      const unsigned slabs = (unsigned)std::min<int64_t>(pl.slabs, 65535), col_blocks = cols ? col_blocks_of(pl) : 0;
      by_width(a, [&](auto sl, auto whole) {
        const size_t lds = (size_t)pl.pw * EPP<T> * 32 + SPLIT_NTH * EPP<T> * 8;
        k_gn_bwd_sums<T, sl.value, whole.value, ACT><<<dim3((unsigned)pl.slots, slabs, G), SPLIT_NTH, lds, st>>>(a, sums, (uint32_t)ranges);
        if (a.out.p)   // dx may overwrite dy
          k_gn_bwd_apply<T, sl.value, whole.value, ACT><<<dim3(grid_of(ranges) + col_blocks, slabs, G), SPLIT_NTH,
              std::max<size_t>(SPLIT_NTH * 8, (size_t)pl.ng * sizeof(float2)), st>>>(a, (uint32_t)ranges, sums, col_blocks);
      });
      if (!a.out.p) k_gn_cols<T><<<dim3(col_blocks, slabs, G), SPLIT_NTH, 0, st>>>(a, sums);
    }
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !cols || pl.slots == 1 || pl.mode == GN_SPLIT) return e;
  return launch_slot_sum((const float*)a.ws, pl.slots * 2 * a.C, (int)pl.slots, 2 * a.C, a.dgamma, a.C, a.dbeta, G, st);
}

#define PIGAN_GN_INST(T) template hipError_t launch_gn_bwd<T>(const GnArgs<T>&, int, hipStream_t);
PIGAN_GN_INST(float)
PIGAN_GN_INST(bf16)
PIGAN_GN_INST(f16)

}  // namespace pigan
