// Group norm with an activation, channels last, forward, for gfx950.
#include "group_norm_parts.h"

namespace pigan {
namespace {

// ---------------------------------------------------------------------------
// Rows: samples of one point.  A group is 2^i <= 64 neighbouring lanes with a piece each,
// the sums are theirs by shuffles; a thread keeps its column over NV rows at a time, so that
// four loads are under way.  Bound by memory: 131,072 x 1024 fp16, 32 groups, 110 us
// (5.2 TB/s with the statistics).
// ---------------------------------------------------------------------------
template <class T, int NV, int ACT>
__global__ void __launch_bounds__(256) k_gn_rows(const GnArgs<T> a) {
  constexpr int E = EPP<T>;
  const GnPlan& pl = a.pl;
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw;
  const Slab b = slab_at(a, blockIdx.y);
  const int64_t g = blockIdx.z;
  const int lanes = pl.span, j = Div(lanes)(col);
  const bool head = threadIdx.x % lanes == 0;
  if (row >= pl.rows || col * E >= b.width) return;   // whole groups of lanes
  const double inv_n = pl.inv_n;
  float ga[E], be[E];
  vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, a.C, 1.0f, ga);
  vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, a.C, 0.0f, be);
  const T* x = a.x.p + g * a.x.gs + b.c0 + col * E;
  T* y = a.out.p + g * a.out.gs + b.c0 + col * E;
  const int64_t step = (int64_t)gridDim.x * pl.rows;
  for (int64_t s0 = (int64_t)blockIdx.x * pl.rows + row; s0 < a.S; s0 += NV * step) {
    piece_t raw[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t s = s0 + v * step;
      raw[v] = load_piece<true>(x + (s < a.S ? s : s0) * a.x.ss, E, pl.stream);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t s = s0 + v * step;
      float f[E];
      piece_floats<T>(raw[v], f);
      const float k = shift_of(__shfl(f[0], (threadIdx.x & 63) & ~(lanes - 1)));
      Pair t = {0.0, 0.0};
#pragma unroll
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
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = value_of<ACT, T>((f[e] - st.mean) * (st.rstd * ga[e]) + be[e]);
        store_piece<true>(y + s * a.out.ss, E, f, pl.stream);
        const int64_t at = (g * a.S + s) * a.n + b.j0 + j;
        if (head && a.mean) a.mean[at] = st.mean;
        if (head && a.rstd) a.rstd[at] = st.rstd;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Samples whose slabs fit a block's registers: read once, written once.  Short samples
// share a block, NV = 1 then.  More than eight pieces a thread spill.  All blocks read, then
// all write, with the vector units busy for three quarters of it: 256 x 1024 x 128 bf16,
// silu, 32 us (4.2 TB/s; 512 threads on 64 bytes of a point 37 us, two passes 42).
// ---------------------------------------------------------------------------
// Whether a block's values lie in LDS for the sums, 4 bytes each: where a thread has one piece
// of several groups, whose sums would be 16 bytes an element.  Else bytes of the sums.
constexpr bool one_values(int nv, int sl) { return nv == 1 && sl > 1; }
constexpr size_t one_lds(int nth, int nv, int sl) {
  return one_values(nv, sl) ? (size_t)nth * (sl + 1) * 4 : (size_t)nth * (sl + 1) * sizeof(Pair);
}

template <class T, int NTH, int NV, int SL, bool WHOLE, int ACT>
__global__ void __launch_bounds__(NTH, NV < 8 ? 1 : SL == 1 && WHOLE ? 4 : 3) k_gn_one(const GnArgs<T> a, int64_t batches, uint32_t slab0) {
  constexpr int E = EPP<T>;
  constexpr bool VALUES = one_values(NV, SL);
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  float* values = (float*)sm;
  Stat* stat = (Stat*)((char*)sm + one_lds(NTH, NV, SL));
  float* shift = (float*)(stat + pl.ns * pl.ng);
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw;
  const bool many = NV == 1 && pl.ns > 1;
  const int si = many ? Div((int)a.P)(row) : 0, pr = many ? row - si * (int)a.P : row;
  const Div by_span(pl.span);
  const int per = row_of(pl.pw * SL);
  const int64_t g = blockIdx.z;
  const Slab b = slab_at(a, slab0 + blockIdx.x);
  const int valid = b.width - col * E, left = (int)a.P - pr;
  for (int64_t bt = blockIdx.y; bt < batches; bt += gridDim.y) {
    const int64_t s0 = bt * pl.ns, s = s0 + si;
    const bool on = row < pl.rows && left > 0 && s < a.S && valid > 0;
    const T* first = a.x.p + g * a.x.gs + (on ? s : s0) * a.x.ss;
    piece_t raw[NV];
    load_rows<WHOLE>(raw, on ? first + b.c0 + col * E + pr * a.x.ld : first + b.c0, pl.rows * a.x.ld, on ? left : 1, pl.rows,
                     on ? valid : b.width);
    auto tell = [&](int i, int j, const Pair& t, float k) {
      const Stat st = stat_of(t, k, pl.inv_n, a.eps);
      stat[i * b.ng + j] = st;
      const int64_t at = (g * a.S + s0 + i) * a.n + b.j0 + j;
      if (s0 + i < a.S) {
        if (a.mean) a.mean[at] = st.mean;
        if (a.rstd) a.rstd[at] = st.rstd;
      }
    };
    if constexpr (VALUES) {
      // one piece of several groups: the values themselves, which the groups' lanes sum
      if (on) {
        float f[E];
        piece_floats<T>(raw[0], f);
#pragma unroll
        for (int e = 0; e < E; ++e) values[row * per + col * E + e] = f[e];
      }
      __syncthreads();
      const int rows = min((int)a.P, pl.rows);
      const Div by_ng(b.ng);
      auto at = [&](int k) { return values + (pl.ns > 1 ? by_ng(k) : 0) * rows * per + (pl.ns > 1 ? k - by_ng(k) * b.ng : k) * pl.span; };
      lane_sums(pl.ns * b.ng, pl.lanes, [&](int k, int l) {
        const float* v = at(k);
        const double base = shift_of(v[0]);
        Pair t = {0.0, 0.0};
#pragma unroll 4
        for (int q = l; q < rows * pl.span; q += pl.lanes) {
          const int r = by_span(q);
          const double d = v[r * per + (q - r * pl.span)] - base;
          t.s += d;
          t.q += d * d;
        }
        return t;
      }, [&](int k, const Pair& t) {
        const int i = pl.ns > 1 ? by_ng(k) : 0;
        tell(i, k - i * b.ng, t, shift_of(at(k)[0]));
      });
    } else {
      float k[SL];
      Pair acc[SL];
#pragma unroll
      for (int e = 0; e < SL; ++e) {
        k[e] = shift_of(Elem<T>::to_f(first[(b.j0 + group_of<T, SL>(b, by_span, col, e)) * pl.cg]));
        acc[e] = {0.0, 0.0};
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (on && v * pl.rows < left) {
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
          const int slot = col * SL + e, j = by_span(slot);
          sm[row * per + slot] = acc[e];
          if (on && pr == 0 && j < b.ng && slot == j * pl.span) shift[si * b.ng + j] = k[e];
        }
      __syncthreads();
      group_sums(sm, pl.ns, pl.ns > 1 ? (int)a.P : pl.rows, per, b.ng, pl.span, pl.lanes,
                 [&](int i, int j, const Pair& t) { tell(i, j, t, shift[i * b.ng + j]); });
    }
    __syncthreads();
    if (!on) continue;
    float mean[SL], sc[E], be[E];
    vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 1.0f, sc);
    vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 0.0f, be);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const Stat st = stat[si * b.ng + group_of<T, SL>(b, by_span, col, SL > 1 ? e : 0)];
      if (e < SL) mean[e] = st.mean;
      sc[e] *= st.rstd;
    }
    T* out = a.out.p + g * a.out.gs + s * a.out.ss + b.c0 + col * E + pr * a.out.ld;
    const int64_t step = pl.rows * a.out.ld;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v * pl.rows < left) {
        float f[E];
        piece_floats<T>(raw[v], f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = value_of<ACT, T>((f[e] - mean[SL > 1 ? e : 0]) * sc[e] + be[e]);
        store_piece<WHOLE>(out + v * step, valid, f, pl.stream);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// ---------------------------------------------------------------------------
// Samples of more points than a block's registers hold: sums of ranges of points, then the
// results.  Blocks: [G][slabs][S * splits].  16 x 65,536 x 128 bf16, gelu: sums 50 us
// (5.4 TB/s, memory), results 99 us (5.4 TB/s, vector units: 20 instructions an element, two
// of them transcendental ones that count twice).
// ---------------------------------------------------------------------------
// ws: Pair [G][S][n][chan_parts * splits], and float [G][S][n] behind them: the values that
// the sums begin at (y may overwrite x while other blocks still apply)
template <class T, int SL, bool WHOLE>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_sums(const GnArgs<T> a, uint32_t ranges, int64_t all_groups) {
  constexpr int E = EPP<T>;
  extern __shared__ Pair sm[];
  const GnPlan& pl = a.pl;
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw, parts = pl.chan_parts * pl.splits;
  const Div by_span(pl.span);
  const int per = row_of(pl.pw * SL);
  const int64_t g = blockIdx.z;
  for (uint32_t slab = blockIdx.y; slab < pl.slabs; slab += gridDim.y) {
    const Slab b = slab_at(a, slab);
    const int valid = b.width - col * E;
    for (uint32_t it = blockIdx.x; it < ranges; it += gridDim.x) {
      const uint32_t s = it / (uint32_t)pl.splits, split = it - s * (uint32_t)pl.splits;
      const T* first = a.x.p + g * a.x.gs + s * a.x.ss;
      Pair acc[SL];
      float k[SL];
#pragma unroll
      for (int e = 0; e < SL; ++e) {
        acc[e] = {0.0, 0.0};
        k[e] = shift_of(Elem<T>::to_f(first[(b.j0 + group_of<T, SL>(b, by_span, col, e)) * pl.cg]));
      }
      if (valid > 0 && row < pl.rows) {
        const Turns tn(pl, a.P, SUM_TURN, split, pl.splits, row);
        const int64_t step = pl.rows * a.x.ld;
        const T* q = first + b.c0 + col * E + tn.first * a.x.ld;
        for (int left = tn.left; left > 0; left -= tn.by, q += tn.by * a.x.ld) {
          piece_t raw[SUM_TURN];
          load_rows<WHOLE>(raw, q, step, left, pl.rows, valid);
#pragma unroll
          for (int v = 0; v < SUM_TURN; ++v) {
            if (v > 0 && v * pl.rows >= left) break;
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
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      if (row < pl.rows)
#pragma unroll
        for (int e = 0; e < SL; ++e) sm[row * per + col * SL + e] = acc[e];
      __syncthreads();
      Pair* part = (Pair*)a.ws;
      float* shifts = (float*)(part + all_groups * parts);
      const int64_t i0 = (g * a.S + s) * a.n + b.j0;
      const int at = pl.chan_parts > 1 ? slab % (uint32_t)pl.chan_parts * pl.splits + split : split;
      group_sums(sm, 1, pl.rows, per, b.ng, pl.span, pl.lanes, [&](int, int j, const Pair& t) {
        part[(i0 + j) * parts + at] = t;
        if (at == 0) shifts[i0 + j] = shift_of(Elem<T>::to_f(first[(b.j0 + j) * pl.cg]));
      });
      __syncthreads();
    }
  }
}

template <class T, int SL, bool WHOLE, int ACT>
__global__ void __launch_bounds__(SPLIT_NTH) k_gn_apply(const GnArgs<T> a, uint32_t ranges, int64_t all_groups) {
  constexpr int E = EPP<T>, U = APPLY_TURN;
  extern __shared__ Pair sm[];   // of Stat
  Stat* stat = (Stat*)sm;
  const GnPlan& pl = a.pl;
  const int row = Div(pl.pw)(threadIdx.x), col = threadIdx.x - row * pl.pw, parts = pl.chan_parts * pl.splits;
  const Div by_span(pl.span);
  const int64_t g = gridDim.z - 1 - blockIdx.z;
  for (uint32_t k = blockIdx.y; k < pl.slabs; k += gridDim.y) {
    const uint32_t slab = (uint32_t)pl.slabs - 1 - k;
    const Slab b = slab_at(a, slab);
    const int valid = b.width - col * E;
    for (uint32_t at = blockIdx.x; at < ranges; at += gridDim.x) {
      const uint32_t it = from_last(at, ranges), s = it / (uint32_t)pl.splits, split = it - s * (uint32_t)pl.splits;
      const Turns tn(pl, a.P, U, split, pl.splits, row);
      const int64_t step = pl.rows * a.x.ld, p0 = tn.first + tn.last();
      int left = valid > 0 && row < pl.rows ? tn.left - tn.last() : 0;
      const T* q = a.x.p + g * a.x.gs + s * a.x.ss + b.c0 + col * E + p0 * a.x.ld;
      piece_t raw[U];
      if (left > 0) load_rows<WHOLE>(raw, q, step, left, pl.rows, valid);
      const int64_t i0 = (g * a.S + s) * a.n + b.j0;
      const Pair* part = (const Pair*)a.ws;
      const float* shifts = (const float*)(part + all_groups * parts) + i0;
      const bool tells = split == 0 && (pl.chan_parts == 1 || slab % (uint32_t)pl.chan_parts == 0);
      range_sums(part + i0 * parts, b.ng, parts, pl.lanes, [&](int j, const Pair& t) {
        const Stat st = stat_of(t, shifts[j], pl.inv_n, a.eps);
        stat[j] = st;
        if (tells && a.mean) a.mean[i0 + j] = st.mean;
        if (tells && a.rstd) a.rstd[i0 + j] = st.rstd;
      });
      __syncthreads();
      if (left > 0) {
        float mean[SL], sc[E], be[E];
        vec_load<E>(a.gamma ? a.gamma + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 1.0f, sc);
        vec_load<E>(a.beta ? a.beta + g * a.C : nullptr, b.c0 + col * E, b.c0 + b.width, 0.0f, be);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const Stat st = stat[group_of<T, SL>(b, by_span, col, SL > 1 ? e : 0)];
          if (e < SL) mean[e] = st.mean;
          sc[e] *= st.rstd;
        }
        T* out = a.out.p + g * a.out.gs + s * a.out.ss + b.c0 + col * E + p0 * a.out.ld;
        const int64_t ostep = pl.rows * a.out.ld;
        for (;;) {
          // the next turn's loads before this one's stores: a wait for them is one for the stores too
          piece_t next[U];
          const bool more = tn.before(left);
          q -= tn.by * a.x.ld;
          if (more) load_rows<WHOLE>(next, q, step, left + tn.by, pl.rows, valid);
#pragma unroll
          for (int v = 0; v < U; ++v) {
            if (v * pl.rows < left) {
              float f[E];
              piece_floats<T>(raw[v], f);
#pragma unroll
              for (int e = 0; e < E; ++e) f[e] = value_of<ACT, T>((f[e] - mean[SL > 1 ? e : 0]) * sc[e] + be[e]);
              store_piece<WHOLE>(out + v * ostep, valid, f, pl.stream);
            }
            __builtin_amdgcn_sched_barrier(0);   // a piece at a time: more would not fit the registers
          }
          if (!more) break;
          left += tn.by;
          out -= tn.by * a.out.ld;
#pragma unroll
          for (int v = 0; v < U; ++v) raw[v] = next[v];
        }
      }
      __syncthreads();
    }
  }
}

}  // namespace

template <class T> hipError_t launch_gn_fwd(const GnArgs<T>& a, int G, hipStream_t st) {
  if (a.S <= 0) return hipSuccess;
  const GnPlan& pl = a.pl;
  by_act(a.act, [&](auto act) {
    constexpr int ACT = act.value;
    if (pl.mode == GN_ROWS) {
      const int64_t turns = cdiv(a.S, (int64_t)pl.rows * 4), most = std::max<int64_t>(1, 4096 / std::min<int64_t>(4096, G * pl.slabs));
      k_gn_rows<T, 4, ACT><<<dim3((unsigned)std::min(turns, most), (unsigned)pl.slabs, G), 256, 0, st>>>(a);
    } else if (pl.mode == GN_ONE) {
      const int64_t batches = cdiv(a.S, pl.ns);
      const int64_t most = int64_t(1) << 21;   // a launch's x dimension holds fewer than 2^32 threads
      by_width(a, [&](auto sl, auto whole) {
        by_shape<sl.value == 1 && whole.value>(pl, [&](auto nth, auto nv) {
          const size_t lds = one_lds(nth.value, nv.value, sl.value) + (size_t)pl.ns * pl.ng * (sizeof(Stat) + 4);
          for (int64_t at = 0; at < pl.slabs; at += most) {
            const dim3 grid((unsigned)std::min(most, pl.slabs - at), (unsigned)std::min<int64_t>(batches, 65535), G);
            k_gn_one<T, nth.value, nv.value, sl.value, whole.value, ACT><<<grid, nth.value, lds, st>>>(a, batches, (uint32_t)at);
          }
        });
      });
    } else {
      const int64_t groups = (int64_t)G * a.S * a.n, ranges = a.S * pl.splits;
      const unsigned slabs = (unsigned)std::min<int64_t>(pl.slabs, 65535);
      by_width(a, [&](auto sl, auto whole) {
        k_gn_sums<T, sl.value, whole.value><<<dim3(grid_of(ranges), slabs, G), SPLIT_NTH, SPLIT_NTH * (sl.value + 1) * sizeof(Pair), st>>>(a, (uint32_t)ranges, groups);
        k_gn_apply<T, sl.value, whole.value, ACT><<<dim3(grid_of(ranges), slabs, G), SPLIT_NTH, (size_t)pl.ng * sizeof(Stat), st>>>(a, (uint32_t)ranges, groups);
      });
    }
  });
  return hipGetLastError();
}

#define PIGAN_GN_INST(T) template hipError_t launch_gn_fwd<T>(const GnArgs<T>&, int, hipStream_t);
PIGAN_GN_INST(float)
PIGAN_GN_INST(bf16)
PIGAN_GN_INST(f16)

}  // namespace pigan
