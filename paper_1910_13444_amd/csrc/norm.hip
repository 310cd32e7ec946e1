// Layer norm (forward, backward with the column sums of its parameter
// gradients) and the reverse pass of an activation, for gfx950.
//
// All of it is bound by memory: a row is read once into registers, its
// statistics are sums over the lanes that hold it, and the results leave from
// the same registers.  TPR threads share a row, NV 16-byte pieces each; rows
// may start at any element (the pieces are under-aligned vector accesses).
#include "norm.h"

#include "act.h"
#include "piece.h"

namespace pigan {
namespace {

// A piece of a row of N columns from column c on.  WHOLE: the columns come in whole
// pieces, so a piece is all there or not at all.
template <bool WHOLE, class T>
__device__ __forceinline__ piece_t row_load(const T* p, int64_t c, int64_t N) {
  if constexpr (!WHOLE) return piece_load(p + c, N - c);
  piece_t v = {0, 0, 0, 0};
  if (c < N) v = *(const piece_u*)(p + c);
  return v;
}
template <bool WHOLE, class T>
__device__ __forceinline__ void row_store(T* p, int64_t c, int64_t N, const float* f) {
  if constexpr (!WHOLE) piece_store(p + c, N - c, f);
  else if (c < N) piece_store(p + c, EPP<T>, f);
}

// v of the lane whose number differs in bit O, where the O lanes of each aligned group
// have one value: any lane of the other group will do, and up to 16 lanes LDS is not
// asked (__shfl_xor becomes a ds_bpermute: 7 % of fp32 16 x 75,770 x 41 forward; the
// swaps of half rows and half waves for 16 and 32 are slower than theirs by 4 %).
template <int O>
__device__ __forceinline__ uint32_t other_group(uint32_t v) {
  if constexpr (O == 1) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true);         // quad 1 0 3 2
  else if constexpr (O == 2) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true);    // quad 2 3 0 1
  else if constexpr (O == 4) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true);   // 8 lanes mirrored
  else if constexpr (O == 8) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true);   // 16 lanes mirrored
  else return (uint32_t)__shfl_xor((int)v, O);
}
template <int O>
__device__ __forceinline__ float other_group(float v) { return __uint_as_float(other_group<O>(__float_as_uint(v))); }
template <int O>
__device__ __forceinline__ double other_group(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)other_group<O>((uint32_t)b) | (uint64_t)other_group<O>((uint32_t)(b >> 32)) << 32);
}

// Sums over the TPR threads of a row, in a fixed order; every one of them gets
// them.  Above a wave, `red` (K entries per wave) passes the waves' sums on; the
// caller alternates between two of them, so one barrier is enough.  MOVES: by lane
// moves (between them the compiler puts other work, and holds its registers).
template <int TPR, bool MOVES = true, int K, class S>
__device__ __forceinline__ void row_sums(S (&v)[K], S* red) {
  if constexpr (MOVES) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] += other_group<1>(v[k]);
      v[k] += other_group<2>(v[k]);
      v[k] += other_group<4>(v[k]);
      if constexpr (TPR > 8) v[k] += other_group<8>(v[k]);
      if constexpr (TPR > 16) v[k] += other_group<16>(v[k]);
      if constexpr (TPR > 32) v[k] += other_group<32>(v[k]);
    }
  } else {
#pragma unroll
    for (int o = 1; o < (TPR < 64 ? TPR : 64); o *= 2)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o);
  }
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) red[wave * K + k] = v[k];
    __syncthreads();
    const S* r = red + wave / NW * NW * K;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = r[k];
#pragma unroll
      for (int i = 1; i < NW; ++i) v[k] += r[i * K + k];
    }
  }
}
template <int TPR, class S>
__device__ __forceinline__ S row_sum(S v, S* red) {
  S s[1] = {v};
  row_sums<TPR>(s, red);
  return s[0];
}

// ---------------------------------------------------------------------------
// Forward.  Two sums over registers (mean, then squared distances from it: no
// cancellation).  The mean is rounded once, so that a constant row's is that constant:
// its sum is held in fp64 where fp32 does not hold up to MAX_PIECES pieces of one
// value, which it does of 8 bits (bf16), and of 11 (fp16) in up to 8192 columns.
// Blocks walk rows; the next row is requested before the present one is worked on,
// gamma and beta stay in registers.
//   bf16, us (TB/s)  524288 x 512: 222 (4.8), 131072 x 2048: 214 (5.0), 32768 x 8192:
//                    209 (5.1), 16384 x 16384: 198 (5.4); 1250 of 2048 pieces a row
//                    (26843 x 10000) 268 (4.0)
//   fp32             128521 x 1152: 230 (5.2), 2048 x 8191: 25 (5.3)
// ---------------------------------------------------------------------------
__device__ __forceinline__ float mean_of(float sum, float n, double) { return sum / n; }   // no rounding of 1 / n
__device__ __forceinline__ float mean_of(double sum, float, double inv_n) { return (float)(sum * inv_n); }

template <class T, int COLS>
using MeanSum = std::conditional_t<sizeof(T) == 4 || (__is_same(T, f16) && COLS > 8192), double, float>;

template <class T, int TPR, int NV, int NTH, bool WHOLE>
__global__ void __launch_bounds__(NTH) k_norm_fwd(const NormArgs<T> p) {
  constexpr int E = EPP<T>, RPB = NTH / TPR;
  typedef MeanSum<T, TPR * NV * E> Sum;
  __shared__ Sum red0[NTH / 64];
  __shared__ float red1[NTH / 64];
  const int g = blockIdx.z;
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const T* x = p.x.p + g * p.x.gs;
  T* y = p.out.p + g * p.out.gs;
  const float* gamma = p.gamma ? p.gamma + g * p.N : nullptr;
  const float* beta = p.beta ? p.beta + g * p.N : nullptr;
  const int64_t step = (int64_t)gridDim.x * RPB;
  const float n = (float)p.N;

  float ga[NV][E], be[NV][E];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int64_t c = (int64_t)(v * TPR + lane) * E;
    vec_load<E>(gamma, c, p.N, 1.0f, ga[v]);
    vec_load<E>(beta, c, p.N, 0.0f, be[v]);
  }
  auto request = [&](piece_t (&raw)[NV], int64_t r) {
    const T* row = x + (r < p.M ? r : p.M - 1) * p.x.ld;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (int64_t)(v * TPR + lane) * E;
      raw[v] = row_load<WHOLE>(row, c, p.N);
    }
  };
  piece_t next[NV];
  int64_t r0 = (int64_t)blockIdx.x * RPB;
  request(next, r0 + sub);
  // every thread of a block takes the same number of turns (barriers above a wave)
  for (; r0 < p.M; r0 += step) {
    const int64_t r = r0 + sub;
    float f[NV][E];
#pragma unroll
    for (int v = 0; v < NV; ++v) piece_floats<T>(next[v], f[v]);
    if (r0 + step < p.M) request(next, r + step);
    std::conditional_t<sizeof(T) == 4, double, float> s = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < E; ++e) s += f[v][e];       // zeros past the end
    const float mean = mean_of(row_sum<TPR>((Sum)s, red0), n, p.inv_n);
    float q = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (int64_t)(v * TPR + lane) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        f[v][e] -= mean;
        if (WHOLE ? c < p.N : c + e < p.N) q += f[v][e] * f[v][e];
      }
    }
    const float var = row_sum<TPR>(q, red1) / n;
    const float rstd = 1.0f / sqrtf(var + p.eps);
    if (r < p.M) {
      T* row = y + r * p.out.ld;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int64_t c = (int64_t)(v * TPR + lane) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) f[v][e] = f[v][e] * rstd * ga[v][e] + be[v][e];
        row_store<WHOLE>(row, c, p.N, f[v]);
      }
      if (lane == 0) {
        if (p.mean) p.mean[g * p.M + r] = mean;
        if (p.rstd) p.rstd[g * p.M + r] = rstd;
      }
    }
  }
}

// Rows too long for registers: the row is read three times (from L2 after the
// first), a block of 1024 threads per row (bf16 16376 x 16392: 392 us, 2.7 TB/s).
template <class T>
__global__ void __launch_bounds__(1024) k_norm_fwd_long(const NormArgs<T> p) {
  constexpr int E = EPP<T>;
  __shared__ double red0[16];
  __shared__ float red1[16];
  const int g = blockIdx.z;
  const float* gamma = p.gamma ? p.gamma + g * p.N : nullptr;
  const float* beta = p.beta ? p.beta + g * p.N : nullptr;
  const float n = (float)p.N;
  for (int64_t r = blockIdx.x; r < p.M; r += gridDim.x) {
    const T* row = p.x.p + g * p.x.gs + r * p.x.ld;
    T* out = p.out.p + g * p.out.gs + r * p.out.ld;
    double s = 0.0;
    float f[E];
    for (int64_t c = (int64_t)threadIdx.x * E; c < p.N; c += 1024 * E) {
      piece_floats<T>(piece_load(row + c, p.N - c), f);
#pragma unroll
      for (int e = 0; e < E; ++e) s += f[e];
    }
    const float mean = mean_of(row_sum<1024>(s, red0), n, p.inv_n);
    float q = 0.0f;
    for (int64_t c = (int64_t)threadIdx.x * E; c < p.N; c += 1024 * E) {
      piece_floats<T>(piece_load(row + c, p.N - c), f);
#pragma unroll
      for (int e = 0; e < E; ++e) q += c + e < p.N ? (f[e] - mean) * (f[e] - mean) : 0.0f;
    }
    const float rstd = 1.0f / sqrtf(row_sum<1024>(q, red1) / n + p.eps);
    for (int64_t c = (int64_t)threadIdx.x * E; c < p.N; c += 1024 * E) {
      float ga[E], be[E];
      piece_floats<T>(piece_load(row + c, p.N - c), f);
      vec_load<E>(gamma, c, p.N, 1.0f, ga);
      vec_load<E>(beta, c, p.N, 0.0f, be);
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = (f[e] - mean) * rstd * ga[e] + be[e];
      piece_store(out + c, p.N - c, f);
    }
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[g * p.M + r] = mean;
      if (p.rstd) p.rstd[g * p.M + r] = rstd;
    }
    // a thread may not begin the next row's sums while another still reads these
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Backward.  As the forward, with two sums per row (h and h xhat); a thread
// keeps the column sums of its NV pieces over all rows of the block in
// registers, the block adds its waves' in order and writes one partial row of
// [dgamma, dbeta] (the final ones, where one block takes all rows).
// ---------------------------------------------------------------------------
// Threads of a block: 1024, which leaves few partial rows, but 256 where a thread
// holds two 16-bit pieces (sixteen columns) of a wave's row: that needs more
// registers than 1024 threads have (131,072 x 1024 with a skip: 312 us spilling,
// 210 us without).  Rows of 8192 to 16384 such columns have no other way and spill
// (17 registers; 16384 x 16384: 370 us, 4.4 TB/s).
template <class T, int TPR, int NV> constexpr int bwd_nth() { return TPR <= 64 && sizeof(T) == 2 && NV == 2 ? 256 : 1024; }

// Nothing is masked by element: past the end of a row dy is loaded as zero, and
// with it everything that a column there adds.
// Several rows of more than a wave in a block leave its loop together, for its
// barriers: past the last row they work on zeros (ROWS_JOIN).
//   bf16, us (TB/s)   no skip      with a skip     one row per 1024 threads
//   262144 x 1024     314 (5.1)    421 (5.1)
//   131072 x 2048     287 (5.6)    388 (5.5)       707, 741
//   65536 x 4096      289 (5.6)    390 (5.5)       390, 449
//   32768 x 8192      300 (5.4)    401 (5.4)
template <class T, int TPR, int NV, bool DX, bool COLS, bool WHOLE>
__global__ void __launch_bounds__((bwd_nth<T, TPR, NV>())) k_norm_bwd(const NormArgs<T> p, float* __restrict__ d0,
                                                      float* __restrict__ d1, int64_t d_g, int64_t d_b) {
  constexpr int E = EPP<T>, BWD_NTH = bwd_nth<T, TPR, NV>(), RPB = BWD_NTH / TPR;
  constexpr bool ROWS_JOIN = TPR > 64 && RPB > 1;
  __shared__ float red[2][2 * BWD_NTH / 64];
  __shared__ float cols[COLS && RPB > 1 ? 2 * TPR * NV * E : 1];
  __shared__ __attribute__((aligned(16))) float ga[TPR * NV * E];
  const int g = blockIdx.z;
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const T* x = p.x.p + g * p.x.gs;
  const T* dy = p.dy.p + g * p.dy.gs;
  const T* add = DX && p.add.p ? p.add.p + g * p.add.gs : nullptr;
  const float* gamma = p.gamma ? p.gamma + g * p.N : nullptr;
  const int64_t step = (int64_t)gridDim.x * RPB;
  const float n = (float)p.N;

  // gamma waits in LDS: beside the column sums it would not fit the registers
  for (int c = threadIdx.x; c < TPR * NV * E; c += BWD_NTH) ga[c] = gamma && c < p.N ? gamma[c] : 1.0f;
  __syncthreads();
  float sg[NV][E], sb[NV][E];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < E; ++e) sg[v][e] = sb[v][e] = 0.0f;
  piece_t rx[NV], rd[NV], ra[NV];
  float mean = 0.0f, rstd = 0.0f;
  auto request = [&](int64_t r) {
    const bool live = !ROWS_JOIN || r < p.M;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = live ? (int64_t)(v * TPR + lane) * E : p.N;
      rx[v] = row_load<WHOLE>(x + r * p.x.ld, c, p.N);
      rd[v] = row_load<WHOLE>(dy + r * p.dy.ld, c, p.N);
    }
    mean = live ? p.mean[g * p.M + r] : 0.0f;
    rstd = live ? p.rstd[g * p.M + r] : 0.0f;
  };
  auto request_add = [&](int64_t r) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = !ROWS_JOIN || r < p.M ? (int64_t)(v * TPR + lane) * E : p.N;
      ra[v] = row_load<WHOLE>(add + r * p.add.ld, c, p.N);
    }
  };
  int turn = 0;
  const int64_t last = p.M + (ROWS_JOIN ? sub : 0);   // as far as this thread's rows go
  int64_t r = (int64_t)blockIdx.x * RPB + sub;
  if (r < last) {
    request(r);
    if (add) request_add(r);
  }
  for (; r < last; r += step, turn ^= 1) {
    asm volatile("" ::: "memory");   // gamma is read again for every row
    float xh[NV][E], h[NV][E], s[2] = {0.0f, 0.0f};
    const float mu = mean, rs = rstd;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      piece_floats<T>(rx[v], xh[v]);
      piece_floats<T>(rd[v], h[v]);
    }
    // the next row is on its way while this one is worked on
    if (r + step < last) request(r + step);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xh[v][e] = (xh[v][e] - mu) * rs;
        if (COLS) {
          sg[v][e] += h[v][e] * xh[v][e];
          sb[v][e] += h[v][e];
        }
        h[v][e] *= ga[(v * TPR + lane) * E + e];
        s[0] += h[v][e];
        s[1] += h[v][e] * xh[v][e];
      }
    }
    if constexpr (DX) {
      // (two pieces of a row of 1024 threads: 63 registers spilled with moves, 697 us at
      // 16384 x 16384)
      row_sums<TPR, !(TPR == 1024 && NV == 2)>(s, red[turn]);
      const float s1 = s[0] / n, s2 = s[1] / n;
      T* row = p.out.p + g * p.out.gs + r * p.out.ld;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int64_t c = !ROWS_JOIN || r < p.M ? (int64_t)(v * TPR + lane) * E : p.N;
#pragma unroll
        for (int e = 0; e < E; ++e) h[v][e] = rs * (h[v][e] - s1 - xh[v][e] * s2);
        if (add) {
          float res[E];
          piece_floats<T>(ra[v], res);
#pragma unroll
          for (int e = 0; e < E; ++e) h[v][e] += res[e];
        }
        row_store<WHOLE>(row, c, p.N, h[v]);
      }
      if (add && r + step < last) request_add(r + step);
    }
  }
  if constexpr (COLS) {
    float* o0 = d0 ? d0 + g * d_g + blockIdx.x * d_b : nullptr;
    float* o1 = d1 ? d1 + g * d_g + blockIdx.x * d_b : nullptr;
    if constexpr (TPR < 64) {
      // lanes of a wave that hold the same columns
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int o = TPR; o < 64; o *= 2) {
            sg[v][e] += __shfl_xor(sg[v][e], o);
            sb[v][e] += __shfl_xor(sb[v][e], o);
          }
    }
    if constexpr (RPB > 1) {
      constexpr int UNIT = TPR < 64 ? 64 : TPR;   // threads that hold a set of sums
      for (int w = 0; w < BWD_NTH / UNIT; ++w) {
        if ((int)(threadIdx.x / UNIT) == w && threadIdx.x % UNIT < TPR) {
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const int c = (v * TPR + lane) * E + e;
              cols[c] = w ? cols[c] + sg[v][e] : sg[v][e];
              cols[TPR * NV * E + c] = w ? cols[TPR * NV * E + c] + sb[v][e] : sb[v][e];
            }
        }
        __syncthreads();
      }
      for (int c = threadIdx.x; c < p.N; c += BWD_NTH) {
        if (o0) o0[c] = cols[c];
        if (o1) o1[c] = cols[TPR * NV * E + c];
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int64_t c = (int64_t)(v * TPR + lane) * E + e;
          if (c < p.N && o0) o0[c] = sg[v][e];
          if (c < p.N && o1) o1[c] = sb[v][e];
        }
    }
  }
}

// Rows too long for registers: two passes over the row (bf16 16376 x 16392, with the
// column sums' own kernel: 604 us, 2.7 TB/s; x and dy are read once more for those).
template <class T>
__global__ void __launch_bounds__(1024) k_norm_bwd_long(const NormArgs<T> p) {
  constexpr int E = EPP<T>;
  __shared__ float red[32];
  const int g = blockIdx.z;
  const float* gamma = p.gamma ? p.gamma + g * p.N : nullptr;
  const float n = (float)p.N;
  for (int64_t r = blockIdx.x; r < p.M; r += gridDim.x) {
    const T* x = p.x.p + g * p.x.gs + r * p.x.ld;
    const T* dy = p.dy.p + g * p.dy.gs + r * p.dy.ld;
    const T* add = p.add.p ? p.add.p + g * p.add.gs + r * p.add.ld : nullptr;
    T* out = p.out.p + g * p.out.gs + r * p.out.ld;
    const float mean = p.mean[g * p.M + r], rstd = p.rstd[g * p.M + r];
    float s[2] = {0.0f, 0.0f}, fx[E], fd[E], ga[E];
    for (int64_t c = (int64_t)threadIdx.x * E; c < p.N; c += 1024 * E) {
      piece_floats<T>(piece_load(x + c, p.N - c), fx);
      piece_floats<T>(piece_load(dy + c, p.N - c), fd);
      vec_load<E>(gamma, c, p.N, 1.0f, ga);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float h = fd[e] * ga[e];
        s[0] += h;
        s[1] += h * ((fx[e] - mean) * rstd);
      }
    }
    row_sums<1024>(s, red);
    const float s1 = s[0] / n, s2 = s[1] / n;
    for (int64_t c = (int64_t)threadIdx.x * E; c < p.N; c += 1024 * E) {
      float o[E];
      piece_floats<T>(piece_load(x + c, p.N - c), fx);
      piece_floats<T>(piece_load(dy + c, p.N - c), fd);
      vec_load<E>(gamma, c, p.N, 1.0f, ga);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = rstd * (fd[e] * ga[e] - s1 - (fx[e] - mean) * rstd * s2);
      if (add) {
        piece_floats<T>(piece_load(add + c, p.N - c), fd);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += fd[e];
      }
      piece_store(out + c, p.N - c, o);
    }
    __syncthreads();
  }
}

// Column sums where the columns of a row do not fit a block's registers: a
// block takes 256 pieces of columns and the rows b, b + gridDim.y, ...
template <class T>
__global__ void __launch_bounds__(256) k_norm_cols(const NormArgs<T> p, float* __restrict__ d0,
                                                   float* __restrict__ d1, int64_t d_g, int64_t d_b) {
  constexpr int E = EPP<T>;
  const int g = blockIdx.z;
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E;
  if (c >= p.N) return;
  const T* x = p.x.p + g * p.x.gs + c;
  const T* dy = p.dy.p + g * p.dy.gs + c;
  float sg[E], sb[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sg[e] = sb[e] = 0.0f;
#pragma unroll 2
  for (int64_t r = blockIdx.y; r < p.M; r += gridDim.y) {
    float fx[E], fd[E];
    piece_floats<T>(piece_load(x + r * p.x.ld, p.N - c), fx);
    piece_floats<T>(piece_load(dy + r * p.dy.ld, p.N - c), fd);
    const float mean = p.mean[g * p.M + r], rstd = p.rstd[g * p.M + r];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sg[e] += fd[e] * ((fx[e] - mean) * rstd);
      sb[e] += fd[e];
    }
  }
  const int64_t o = g * d_g + blockIdx.y * d_b + c;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (c + e < p.N) {
      if (d0) d0[o + e] = sg[e];
      if (d1) d1[o + e] = sb[e];
    }
}

template <class T>
__global__ void __launch_bounds__(256) k_colsum_rows(const Mat<const T> m, int64_t M, int64_t N,
                                                     float* __restrict__ part) {
  constexpr int E = EPP<T>;
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E;
  if (c >= N) return;
  const T* p = m.p + blockIdx.z * m.gs + c;
  float s[E], f[E];
#pragma unroll
  for (int e = 0; e < E; ++e) s[e] = 0.0f;
#pragma unroll 4
  for (int64_t r = blockIdx.y; r < M; r += gridDim.y) {
    piece_floats<T>(piece_load(p + r * m.ld, N - c), f);
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] += f[e];
  }
  float* o = part + ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * N + c;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (c + e < N) o[e] = s[e];
}

// Slot sums: 32 columns x 32 slot lanes per block; a slot lane adds every 32nd slot
// in fp64, the 32 lanes' sums are added in order.  Bound by latency (256 slots of
// 16,382 columns: 5.8 us, 2.9 TB/s).  WIDE: more columns than a launch's x dimension
// holds, 2^25 for every y (a kernel by itself: the blocks are so short that its
// arithmetic shows; bf16 reverse of 16 x 4 x 7216 28.8 us, 32.1 with it).
constexpr int64_t SLOT_RANGE = int64_t(1) << 25;

template <bool WIDE>
__global__ void __launch_bounds__(1024) k_slot_sum(const float* __restrict__ part, int64_t p_g, int n_slots, int64_t n,
                                                   float* __restrict__ dst, int64_t n1, float* __restrict__ dst2) {
  __shared__ double sums[32][33];
  const int cl = threadIdx.x & 31, sl = threadIdx.x >> 5;
  const int64_t c = (WIDE ? blockIdx.y * SLOT_RANGE : 0) + (int64_t)blockIdx.x * 32 + cl;
  const int g = blockIdx.z;
  double s = 0.0;
  if (c < n) {
    const float* q = part + g * p_g + c;
#pragma unroll 4
    for (int i = sl; i < n_slots; i += 32) s += (double)q[(int64_t)i * n];
  }
  sums[sl][cl] = s;
  __syncthreads();
  if (sl == 0 && c < n) {
    for (int i = 1; i < 32; ++i) s += sums[i][cl];
    if (c < n1) {
      if (dst) dst[g * n1 + c] = (float)s;
    } else if (dst2) {
      dst2[g * (n - n1) + c - n1] = (float)s;
    }
  }
}

__global__ void __launch_bounds__(256) k_zeros(float* __restrict__ dst, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) dst[i] = 0.0f;
}

// g = dy act'(pre), a piece per thread and turn; `vpr` pieces per row.  Bound by
// memory: 65,536 x 1024 bf16, silu, 72 us (5.6 TB/s), fp32, gelu, 158 (5.1); in the
// caches by the fp64 slope (16 x 926 x 1024 fp32, gelu, 39 us, 4.7 TB/s).
template <class T, class I>
__global__ void __launch_bounds__(256) k_act_bwd(int act, const Mat<const T> dy, const Mat<const T> pre, const Mat<T> out,
                                                 int64_t M, int64_t N, I vpr) {
  constexpr int E = EPP<T>;
  const int g = blockIdx.z;
  const I total = (I)M * vpr, stride = (I)gridDim.x * 256;
  const T* pd = dy.p + g * dy.gs;
  const T* pa = pre.p + g * pre.gs;
  T* po = out.p + g * out.gs;
  PIGAN_ACT_SWITCH(act, {
    for (I i = (I)blockIdx.x * 256 + threadIdx.x; i < total; i += stride) {
      const I r = i / vpr;
      const int64_t c = (int64_t)(i - r * vpr) * E;
      float fd[E], fa[E];
      piece_floats<T>(piece_load(pd + (int64_t)r * dy.ld + c, N - c), fd);
      piece_floats<T>(piece_load(pa + (int64_t)r * pre.ld + c, N - c), fa);
      for (int e = 0; e < E; ++e) fd[e] *= act_slope<ACT, T>(fa[e]);
      piece_store(po + (int64_t)r * out.ld + c, N - c, fd);
    }
  })
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// pieces of a row that a block's registers hold at most: 1024 threads, two each
constexpr int64_t MAX_PIECES = 2048;

template <class T, int TPR, int NV, int NTH>
void fwd(const NormArgs<T>& a, int G, hipStream_t st) {
  // 32 waves per CU and row of the grid: enough loads in flight, and gamma and
  // beta are read once for many rows
  const int64_t most = cdiv(int64_t(256) * 2048 / NTH, G);
  const int64_t blocks = cdiv(a.M, NTH / TPR);
  const dim3 grid((unsigned)(blocks < most ? blocks : most), 1, G);
  if (a.N % EPP<T> == 0) k_norm_fwd<T, TPR, NV, NTH, true><<<grid, NTH, 0, st>>>(a);
  else k_norm_fwd<T, TPR, NV, NTH, false><<<grid, NTH, 0, st>>>(a);
}

// blocks of the backward kernel per group: each is another partial row, so no
// more than fill the CUs (one of 1024 threads, three of 256)
int64_t bwd_blocks(int elem_bytes, int64_t pieces, int64_t M) {
  const int tpr = pieces <= 8 ? 8 : pieces <= 32 ? 32 : pieces <= 128 ? 64 : pieces <= 256 ? 256
                  : pieces <= 512 ? 512 : 1024;
  const bool small = pieces > 64 && pieces <= 128 && elem_bytes == 2;
  const int64_t most = small ? 768 : 256, want = cdiv(M, (small ? 256 : 1024) / tpr);
  return want < most ? want : most;
}
int64_t cols_splits(int64_t M) { return M < 64 ? M : 64; }

template <class T, int TPR, int NV, bool WHOLE>
void bwd_of(const NormArgs<T>& a, int64_t nb, int G, hipStream_t st) {
  constexpr int BWD_NTH = bwd_nth<T, TPR, NV>();
  const dim3 grid((unsigned)nb, 1, G);
  const bool cols = a.dgamma || a.dbeta;
  float* d0 = !cols ? nullptr : nb > 1 ? a.part : a.dgamma;
  float* d1 = !cols ? nullptr : nb > 1 ? a.part + a.N : a.dbeta;
  const int64_t d_g = nb > 1 ? nb * 2 * a.N : a.N, d_b = 2 * a.N;
  if (a.out.p && cols) k_norm_bwd<T, TPR, NV, true, true, WHOLE><<<grid, BWD_NTH, 0, st>>>(a, d0, d1, d_g, d_b);
  else if (cols) k_norm_bwd<T, TPR, NV, false, true, WHOLE><<<grid, BWD_NTH, 0, st>>>(a, d0, d1, d_g, d_b);
  else if (a.out.p) k_norm_bwd<T, TPR, NV, true, false, WHOLE><<<grid, BWD_NTH, 0, st>>>(a, d0, d1, d_g, d_b);
}

template <class T, int TPR, int NV>
void bwd(const NormArgs<T>& a, int64_t nb, int G, hipStream_t st) {
  if (a.N % EPP<T> == 0) bwd_of<T, TPR, NV, true>(a, nb, G, st);
  else bwd_of<T, TPR, NV, false>(a, nb, G, st);
}

}  // namespace

template <class T>
hipError_t launch_norm_fwd(const NormArgs<T>& args, int G, hipStream_t st) {
  if (args.M <= 0) return hipSuccess;
  NormArgs<T> a = args;
  a.inv_n = 1.0 / (double)a.N;
  const int64_t pc = cdiv(a.N, EPP<T>);
  if (pc <= 8) fwd<T, 8, 1, 256>(a, G, st);
  else if (pc <= 32) fwd<T, 32, 1, 256>(a, G, st);
  else if (pc <= 64) fwd<T, 64, 1, 256>(a, G, st);
  else if (pc <= 128) fwd<T, 64, 2, 256>(a, G, st);
  else if (pc <= 256) fwd<T, 256, 1, 256>(a, G, st);
  else if (pc <= 512) fwd<T, 256, 2, 256>(a, G, st);
  else if (pc <= 1024) fwd<T, 1024, 1, 1024>(a, G, st);
  else if (pc <= MAX_PIECES) fwd<T, 1024, 2, 1024>(a, G, st);
  else k_norm_fwd_long<T><<<dim3((unsigned)(a.M < 65536 ? a.M : 65536), 1, G), 1024, 0, st>>>(a);
  return hipGetLastError();
}

int64_t norm_part_floats(int elem_bytes, int64_t M, int64_t N) {
  const int64_t pc = cdiv(N, 16 / elem_bytes);
  const int64_t nb = pc <= MAX_PIECES ? bwd_blocks(elem_bytes, pc, M) : cols_splits(M);
  return nb > 1 ? nb * 2 * N : 0;
}

template <class T>
hipError_t launch_norm_bwd(const NormArgs<T>& a, int G, hipStream_t st) {
  const bool cols = a.dgamma || a.dbeta;
  if (a.M <= 0) {
    // sums over no rows
    for (float* sum : {a.dgamma, a.dbeta})
      if (sum)
        if (const hipError_t e = launch_zeros(sum, G * a.N, st); e != hipSuccess) return e;
    return hipSuccess;
  }
  const int64_t pc = cdiv(a.N, EPP<T>);
  int64_t nb;
  if (pc <= MAX_PIECES) {
    nb = bwd_blocks((int)sizeof(T), pc, a.M);
    if (pc <= 8) bwd<T, 8, 1>(a, nb, G, st);
    else if (pc <= 32) bwd<T, 32, 1>(a, nb, G, st);
    else if (pc <= 64) bwd<T, 64, 1>(a, nb, G, st);
    else if (pc <= 128) bwd<T, 64, 2>(a, nb, G, st);
    else if (pc <= 256) bwd<T, 256, 1>(a, nb, G, st);
    else if (pc <= 512) bwd<T, 512, 1>(a, nb, G, st);
    else if (pc <= 1024) bwd<T, 1024, 1>(a, nb, G, st);
    else bwd<T, 1024, 2>(a, nb, G, st);
  } else {
    nb = cols_splits(a.M);
    if (cols) {
      float* d0 = nb > 1 ? a.part : a.dgamma;
      float* d1 = nb > 1 ? a.part + a.N : a.dbeta;
      k_norm_cols<T><<<dim3((unsigned)cdiv(pc, 256), (unsigned)nb, G), 256, 0, st>>>(
          a, d0, d1, nb > 1 ? nb * 2 * a.N : a.N, 2 * a.N);
    }
    // after the column sums: dx may overwrite dy
    if (a.out.p) k_norm_bwd_long<T><<<dim3((unsigned)(a.M < 65536 ? a.M : 65536), 1, G), 1024, 0, st>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !cols || nb == 1) return e;
  return launch_slot_sum(a.part, nb * 2 * a.N, (int)nb, 2 * a.N, a.dgamma, a.N, a.dbeta, G, st);
}

hipError_t launch_slot_sum(const float* part, int64_t p_g, int n_slots, int64_t n, float* dst, int64_t n1, float* dst2,
                           int G, hipStream_t st) {
  // a launch's x dimension holds fewer than 2^32 threads
  const int64_t most = SLOT_RANGE / 32, blocks = cdiv(n, 32), ranges = cdiv(blocks, most);
  if (ranges > 65535) return hipErrorInvalidValue;
  if (ranges > 1)
    k_slot_sum<true><<<dim3((unsigned)most, (unsigned)ranges, G), 1024, 0, st>>>(part, p_g, n_slots, n, dst, n1, dst2);
  else
    k_slot_sum<false><<<dim3((unsigned)blocks, 1, G), 1024, 0, st>>>(part, p_g, n_slots, n, dst, n1, dst2);
  return hipGetLastError();
}

hipError_t launch_zeros(float* dst, int64_t n, hipStream_t st) {
  const int64_t most = 8192, blocks = cdiv(n, 256);
  k_zeros<<<(unsigned)(blocks < most ? blocks : most), 256, 0, st>>>(dst, n);
  return hipGetLastError();
}

template <class T>
hipError_t launch_colsum_rows(const Mat<const T>& m, int64_t M, int64_t N, int slots, float* part, int G,
                              hipStream_t st) {
  k_colsum_rows<T><<<dim3((unsigned)cdiv(cdiv(N, EPP<T>), 256), slots, G), 256, 0, st>>>(m, M, N, part);
  return hipGetLastError();
}

template <class T>
hipError_t launch_act_bwd(int act, const Mat<const T>& dy, const Mat<const T>& pre, const Mat<T>& g, int64_t M,
                          int64_t N, int G, hipStream_t st) {
  if (M <= 0) return hipSuccess;
  const bool flat = dy.ld == N && pre.ld == N && g.ld == N;   // one long row
  const int64_t rows = flat ? 1 : M, cols = flat ? M * N : N;
  const int64_t vpr = cdiv(cols, EPP<T>), total = rows * vpr;
  const int64_t most = cdiv(8192, G), blocks = cdiv(total, 256);
  const dim3 grid((unsigned)(blocks < most ? blocks : most), 1, G);
  // a turn adds up to 2^21 to the index
  if (total < (int64_t(1) << 31))
    k_act_bwd<T, uint32_t><<<grid, 256, 0, st>>>(act, dy, pre, g, rows, cols, (uint32_t)vpr);
  else
    k_act_bwd<T, uint64_t><<<grid, 256, 0, st>>>(act, dy, pre, g, rows, cols, (uint64_t)vpr);
  return hipGetLastError();
}

#define PIGAN_NORM_INST(T)                                                                                          \
  template hipError_t launch_norm_fwd<T>(const NormArgs<T>&, int, hipStream_t);                                     \
  template hipError_t launch_norm_bwd<T>(const NormArgs<T>&, int, hipStream_t);                                     \
  template hipError_t launch_colsum_rows<T>(const Mat<const T>&, int64_t, int64_t, int, float*, int, hipStream_t);    \
  template hipError_t launch_act_bwd<T>(int, const Mat<const T>&, const Mat<const T>&, const Mat<T>&, int64_t, int64_t, \
                                        int, hipStream_t);
PIGAN_NORM_INST(float)
PIGAN_NORM_INST(bf16)
PIGAN_NORM_INST(f16)

}  // namespace pigan
