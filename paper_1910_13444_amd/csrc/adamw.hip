// AdamW over many tensors at once, with states in 32 or in 8 bits, the norm of their
// gradients, and the values of 8-bit states, for gfx950.
//
//   g' = coef g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p -= lr (m c1 / (sqrt(v c2) + eps) + decay p),   c = 1 / (1 - b^t)
//
// A table says which piece of which tensor a block takes, so one launch does all.
// States are fp32 values; everything between is formed in fp64 and rounded once: a step
// moves 16 to 30 bytes an element, which leaves the time, and what an 8-bit state rounds
// to does not depend on the order of a sum.
//
// 8-bit states are codes of QBLOCK elements with the largest size s among them:
//   m = s q |q| / 127^2,  q = sign(m) round(127 sqrt(|m| / s)),
//   v = s q^4 / 255^4,    q = round(255 (v / s)^(1/4)), at least 1 for v > 0.
// The root of v is what divides m: in it both codes are squares, whose steps are fine near
// the block's largest (0.8 % of it) and reach down to 2^-14 and 2^-16 of it.  A v of 0
// beside an m that is not would divide by eps alone.  A block that holds a state that is
// not finite has the scale NaN and codes 0.
#include "adamw.h"

#include <algorithm>
#include <type_traits>

#include "piece.h"

namespace pigan {
namespace {

constexpr int NTH = 256;

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
  return v;
}
// of values >= 0, by lane permutes: rows of 16 lanes, then rows to the ones behind them
__device__ __forceinline__ float wave_max(float v) {
  auto with = [&](auto ctrl, auto rows) {
    const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl.value, rows.value, 0xf, false);
    v = fmaxf(v, __builtin_bit_cast(float, o));
  };
  using std::integral_constant;
  with(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // row_shr 1, 2, 4, 8
  with(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  with(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  with(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  with(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // row_bcast 15, 31
  with(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

typedef uint32_t half4 __attribute__((ext_vector_type(2), aligned(2)));

// Pointers to global memory: those that a table holds would else be taken for any memory's,
// whose accesses wait for LDS too.
template <class T> using G = __attribute__((address_space(1))) T*;

// Vectors that may start at any element.  `stream`: past the caches, AdamwArgs::stream.
template <class V, class T> __device__ __forceinline__ V get(G<const T> p, bool stream) {
  V v;
  if (stream) {
    asm volatile("; streamed");   // else the compiler joins both to a plain access
    v = __builtin_nontemporal_load((G<const V>)p);
    asm volatile("; streamed");
  } else {
    v = *(G<const V>)p;
  }
  return v;
}
template <class V, class T> __device__ __forceinline__ void put(G<T> p, const V& v, bool stream) {
  if (stream) {
    asm volatile("; streamed");
    __builtin_nontemporal_store(v, (G<V>)p);
    asm volatile("; streamed");
  } else {
    *(G<V>)p = v;
  }
}

// four elements of a gradient, zeros past `valid`
__device__ __forceinline__ void load_grad(G<const void> g, int dt, int64_t i, int64_t valid, float (&f)[4], bool stream = false) {
  if (dt == PIGAN_FP32) {
    const G<const float> p = (G<const float>)g + i;
    if (valid >= 4) {
      const f32x4u v = get<f32x4u>(p, stream);
      for (int e = 0; e < 4; ++e) f[e] = v[e];
    } else {
      for (int e = 0; e < 4; ++e) f[e] = e < valid ? p[e] : 0.0f;
    }
    return;
  }
  const G<const uint16_t> p = (G<const uint16_t>)g + i;
  uint16_t h[4];
  if (valid >= 4) {
    const half4 v = get<half4>(p, stream);
    __builtin_memcpy(h, &v, 8);
  } else {
    for (int e = 0; e < 4; ++e) h[e] = e < valid ? p[e] : 0;
  }
  for (int e = 0; e < 4; ++e)
    f[e] = dt == PIGAN_BF16 ? __uint_as_float((uint32_t)h[e] << 16) : (float)__builtin_bit_cast(f16, h[e]);
}

__device__ __forceinline__ void load4(G<const float> p, int64_t valid, float (&f)[4], bool stream) {
  if (valid >= 4) {
    const f32x4u v = get<f32x4u>(p, stream);
    for (int e = 0; e < 4; ++e) f[e] = v[e];
  } else {
    for (int e = 0; e < 4; ++e) f[e] = e < valid ? p[e] : 0.0f;
  }
}
__device__ __forceinline__ void store4(G<float> p, int64_t valid, const float (&f)[4], bool stream) {
  if (valid >= 4) {
    f32x4u v;
    for (int e = 0; e < 4; ++e) v[e] = f[e];
    put<f32x4u>(p, v, stream);
  } else {
    for (int e = 0; e < 4; ++e)
      if (e < valid) p[e] = f[e];
  }
}
template <class T>
__device__ __forceinline__ void store_copy4(G<T> p, int64_t valid, const float (&f)[4], bool stream) {
  T h[4];
  for (int e = 0; e < 4; ++e) h[e] = Elem<T>::from_f(f[e]);
  if (valid >= 4) {
    half4 v;
    __builtin_memcpy(&v, h, 8);
    put<half4>(p, v, stream);
  } else {
    for (int e = 0; e < 4; ++e)
      if (e < valid) p[e] = h[e];
  }
}
__device__ __forceinline__ void store_copy(const TensorEntry& t, int64_t i, int64_t valid, const float (&f)[4], bool stream) {
  if (!t.copy) return;
  if (t.copy_dt == PIGAN_BF16) store_copy4((G<bf16>)t.copy + i, valid, f, stream);
  else store_copy4((G<f16>)t.copy + i, valid, f, stream);
}

// ---------------------------------------------------------------------------
// The step.
// ---------------------------------------------------------------------------
// 1 / d in fp64 from the hardware's (2^-24): two Newton steps
__device__ __forceinline__ double rcp64_full(double d) {
  double r = __builtin_amdgcn_rcp(d);
  r += r * (1.0 - d * r);
  return r + r * (1.0 - d * r);
}

constexpr double TOP_M = 127.0 * 127.0, TOP_V = 255.0 * 255.0 * 255.0 * 255.0;
// s / top, rounded once: top times it is s again, as sums of short numbers m and v may lie
// halfway between two fp32 values
__device__ __forceinline__ double unit_of(float s, double top) {
  const double inv = 1.0 / top, q = s * inv;   // a constant
  return __builtin_fma(__builtin_fma(-top, q, (double)s), inv, q);
}

// of a tensor: p' = keep p - by m / (sqrt(c2 v) + eps)
struct Coefs { double coef, c2, keep, by; };
__device__ __forceinline__ Coefs coefs_of(const AdamwArgs& a, double decay) {
  const double c1 = a.corr ? a.corr[0] : a.c1, c2 = a.corr ? a.corr[1] : a.c2;
  return {a.coef ? a.scale * (double)*a.coef : a.scale, c2, 1.0 - a.lr * decay, a.lr * c1};
}

// the new states, as fp32 values, and the new parameter.  Root and quotient are the
// hardware's fp64 approximations (2^-24.2, 2^-24.4) with a Newton step each (1e-14).
__device__ __forceinline__ void update(const AdamwArgs& a, const Coefs& k, float g, double m, double v, float& p, float& mn,
                                       float& vn) {
  const double gs = k.coef * g;
  mn = (float)(a.b1 * m + a.nb1 * gs);
  vn = (float)(a.b2 * v + a.nb2 * gs * gs);
  // a v of 0 is a number with a root's reciprocal; of an infinite one, whose root comes out as
  // NaN, update_over sees
  const double s = (double)vn * k.c2 + 1e-300;
  const double r = __builtin_amdgcn_rsq(s), root = s * r, d = root + root * (0.5 - root * (0.5 * r)) + a.eps;
  double q = __builtin_amdgcn_rcp(d);
  q += q * (1.0 - d * q);
  p = (float)(k.keep * (double)p - k.by * (double)mn * q);
}

// Parameters beside a v that has passed fp32: m / sqrt(v) is 0, NaN for an infinite m.  One
// branch for four elements, and p read again: a branch in `update` cost 33.6 M parameters
// 2.5 us of 165, selects there 21.2 M with 8-bit states 3 of 70.
__device__ __forceinline__ void update_over(const Coefs& k, G<const float> p, int64_t valid, const float (&mf)[4],
                                            const float (&vf)[4], float (&pf)[4]) {
  if (fmaxf(fmaxf(vf[0], vf[1]), fmaxf(vf[2], vf[3])) <= 3.4028234663852886e38f) return;
  for (int e = 0; e < 4; ++e)
    if (e < valid && vf[e] > 3.4028234663852886e38f) pf[e] = (float)(k.keep * (double)p[e] - 0.0 * (double)mf[e]);
}

// Four elements a thread, one turn a block, in order: as a copy, which is fastest that way
// (1 GiB: 6.2 TB/s, blocks of four turns 4.9).  Bound by memory: 33.6 M parameters with bf16
// copies 174 us (5.8 TB/s; in blocks of 4096 elements 190).
__global__ void __launch_bounds__(NTH) k_adamw32(const AdamwArgs a) {
  if (a.skip && *a.skip) return;   // one flag for the whole launch
  const TensorPiece w = a.pieces[blockIdx.x];
  const TensorEntry t = a.entries[w.tensor];
  const Coefs k = coefs_of(a, t.decay);
  const int64_t i = (int64_t)w.piece * PIECE + threadIdx.x * 4, valid = t.n - i;
  if (valid <= 0) return;
  const G<float> m = (G<float>)a.m + t.state, v = (G<float>)a.v + t.state;
  float pf[4], gf[4], mf[4], vf[4];
  load4((G<const float>)t.p + i, valid, pf, a.stream);
  load_grad((G<const void>)t.g, t.g_dt, i, valid, gf, a.stream);
  load4(m + i, valid, mf, a.stream);
  load4(v + i, valid, vf, a.stream);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double mo = mf[e], vo = vf[e];
    update(a, k, gf[e], mo, vo, pf[e], mf[e], vf[e]);
  }
  update_over(k, (G<const float>)t.p + i, valid, mf, vf, pf);
  store4((G<float>)t.p + i, valid, pf, a.stream);
  store4(m + i, valid, mf, a.stream);
  store4(v + i, valid, vf, a.stream);
  store_copy(t, i, valid, pf, a.stream);
}

// a b - c d, its sign exact: |a|, |c| are fp32 values and b, d whole numbers below 2^53
__device__ __forceinline__ double difference(double a, double b, double c, double d) {
#pragma clang fp contract(off)
  const double p = a * b, q = c * d;
  return (p - q) + (__builtin_fma(a, b, -p) - __builtin_fma(c, d, -q));
}

// The code of size x among a largest of s: the nearest whole number to top (x / s)^(1/2), or
// 255 (x / s)^(1/4), an even one where two are as near (x = s / 4 is halfway between 63 and
// 64, s / 16 between 127 and 128); inv = top^2 / s or top^4 / s.  The fp32 root y is off by
// less than 6e-5 codes (2e-7 of 255), so only within 2^-12 of a halfway point n + 1/2 the
// whole powers decide, x (2 top)^2 against s (2 n + 1)^2.
template <bool FOURTH>
__device__ __forceinline__ int code_of(float x, float s, double inv) {
  float y = __builtin_amdgcn_sqrtf((float)((double)x * inv));
  if constexpr (FOURTH) y = __builtin_amdgcn_sqrtf(y);
  const float c = rintf(y);
  int q = (int)c;
  if (fabsf(y - c) > 0.5f - 0x1p-12f) {
    const int n = (int)floorf(y);
    const double h = 2 * n + 1, h2 = h * h;
    const double d = FOURTH ? difference(x, 16.0 * TOP_V, s, h2 * h2) : difference(x, 4.0 * TOP_M, s, h2);
    q = d > 0.0 || (d == 0.0 && (n & 1)) ? n + 1 : n;
  }
  return q;
}

// A wave takes a block of states at a time, four elements a lane.  Memory and the vector units
// (a hundred instructions an element, most in fp64) take the same time: 21.2 M parameters with
// bf16 copies 72 us (5.3 TB/s); with library roots and quotients and every code's borders in
// fp64 131 us.
__global__ void __launch_bounds__(NTH) k_adamw8(const AdamwArgs a) {
  if (a.skip && *a.skip) return;
  const TensorPiece w = a.pieces[blockIdx.x];
  const TensorEntry t = a.entries[w.tensor];
  const Coefs k = coefs_of(a, t.decay);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = (int64_t)w.piece * PIECE + wave * QBLOCK;
  if (b >= t.n) return;
  const int64_t i = b + lane * 4, valid = t.n - i, at = t.state + i, qb = (t.state + b) / QBLOCK;
  float pf[4] = {0, 0, 0, 0}, gf[4] = {0, 0, 0, 0}, mf[4], vf[4];
  if (valid > 0) {
    load4((G<const float>)t.p + i, valid, pf, a.stream);
    load_grad((G<const void>)t.g, t.g_dt, i, valid, gf, a.stream);
  }
  // states are there to the end of the block
  const uint32_t mq = get<uint32_t>((G<const int8_t>)a.m + at, a.stream), vq = get<uint32_t>((G<const uint8_t>)a.v + at, a.stream);
  const double ms = unit_of(a.m_scale[qb], TOP_M), vs = unit_of(a.v_scale[qb], TOP_V);
  float mmax = 0.0f, vmax = 0.0f, none = 0.0f;   // `none` is 0 unless a state is not finite
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int qm = (int)(int8_t)(mq >> (8 * e));
    const uint32_t qv = (vq >> (8 * e)) & 255, q2 = qv * qv;
    update(a, k, gf[e], (double)(qm * abs(qm)) * ms, (double)(q2 * q2) * vs, pf[e], mf[e], vf[e]);
    if (e >= valid) mf[e] = vf[e] = 0.0f;
    mmax = fmaxf(mmax, fabsf(mf[e]));
    vmax = fmaxf(vmax, vf[e]);
    none += 0.0f * mf[e];
    none += 0.0f * vf[e];
  }
  mmax = wave_max(mmax);
  vmax = wave_max(vmax);
  const bool all = __all(none == 0.0f);
  const double mi = mmax > 0.0f ? TOP_M * rcp64_full((double)mmax) : 0.0, vi = vmax > 0.0f ? TOP_V * rcp64_full((double)vmax) : 0.0;
  uint32_t mo = 0, vo = 0;
  if (all) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int q = min(code_of<false>(fabsf(mf[e]), mmax, mi), 127), u = min(code_of<true>(vf[e], vmax, vi), 255);
      mo |= (uint32_t)(uint8_t)(mf[e] < 0.0f ? -q : q) << (8 * e);
      vo |= (uint32_t)(vf[e] > 0.0f ? max(u, 1) : 0) << (8 * e);
    }
  }
  put<uint32_t>((G<int8_t>)a.m + at, mo, a.stream);
  put<uint32_t>((G<uint8_t>)a.v + at, vo, a.stream);
  if (lane == 0) {
    a.m_scale[qb] = all ? mmax : __builtin_nanf("");
    a.v_scale[qb] = all ? vmax : __builtin_nanf("");
  }
  if (valid > 0) {
    if (!all) update_over(k, (G<const float>)t.p + i, valid, mf, vf, pf);
    store4((G<float>)t.p + i, valid, pf, a.stream);
    store_copy(t, i, valid, pf, a.stream);
  }
}

__global__ void k_adamw_begin(double b1, double b2, int32_t* step, const int32_t* skip, double* corr) {
  int32_t t = *step;
  if (!(skip && *skip)) *step = ++t;
  const double n = t < 1 ? 1.0 : (double)t;
  corr[0] = 1.0 / (1.0 - pow(b1, n));
  corr[1] = 1.0 / (1.0 - pow(b2, n));
}

// ---------------------------------------------------------------------------
// The gradients' norm: a sum of squares per block in fp64, joined in a fixed order.  Bound by
// memory: 33.6 M fp32 24 us (5.6 TB/s) and 4 us for the join, a launch of one block.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(NTH) k_grad_squares(const TensorEntry* __restrict__ entries,
                                                      const TensorPiece* __restrict__ pieces, int64_t n_pieces,
                                                      double* __restrict__ part) {
  __shared__ double sums[NTH / 64];
  constexpr int U = 4;   // pieces under way
  double s = 0.0;
  for (int64_t b = (int64_t)blockIdx.x * U; b < n_pieces; b += (int64_t)gridDim.x * U) {
    float f[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const TensorPiece w = pieces[min(b + u, n_pieces - 1)];
      const TensorEntry& t = entries[w.tensor];
      const int64_t i = (int64_t)w.piece * PIECE + threadIdx.x * 4;
      load_grad((G<const void>)t.g, t.g_dt, i, b + u < n_pieces ? t.n - i : 0, f[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) s += (double)f[u][e] * (double)f[u][e];
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < NTH / 64; ++i) s += sums[i];
    part[blockIdx.x] = s;
  }
}

__global__ void __launch_bounds__(1024) k_grad_norm(const double* __restrict__ part, int n, double max_norm, double scale,
                                                    float* norm, float* coef, int32_t* nonfinite) {
  __shared__ double sums[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) s += sums[i];
    const double v = scale * sqrt(s);
    if (norm) *norm = (float)v;
    if (coef) *coef = (float)(v > max_norm ? scale * (max_norm / v) : scale);
    if (nonfinite) *nonfinite = !__builtin_isfinite(v);
  }
}

// Bound by memory: 21.2 M values of m and v 38 us (5.6 TB/s).
__global__ void __launch_bounds__(NTH) k_state_values(int64_t n, const int8_t* __restrict__ m, const float* __restrict__ m_scale,
                                                      const uint8_t* __restrict__ v, const float* __restrict__ v_scale,
                                                      float* __restrict__ m_out, float* __restrict__ v_out, bool stream) {
  for (int64_t i = ((int64_t)blockIdx.x * NTH + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * NTH * 4) {
    float f[4];
    if (m_out) {
      const uint32_t q = get<uint32_t>((G<const int8_t>)m + i, stream);
      const double s = unit_of(m_scale[i / QBLOCK], TOP_M);
      for (int e = 0; e < 4; ++e) {
        const int c = (int)(int8_t)(q >> (8 * e));
        f[e] = (float)((double)(c * abs(c)) * s);
      }
      store4((G<float>)m_out + i, 4, f, stream);
    }
    if (v_out) {
      const uint32_t q = get<uint32_t>((G<const uint8_t>)v + i, stream);
      const double s = unit_of(v_scale[i / QBLOCK], TOP_V);
      for (int e = 0; e < 4; ++e) {
        const uint32_t c = (q >> (8 * e)) & 255;
        f[e] = (float)((double)(c * c * c * c) * s);
      }
      store4((G<float>)v_out + i, 4, f, stream);
    }
  }
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, int bits, int64_t n_pieces, hipStream_t st) {
  // a launch's x dimension holds fewer than 2^32 threads
  const int64_t most = int64_t(1) << 23;
  for (int64_t at = 0; at < n_pieces; at += most) {
    AdamwArgs part = a;
    part.pieces += at;
    const unsigned blocks = (unsigned)std::min(most, n_pieces - at);
    if (bits == 8) k_adamw8<<<blocks, NTH, 0, st>>>(part);
    else k_adamw32<<<blocks, NTH, 0, st>>>(part);
  }
  return hipGetLastError();
}

hipError_t launch_adamw_begin(double b1, double b2, int32_t* step, const int32_t* skip, double* corr, hipStream_t st) {
  k_adamw_begin<<<1, 1, 0, st>>>(b1, b2, step, skip, corr);
  return hipGetLastError();
}

int64_t grad_norm_blocks(int64_t n_pieces) { return std::max<int64_t>(1, std::min<int64_t>((n_pieces + 3) / 4, 2048)); }

hipError_t launch_grad_norm(const TensorEntry* entries, const TensorPiece* pieces, int64_t n_pieces, double max_norm,
                            double scale, double* part, float* norm, float* coef, int32_t* nonfinite, hipStream_t st) {
  const int blocks = (int)grad_norm_blocks(n_pieces);
  k_grad_squares<<<blocks, NTH, 0, st>>>(entries, pieces, n_pieces, part);
  k_grad_norm<<<1, 1024, 0, st>>>(part, blocks, max_norm, scale, norm, coef, nonfinite);
  return hipGetLastError();
}

hipError_t launch_state_values(int64_t n, const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale,
                               float* m_out, float* v_out, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const int64_t blocks = std::min<int64_t>((n + NTH * 4 - 1) / (NTH * 4), 1 << 20);
  k_state_values<<<(unsigned)blocks, NTH, 0, st>>>(n, m, m_scale, v, v_scale, m_out, v_out, n * 5.0 * (!!m_out + !!v_out) > STREAM_BYTES);
  return hipGetLastError();
}

}  // namespace pigan
