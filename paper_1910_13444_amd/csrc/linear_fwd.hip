// Forward pass of the linear layer: y = act(x w^T + bias) + add, on tiles
// (mm.h) and on few rows; bf16 planes of fp32 matrices.
#include "mm.h"

namespace pigan {
namespace {

// ---------------------------------------------------------------------------
// Few rows.  A block forms 16 x 16 results; its waves take chunks of k in turn
// and read both operands' fragments from memory (w streams through once, 16
// bytes a lane), U chunks in flight.  Their sums meet in LDS, in order.
// ---------------------------------------------------------------------------
template <class T> struct ShortMma;
template <> struct ShortMma<bf16> {
  static constexpr int CK = 32;   // k per chunk: 8 values in each of four lane groups
  static __device__ __forceinline__ f32x4 mma(const piece_t& a, const piece_t& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct ShortMma<f16> {
  static constexpr int CK = 32;
  static __device__ __forceinline__ f32x4 mma(const piece_t& a, const piece_t& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <> struct ShortMma<float> {
  static constexpr int CK = 16;   // 4 values in each group: four products of 4 k
  static __device__ __forceinline__ f32x4 mma(const piece_t& a, const piece_t& b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
};

template <class T, int NW, int U>
__global__ void __launch_bounds__(64 * NW) k_short_fwd(const MmArgs<T, T> p) {
  constexpr int CK = ShortMma<T>::CK;
  __shared__ float sums[NW][16][17];
  const int g = blockIdx.z;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i0 = (int64_t)blockIdx.y * 16, j0 = (int64_t)blockIdx.x * 16;
  const int64_t i = i0 + (lane & 15), j = j0 + (lane & 15);
  // rows past the end repeat the last one; their results are not stored
  const T* pa = p.a.p + g * p.a.gs + (i < p.o.I ? i : p.o.I - 1) * p.a.ld;
  const T* pb = p.b.p + g * p.b.gs + (j < p.o.J ? j : p.o.J - 1) * p.b.ld;
  const int kl = (lane >> 4) * EPP<T>;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  // whole turns of U chunks for every wave, then the rest with zeros past the end
  const int64_t whole = p.K / (NW * CK * U) * (NW * CK * U);
  pa += wave * CK + kl;
  pb += wave * CK + kl;
  for (int64_t k0 = 0; k0 < whole; k0 += NW * CK * U) {
    piece_t a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      b[u] = *(const piece_u*)(pb + k0 + u * NW * CK);
      a[u] = *(const piece_u*)(pa + k0 + u * NW * CK);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) acc = ShortMma<T>::mma(b[u], a[u], acc);
  }
  for (int64_t k0 = whole; k0 < p.K; k0 += NW * CK) {
    const int64_t left = p.K - k0 - wave * CK - kl;
    acc = ShortMma<T>::mma(piece_load(pb + k0, left), piece_load(pa + k0, left), acc);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) sums[wave][lane & 15][4 * (lane >> 4) + r] = acc[r];
  __syncthreads();
  if (threadIdx.x < 32) {
    const int row = threadIdx.x >> 1, c = 8 * (threadIdx.x & 1);
    float v[8], bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = sums[0][row][c + e];
    for (int w = 1; w < NW; ++w)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += sums[w][row][c + e];
    if (i0 + row < p.o.I && j0 + c < p.o.J) {
      vec_load<8>(p.o.bias ? p.o.bias + g * p.o.J : nullptr, j0 + c, p.o.J, 0.0f, bias);
      mm_finish<MM_FWD>(p.o, g, i0 + row, j0 + c, bias, v);
    }
  }
}

// ---------------------------------------------------------------------------
// bf16 planes of fp32 matrices: x0 and x1 are x and the rest cut to eight
// significand bits (towards zero, so that no plane overflows), x2 what is left:
// all 24 bits.  An infinity or NaN goes to x0 alone.
// ---------------------------------------------------------------------------
struct SplitSets {
  SplitSet s[3];
};

__device__ __forceinline__ float cut8(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

__global__ void __launch_bounds__(256) k_split3(const SplitSets sets, int G) {
  const SplitSet s = sets.s[blockIdx.y];
  const int g = blockIdx.z;
  const int64_t vpr = s.Kp / 8, total = s.rows * vpr, plane = G * s.rows * s.Kp;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t r = q / vpr, c = (q - r * vpr) * 8;
    float f[8];
    load8(s.src + g * s.gs + r * s.ld + c, s.cols - c, f);
    bf16* d = s.dst + (g * s.rows + r) * s.Kp + c;
    float p0[8], p1[8], p2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool fin = __builtin_isfinite(f[e]);
      p0[e] = fin ? cut8(f[e]) : f[e];
      const float rest = fin ? f[e] - p0[e] : 0.0f;
      p1[e] = cut8(rest);
      p2[e] = rest - p1[e];
    }
    store8(d, 8, p0);
    store8(d + plane, 8, p1);
    store8(d + 2 * plane, 8, p2);
  }
}

}  // namespace

template <class T>
hipError_t launch_short_fwd(const MmArgs<T, T>& a, int G, hipStream_t st) {
  const int64_t bx = (a.o.J + 15) / 16, by = (a.o.I + 15) / 16;
  if (a.o.I < 1 || a.o.J < 1 || a.K < 1 || by > 65535 || bx > 0x7fffffff || G < 1 || G > 65535)
    return hipErrorInvalidValue;
  const dim3 grid((unsigned)bx, (unsigned)by, G);
  if (a.K > 1024) k_short_fwd<T, 16, 4><<<grid, 1024, 0, st>>>(a);
  else k_short_fwd<T, 4, 2><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_split3(const SplitSet* sets, int n, int G, hipStream_t st) {
  if (n < 1 || n > 3) return hipErrorInvalidValue;
  SplitSets s{};
  int64_t most = 1;
  for (int i = 0; i < n; ++i) {
    s.s[i] = sets[i];
    const int64_t blocks = (sets[i].rows * (sets[i].Kp / 8) + 255) / 256;
    if (sets[i].Kp % 8 || sets[i].Kp < sets[i].cols) return hipErrorInvalidValue;
    if (blocks > most) most = blocks;
  }
  k_split3<<<dim3((unsigned)(most < 4096 ? most : 4096), n, G), 256, 0, st>>>(s, G);
  return hipGetLastError();
}

template <class T, class TO>
hipError_t launch_mm_fwd(const MmArgs<T, TO>& a, int tile, bool direct, int G, hipStream_t st) {
  return mm_launch<T, TO, MM_FWD>(a, tile, direct, G, st);
}
template <class TO> hipError_t launch_mm_join_fwd(const MmOut<TO>& o, int G, hipStream_t st) {
  return join_launch<MM_FWD>(o, G, st);
}

template hipError_t launch_short_fwd<float>(const MmArgs<float, float>&, int, hipStream_t);
template hipError_t launch_short_fwd<bf16>(const MmArgs<bf16, bf16>&, int, hipStream_t);
template hipError_t launch_short_fwd<f16>(const MmArgs<f16, f16>&, int, hipStream_t);
template hipError_t launch_mm_fwd<bf16, bf16>(const MmArgs<bf16, bf16>&, int, bool, int, hipStream_t);
template hipError_t launch_mm_fwd<f16, f16>(const MmArgs<f16, f16>&, int, bool, int, hipStream_t);
template hipError_t launch_mm_fwd<bf16, float>(const MmArgs<bf16, float>&, int, bool, int, hipStream_t);
template hipError_t launch_mm_join_fwd<bf16>(const MmOut<bf16>&, int, hipStream_t);
template hipError_t launch_mm_join_fwd<f16>(const MmOut<f16>&, int, hipStream_t);
template hipError_t launch_mm_join_fwd<float>(const MmOut<float>&, int, hipStream_t);

}  // namespace pigan
