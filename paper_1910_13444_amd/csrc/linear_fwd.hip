// Forward pass of the linear layer: y = act(x w^T + bias) + add, on tiles
// (mm.h) and on few rows; bf16 planes of fp32 matrices.
#include "mm.h"

namespace pigan {
namespace {

// ---------------------------------------------------------------------------
// Few rows.  A block forms a strip of 16 / P columns for up to 16 / P rows at a
// time; its waves take chunks of k in turn and read both operands' fragments
// straight from memory, U chunks in flight, so w streams through once and no wave
// waits for another before the end.  With P > 1 the 16 rows and columns of the
// matrix instruction hold P chunks of k at once, 16 / P rows and columns each:
// only the blocks on its diagonal, which pair a chunk with itself, are used.  The
// lanes of a load then cover 64 P consecutive bytes of a row of w, and there are P
// times as many blocks.  The waves' sums meet in LDS, in order.
// Four waves and P = 1 (many strips) are held to the registers of eight waves per
// SIMD: 2048 blocks are then on the chip at once (fp32 64 x 1024 x 8192 31 us, 34 with
// seven).
// Bound by the bytes of w (one row of x, 8192 -> 2048 bf16: 9.8 us, 3.4 TB/s, of
// which a launch by itself is 2; P = 1 15.6 us; fp32 14.9 us, 4.5 TB/s).
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

template <class T, int P, int NW, int U>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(P == 1 && NW == 4 ? 8 : 2)))
k_short_fwd(const MmArgs<T, T> p, uint32_t row_tiles, uint32_t ranges) {
  constexpr int CK = ShortMma<T>::CK, S = 16 / P, TURN = NW * P * CK;   // k per turn of all waves
  __shared__ float sums[NW][16][17];
  const int g = blockIdx.z;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // strips beyond a launch's x dimension: their range of gridDim.x strips is in y
  uint32_t tile = blockIdx.y;
  int64_t strip = blockIdx.x;
  if (ranges > 1) {
    const uint32_t range = tile / row_tiles;
    tile -= range * row_tiles;
    strip += (int64_t)range * gridDim.x;
  }
  const int64_t i0 = (int64_t)tile * S, j0 = strip * S;
  const int64_t i = i0 + (lane & (S - 1)), j = j0 + (lane & (S - 1));
  // rows past the end repeat the last one; their results are not stored
  const int64_t kl = (wave * P + ((lane & 15) / S)) * CK + (lane >> 4) * EPP<T>;
  const T* pa = p.a.p + g * p.a.gs + (i < p.o.I ? i : p.o.I - 1) * p.a.ld + kl;
  const T* pb = p.b.p + g * p.b.gs + (j < p.o.J ? j : p.o.J - 1) * p.b.ld + kl;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  // turns of U chunks that are whole for every wave, then the rest with zeros past the end
  const int64_t whole = p.K / (TURN * U) * (TURN * U);
  for (int64_t k0 = 0; k0 < whole; k0 += TURN * U) {
    piece_t a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) b[u] = *(const piece_u*)(pb + k0 + u * TURN);
#pragma unroll
    for (int u = 0; u < U; ++u) a[u] = *(const piece_u*)(pa + k0 + u * TURN);
#pragma unroll
    for (int u = 0; u < U; ++u) acc = ShortMma<T>::mma(b[u], a[u], acc);
  }
  for (int64_t k0 = whole; k0 < p.K; k0 += TURN) {
    const int64_t left = p.K - k0 - kl;
    acc = ShortMma<T>::mma(piece_load(pb + k0, left), piece_load(pa + k0, left), acc);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) sums[wave][lane & 15][4 * (lane >> 4) + r] = acc[r];
  __syncthreads();
  constexpr int OC = S < 8 ? 1 : S / 8;   // octets per row of the strip
  if (threadIdx.x < S * OC) {
    const int row = threadIdx.x / OC, c = 8 * (threadIdx.x % OC);
    float v[8], bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    for (int w = 0; w < NW; ++w)
#pragma unroll
      for (int q = 0; q < P; ++q)
#pragma unroll
        for (int e = 0; e < (S < 8 ? S : 8); ++e) v[e] += sums[w][q * S + row][q * S + c + e];
    const int64_t left = p.o.J - j0 - c, valid = left < S - c ? left : S - c;
    if (i0 + row < p.o.I && valid > 0) {
      vec_load<8>(p.o.bias ? p.o.bias + g * p.o.J : nullptr, j0 + c, p.o.J, 0.0f, bias);
      mm_finish<MM_FWD>(p.o, g, i0 + row, j0 + c, valid < 8 ? valid : 8, bias, v);
    }
  }
}

// ---------------------------------------------------------------------------
// bf16 planes of fp32 matrices: x0 and x1 are x and the rest rounded to eight
// significand bits (to nearest; towards zero where x0 would overflow), x2 what is
// left: all 24 bits.  With |x1| <= 2^-8 and |x2| <= 2^-17 for x in [1, 2), the three
// products that are left out (x1 y2, x2 y1, x2 y2) are at most 2^-24 of x y, of either
// sign.  (Planes cut towards zero lose up to 2^-21, always of the product's sign.)
// An infinity is (1, 0, inf) with its sign: x2 meets y0 alone, so it is multiplied by
// no zero but y's own, and x0 y2 is infinite with the right sign where y is, too.
// Bound by memory: 4 bytes read and 6 written per value (1001 x 2000, 513 x 2000 and
// 1001 x 513 in 7.4 us, 4.7 TB/s).
// ---------------------------------------------------------------------------
struct SplitSets {
  SplitSet s[3];
};

__device__ __forceinline__ float nearest8(float x) { return (float)(bf16)x; }

__device__ __forceinline__ void planes(float x, float& p0, float& p1, float& p2) {
  const bool inf = fabsf(x) == __builtin_inff();
  p0 = nearest8(x);
  if (fabsf(p0) == __builtin_inff()) p0 = inf ? copysignf(1.0f, x) : __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  const float rest = inf ? 0.0f : x - p0;
  p1 = nearest8(rest);
  p2 = inf ? x : rest - p1;
}

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
    for (int e = 0; e < 8; ++e) planes(f[e], p0[e], p1[e], p2[e]);
    store8(d, 8, p0);
    store8(d + plane, 8, p1);
    store8(d + 2 * plane, 8, p2);
  }
}

struct PackSets {
  PackSet s[3];
};

// Bound by memory; copies bits, so bf16 stands for either type (two of 4096 x 4096
// in the 11 us between the product's 107 and 118).
__global__ void __launch_bounds__(256) k_pack(const PackSets sets) {
  const PackSet s = sets.s[blockIdx.y];
  const int g = blockIdx.z;
  const int64_t vpr = s.Kp / 8, total = s.rows * vpr;
  const bf16* src = (const bf16*)s.src + g * s.gs;
  bf16* dst = (bf16*)s.dst + g * s.rows * s.Kp;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t r = q / vpr, c = (q - r * vpr) * 8;
    *(piece_t*)(dst + r * s.Kp + c) = piece_load(src + r * s.ld + c, s.cols - c);
  }
}

}  // namespace

// (a launch's x dimension holds fewer than 2^32 threads)
template <class T, int P, int NW, int U>
hipError_t short_of(const MmArgs<T, T>& a, int G, hipStream_t st) {
  constexpr int S = 16 / P;
  constexpr int64_t MOST = (int64_t(1) << 32) / (64 * NW) - 1;
  const int64_t strips = (a.o.J + S - 1) / S, tiles = (a.o.I + S - 1) / S, ranges = (strips + MOST - 1) / MOST;
  if (tiles * ranges > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((strips + ranges - 1) / ranges), (unsigned)(tiles * ranges), G);
  k_short_fwd<T, P, NW, U><<<grid, 64 * NW, 0, st>>>(a, (uint32_t)tiles, (uint32_t)ranges);
  return hipGetLastError();
}
template <class T, int P>
hipError_t short_of(const MmArgs<T, T>& a, int G, hipStream_t st) {
  // waves for the length of k, so that all of a row is in flight at once up to 8192
  return a.K > 2048 ? short_of<T, P, 8, 8>(a, G, st) : short_of<T, P, 4, 4>(a, G, st);
}

template <class T>
hipError_t launch_short_fwd(const MmArgs<T, T>& a, int G, hipStream_t st) {
  if (a.o.I < 1 || a.o.J < 1 || a.K < 1 || a.o.J > 0x7fffffff || G < 1 || G > 65535) return hipErrorInvalidValue;
  return a.o.I <= 4 ? short_of<T, 4>(a, G, st) : a.o.I <= 8 ? short_of<T, 2>(a, G, st) : short_of<T, 1>(a, G, st);
}

// the sets of a launch, and blocks for the largest of them; 0 where one cannot be
template <class Sets, class Set> unsigned sets_of(Sets& all, const Set* sets, int n) {
  int64_t most = 1;
  if (n < 1 || n > 3) return 0;
  for (int i = 0; i < n; ++i) {
    all.s[i] = sets[i];
    const int64_t blocks = (sets[i].rows * (sets[i].Kp / 8) + 255) / 256;
    if (sets[i].Kp % 8 || sets[i].Kp < sets[i].cols) return 0;
    if (blocks > most) most = blocks;
  }
  return (unsigned)(most < 4096 ? most : 4096);
}
hipError_t launch_split3(const SplitSet* sets, int n, int G, hipStream_t st) {
  SplitSets s{};
  const unsigned blocks = sets_of(s, sets, n);
  if (!blocks) return hipErrorInvalidValue;
  k_split3<<<dim3(blocks, n, G), 256, 0, st>>>(s, G);
  return hipGetLastError();
}
hipError_t launch_pack(const PackSet* sets, int n, int G, hipStream_t st) {
  PackSets s{};
  const unsigned blocks = sets_of(s, sets, n);
  if (!blocks) return hipErrorInvalidValue;
  k_pack<<<dim3(blocks, n, G), 256, 0, st>>>(s);
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
