// Device helpers of the matrix-core kernels: how tiles are dealt to the XCDs,
// product fragments against rows in memory, waits and barriers of staged
// operands, the transposing LDS read.
#pragma once
#include "common.h"

namespace pigan {

typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Workgroups are dispatched round-robin over the 8 XCDs (each with its own
// L2).  Map hardware block b to a logical tile so that every XCD walks one
// contiguous range of logical tiles: blocks that share an operand tile run on
// the same XCD at about the same time.  Bijective for any block count.
__device__ __forceinline__ int64_t xcd_remap(int64_t b, int64_t nb) {
  const int64_t q = nb / 8, r = nb % 8;
  const int64_t x = b % 8, local = b / 8;
  return x < r ? x * (q + 1) + local : r * (q + 1) + (x - r) * q + local;
}

// A 32 x 32 product fragment against rows in memory.  The matrix core leaves
// lane l with point l & 31 and four consecutive columns per register group q
// (8 q + 4 (l >> 5) ..).  Two lane exchanges turn that into 16-byte row pieces
// of which four lanes (l, l + 32, l + 16, l + 48) cover 64 consecutive bytes:
// v_permlane32_swap_b32 (16-bit storage only: gathers eight columns per lane),
// then v_permlane16_swap_b32, which trades the second piece of point p with
// the first piece of point p + 16.  Piece pair i, half j of a lane is then
// point (l & 15) + 16 j, columns FragPos::col(i) ...  Both swaps are their own
// inverse, so loads run the same steps backwards.  (32-byte pieces, without
// the second exchange, made the forward stores of five streams slower than
// staging whole rows through LDS: 1.82 against 1.76 ms at K = N = 512,
// 256,064 points; 64-byte pieces take neither barrier nor LDS.)
template <class T> struct FragRaw { u32x4 w[sizeof(T) == 2 ? 1 : 2][2]; };

__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ __forceinline__ void swap16(u32x4& a, u32x4& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto r = __builtin_amdgcn_permlane16_swap(a[e], b[e], false, false);
    a[e] = r[0];
    b[e] = r[1];
  }
}

// first column of the lane's piece in pair i (of a fragment's 32 columns)
template <class T>
__device__ __forceinline__ int frag_col(int lane, int i) {
  return sizeof(T) == 2 ? 16 * ((lane >> 4) & 1) + 8 * (lane >> 5) : 16 * i + 8 * ((lane >> 4) & 1) + 4 * (lane >> 5);
}

// both values rounded to the storage type, together: converted one at a time,
// fp16 results come from v_fma_mixlo_f16, which rounds the last operation to
// 16 bits at once and not after its fp32 rounding (80 of them in the five-stream
// reverse epilogue: other values in rare cases, and two instructions a pair)
template <class T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), T2));
}

// products layout -> pieces
template <class T>
__device__ __forceinline__ void frag_pack(FragRaw<T>& f, const f32x16& v) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int b = 8 * j;
      uint32_t a0 = pack2<T>(v[b], v[b + 1]), a1 = pack2<T>(v[b + 2], v[b + 3]);
      uint32_t b0 = pack2<T>(v[b + 4], v[b + 5]), b1 = pack2<T>(v[b + 6], v[b + 7]);
      swap32(a0, b0);
      swap32(a1, b1);
      f.w[0][j] = u32x4{a0, a1, b0, b1};
    }
    swap16(f.w[0][0], f.w[0][1]);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) f.w[i][j][e] = __float_as_uint(v[8 * i + 4 * j + e]);
      swap16(f.w[i][0], f.w[i][1]);
    }
  }
}

// pieces -> products layout: first the lane exchanges of the whole fragment,
// then the lane's values of register group q
template <class T>
__device__ __forceinline__ void frag_unswap(FragRaw<T>& f) {
#pragma unroll
  for (int i = 0; i < (sizeof(T) == 2 ? 1 : 2); ++i) swap16(f.w[i][0], f.w[i][1]);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t x = f.w[0][j][c], y = f.w[0][j][2 + c];
        swap32(x, y);
        f.w[0][j][c] = x;
        f.w[0][j][2 + c] = y;
      }
  }
}
template <class T>
__device__ __forceinline__ void frag_group(const FragRaw<T>& f, int q, float* v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2)
      v[e] = Elem<T>::to_f(__builtin_bit_cast(T, (uint16_t)(f.w[0][q >> 1][2 * (q & 1) + (e >> 1)] >> (16 * (e & 1)))));
    else
      v[e] = __uint_as_float(f.w[q >> 1][q & 1][e]);
  }
}

// Barrier for data exchanged through LDS only.  __syncthreads() also fences
// global memory, which makes every wave wait for all of its outstanding global
// loads (s_waitcnt vmcnt(0)) and so defeats loads prefetched stages ahead;
// here only the LDS writes must be complete before the barrier.
__device__ __forceinline__ void lds_sync() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Wait until at most N vector-memory operations of this wave are outstanding
// (N is an immediate).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

typedef __attribute__((address_space(3))) void* lds_ptr_t;

// Transposing LDS read of 16-bit elements: within each 16-lane group, lanes
// 4r..4r+3 address the four 8-byte pieces of row r of a 4 x 16 block and lane i
// receives column i of the block.
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 tr_bf16x4;
typedef __attribute__((__vector_size__(4 * sizeof(__fp16)))) __fp16 tr_f16x4;

template <class T>
__device__ __forceinline__ u32x2 lds_read_tr(const char* p) {
  if constexpr (__is_same(T, bf16)) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                                         (__attribute__((address_space(3))) tr_bf16x4*)(p)));
  } else {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4f16(
                                         (__attribute__((address_space(3))) tr_f16x4*)(p)));
  }
}

}  // namespace pigan
