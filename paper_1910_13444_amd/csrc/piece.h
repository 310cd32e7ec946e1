// 16-byte pieces of matrix rows that may start at any element address: the
// accesses are under-aligned vector types, the last piece of a row goes
// element by element.
#pragma once
#include "common.h"

namespace pigan {

typedef uint32_t piece_t __attribute__((ext_vector_type(4)));
typedef uint32_t piece_u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

template <class T> constexpr int EPP = 16 / (int)sizeof(T);   // elements per piece

// the first `valid` elements of a piece (any number, also none), zeros behind them
template <class T>
__device__ __forceinline__ piece_t piece_load(const T* p, int64_t valid) {
  if (valid >= EPP<T>) return *(const piece_u*)p;
  piece_t v;
  T e[EPP<T>];
#pragma unroll
  for (int i = 0; i < EPP<T>; ++i) e[i] = i < valid ? p[i] : Elem<T>::from_f(0.0f);
  __builtin_memcpy(&v, e, 16);
  return v;
}

template <class T>
__device__ __forceinline__ void piece_store(T* p, int64_t valid, const float* f) {
  T e[EPP<T>];
#pragma unroll
  for (int i = 0; i < EPP<T>; ++i) e[i] = Elem<T>::from_f(f[i]);
  if (valid >= EPP<T>) {
    piece_t v;
    __builtin_memcpy(&v, e, 16);
    *(piece_u*)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < EPP<T>; ++i)
      if (i < valid) p[i] = e[i];
  }
}

template <class T>
__device__ __forceinline__ void piece_floats(const piece_t& v, float* f) {
  T e[EPP<T>];
  __builtin_memcpy(e, &v, 16);
#pragma unroll
  for (int i = 0; i < EPP<T>; ++i) f[i] = Elem<T>::to_f(e[i]);
}

// E entries from column c of an fp32 vector of N (`fill` past the end, and
// where there is no vector)
template <int E>
__device__ __forceinline__ void vec_load(const float* p, int64_t c, int64_t N, float fill, float* f) {
  if (p && c + E <= N) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const f32x4u v = *(const f32x4u*)(p + c + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[i + j] = v[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = p && c + i < N ? p[c + i] : fill;
  }
}

// eight consecutive elements of a row, as one or two pieces
template <class T>
__device__ __forceinline__ void load8(const T* p, int64_t valid, float* f) {
#pragma unroll
  for (int i = 0; i < 8; i += EPP<T>) piece_floats<T>(piece_load(p + i, valid - i), f + i);
}
template <class T>
__device__ __forceinline__ void store8(T* p, int64_t valid, const float* f) {
#pragma unroll
  for (int i = 0; i < 8; i += EPP<T>) piece_store(p + i, valid - i, f + i);
}

}  // namespace pigan
