// Launchers of layer norm and of the elementwise reverse pass (norm.hip).
#pragma once
#include "common.h"

namespace pigan {

// A matrix operand of a launch; row r of group g at p + g * gs + r * ld.
template <class T> struct Mat {
  T* p; int64_t ld; int64_t gs;
};

template <class T> struct NormArgs {
  Mat<const T> x; Mat<const T> dy; Mat<const T> add;   // add.p may be null
  Mat<T> out;                                          // y, or dx (null: not wanted)
  const float* gamma; const float* beta;               // null: ones, zeros
  float* mean; float* rstd;                            // forward: outputs or null; backward: inputs
  float* dgamma; float* dbeta;                         // backward: outputs or null
  float* part;                                         // backward: partial column sums
  int64_t M, N;
  float eps;
  double inv_n;                                        // forward: 1 / N, set by the launcher
};

template <class T> hipError_t launch_norm_fwd(const NormArgs<T>& a, int G, hipStream_t st);
// floats of NormArgs::part per group (0: none)
int64_t norm_part_floats(int elem_bytes, int64_t M, int64_t N);
template <class T> hipError_t launch_norm_bwd(const NormArgs<T>& a, int G, hipStream_t st);

template <class T>
hipError_t launch_act_bwd(int act, const Mat<const T>& dy, const Mat<const T>& pre, const Mat<T>& g, int64_t M,
                          int64_t N, int G, hipStream_t st);

// part[g][s][c] = sum of rows s, s + slots, ... of column c
template <class T>
hipError_t launch_colsum_rows(const Mat<const T>& m, int64_t M, int64_t N, int slots, float* part, int G,
                              hipStream_t st);

// dst[g][c] = sum over slots s, in order, of part[g][s][c]  (fp64 sums); a
// second array of columns behind the first may go to dst2 (columns [n1, n))
hipError_t launch_slot_sum(const float* part, int64_t p_g, int n_slots, int64_t n, float* dst, int64_t n1, float* dst2,
                           int G, hipStream_t st);

// n zeros
hipError_t launch_zeros(float* dst, int64_t n, hipStream_t st);

}  // namespace pigan
