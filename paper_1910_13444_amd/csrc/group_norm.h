// Launchers of group norm with an activation (group_norm.hip).
#pragma once
#include "common.h"

namespace pigan {

// Points of C channels; point p of sample s of group g at ptr + g * gs + s * ss + p * ld.
template <class T> struct Field {
  T* p; int64_t ld; int64_t ss; int64_t gs;
};

// How a call's samples are cut.  A slab is the channels that a block works on: whole
// channel groups, or a part of one that is wider than a block's threads reach.
enum GnMode {
  GN_ROWS = 0,          // one point a sample, a channel group in 2^i <= 64 lanes
  GN_ONE = 1,           // a sample's slab stays in a block's registers
  GN_SPLIT = 2          // ranges of points, a pass for sums and one for results
};
struct GnPlan {
  int32_t mode;
  int64_t W;            // channels of a slab (the last may have fewer)
  int64_t slabs;        // of a sample
  int64_t ng;           // channel groups of a slab
  int64_t chan_parts;   // slabs of a channel group (1: whole ones)
  int32_t nth, nv;      // threads of a block, pieces of a thread (one pass)
  int32_t pw;           // pieces of a slab's point
  int32_t rows;         // points of a block's threads at a time
  int32_t ns;           // samples of a block at a time; above 1 rows = ns P
  int32_t lanes;        // that sum one channel group of one sample
  int64_t splits;       // ranges of a sample's points
  int64_t split_rows;   // points of a range
  int64_t slots;        // reverse pass: partial rows of [dgamma, dbeta]
};

template <class T> struct GnArgs {
  Field<const T> x; Field<const T> dy; Field<const T> add;   // add.p may be null
  Field<T> out;                                              // y, or dx (null: not wanted)
  const float* gamma; const float* beta;                     // null: ones, zeros
  float* mean; float* rstd;                                  // forward: outputs or null; backward: inputs
  float* dgamma; float* dbeta;                               // backward: outputs or null
  char* ws;
  int64_t S, P, C, n;
  float eps;
  int32_t act;
  GnPlan pl;
};

GnPlan gn_plan(bool backward, int elem_bytes, int64_t G, int64_t S, int64_t P, int64_t C, int64_t n);
// workspace of a call (0: none); `cols`: dgamma or dbeta is wanted
size_t gn_forward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t n);
size_t gn_backward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t C, int64_t n, bool cols);

template <class T> hipError_t launch_gn_fwd(const GnArgs<T>& a, int G, hipStream_t st);
template <class T> hipError_t launch_gn_bwd(const GnArgs<T>& a, int G, hipStream_t st);

}  // namespace pigan
