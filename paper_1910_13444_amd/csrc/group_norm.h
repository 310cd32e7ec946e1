// Launchers of group norm with an activation (group_norm_fwd.hip, group_norm_bwd.hip) and how
// a call is cut (group_norm_plan.cpp).
#pragma once
#include "common.h"

namespace pigan {

// Points of C channels; point p of sample s of group g at ptr + g * gs + s * ss + p * ld.
template <class T> struct Field {
  T* p; int64_t ld; int64_t ss; int64_t gs;
};

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline unsigned grid_of(int64_t blocks) { return (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20); }

// How a call's samples are cut.  A slab is the channels that a block works on: whole
// channel groups, or a part of one that is wider than a block's threads reach.
enum GnMode {
  GN_ROWS = 0,          // one point a sample, a channel group in 2^i <= 64 lanes
  GN_ONE = 1,           // a sample's slab stays in a block's registers
  GN_SPLIT = 2          // blocks share a sample, a pass for sums and one for results
};
struct GnPlan {
  int32_t mode;
  bool stream;          // operands past the last-level cache
  int32_t nth, nv;      // threads of a block, pieces of a thread (one pass)
  int32_t pw;           // pieces of a slab's point
  int32_t rows;         // points of a block's threads at a time
  int32_t ns;           // samples of a block at a time; above 1 rows = ns P
  int32_t lanes;        // that sum one channel group of one sample
  int32_t span;         // slots of a channel group in a slab: pieces, or channels where pieces are of several groups
  int32_t chan_parts;   // slabs of a channel group (1: whole ones)
  int32_t splits;       // blocks that share a sample's points
  int32_t slots;        // reverse pass: partial rows of [dgamma, dbeta]
  int64_t cg;           // channels of a channel group
  int64_t W;            // channels of a slab (the last may have fewer)
  int64_t slabs;        // of a sample
  int64_t ng;           // channel groups of a slab
  double inv_n;         // 1 / values of a channel group
};

// Threads and pieces of a thread of the one-pass kernels, by what they hold.
struct Shape { int nth, nv; };
constexpr Shape FWD_SHAPES[] = {{256, 1}, {256, 4}, {1024, 2}, {256, 8}, {512, 8}, {1024, 8}};
constexpr Shape FWD_ODD[] = {{256, 1}, {512, 1}, {256, 4}, {256, 8}};   // channel groups that are no whole pieces
constexpr Shape BWD_SHAPES[] = {{256, 1}, {512, 1}};
constexpr int SPLIT_NTH = 256;   // threads of a block that takes a range of points
// Terms that the reverse pass sums in fp32 at most, before it joins in fp64: of a channel's
// gradients those of a thread, of a channel group's means those of a row's lanes (64 pieces).
// A sum is off by BWD_TERMS 2^-24 of its terms' sizes at most.
constexpr int64_t BWD_TERMS = 512;

struct Pair { double s, q; };    // of two sums

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

// `fields`: how many of them the call reads and writes
GnPlan gn_plan(bool backward, int fields, int elem_bytes, int64_t G, int64_t S, int64_t P, int64_t C, int64_t n);
// bytes of ranges' sums; workspace of a call (0: none); `cols`: dgamma or dbeta is wanted
size_t gn_pairs_bytes(const GnPlan& pl, int64_t G, int64_t S, int64_t n);
size_t gn_forward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t n);
size_t gn_backward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t C, int64_t n, bool cols);

template <class T> hipError_t launch_gn_fwd(const GnArgs<T>& a, int G, hipStream_t st);
template <class T> hipError_t launch_gn_bwd(const GnArgs<T>& a, int G, hipStream_t st);

}  // namespace pigan
