// Launchers of the linear layer's products (linear_fwd.hip, linear_dx.hip,
// linear_dw.hip).
//
// Every product is C[i][j] = sum_k A(i, k) B(j, k) on matrices stored in rows:
//   forward   A = x   (k along the row),  B = w (k along the row)
//   dx        A = g   (k along the row),  B = w (k down the rows)
//   dw        A = g,  B = x               (k down the rows of both)
#pragma once
#include "common.h"

namespace pigan {

// One operand; element (i, k) of group g at p + g gs + i ld + k, or + k ld + i
template <class T> struct MmOperand {
  const T* p; int64_t ld; int64_t gs; int64_t plane;   // elements between planes (MmArgs::pairs > 1)
};

// The result and its epilogue; TO: type of the outputs and of the epilogue's matrices
template <class TO> struct MmOut {
  int64_t I, J;
  int32_t act;
  int32_t n_split;          // blocks that share the contraction of a tile
  // forward: out = act(C + bias) + add, pre = C + bias;  dx: out = C act'(pre) + add
  const float* bias;        // [G][J], or null
  TO* pre; int64_t ldp, gsp;          // or null
  const TO* add; int64_t lda, gsa;    // or null
  TO* out; int64_t ldo, gso;
  float* part;              // partial sums [G][n_split][I][J]: stored instead of the epilogue's results
};

template <class T, class TO> struct MmArgs {
  MmOperand<T> a, b;
  int64_t K;
  int32_t pairs;            // 1; 6: three bf16 planes per operand (fp32 products)
  MmOut<TO> o;
  float* part_db;           // dw: sums of A over k, [G][I], with splits [G][n_split * column tiles][I]; or null
};

// MM_64K: 64 with the contraction shared by four groups of waves
enum MmTile { MM_64 = 0, MM_128 = 1, MM_256 = 2, MM_64K = 3 };
inline int mm_tile_side(int t) { return t == MM_128 ? 128 : t == MM_256 ? 256 : 64; }

inline int mm_tile_threads(int t) { return t == MM_64K ? 1024 : t == MM_256 ? 512 : 256; }

// direct: both operands may go straight to LDS: 16-byte aligned rows (a tile's
// extent below 2^31 bytes) of whole pieces; copies (pack) and planes (split3), which
// pairs = 6 needs, hold zeros behind their rows up to a whole piece
template <class T> bool mm_whole(const MmOperand<T>& m, int64_t cols, int G) {
  return (uintptr_t)m.p % 16 == 0 && m.ld % 8 == 0 && (G == 1 || m.gs % 8 == 0) && m.plane % 8 == 0 &&
         (cols + 7) / 8 * 8 <= m.ld && m.ld < (int64_t(1) << 21);
}
template <class T, class TO>
hipError_t launch_mm_fwd(const MmArgs<T, TO>& a, int tile, bool direct, int G, hipStream_t st);
template <class T, class TO>
hipError_t launch_mm_dx(const MmArgs<T, TO>& a, int tile, bool direct, int G, hipStream_t st);
template <class T>
hipError_t launch_mm_dw(const MmArgs<T, float>& a, int tile, bool direct, int G, hipStream_t st);

// dx and dw of aligned operands in one launch (tiles of 64 and 128)
template <class T, class TO>
hipError_t launch_mm_both(const MmArgs<T, TO>& dx, const MmArgs<T, float>& dw, int tile, bool dw_first, int G,
                          hipStream_t st);

// sums the partials of split products in order and applies the epilogue
template <class TO> hipError_t launch_mm_join_fwd(const MmOut<TO>& o, int G, hipStream_t st);
template <class TO> hipError_t launch_mm_join_dx(const MmOut<TO>& o, int G, hipStream_t st);
// (and of db, where it is wanted: [G][slots][I])
hipError_t launch_mm_join_dw(const MmOut<float>& o, const float* part_db, int slots, float* db, int G, hipStream_t st);

// forward on few rows or few outputs, no LDS stages
template <class T> hipError_t launch_short_fwd(const MmArgs<T, T>& a, int G, hipStream_t st);

// fp32 matrices to three bf16 planes x = x0 + x1 + x2, rows of Kp >= cols
// elements (zeros behind the row): up to three matrices in one launch
struct SplitSet {
  const float* src; int64_t ld, gs; int64_t rows, cols, Kp;
  bf16* dst;                 // [3][G][rows][Kp]
};
hipError_t launch_split3(const SplitSet* sets, int n, int G, hipStream_t st);

// 16-bit matrices with rows at any address to rows of whole, aligned pieces, zeros
// behind them: up to three in one launch
struct PackSet {
  const void* src; int64_t ld, gs; int64_t rows, cols, Kp;
  void* dst;                 // [G][rows][Kp]
};
hipError_t launch_pack(const PackSet* sets, int n, int G, hipStream_t st);

}  // namespace pigan
