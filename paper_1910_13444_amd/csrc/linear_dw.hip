// Parameter gradients of the linear layer: dw = g^T x, db = sum of g.
#include "mm.h"

namespace pigan {

template <class T>
hipError_t launch_mm_dw(const MmArgs<T, float>& a, int tile, bool direct, int G, hipStream_t st) {
  return mm_launch<T, float, MM_DW>(a, tile, direct, G, st);
}
hipError_t launch_mm_join_dw(const MmOut<float>& o, const float* part_db, int slots, float* db, int G, hipStream_t st) {
  return join_launch<MM_DW>(o, G, st, part_db, slots, db);
}

template hipError_t launch_mm_dw<bf16>(const MmArgs<bf16, float>&, int, bool, int, hipStream_t);
template hipError_t launch_mm_dw<f16>(const MmArgs<f16, float>&, int, bool, int, hipStream_t);

}  // namespace pigan
