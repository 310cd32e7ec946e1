// Input gradient of the linear layer: dx = (g w) act'(pre) + add.
#include "mm.h"

namespace pigan {

template <class T, class TO>
hipError_t launch_mm_dx(const MmArgs<T, TO>& a, int tile, bool direct, int G, hipStream_t st) {
  return mm_launch<T, TO, MM_DX>(a, tile, direct, G, st);
}
template <class TO> hipError_t launch_mm_join_dx(const MmOut<TO>& o, int G, hipStream_t st) {
  return join_launch<MM_DX>(o, G, st);
}

template hipError_t launch_mm_dx<bf16, bf16>(const MmArgs<bf16, bf16>&, int, bool, int, hipStream_t);
template hipError_t launch_mm_dx<f16, f16>(const MmArgs<f16, f16>&, int, bool, int, hipStream_t);
template hipError_t launch_mm_dx<bf16, float>(const MmArgs<bf16, float>&, int, bool, int, hipStream_t);
template hipError_t launch_mm_join_dx<bf16>(const MmOut<bf16>&, int, hipStream_t);
template hipError_t launch_mm_join_dx<f16>(const MmOut<f16>&, int, hipStream_t);
template hipError_t launch_mm_join_dx<float>(const MmOut<float>&, int, hipStream_t);

}  // namespace pigan
