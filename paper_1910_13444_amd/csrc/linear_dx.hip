// Input gradient of the linear layer, dx = (g w) act'(pre) + add, by itself and in
// one launch with the weight gradient.
#include "mm.h"

namespace pigan {

// Both products of a small layer's reverse pass: neither fills the chip for long,
// and side by side they fill each other's waits (21 layers of 512 x 256 x 256 fp16:
// 13 us; 10.4 us and 11.2 us apart).  The one with the longer blocks comes first.
template <class T, class TO, int MT, int NT, int OCC, bool WHOLE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
k_mm_both(const MmArgs<T, TO> dx, const MmArgs<T, float> dw, uint32_t n_dx, uint32_t n_dw, int dw_first) {
  __shared__ __attribute__((aligned(1024))) char s0[mm_stage<MT, NT, 2>()];
  __shared__ __attribute__((aligned(1024))) char s1[mm_stage<MT, NT, 2>()];
  const uint32_t n = blockIdx.x, begin = dw_first ? n_dw : 0;
  if (n >= begin && n - begin < n_dx) mm_piped<T, TO, MM_DX, MT, NT, 2, WHOLE>(dx, n - begin, n_dx, s0, s1);
  else mm_piped<T, float, MM_DW, MT, NT, 2, WHOLE>(dw, dw_first ? n : n - n_dx, n_dw, s0, s1);
}

template <class T, class TO, bool WHOLE>
void both_of(const MmArgs<T, TO>& dx, const MmArgs<T, float>& dw, int tile, uint32_t n_dx, uint32_t n_dw, bool dw_first,
             hipStream_t st) {
  if (tile == MM_128) k_mm_both<T, TO, 2, 2, 2, WHOLE><<<n_dx + n_dw, 256, 0, st>>>(dx, dw, n_dx, n_dw, dw_first);
  else k_mm_both<T, TO, 1, 1, 4, WHOLE><<<n_dx + n_dw, 256, 0, st>>>(dx, dw, n_dx, n_dw, dw_first);
}

template <class T, class TO>
hipError_t launch_mm_both(const MmArgs<T, TO>& dx, const MmArgs<T, float>& dw, int tile, bool dw_first, int G,
                          hipStream_t st) {
  const uint32_t n_dx = mm_blocks<T, TO, MM_DX>(dx, tile, true, G), n_dw = mm_blocks<T, float, MM_DW>(dw, tile, true, G);
  if (!n_dx || !n_dw || dx.o.J != dw.o.J || ((uint64_t)n_dx + n_dw) * 256 >> 32 || (tile != MM_64 && tile != MM_128)) return hipErrorInvalidValue;
  if (dx.o.J % 8 == 0) both_of<T, TO, true>(dx, dw, tile, n_dx, n_dw, dw_first, st);
  else both_of<T, TO, false>(dx, dw, tile, n_dx, n_dw, dw_first, st);
  return hipGetLastError();
}

template hipError_t launch_mm_both<bf16, bf16>(const MmArgs<bf16, bf16>&, const MmArgs<bf16, float>&, int, bool, int,
                                               hipStream_t);
template hipError_t launch_mm_both<f16, f16>(const MmArgs<f16, f16>&, const MmArgs<f16, float>&, int, bool, int,
                                             hipStream_t);
template hipError_t launch_mm_both<bf16, float>(const MmArgs<bf16, float>&, const MmArgs<bf16, float>&, int, bool, int,
                                                hipStream_t);

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
