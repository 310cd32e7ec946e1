// Host helpers shared by the files of C entry points.
#pragma once
#include "common.h"

namespace pigan {

// records the thread's error text and returns st; clear_error() empties it
pigan_status fail(pigan_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

#define HIP_TRY(expr)                                                                       \
  do {                                                                                      \
    hipError_t e_ = (expr);                                                                 \
    if (e_ != hipSuccess) return fail(PIGAN_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

struct ProfScope {
  hipStream_t st;
  ProfScope(hipStream_t s, const char* name, double flops, double bytes) : st(s) {
    prof_begin(s, name, flops, bytes);
  }
  ~ProfScope() { prof_end(st); }
};

inline int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

struct Carver {
  size_t off = 0;
  size_t take(size_t bytes) {
    off = (size_t)round_up((int64_t)off, 256);
    const size_t o = off;
    off += bytes;
    return o;
  }
};

inline size_t esize(int32_t dt) { return dt == PIGAN_FP32 ? 4 : 2; }

inline pigan_status check_dtype(int32_t dt) {
  if (dt != PIGAN_FP32 && dt != PIGAN_BF16 && dt != PIGAN_FP16) return fail(PIGAN_EINVAL, "unknown dtype %d", (int)dt);
  return PIGAN_OK;
}

}  // namespace pigan
