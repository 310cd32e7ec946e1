// Checks of operands that the files of C entry points share: vectors, activations,
// the workspace, and nested blocks of memory that may overlap.
#pragma once
#include <algorithm>

#include "api.h"

namespace pigan {

inline pigan_status check_vec(const void* p, const char* name) {
  if ((uintptr_t)p % 4) return fail(PIGAN_EINVAL, "%s: pointer is not aligned to its elements", name);
  return PIGAN_OK;
}

inline pigan_status check_act(int32_t act) {
  if (act < PIGAN_ACT_NONE || act > PIGAN_ACT_SILU) return fail(PIGAN_EINVAL, "unknown activation %d", (int)act);
  return PIGAN_OK;
}

inline pigan_status check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return PIGAN_OK;
  if (!ws) return fail(PIGAN_EWORKSPACE, "null workspace, %zu bytes are needed", need);
  if (have < need) return fail(PIGAN_EWORKSPACE, "workspace of %zu bytes, %zu are needed", have, need);
  if ((uintptr_t)ws % 256) return fail(PIGAN_EINVAL, "the workspace must be 256-byte aligned");
  return PIGAN_OK;
}

// an exception may not leave a C entry point
template <class F> pigan_status guarded(F&& f) noexcept {
  try {
    clear_error();
    return f();
  } catch (...) {
    return PIGAN_EDEVICE;
  }
}

// f(element of the storage type)
template <class F> pigan_status by_dtype(int32_t dt, F&& f) {
  switch (dt) {
    case PIGAN_BF16: return f(bf16{});
    case PIGAN_FP16: return f(f16{});
    default: return f(float{});
  }
}

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }

// ---------------------------------------------------------------------------
// Memory of an operand: runs of `len` bytes, up to three times repeated, level 0
// innermost; a level's stride is at least the extent of what it repeats.  Levels
// that continue the one below are joined, so equal memory has equal fields.
// ---------------------------------------------------------------------------
struct Runs {
  const char* name;
  int64_t p, len;
  int levels;
  int64_t n[3], st[3];

  // p = 0: no operand
  Runs(const char* nm, const void* q, int64_t bytes) : name(nm), p((int64_t)(uintptr_t)q), len(bytes), levels(0), n{}, st{} {
    if (bytes <= 0) p = 0;
  }
  Runs& repeat(int64_t count, int64_t stride) {
    if (count < 1) p = 0;
    if (!p || count == 1) return *this;
    if (levels == 0 && stride == len) len *= count;
    else if (levels > 0 && stride == n[levels - 1] * st[levels - 1]) n[levels - 1] *= count;
    else { n[levels] = count; st[levels++] = stride; }
    return *this;
  }
  __int128 end() const {
    __int128 e = (__int128)p + len;
    for (int i = 0; i < levels; ++i) e += (__int128)(n[i] - 1) * st[i];
    return e;
  }
  bool same(const Runs& o) const {
    if (p != o.p || len != o.len || levels != o.levels) return false;
    for (int i = 0; i < levels; ++i)
      if (n[i] != o.n[i] || st[i] != o.st[i]) return false;
    return true;
  }
};

// the interval [from, to) and b's levels below `level`, begun at `at`: of a level's
// repetitions the last one that begins at or before `from` and the next one may meet it
inline bool interval_meets(__int128 from, __int128 to, const Runs& b, int level, __int128 at) {
  if (level == 0) return at < to && from < at + b.len;
  const __int128 st = b.st[level - 1], last = b.n[level - 1] - 1;
  const __int128 i = from < at ? 0 : std::min<__int128>((from - at) / st, last);
  return interval_meets(from, to, b, level - 1, at + i * st) ||
         (i < last && interval_meets(from, to, b, level - 1, at + (i + 1) * st));
}

// a from 0 on and b from d on, of equal strides: repetition j of b can only meet those
// of a that are less than a stride away
inline bool alike_meet(const Runs& a, const Runs& b, int level, int64_t d) {
  if (level == 0) return d < a.len && -d < b.len;
  const int64_t st = a.st[level - 1];
  for (int64_t s = floor_div(-d, st), k = 0; k < 2; ++k, ++s)
    if (s > -a.n[level - 1] && s < b.n[level - 1] && alike_meet(a, b, level - 1, d + s * st)) return true;
  return false;
}

// Whether a and b have a byte in common; of two that are both apart in runs, by
// different strides, it is only told where they begin at the same address.
inline bool share(const Runs& a, const Runs& b) {
  if (!a.p || !b.p || a.end() <= b.p || b.end() <= a.p) return false;
  if (a.levels == 0) return interval_meets(a.p, a.end(), b, b.levels, b.p);
  if (b.levels == 0) return interval_meets(b.p, b.end(), a, a.levels, a.p);
  bool alike = a.levels == b.levels;
  for (int i = 0; i < a.levels && alike; ++i) alike = a.st[i] == b.st[i];
  return alike ? alike_meet(a, b, a.levels, b.p - a.p) : a.p == b.p;
}

// No output shares memory with another operand, but for the same one where
// same_ok(output, input) says so.
template <int NO, int NI, class F>
pigan_status check_apart(const Runs (&outs)[NO], const Runs (&ins)[NI], F&& same_ok) {
  for (int o = 0; o < NO; ++o) {
    for (int q = 0; q < o; ++q)
      if (share(outs[o], outs[q])) return fail(PIGAN_EINVAL, "%s overlaps %s", outs[o].name, outs[q].name);
    for (int i = 0; i < NI; ++i)
      if (share(outs[o], ins[i]) && !(same_ok(o, i) && outs[o].same(ins[i])))
        return fail(PIGAN_EINVAL, "%s overlaps %s", outs[o].name, ins[i].name);
  }
  return PIGAN_OK;
}

}  // namespace pigan
