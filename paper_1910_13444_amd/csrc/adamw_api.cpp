// C entry points of the gradients' norm and of AdamW over many tensors: argument
// checks, the table.
#include "adamw.h"

#include <cmath>
#include <cstring>
#include <vector>

#include "operands.h"

namespace pigan {
namespace {

constexpr int64_t MOST = int64_t(1) << 40;   // elements of a table

// what the sizes alone decide
struct Counts { int64_t elements, states, pieces, g_bytes, copy_bytes; };

pigan_status check_tensors(const pigan_tensors* a, Counts& c) {
  if (!a) return fail(PIGAN_EINVAL, "null arguments");
  if (a->n_tensors < 0) return fail(PIGAN_EINVAL, "n_tensors=%d must be >= 0", (int)a->n_tensors);
  if (a->bits != 0 && a->bits != 8 && a->bits != 32) return fail(PIGAN_EINVAL, "bits=%d must be 0, 8 or 32", (int)a->bits);
  if (a->n_tensors > 0 && !a->tensors) return fail(PIGAN_EINVAL, "tensors: null pointer");
  c = {};
  for (int32_t i = 0; i < a->n_tensors; ++i) {
    const pigan_tensor& t = a->tensors[i];
    if (t.n < 0 || t.n > MOST) return fail(PIGAN_EINVAL, "tensor %d: n=%lld out of [0, 2^40]", (int)i, (long long)t.n);
    if (pigan_status st = check_dtype(t.g_dt)) return st;
    if (t.n > 0 && !t.g) return fail(PIGAN_EINVAL, "tensor %d: null gradient", (int)i);
    if ((uintptr_t)t.g % esize(t.g_dt)) return fail(PIGAN_EINVAL, "tensor %d: gradient not aligned to its elements", (int)i);
    if (a->bits) {
      if (t.n > 0 && !t.p) return fail(PIGAN_EINVAL, "tensor %d: null parameter", (int)i);
      if ((uintptr_t)t.p % 4) return fail(PIGAN_EINVAL, "tensor %d: parameter not aligned to its elements", (int)i);
      if (t.copy && t.copy_dt != PIGAN_BF16 && t.copy_dt != PIGAN_FP16)
        return fail(PIGAN_EINVAL, "tensor %d: copy_dt=%d must be bf16 or fp16", (int)i, (int)t.copy_dt);
      if ((uintptr_t)t.copy % 2) return fail(PIGAN_EINVAL, "tensor %d: copy not aligned to its elements", (int)i);
      if (!(t.decay >= 0.0) || !std::isfinite(t.decay))
        return fail(PIGAN_EINVAL, "tensor %d: decay=%g must be finite and >= 0", (int)i, t.decay);
    }
    c.elements += t.n;
    if (c.elements >= MOST) return fail(PIGAN_EINVAL, "2^40 elements and more");
    c.states += a->bits == 8 ? round_up(t.n, QBLOCK) : t.n;
    c.pieces += (t.n + PIECE - 1) / PIECE;
    c.g_bytes += t.n * (int64_t)esize(t.g_dt);
    if (a->bits && t.copy) c.copy_bytes += 2 * t.n;
  }
  if (!a->bits) c.states = 0;
  return PIGAN_OK;
}

pigan_status check_states(const pigan_tensors* a, const Counts& c) {
  if (!a->bits || c.states == 0) return PIGAN_OK;
  if (!a->m || !a->v) return fail(PIGAN_EINVAL, "m and v: null pointer");
  // 8-bit codes are read four at a time
  if ((uintptr_t)a->m % 4 || (uintptr_t)a->v % 4) return fail(PIGAN_EINVAL, "m and v must be 4-byte aligned");
  if (a->bits == 8) {
    if (!a->m_scale || !a->v_scale) return fail(PIGAN_EINVAL, "m_scale and v_scale: null pointer");
    if ((uintptr_t)a->m_scale % 4 || (uintptr_t)a->v_scale % 4)
      return fail(PIGAN_EINVAL, "m_scale and v_scale: not aligned to their elements");
  }
  return PIGAN_OK;
}

struct Span { uintptr_t from, to; const char* what; int32_t tensor; };

// parameters, copies and states
std::vector<Span> written(const pigan_tensors* a, const Counts& c) {
  std::vector<Span> outs;
  auto add = [&](const void* p, int64_t bytes, const char* what, int32_t i) {
    if (p && bytes > 0) outs.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, what, i});
  };
  if (!a->bits) return outs;
  for (int32_t i = 0; i < a->n_tensors; ++i) {
    add(a->tensors[i].p, a->tensors[i].n * 4, "parameter", i);
    add(a->tensors[i].copy, a->tensors[i].n * 2, "copy", i);
  }
  const int64_t bytes = c.states * (a->bits / 8);
  add(a->m, bytes, "m", -1);
  add(a->v, bytes, "v", -1);
  if (a->bits == 8) {
    add(a->m_scale, c.states / QBLOCK * 4, "m_scale", -1);
    add(a->v_scale, c.states / QBLOCK * 4, "v_scale", -1);
  }
  return outs;
}

std::vector<Span> gradients(const pigan_tensors* a) {
  std::vector<Span> ins;
  for (int32_t i = 0; i < a->n_tensors; ++i) {
    const pigan_tensor& t = a->tensors[i];
    if (t.n > 0) ins.push_back({(uintptr_t)t.g, (uintptr_t)t.g + (uintptr_t)(t.n * (int64_t)esize(t.g_dt)), "gradient", i});
  }
  return ins;
}

std::vector<Span> in_order(std::vector<Span> v) {
  std::sort(v.begin(), v.end(), [](const Span& x, const Span& y) { return x.from < y.from; });
  return v;
}

// joined, behind each other to `to`; their number
int64_t extents(const std::vector<Span>& v, Extent* to) {
  int64_t n = 0;
  for (const Span& s : v) {
    if (n > 0 && s.from <= to[n - 1].to) to[n - 1].to = std::max<uint64_t>(to[n - 1].to, s.to);
    else to[n++] = {s.from, s.to};
  }
  return n;
}

// every output lies apart from every other one and from every gradient
pigan_status check_spans(const std::vector<Span>& outs, const std::vector<Span>& grads) {
  for (size_t i = 1; i < outs.size(); ++i)
    if (outs[i].from < outs[i - 1].to)
      return fail(PIGAN_EINVAL, "%s (tensor %d) overlaps %s (tensor %d)", outs[i].what, (int)outs[i].tensor, outs[i - 1].what,
                  (int)outs[i - 1].tensor);
  for (const Span& g : grads) {
    // the last output that begins before the gradient ends
    auto it = std::lower_bound(outs.begin(), outs.end(), g.to, [](const Span& s, uintptr_t v) { return s.from < v; });
    if (it != outs.begin() && (--it)->to > g.from)
      return fail(PIGAN_EINVAL, "gradient of tensor %d overlaps %s (tensor %d)", (int)g.tensor, it->what, (int)it->tensor);
  }
  return PIGAN_OK;
}

TableHeader header_of(const pigan_tensors* a, const Counts& c) {
  TableHeader h{};
  h.magic = TABLE_MAGIC;
  h.n_tensors = a->n_tensors;
  h.bits = a->bits;
  h.n_pieces = c.pieces;
  h.states = c.states;
  h.entries_at = round_up(sizeof(TableHeader), 16);
  h.pieces_at = h.entries_at + (int64_t)a->n_tensors * (int64_t)sizeof(TensorEntry);
  h.extents_at = h.pieces_at + c.pieces * (int64_t)sizeof(TensorPiece);
  // as many as there are where none are joined
  h.bytes = h.extents_at + ((int64_t)a->n_tensors * (a->bits ? 3 : 1) + (a->bits ? 4 : 0)) * (int64_t)sizeof(Extent);
  h.m = a->m;
  h.v = a->v;
  h.m_scale = a->m_scale;
  h.v_scale = a->v_scale;
  h.elements = c.elements;
  h.g_bytes = c.g_bytes;
  h.copy_bytes = c.copy_bytes;
  return h;
}

pigan_status check_table(const void* table, const void* device_table) {
  if (!table || !device_table) return fail(PIGAN_EINVAL, "null table");
  if ((uintptr_t)table % 8 || (uintptr_t)device_table % 8) return fail(PIGAN_EINVAL, "the table must be 8-byte aligned");
  if (((const TableHeader*)table)->magic != TABLE_MAGIC) return fail(PIGAN_EINVAL, "not a table of pigan_tensors_table");
  return PIGAN_OK;
}

template <class T> const T* at(const void* table, int64_t off) { return (const T*)((const char*)table + off); }

bool meets(const Extent* e, int64_t n, const Runs& r) {
  const uint64_t from = (uint64_t)r.p, to = from + (uint64_t)r.len;
  const Extent* it = std::upper_bound(e, e + n, from, [](uint64_t v, const Extent& x) { return v < x.to; });
  return it != e + n && it->from < to;
}

// `r` apart from the tables' tensors: those that a call writes, and their gradients, and, where
// the call writes r, from the table
pigan_status check_off_tensors(const void* table, const void* device_table, const Runs& r, bool is_written, bool with_written,
                               bool with_gradients) {
  if (!r.p) return PIGAN_OK;
  const TableHeader& h = *(const TableHeader*)table;
  const Extent* e = at<Extent>(table, h.extents_at);
  if (with_written && meets(e, h.n_written, r)) return fail(PIGAN_EINVAL, "%s overlaps a parameter, copy or state", r.name);
  if (with_gradients && meets(e + h.n_written, h.n_read, r)) return fail(PIGAN_EINVAL, "%s overlaps a gradient", r.name);
  const Extent own = {(uint64_t)(uintptr_t)device_table, (uint64_t)(uintptr_t)device_table + (uint64_t)h.bytes};
  if (is_written && meets(&own, 1, r)) return fail(PIGAN_EINVAL, "%s overlaps the table", r.name);
  return PIGAN_OK;
}

pigan_status check_device_word(const void* p, const char* name) {
  if ((uintptr_t)p % 4) return fail(PIGAN_EINVAL, "%s: not aligned to its elements", name);
  return PIGAN_OK;
}

}  // namespace
}  // namespace pigan

using namespace pigan;

extern "C" {

int64_t pigan_tensors_states(const pigan_tensors* a) {
  int64_t n = -1;
  guarded([&]() -> pigan_status {
    Counts c;
    if (pigan_status st = check_tensors(a, c)) return st;
    n = c.states;
    return PIGAN_OK;
  });
  return n;
}

size_t pigan_tensors_table_bytes(const pigan_tensors* a) {
  size_t n = 0;
  guarded([&]() -> pigan_status {
    Counts c;
    if (pigan_status st = check_tensors(a, c)) return st;
    n = (size_t)header_of(a, c).bytes;
    return PIGAN_OK;
  });
  return n;
}

pigan_status pigan_tensors_table(const pigan_tensors* a, void* table, size_t bytes) {
  return guarded([&]() -> pigan_status {
    Counts c;
    if (pigan_status st = check_tensors(a, c)) return st;
    if (pigan_status st = check_states(a, c)) return st;
    const std::vector<Span> outs = in_order(written(a, c)), grads = in_order(gradients(a));
    if (pigan_status st = check_spans(outs, grads)) return st;
    TableHeader h = header_of(a, c);
    if (!table || (uintptr_t)table % 8) return fail(PIGAN_EINVAL, "the table must be 8-byte aligned");
    if (bytes < (size_t)h.bytes) return fail(PIGAN_EINVAL, "table of %zu bytes, %lld are needed", bytes, (long long)h.bytes);
    Extent* const to = (Extent*)((char*)table + h.extents_at);
    h.n_written = extents(outs, to);
    h.n_read = extents(grads, to + h.n_written);
    memset(to + h.n_written + h.n_read, 0, (size_t)(h.bytes - h.extents_at) - (size_t)(h.n_written + h.n_read) * sizeof(Extent));
    memcpy(table, &h, sizeof h);
    TensorEntry* entries = (TensorEntry*)((char*)table + h.entries_at);
    TensorPiece* pieces = (TensorPiece*)((char*)table + h.pieces_at);
    int64_t state = 0;
    for (int32_t i = 0; i < a->n_tensors; ++i) {
      const pigan_tensor& t = a->tensors[i];
      entries[i] = {a->bits ? t.p : nullptr, t.g, a->bits ? t.copy : nullptr, t.n, state, t.decay, t.g_dt, t.copy_dt};
      state += a->bits == 8 ? round_up(t.n, QBLOCK) : t.n;
      for (int64_t k = 0; k * PIECE < t.n; ++k) *pieces++ = {(uint32_t)i, (uint32_t)k};
    }
    return PIGAN_OK;
  });
}

size_t pigan_grad_norm_workspace(const void* table) {
  size_t n = 0;
  guarded([&]() -> pigan_status {
    if (pigan_status st = check_table(table, table)) return st;
    n = (size_t)grad_norm_blocks(((const TableHeader*)table)->n_pieces) * 8;
    return PIGAN_OK;
  });
  return n;
}

pigan_status pigan_grad_norm(const void* table, const void* device_table, double max_norm, double scale, float* norm,
                             float* coef, int32_t* nonfinite, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> pigan_status {
    if (pigan_status st = check_table(table, device_table)) return st;
    const TableHeader& h = *(const TableHeader*)table;
    if (!(max_norm > 0.0)) return fail(PIGAN_EINVAL, "max_norm=%g must be > 0", max_norm);
    if (!(scale > 0.0) || !std::isfinite(scale)) return fail(PIGAN_EINVAL, "scale=%g must be finite and > 0", scale);
    if (!norm && !coef && !nonfinite) return fail(PIGAN_EINVAL, "no output: norm, coef and nonfinite are null");
    const Runs outs[] = {{"norm", norm, 4}, {"coef", coef, 4}, {"nonfinite", nonfinite, 4}};
    for (const Runs& o : outs)
      if (pigan_status st = check_device_word((const void*)o.p, o.name)) return st;
    const size_t need = (size_t)grad_norm_blocks(h.n_pieces) * 8;
    if (pigan_status st = check_ws(ws, ws_bytes, need)) return st;
    const Runs none[] = {{"the workspace", ws, (int64_t)need}};
    if (pigan_status st = check_apart(outs, none, [](int, int) { return false; })) return st;
    for (const Runs& o : {outs[0], outs[1], outs[2], none[0]})
      if (pigan_status st = check_off_tensors(table, device_table, o, true, false, true)) return st;
    const hipStream_t st = (hipStream_t)stream;
    ProfScope prof(st, "grad_norm", 0.0, (double)h.g_bytes);
    HIP_TRY(launch_grad_norm(at<TensorEntry>(device_table, h.entries_at), at<TensorPiece>(device_table, h.pieces_at), h.n_pieces,
                             max_norm, scale, (double*)ws, norm, coef, nonfinite, st));
    return PIGAN_OK;
  });
}

pigan_status pigan_adamw_update(const pigan_adamw* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> pigan_status {
    if (!a) return fail(PIGAN_EINVAL, "null arguments");
    if (pigan_status st = check_table(a->table, a->device_table)) return st;
    const TableHeader& h = *(const TableHeader*)a->table;
    if (!h.bits) return fail(PIGAN_EINVAL, "the table is one of gradients alone");
    if (a->reserved) return fail(PIGAN_EINVAL, "reserved=%d must be 0", (int)a->reserved);
    for (double b : {a->beta1, a->beta2})
      if (!(b >= 0.0 && b < 1.0)) return fail(PIGAN_EINVAL, "beta1=%g and beta2=%g must lie in [0, 1)", a->beta1, a->beta2);
    if (!std::isfinite(a->lr) || !(a->eps >= 0.0) || !std::isfinite(a->eps))
      return fail(PIGAN_EINVAL, "lr must be finite and eps finite and >= 0");
    if (!(a->scale > 0.0) || !std::isfinite(a->scale)) return fail(PIGAN_EINVAL, "scale=%g must be finite and > 0", a->scale);
    if (!a->step && a->t < 1) return fail(PIGAN_EINVAL, "t=%d must be >= 1", (int)a->t);
    if (pigan_status st = check_device_word(a->coef, "coef")) return st;
    if (pigan_status st = check_device_word(a->skip, "skip")) return st;
    if (pigan_status st = check_device_word(a->step, "step")) return st;
    if (pigan_status st = check_ws(ws, ws_bytes, a->step ? PIGAN_ADAMW_WORKSPACE : 0)) return st;
    const Runs outs[] = {{"step", a->step, 4}, {"the workspace", a->step ? ws : nullptr, PIGAN_ADAMW_WORKSPACE}};
    const Runs ins[] = {{"coef", a->coef, 4}, {"skip", a->skip, 4}};
    if (pigan_status st = check_apart(outs, ins, [](int, int) { return false; })) return st;
    for (const Runs& r : ins)
      if (pigan_status st = check_off_tensors(a->table, a->device_table, r, false, true, false)) return st;
    for (const Runs& r : outs)
      if (pigan_status st = check_off_tensors(a->table, a->device_table, r, true, true, true)) return st;
    const hipStream_t st = (hipStream_t)stream;
    AdamwArgs k{};
    k.entries = at<TensorEntry>(a->device_table, h.entries_at);
    k.pieces = at<TensorPiece>(a->device_table, h.pieces_at);
    k.m = h.m;
    k.v = h.v;
    k.m_scale = h.m_scale;
    k.v_scale = h.v_scale;
    k.lr = a->lr;
    k.b1 = a->beta1;
    k.b2 = a->beta2;
    k.nb1 = 1.0 - a->beta1;
    k.nb2 = 1.0 - a->beta2;
    k.eps = a->eps;
    k.scale = a->scale;
    k.coef = a->coef;
    k.skip = a->skip;
    if (a->step) {
      HIP_TRY(launch_adamw_begin(a->beta1, a->beta2, a->step, a->skip, (double*)ws, st));
      k.corr = (const double*)ws;
    } else {
      k.c1 = 1.0 / (1.0 - std::pow(a->beta1, (double)a->t));
      k.c2 = 1.0 / (1.0 - std::pow(a->beta2, (double)a->t));
    }
    if (h.n_pieces == 0) return PIGAN_OK;
    const double bytes = (double)h.elements * 8 + h.states * (h.bits == 8 ? 4.0 + 16.0 / QBLOCK : 16.0) + h.g_bytes + h.copy_bytes;
    k.stream = bytes > STREAM_BYTES;
    ProfScope prof(st, h.bits == 8 ? "adamw8" : "adamw", 0.0, bytes);
    HIP_TRY(launch_adamw(k, h.bits, h.n_pieces, st));
    return PIGAN_OK;
  });
}

pigan_status pigan_state_values(int64_t n, const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale,
                                float* m_out, float* v_out, void* stream) {
  return guarded([&]() -> pigan_status {
    if (n < 0 || n % QBLOCK || n > MOST) return fail(PIGAN_EINVAL, "n=%lld must be a multiple of 256 in [0, 2^40]", (long long)n);
    if (n == 0) return PIGAN_OK;   // outputs of no elements may have no address
    if (!m_out && !v_out) return fail(PIGAN_EINVAL, "no output: m_out and v_out are null");
    if ((m_out && (!m || !m_scale)) || (v_out && (!v || !v_scale))) return fail(PIGAN_EINVAL, "null codes or scales");
    if ((uintptr_t)m % 4 || (uintptr_t)v % 4) return fail(PIGAN_EINVAL, "m and v must be 4-byte aligned");
    if ((uintptr_t)m_scale % 4 || (uintptr_t)v_scale % 4 || (uintptr_t)m_out % 4 || (uintptr_t)v_out % 4)
      return fail(PIGAN_EINVAL, "scales or outputs: not aligned to their elements");
    const Runs outs[] = {{"m_out", m_out, n * 4}, {"v_out", v_out, n * 4}};
    const Runs ins[] = {{"m", m_out ? m : nullptr, n}, {"m_scale", m_out ? m_scale : nullptr, n / QBLOCK * 4},
                        {"v", v_out ? v : nullptr, n}, {"v_scale", v_out ? v_scale : nullptr, n / QBLOCK * 4}};
    if (pigan_status st = check_apart(outs, ins, [](int, int) { return false; })) return st;
    const hipStream_t st = (hipStream_t)stream;
    ProfScope prof(st, "state_values", 0.0, n * (5.0 + 4.0 / QBLOCK) * (!!m_out + !!v_out));
    HIP_TRY(launch_state_values(n, m, m_scale, v, v_scale, m_out, v_out, st));
    return PIGAN_OK;
  });
}

}  // extern "C"
