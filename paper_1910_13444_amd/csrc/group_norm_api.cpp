// C entry points of group norm: argument checks, plan, workspace.
#include "group_norm.h"
#include "operands.h"

namespace pigan {
namespace {

constexpr int64_t MAX_DIM = 0x7fffffff;
const pigan_field NO_FIELD = {nullptr, 0, 0, 0};

pigan_status check_field(const pigan_field& f, const char* name, const pigan_group_norm* a) {
  const __int128 most = __int128(1) << 46;
  if (!f.p) return fail(PIGAN_EINVAL, "%s: null pointer", name);
  if ((uintptr_t)f.p % esize(a->dt)) return fail(PIGAN_EINVAL, "%s: pointer is not aligned to its elements", name);
  __int128 extent = a->C;
  const int64_t counts[3] = {a->P, a->S, a->n_groups}, strides[3] = {f.ld, f.ss, f.gs};
  const char* of[3] = {"point", "sample", "group"};
  for (int i = 0; i < 3; ++i) {
    if (counts[i] < 2) continue;
    if (strides[i] < (int64_t)extent || (counts[i] - 1) * (__int128)strides[i] + extent > most)
      return fail(PIGAN_EINVAL, "%s: %s stride %lld does not hold a %s of %lld elements, or %lld of them pass 2^46", name, of[i],
                  (long long)strides[i], of[i], (long long)extent, (long long)counts[i]);
    extent += (counts[i] - 1) * (__int128)strides[i];
  }
  return PIGAN_OK;
}

pigan_status check_sizes(const pigan_group_norm* a) {
  if (!a) return fail(PIGAN_EINVAL, "null arguments");
  if (a->n_groups < 1 || a->n_groups > 65535) return fail(PIGAN_EINVAL, "n_groups=%d out of [1, 65535]", (int)a->n_groups);
  if (pigan_status st = check_dtype(a->dt)) return st;
  if (pigan_status st = check_act(a->act)) return st;
  if (a->S < 0 || a->S > MAX_DIM) return fail(PIGAN_EINVAL, "S=%lld out of [0, 2^31 - 1]", (long long)a->S);
  if (a->P < 1 || a->P > MAX_DIM) return fail(PIGAN_EINVAL, "P=%lld out of [1, 2^31 - 1]", (long long)a->P);
  if (a->C < 1 || a->C > MAX_DIM) return fail(PIGAN_EINVAL, "C=%lld out of [1, 2^31 - 1]", (long long)a->C);
  if (a->n < 1 || a->n > a->C || a->C % a->n)
    return fail(PIGAN_EINVAL, "n=%lld channel groups do not divide C=%lld channels", (long long)a->n, (long long)a->C);
  // so that a field's elements, and with them every count of the plan, fit 64 bits
  if ((__int128)a->n_groups * std::max<int64_t>(a->S, 1) * a->P * a->C > __int128(1) << 46)
    return fail(PIGAN_EINVAL, "%d x %lld x %lld x %lld elements, more than 2^46", (int)a->n_groups, (long long)a->S,
                (long long)a->P, (long long)a->C);
  return PIGAN_OK;
}

pigan_status check_common(const pigan_group_norm* a) {
  if (pigan_status st = check_sizes(a)) return st;
  const void* vecs[6] = {a->gamma, a->beta, a->mean, a->rstd, a->dgamma, a->dbeta};
  const char* names[6] = {"gamma", "beta", "mean", "rstd", "dgamma", "dbeta"};
  for (int i = 0; i < 6; ++i)
    if (pigan_status st = check_vec(vecs[i], names[i])) return st;
  return a->S > 0 ? check_field(a->x, "x", a) : PIGAN_OK;
}

pigan_status check_backward(const pigan_group_norm* a) {
  if (pigan_status st = check_common(a)) return st;
  if (a->S == 0) return PIGAN_OK;   // dx has no elements, and may have no address
  if (!a->dx.p && !a->dgamma && !a->dbeta) return fail(PIGAN_EINVAL, "no output: dx, dgamma and dbeta are null");
  if (!a->mean || !a->rstd) return fail(PIGAN_EINVAL, "mean and rstd: null pointer");
  if (pigan_status st = check_field(a->dy, "dy", a)) return st;
  if (a->add.p)
    if (pigan_status st = check_field(a->add, "add", a)) return st;
  return a->dx.p ? check_field(a->dx, "dx", a) : PIGAN_OK;
}

// strides of what there is one of may be any: 0, so that no product with them passes 64 bits
pigan_field used(pigan_field f, const pigan_group_norm* a) {
  if (a->P < 2) f.ld = 0;
  if (a->S < 2) f.ss = 0;
  if (a->n_groups < 2) f.gs = 0;
  return f;
}

Runs runs(const char* name, const pigan_field& field, const pigan_group_norm* a) {
  const int64_t es = (int64_t)esize(a->dt);
  const pigan_field f = used(field, a);
  return Runs(name, f.p, a->C * es).repeat(a->P, f.ld * es).repeat(a->S, f.ss * es).repeat(a->n_groups, f.gs * es);
}

pigan_status check_forward_apart(const pigan_group_norm* a, const void* ws, size_t need) {
  const int64_t chans = a->n_groups * a->C * 4, stats = a->n_groups * a->S * a->n * 4;
  const Runs outs[] = {runs("y", a->y, a), {"mean", a->mean, stats}, {"rstd", a->rstd, stats},
                       {"the workspace", need ? ws : nullptr, (int64_t)need}};
  const Runs ins[] = {runs("x", a->x, a), {"gamma", a->gamma, chans}, {"beta", a->beta, chans}};
  return check_apart(outs, ins, [](int o, int i) { return o == 0 && i == 0; });
}

pigan_status check_backward_apart(const pigan_group_norm* a, const void* ws, size_t need) {
  const int64_t chans = a->n_groups * a->C * 4, stats = a->n_groups * a->S * a->n * 4;
  const Runs outs[] = {runs("dx", a->dx, a), {"dgamma", a->dgamma, chans}, {"dbeta", a->dbeta, chans},
                       {"the workspace", need ? ws : nullptr, (int64_t)need}};
  const Runs ins[] = {runs("dy", a->dy, a), runs("add", a->dx.p ? a->add : NO_FIELD, a), runs("x", a->x, a),
                      {"gamma", a->gamma, chans}, {"beta", a->act != PIGAN_ACT_NONE ? a->beta : nullptr, chans},
                      {"mean", a->mean, stats}, {"rstd", a->rstd, stats}};
  return check_apart(outs, ins, [](int o, int i) { return o == 0 && i < 2; });
}

GnPlan plan(const pigan_group_norm* a, bool backward) {
  const int fields = backward ? 2 + !!a->dx.p + (a->dx.p && a->add.p) : 2;
  return gn_plan(backward, fields, (int)esize(a->dt), a->n_groups, a->S, a->P, a->C, a->n);
}
size_t forward_ws(const pigan_group_norm* a, const GnPlan& pl) {
  return a->S > 0 ? gn_forward_ws(pl, a->n_groups, a->S, a->n) : 0;
}
size_t backward_ws(const pigan_group_norm* a, const GnPlan& pl) {
  return a->S > 0 ? gn_backward_ws(pl, a->n_groups, a->S, a->C, a->n, a->dgamma || a->dbeta) : 0;
}

template <class T> Field<T> field(const pigan_field& f, const pigan_group_norm* a) {
  const pigan_field u = used(f, a);
  return {(T*)u.p, u.ld, u.ss, u.gs};
}

template <class T> GnArgs<T> args(const pigan_group_norm* a, const GnPlan& pl, void* ws) {
  GnArgs<T> k{};
  k.x = field<const T>(a->x, a);
  k.gamma = a->gamma;
  k.beta = a->beta;
  k.mean = a->mean;
  k.rstd = a->rstd;
  k.ws = (char*)ws;
  k.S = a->S;
  k.P = a->P;
  k.C = a->C;
  k.n = a->n;
  k.eps = a->eps;
  k.act = a->act;
  k.pl = pl;
  return k;
}

double field_bytes(const pigan_group_norm* a) { return (double)esize(a->dt) * a->n_groups * a->S * a->P * a->C; }

}  // namespace
}  // namespace pigan

using namespace pigan;

extern "C" {

size_t pigan_group_norm_forward_workspace(const pigan_group_norm* a) {
  size_t n = 0;
  guarded([&]() -> pigan_status {
    if (pigan_status st = check_sizes(a)) return st;
    n = std::max<size_t>(forward_ws(a, plan(a, false)), 1);
    return PIGAN_OK;
  });
  return n;
}

pigan_status pigan_group_norm_forward(const pigan_group_norm* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> pigan_status {
    if (pigan_status st = check_common(a)) return st;
    if (!(a->eps > 0.0f) || !__builtin_isfinite(a->eps)) return fail(PIGAN_EINVAL, "eps=%g must be finite and > 0", a->eps);
    if (a->S == 0) return PIGAN_OK;
    const GnPlan pl = plan(a, false);
    const size_t need = forward_ws(a, pl);
    if (pigan_status st = check_field(a->y, "y", a)) return st;
    if (pigan_status st = check_ws(ws, ws_bytes, need)) return st;
    if (pigan_status st = check_forward_apart(a, ws, need)) return st;
    const hipStream_t st = (hipStream_t)stream;
    ProfScope prof(st, "group_norm_fwd", 0.0, 2.0 * field_bytes(a));
    return by_dtype(a->dt, [&](auto t) -> pigan_status {
      typedef decltype(t) T;
      GnArgs<T> k = args<T>(a, pl, ws);
      k.out = field<T>(a->y, a);
      HIP_TRY(launch_gn_fwd(k, a->n_groups, st));
      return PIGAN_OK;
    });
  });
}

size_t pigan_group_norm_backward_workspace(const pigan_group_norm* a) {
  size_t n = 0;
  guarded([&]() -> pigan_status {
    if (pigan_status st = check_sizes(a)) return st;
    n = std::max<size_t>(backward_ws(a, plan(a, true)), 1);
    return PIGAN_OK;
  });
  return n;
}

pigan_status pigan_group_norm_backward(const pigan_group_norm* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> pigan_status {
    if (pigan_status st = check_backward(a)) return st;
    const GnPlan pl = plan(a, true);
    const size_t need = backward_ws(a, pl);
    if (pigan_status st = check_ws(ws, ws_bytes, need)) return st;
    if (a->S > 0)
      if (pigan_status st = check_backward_apart(a, ws, need)) return st;
    const hipStream_t st = (hipStream_t)stream;
    ProfScope prof(st, "group_norm_bwd", 0.0, (2.0 + !!a->dx.p + !!a->add.p) * field_bytes(a));
    return by_dtype(a->dt, [&](auto t) -> pigan_status {
      typedef decltype(t) T;
      GnArgs<T> k = args<T>(a, pl, ws);
      k.dy = field<const T>(a->dy, a);
      k.add = field<const T>(a->add, a);
      k.out = field<T>(a->dx, a);
      k.dgamma = a->dgamma;
      k.dbeta = a->dbeta;
      HIP_TRY(launch_gn_bwd(k, a->n_groups, st));
      return PIGAN_OK;
    });
  });
}

}  // extern "C"
