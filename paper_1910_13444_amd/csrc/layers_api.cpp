// C entry points of the linear layer, layer norm and the elementwise reverse
// pass: argument checks, choice of kernels, workspace.
#include <math.h>

#include <algorithm>

#include "api.h"
#include "linear.h"
#include "norm.h"
#include "operands.h"

namespace pigan {
namespace {

constexpr int64_t MAX_DIM = 0x7fffffff;

// [rows, cols] matrices of `groups` groups; p = NULL is left to the caller
pigan_status check_mat(const pigan_mat& m, const char* name, int32_t groups, int64_t rows, int64_t cols, size_t es) {
  if (!m.p) return fail(PIGAN_EINVAL, "%s: null pointer", name);
  if ((uintptr_t)m.p % es) return fail(PIGAN_EINVAL, "%s: pointer is not aligned to its elements", name);
  if (m.ld < cols || m.ld > (int64_t(1) << 40))
    return fail(PIGAN_EINVAL, "%s: row stride %lld out of [%lld, 2^40]", name, (long long)m.ld, (long long)cols);
  // (rows - 1) ld may reach 2^71
  const __int128 extent = rows > 0 ? (__int128)(rows - 1) * m.ld + cols : 0, most = __int128(1) << 46;
  if (extent > most) return fail(PIGAN_EINVAL, "%s: %lld rows of stride %lld, more than 2^46 elements", name,
                                 (long long)rows, (long long)m.ld);
  if (groups > 1 && (m.gs < (int64_t)extent || (groups - 1) * (__int128)m.gs + extent > most))
    return fail(PIGAN_EINVAL, "%s: group stride %lld does not hold a group of %lld elements, or %d of them pass 2^46", name,
                (long long)m.gs, (long long)extent, (int)groups);
  return PIGAN_OK;
}

pigan_status check_dims(int32_t groups, int32_t dt, int64_t M, int64_t N) {
  if (groups < 1 || groups > 65535) return fail(PIGAN_EINVAL, "n_groups=%d out of [1, 65535]", (int)groups);
  if (pigan_status st = check_dtype(dt)) return st;
  if (M < 0 || M > MAX_DIM) return fail(PIGAN_EINVAL, "M=%lld out of [0, 2^31 - 1]", (long long)M);
  if (N < 1 || N > MAX_DIM) return fail(PIGAN_EINVAL, "N=%lld out of [1, 2^31 - 1]", (long long)N);
  return PIGAN_OK;
}

// ---------------------------------------------------------------------------
// Operands that share memory.  A kernel's blocks read their inputs while others
// already store, so an output may be an input only where each element is read by
// the thread that then stores it, and the two are the same matrix.
// ---------------------------------------------------------------------------
// in bytes: `groups` groups of `rows` pieces of `len`; p = 0: none
struct Region {
  const char* name;
  int64_t p, len, rows, ld, groups, gs;
  Region(const char* n, const pigan_mat& m, int64_t M, int64_t N, int32_t G, size_t es)
      : name(n), p((int64_t)(uintptr_t)m.p), len(0), rows(1), ld(0), groups(1), gs(0) {
    if (!p) return;
    len = N * es; rows = M; ld = m.ld * es; groups = G; gs = G > 1 ? m.gs * es : 0;
    // the fewest levels that say the same, so that equal memory has equal fields
    if (rows == 1) { rows = groups; ld = gs; groups = 1; }
    if (groups > 1 && gs == rows * ld) { rows *= groups; groups = 1; }
    if (rows == 1 || (groups == 1 && ld == len)) { len *= rows; rows = 1; }
    if (rows == 1) ld = len;
    if (groups == 1) gs = 0;
  }
  Region(const char* n, const void* q, int64_t bytes) : Region(n, pigan_mat{(void*)q, bytes, 0}, 1, bytes, 1, 1) {}
  __int128 end() const { return (__int128)(groups - 1) * gs + (__int128)(rows - 1) * ld + len + p; }
  bool dense() const { return rows == 1 && groups == 1; }
  bool same(const Region& o) const {
    return p == o.p && len == o.len && rows == o.rows && ld == o.ld && groups == o.groups && gs == o.gs;
  }
};

// pieces of a (from 0 on) and of b (from d on), both ld apart
bool rows_meet(const Region& a, const Region& b, int64_t d) {
  for (int64_t s = floor_div(-d, a.ld), n = 0; n < 2; ++n, ++s)   // row j of b, row j + s of a: |distance| < ld
    if (s > -a.rows && s < b.rows && d + s * a.ld < a.len && -(d + s * a.ld) < b.len) return true;
  return false;
}

// the interval [from, to) and the pieces of b; where it does not meet the last piece
// that starts at or before `from`, it meets the next one or none
bool interval_meets(__int128 from, __int128 to, const Region& b) {
  const int64_t last_g = b.groups - 1, last_r = b.rows - 1;
  for (int64_t n = 0; n < 2; ++n) {
    int64_t g = b.groups > 1 ? (int64_t)((from - b.p) / b.gs) + n : 0;
    g = std::min(std::max<int64_t>(from < b.p ? 0 : g, 0), last_g);
    const __int128 at = (__int128)b.p + (__int128)g * b.gs;
    for (int64_t m = 0; m < 2; ++m) {
      __int128 r = from < at ? 0 : (from - at) / b.ld + m;
      r = std::min<__int128>(r, last_r);
      const __int128 q = at + r * b.ld;
      if (q < to && from < q + b.len) return true;
    }
  }
  return false;
}

// whether a and b have a byte in common; of two that are both apart in rows, by
// different strides, it is only told where they begin at the same address
bool share(const Region& a, const Region& b) {
  if (!a.p || !b.p || a.end() <= b.p || b.end() <= a.p) return false;
  if (a.dense()) return interval_meets(a.p, a.end(), b);
  if (b.dense()) return interval_meets(b.p, b.end(), a);
  if (a.ld != b.ld || a.gs != b.gs) return a.p == b.p;
  const int64_t d = b.p - a.p;
  if (a.groups == 1 && b.groups == 1) return rows_meet(a, b, d);
  for (int64_t t = floor_div(-d, a.gs), n = 0; n < 2; ++n, ++t)
    if (t > -a.groups && t < b.groups && rows_meet(a, b, d + t * a.gs)) return true;
  return false;
}

// No output shares memory with another operand, but for the same matrix where
// same_ok(output, input) says so.
template <int NO, int NI, class F>
pigan_status check_apart(const Region (&outs)[NO], const Region (&ins)[NI], F&& same_ok) {
  for (int o = 0; o < NO; ++o) {
    for (int q = 0; q < o; ++q)
      if (share(outs[o], outs[q])) return fail(PIGAN_EINVAL, "%s overlaps %s", outs[o].name, outs[q].name);
    for (int i = 0; i < NI; ++i)
      if (share(outs[o], ins[i]) && !(same_ok(o, i) && outs[o].same(ins[i])))
        return fail(PIGAN_EINVAL, "%s overlaps %s", outs[o].name, ins[i].name);
  }
  return PIGAN_OK;
}

template <class T> Mat<const T> in(const pigan_mat& m) { return {(const T*)m.p, m.ld, m.gs}; }
template <class T> Mat<T> out(const pigan_mat& m) { return {(T*)m.p, m.ld, m.gs}; }

// ---------------------------------------------------------------------------
// linear layer: checks
// ---------------------------------------------------------------------------
pigan_status check_linear(const pigan_linear* a) {
  if (!a) return fail(PIGAN_EINVAL, "null arguments");
  if (pigan_status st = check_dims(a->n_groups, a->dt, a->M, a->N)) return st;
  if (a->K < 1 || a->K > MAX_DIM) return fail(PIGAN_EINVAL, "K=%lld out of [1, 2^31 - 1]", (long long)a->K);
  if (pigan_status st = check_act(a->act)) return st;
  if (a->reserved) return fail(PIGAN_EINVAL, "reserved=%d must be 0", (int)a->reserved);
  return PIGAN_OK;
}

pigan_status check_forward(const pigan_linear* a) {
  if (pigan_status st = check_linear(a)) return st;
  const size_t es = esize(a->dt);
  const int32_t G = a->n_groups;
  if (pigan_status st = check_mat(a->w, "w", G, a->N, a->K, es)) return st;
  if (pigan_status st = check_vec(a->bias, "bias")) return st;
  if (a->M > 0 || a->x.p)
    if (pigan_status st = check_mat(a->x, "x", G, a->M, a->K, es)) return st;
  if (a->M > 0 || a->y.p)
    if (pigan_status st = check_mat(a->y, "y", G, a->M, a->N, es)) return st;
  if (a->pre.p)
    if (pigan_status st = check_mat(a->pre, "pre", G, a->M, a->N, es)) return st;
  if (a->add.p)
    if (pigan_status st = check_mat(a->add, "add", G, a->M, a->N, es)) return st;
  return PIGAN_OK;
}

pigan_status check_backward(const pigan_linear* a) {
  if (pigan_status st = check_linear(a)) return st;
  const size_t es = esize(a->dt);
  const int32_t G = a->n_groups;
  const bool rows = a->M > 0;
  // without rows dx has no elements, and may have no address
  if (rows && !a->dx.p && !a->dw && !a->db) return fail(PIGAN_EINVAL, "no output: dx, dw and db are null");
  if (rows || a->g.p)
    if (pigan_status st = check_mat(a->g, "g", G, a->M, a->N, es)) return st;
  if (a->dx.p) {
    if (pigan_status st = check_mat(a->dx, "dx", G, a->M, a->K, es)) return st;
    if (pigan_status st = check_mat(a->w, "w", G, a->N, a->K, es)) return st;
    if (a->act != PIGAN_ACT_NONE && !a->pre.p && rows)
      return fail(PIGAN_EINVAL, "pre: the derivative of activation %d needs the pre-activation", (int)a->act);
    if (a->act == PIGAN_ACT_NONE && a->pre.p) return fail(PIGAN_EINVAL, "pre: given without an activation");
    if (a->pre.p)
      if (pigan_status st = check_mat(a->pre, "pre", G, a->M, a->K, es)) return st;
    if (a->add.p)
      if (pigan_status st = check_mat(a->add, "add", G, a->M, a->K, es)) return st;
  }
  if (a->dw && rows)
    if (pigan_status st = check_mat(a->x, "x", G, a->M, a->K, es)) return st;
  if (a->dw && (__int128)a->N * a->K * G > (__int128(1) << 46))
    return fail(PIGAN_EINVAL, "dw: %d of %lld x %lld, more than 2^46 elements", (int)G, (long long)a->N, (long long)a->K);
  if (pigan_status st = check_vec(a->dw, "dw")) return st;
  return check_vec(a->db, "db");
}

const pigan_mat NO_MAT = {};

pigan_status check_forward_apart(const pigan_linear* a, const void* ws, size_t need) {
  const size_t es = esize(a->dt);
  const int32_t G = a->n_groups;
  const Region outs[] = {{"y", a->y, a->M, a->N, G, es}, {"pre", a->pre, a->M, a->N, G, es},
                         {"the workspace", need ? ws : nullptr, (int64_t)need}};
  const Region ins[] = {{"add", a->add, a->M, a->N, G, es}, {"x", a->x, a->M, a->K, G, es}, {"w", a->w, a->N, a->K, G, es},
                        {"bias", a->bias, G * a->N * 4}};
  return check_apart(outs, ins, [](int o, int i) { return o == 0 && i == 0; });
}

// (what a call does not read may be anywhere)
pigan_status check_backward_apart(const pigan_linear* a, const void* ws, size_t need) {
  const size_t es = esize(a->dt);
  const int32_t G = a->n_groups;
  const bool dx = a->dx.p;
  const Region outs[] = {{"dx", a->dx, a->M, a->K, G, es}, {"dw", a->dw, G * a->N * a->K * 4}, {"db", a->db, G * a->N * 4},
                         {"the workspace", need ? ws : nullptr, (int64_t)need}};
  const Region ins[] = {{"pre", dx ? a->pre : NO_MAT, a->M, a->K, G, es}, {"add", dx ? a->add : NO_MAT, a->M, a->K, G, es},
                        {"g", a->g, a->M, a->N, G, es}, {"w", dx ? a->w : NO_MAT, a->N, a->K, G, es},
                        {"x", a->dw ? a->x : NO_MAT, a->M, a->K, G, es}};
  return check_apart(outs, ins, [](int o, int i) { return o == 0 && i < 2; });
}

// ---------------------------------------------------------------------------
// linear layer: choice of tile and split
// ---------------------------------------------------------------------------
struct MmPlan {
  int tile = MM_64;
  int n_split = 1;
  double us = 1e30;   // modelled
};

// Modelled time of a launch on 256 CUs, from measured times: of a stage (64 values
// of k) with 1, 2, .. blocks on a CU, of a block's start and epilogue, and of a
// kernel's first blocks (the 256 tile's unrolled epilogue has to be fetched).  The
// splits of a contraction add a launch and the partials' way through memory.
//   M x K x N, us            taken, modelled | measured    the others measured
//   fwd 4096 x 2048 x 2048   128    49 | 38                256: 53, 64: 56
//   fwd 20000 x 1032 x 1000  128    85 | 81                256: 85, 64: 105
//   fwd 512 x 2048 x 2048    64K    13 | 13                64: 13, 128: 20
//   dx 32768 x 512 x 512     128    38 | 39                256: 40, 64: 45
//   dw 20000 x 1032 x 1000   128/4  81 | 78                256/8: 75, 128/2: 118
//   dw 32768 x 512 x 512     128/16 46 | 38                64/16: 45, 256: over 46
// (64 with k down the rows of an operand: 8192^3 in 2066 and 2275 us, forward 1605)
constexpr double STAGE_FWD[3][4] = {{0.33, 0.5, 0.68, 0.85}, {0.6, 1.16, 0, 0}, {1.7, 0, 0, 0}};
constexpr double STAGE_BWD[3][4] = {{0.42, 0.63, 0.84, 1.05}, {0.6, 1.16, 0, 0}, {1.7, 0, 0, 0}};
constexpr double BLOCK_US[3] = {3.0, 7.0, 14.0}, FIRST_US[3] = {2.0, 5.0, 14.0};
constexpr int PER_CU[3] = {4, 2, 1};

double tiles_of(int64_t I, int64_t J, int G, int t) {
  const int64_t s = mm_tile_side(t);
  return (double)((I + s - 1) / s) * (double)((J + s - 1) / s) * G;
}
// a launch's x dimension holds fewer than 2^32 threads
bool grid_holds(double blocks, int t) { return blocks * mm_tile_threads(t) < 4294967296.0; }
double split_us(int64_t I, int64_t J, int G, int split) {
  return split > 1 ? 8.0 + (double)G * I * J * 4.0 * (split * 2 + 1) / 5e6 : 0.0;
}

// a stage with `blocks` blocks spread over the chip, and how full they make a CU
double stage_of(const double (&stage)[3][4], int t, double blocks, double& load) {
  load = std::min<double>(PER_CU[t], std::max(1.0, blocks / 256));
  const int lo = (int)load, hi = std::min(lo + 1, PER_CU[t]);
  return stage[t][lo - 1] + (load - lo) * (stage[t][hi - 1] - stage[t][lo - 1]);
}

MmPlan plan_mm(const double (&STAGE_US)[3][4], int64_t I, int64_t J, int64_t K, int pairs, int G) {
  const int64_t nk = (K + 63) / 64;
  MmPlan best;
  double load;
  for (int t = MM_64; t <= MM_256; ++t)
    for (int split = 1; split <= 64 && split <= nk; split *= 2) {
      if (split > 1 && nk * pairs / split < 4) break;
      const double blocks = tiles_of(I, J, G, t) * split, rounds = ceil(blocks / (256.0 * PER_CU[t]));
      if (!grid_holds(blocks, t)) break;
      const double stages = (double)((nk + split - 1) / split) * pairs;
      const double us = rounds * (stages * stage_of(STAGE_US, t, blocks, load) + BLOCK_US[t]) + FIRST_US[t] +
                        split_us(I, J, G, split);
      if (us < best.us) best = {t, split, us};
    }
  // 64 tiles of four groups, one on a CU: a stage of each group in the time of four blocks' stages
  const double us = ceil(tiles_of(I, J, G, MM_64) / 256) * ((double)((nk + 3) / 4) * pairs * STAGE_US[MM_64][3] + 4.0) +
                    FIRST_US[MM_64];
  if (nk >= 8 && us < best.us && grid_holds(tiles_of(I, J, G, MM_64), MM_64K)) best = {MM_64K, 1, us};
  return best;
}

// Both products of a reverse pass in one launch, dx on whole contractions: the
// time is that of the longest block, or of all of them spread over the chip.
// Taken where it is shorter than one launch after the other (2 us between them).
bool plan_both(int64_t M, int64_t N, int64_t K, int pairs, int G, MmPlan& dx, MmPlan& dw, double& best) {
  const int64_t nx = (N + 63) / 64, nw = (M + 63) / 64;
  best = dx.us + dw.us + 2.0;
  bool both = false;
  for (int t = MM_64; t <= MM_128; ++t)
    for (int split = 1; split <= 64 && split <= nw; split *= 2) {
      if (split > 1 && nw * pairs / split < 4) break;
      const double b1 = tiles_of(M, K, G, t), b2 = tiles_of(N, K, G, t) * split;
      if (!grid_holds(b1 + b2, t)) break;
      double load;
      const double stage = stage_of(STAGE_BWD, t, b1 + b2, load);
      const double t1 = nx * pairs * stage + BLOCK_US[t], t2 = (double)((nw + split - 1) / split) * pairs * stage + BLOCK_US[t];
      const double us = std::max(std::max(t1, t2), (b1 * t1 + b2 * t2) / (256.0 * load)) + FIRST_US[t] + split_us(N, K, G, split);
      if (us < best) {
        best = us;
        both = true;
        dx = {t, 1, t1};
        dw = {t, split, t2};
      }
    }
  return both;
}

// Strips (k_short_fwd) against tiles.  Up to 8 rows w is read once, and little work
// is over before a tile is full: strips.  Up to 64 rows it is read by up to four
// strips of 16 rows, and the shorter modelled time decides.
//   us, strips | tiles (with their planes in fp32)
//   M x K x N             bf16           fp32
//   16 x 1024 x 1024      4.6 |  8.2     6.3 | 19.5
//   64 x 1024 x 1024      4.8 |  8.4     6.4 | 20.8
//   64 x 2048 x 2048      9.9 | 10.7    16.8 | 28.8
//   16 x 8192 x 2048     17.1 | 17.0    30.4 | 69.7
//   64 x 8192 x 2048     31.2 | 16.8    58.7 | 75.0
//   16 x 1024 x 8192      6.3 |  8.2    10.0 | 36.0
//   64 x 1024 x 8192     17.0 |  8.8    31.1 | 42.6
//   19531 x 32 x 32       5.3 |  4.8     5.1 | 10.8    (work 2e7)
//   1220 x 128 x 128      3.8 |  4.3     4.4 | 10.7    (2e7)
//   24414 x 64 x 64       8.6 |  5.2     9.9 | 14.8    (1e8)
//   3333 x 100 x 300      7.0 |  6.2     9.1 | 12.4    (1e8)
// (1000 random layers of 9 to 64 rows: up to 4.7 times as fast as strips alone, one of
// them slower by 20 %)
bool short_ok(const pigan_linear* a) {
  if (a->M <= 8) return true;
  const double work = (double)a->n_groups * a->M * a->K * a->N;
  return work <= (a->dt == PIGAN_FP32 ? 1e8 : 2e7) && (a->M + 15) / 16 <= 65535;
}

// Modelled time of strips of 16 rows and columns: a launch, and rounds of 256 blocks
// that stream K values of their rows (64 x 8192 x 2048: 30 and 57 us)
double short_us(const pigan_linear* a) {
  const double blocks = (double)((a->M + 15) / 16) * (double)((a->N + 15) / 16) * a->n_groups;
  const double round = std::max(0.23, 0.05 + (a->dt == PIGAN_FP32 ? 3.4 : 1.7) * a->K / 1024.0);
  return 3.0 + std::max(1.0, blocks / 256) * round;
}
double split3_us(const pigan_linear* a) {
  return 2.0 + 10.0 * a->n_groups * a->K * ((double)a->M + a->N) / 4.7e6;
}

// A matrix of a product, or its form in the workspace: rows of whole, aligned
// pieces, zeros behind them; of fp32 three bf16 planes.
struct Operand {
  const pigan_mat* m = nullptr;
  int64_t rows = 0, cols = 0, Kp = 0;   // Kp > 0: in the workspace
  size_t at = 0;
  // as it is, its rows may go straight to LDS
  bool whole(int G) const { return cols % 8 == 0 && mm_whole(MmOperand<bf16>{(const bf16*)m->p, m->ld, m->gs, 0}, cols, G); }
  double bytes(int G) const { return 2.0 * G * rows * cols; }
  void take(Carver& cv, int G, int planes) {
    Kp = round_up(cols, 8);
    at = cv.take((size_t)planes * G * rows * Kp * 2);
  }
  template <class T> MmOperand<T> get(char* ws, int G) const {
    if (Kp) return {(const T*)(ws + at), Kp, rows * Kp, (int64_t)G * rows * Kp};
    return {(const T*)m->p, m->ld, m->gs, 0};
  }
  bool direct(char* ws, int G) const { return Kp ? mm_whole(get<bf16>(ws, G), cols, G) : whole(G); }
};

// 16-bit operands that have to be read element by element or in unaligned pieces
// are copied first where that costs less than it saves: `us` is what the products
// take on aligned rows, `ratio` how much longer they take without.
//   bf16, us: whole pieces | copied | as they are
//   fwd 4096 x 4096 x 4096    107 | 118 | 193     bwd  227 | 247 | 415
//   fwd 20000 x 1032 x 1000    70 |     |  83     bwd  122 | 140 | 351
//   fwd 131072 x 1024 x 1024  284 |     | 466     bwd  529 | 736 | 913
// (the second and third forward are not copied: x alone would take 20 and 120 us.  The
// ratios are those of the sizes that lose least: at the third, and at the first, where
// the unaligned kernel takes 1.6 to 1.8 times as long, a copy would still pay)
constexpr double LOOSE_FWD = 1.35, LOOSE_BWD = 2.0;

template <int N> void plan_copies(Operand* (&ops)[N], int G, double us, double ratio, Carver& cv) {
  double cost = 4.0;
  for (Operand* o : ops)
    if (o->m && !o->whole(G)) cost += 2 * o->bytes(G) / 4.5e6;
  if (cost == 4.0 || cost > us * (ratio - 1.0)) return;
  for (Operand* o : ops)
    if (o->m && !o->whole(G)) o->take(cv, G, 1);
}

// fills the workspace forms of the operands that have one
template <int N> hipError_t fill_operands(const Operand* const (&ops)[N], bool fp32, int G, char* ws, hipStream_t st) {
  SplitSet split[N];
  PackSet pack[N];
  int n = 0;
  for (const Operand* o : ops)
    if (o->Kp) {
      split[n] = {(const float*)o->m->p, o->m->ld, o->m->gs, o->rows, o->cols, o->Kp, (bf16*)(ws + o->at)};
      pack[n++] = {o->m->p, o->m->ld, o->m->gs, o->rows, o->cols, o->Kp, ws + o->at};
    }
  if (!n) return hipSuccess;
  return fp32 ? launch_split3(split, n, G, st) : launch_pack(pack, n, G, st);
}

struct ForwardPlan {
  bool brief = false;
  MmPlan mm;
  Operand x, w;
  size_t part = 0, total = 0;
};

ForwardPlan plan_forward(const pigan_linear* a) {
  ForwardPlan p;
  if (a->M == 0 || (p.brief = short_ok(a))) return p;
  Carver cv;
  const int G = a->n_groups;
  const bool fp32 = a->dt == PIGAN_FP32;
  p.mm = plan_mm(STAGE_FWD, a->M, a->N, a->K, fp32 ? 6 : 1, G);
  p.x = {&a->x, a->M, a->K};
  p.w = {&a->w, a->N, a->K};
  if (a->M <= 64) {
    // (16-bit operands without whole pieces have no tile of four groups)
    const bool whole = fp32 || (p.x.whole(G) && p.w.whole(G));
    double tiles = p.mm.us;
    if (!whole && p.mm.tile == MM_64K) tiles = (double)((a->K + 63) / 64) * STAGE_FWD[MM_64][0] + BLOCK_US[MM_64] + FIRST_US[MM_64];
    tiles = tiles * (whole ? 1.0 : LOOSE_FWD) + (fp32 ? split3_us(a) : 0.0);
    if ((p.brief = short_us(a) <= 1.1 * tiles)) return p;   // what the model is off by
  }
  Operand* ops[2] = {&p.x, &p.w};
  if (!fp32) plan_copies(ops, G, p.mm.us, LOOSE_FWD, cv);
  else for (Operand* o : ops) o->take(cv, G, 3);
  if (p.mm.n_split > 1) p.part = cv.take((size_t)G * p.mm.n_split * a->M * a->N * 4);
  p.total = cv.off;
  return p;
}

struct BackwardPlan {
  MmPlan dx, dw;
  Operand g, w, x;   // those that are used
  size_t part_dx = 0, part_dw = 0, part_db = 0, total = 0;
  int db_slots = 0;
  bool both = false;   // dx and dw in one launch
};

constexpr int COLSUM_SPLITS = 64;

BackwardPlan plan_backward(const pigan_linear* a) {
  BackwardPlan p;
  if (a->M == 0) return p;
  Carver cv;
  const int G = a->n_groups;
  const bool fp32 = a->dt == PIGAN_FP32;
  const int pairs = fp32 ? 6 : 1;
  // tiles and splits do not depend on which gradients are wanted: the same sums for each of them
  p.dx = plan_mm(STAGE_BWD, a->M, a->K, a->N, pairs, G);
  p.dw = plan_mm(STAGE_BWD, a->N, a->K, a->M, pairs, G);
  double us;
  p.both = plan_both(a->M, a->N, a->K, pairs, G, p.dx, p.dw, us) && a->dx.p && a->dw;
  if (a->dx.p || a->dw) p.g = {&a->g, a->M, a->N};
  if (a->dx.p) p.w = {&a->w, a->N, a->K};
  if (a->dw) p.x = {&a->x, a->M, a->K};
  Operand* ops[3] = {&p.g, &p.w, &p.x};
  if (!fp32) plan_copies(ops, G, us, LOOSE_BWD, cv);
  else for (Operand* o : ops) if (o->m) o->take(cv, G, 3);
  if (a->dx.p) {
    if (p.dx.n_split > 1) p.part_dx = cv.take((size_t)G * p.dx.n_split * a->M * a->K * 4);
  }
  if (a->dw) {
    if (p.dw.n_split > 1) p.part_dw = cv.take((size_t)G * p.dw.n_split * a->N * a->K * 4);
    const int64_t side = std::min(mm_tile_side(p.dw.tile), 128);   // the smaller of the tiles that it may become
    p.db_slots = p.dw.n_split * (int)((a->K + side - 1) / side);
  } else {
    p.db_slots = (int)std::min<int64_t>(a->M, COLSUM_SPLITS);
  }
  if (a->db && (!a->dw || p.dw.n_split > 1)) p.part_db = cv.take((size_t)G * p.db_slots * a->N * 4);
  p.total = cv.off;
  return p;
}

// ---------------------------------------------------------------------------
// linear layer: launches
// ---------------------------------------------------------------------------
template <class TO> MmOut<TO> forward_out(const pigan_linear* a, const MmPlan& mm, float* part) {
  MmOut<TO> o{};
  o.I = a->M;
  o.J = a->N;
  o.act = a->act;
  o.n_split = mm.n_split;
  o.bias = a->bias;
  o.pre = (TO*)a->pre.p; o.ldp = a->pre.ld; o.gsp = a->pre.gs;
  o.add = (const TO*)a->add.p; o.lda = a->add.ld; o.gsa = a->add.gs;
  o.out = (TO*)a->y.p; o.ldo = a->y.ld; o.gso = a->y.gs;
  o.part = mm.n_split > 1 ? part : nullptr;
  return o;
}

template <class T> MmOperand<T> operand(const pigan_mat& m) { return {(const T*)m.p, m.ld, m.gs, 0}; }

// the largest tile and the shared one are there for aligned operands only
int tile_for(const MmPlan& mm, bool direct) {
  return direct ? mm.tile : mm.tile == MM_256 ? (int)MM_128 : mm.tile == MM_64K ? (int)MM_64 : mm.tile;
}

// T: operands of the products; TO: storage type of the layer
template <class T, class TO>
pigan_status forward_tiles(const pigan_linear* a, const ForwardPlan& p, char* ws, hipStream_t st) {
  const int G = a->n_groups;
  const Operand* ops[2] = {&p.x, &p.w};
  HIP_TRY(fill_operands(ops, sizeof(TO) == 4, G, ws, st));
  const bool direct = p.x.direct(ws, G) && p.w.direct(ws, G);
  MmArgs<T, TO> m{p.x.get<T>(ws, G), p.w.get<T>(ws, G), a->K, sizeof(TO) == 4 ? 6 : 1,
                  forward_out<TO>(a, p.mm, (float*)(ws + p.part)), nullptr};
  HIP_TRY(launch_mm_fwd(m, tile_for(p.mm, direct), direct, G, st));
  if (p.mm.n_split > 1) HIP_TRY(launch_mm_join_fwd(m.o, G, st));
  return PIGAN_OK;
}

pigan_status run_forward(const pigan_linear* a, const ForwardPlan& p, char* ws, hipStream_t st) {
  const int G = a->n_groups;
  const double es = (double)esize(a->dt), MN = (double)a->M * a->N;
  ProfScope prof(st, "linear_fwd", 2.0 * G * MN * a->K,
                 G * (es * ((double)a->M * a->K + (double)a->N * a->K + MN * (1 + !!a->pre.p + !!a->add.p)) + 4.0 * a->N));
  if (p.brief)
    return by_dtype(a->dt, [&](auto t) -> pigan_status {
      typedef decltype(t) T;
      MmArgs<T, T> m{operand<T>(a->x), operand<T>(a->w), a->K, 1, forward_out<T>(a, MmPlan{}, nullptr), nullptr};
      HIP_TRY(launch_short_fwd(m, G, st));
      return PIGAN_OK;
    });
  return a->dt == PIGAN_FP32 ? forward_tiles<bf16, float>(a, p, ws, st)
         : a->dt == PIGAN_BF16 ? forward_tiles<bf16, bf16>(a, p, ws, st)
                               : forward_tiles<f16, f16>(a, p, ws, st);
}

// T: operands of the products; TO: storage type of the layer
template <class T, class TO>
pigan_status backward_products(const pigan_linear* a, const BackwardPlan& p, char* ws, hipStream_t st) {
  const int G = a->n_groups;
  const double es = (double)esize(a->dt), MN = (double)a->M * a->N, MK = (double)a->M * a->K, NK = (double)a->N * a->K;
  const Operand* ops[3] = {&p.g, &p.w, &p.x};
  HIP_TRY(fill_operands(ops, sizeof(TO) == 4, G, ws, st));
  const bool direct_dx = a->dx.p && p.g.direct(ws, G) && p.w.direct(ws, G);
  const bool direct_dw = a->dw && p.g.direct(ws, G) && p.x.direct(ws, G);
  const int pairs = sizeof(TO) == 4 ? 6 : 1;
  MmArgs<T, TO> dx{};
  MmArgs<T, float> dw{};
  dx.pairs = dw.pairs = pairs;
  dx.a = dw.a = p.g.get<T>(ws, G);
  dx.K = a->N;
  dw.K = a->M;
  const int tile_dw = tile_for(p.dw, direct_dw), side = mm_tile_side(tile_dw);
  const int slots = p.dw.n_split * (int)((a->K + side - 1) / side);
  if (a->dx.p) {
    dx.b = p.w.get<T>(ws, G);
    dx.o.I = a->M;
    dx.o.J = a->K;
    dx.o.act = a->act;
    dx.o.n_split = p.dx.n_split;
    dx.o.pre = (TO*)a->pre.p; dx.o.ldp = a->pre.ld; dx.o.gsp = a->pre.gs;
    dx.o.add = (const TO*)a->add.p; dx.o.lda = a->add.ld; dx.o.gsa = a->add.gs;
    dx.o.out = (TO*)a->dx.p; dx.o.ldo = a->dx.ld; dx.o.gso = a->dx.gs;
    dx.o.part = p.dx.n_split > 1 ? (float*)(ws + p.part_dx) : nullptr;
  }
  if (a->dw) {
    dw.b = p.x.get<T>(ws, G);
    dw.o.I = a->N;
    dw.o.J = a->K;
    dw.o.n_split = p.dw.n_split;
    dw.o.out = a->dw; dw.o.ldo = a->K; dw.o.gso = a->N * a->K;
    dw.o.part = p.dw.n_split > 1 ? (float*)(ws + p.part_dw) : nullptr;
    dw.part_db = !a->db ? nullptr : p.dw.n_split == 1 ? a->db : (float*)(ws + p.part_db);
  }
  const double fl = 2.0 * G * MN * a->K, bx = G * es * (MN + NK + MK * (1 + !!a->pre.p + !!a->add.p));
  const double bw = G * (es * (MN + MK) + 4.0 * NK);
  if (p.both && direct_dx && direct_dw) {
    ProfScope prof(st, "linear_bwd", 2 * fl, bx + bw);
    HIP_TRY(launch_mm_both(dx, dw, p.dx.tile, p.dw.us > p.dx.us, G, st));
    if (p.dw.n_split > 1) HIP_TRY(launch_mm_join_dw(dw.o, dw.part_db, slots, a->db, G, st));
    return PIGAN_OK;
  }
  if (a->dx.p) {
    ProfScope prof(st, "linear_dx", fl, bx);
    HIP_TRY(launch_mm_dx(dx, tile_for(p.dx, direct_dx), direct_dx, G, st));
    if (p.dx.n_split > 1) HIP_TRY(launch_mm_join_dx(dx.o, G, st));
  }
  if (a->dw) {
    ProfScope prof(st, "linear_dw", fl, bw);
    HIP_TRY(launch_mm_dw(dw, tile_dw, direct_dw, G, st));
    if (p.dw.n_split > 1) HIP_TRY(launch_mm_join_dw(dw.o, dw.part_db, slots, a->db, G, st));
  }
  return PIGAN_OK;
}

pigan_status run_backward(const pigan_linear* a, const BackwardPlan& p, char* ws, hipStream_t st) {
  const int G = a->n_groups;
  if (a->M == 0) {   // sums over no rows
    if (a->dw) HIP_TRY(launch_zeros(a->dw, G * a->N * a->K, st));
    if (a->db) HIP_TRY(launch_zeros(a->db, G * a->N, st));
    return PIGAN_OK;
  }
  if (a->dx.p || a->dw) {
    const pigan_status s = a->dt == PIGAN_FP32   ? backward_products<bf16, float>(a, p, ws, st)
                           : a->dt == PIGAN_BF16 ? backward_products<bf16, bf16>(a, p, ws, st)
                                                 : backward_products<f16, f16>(a, p, ws, st);
    if (s != PIGAN_OK) return s;
  }
  if (a->db && !a->dw) {   // by themselves
    float* part = (float*)(ws + p.part_db);
    pigan_status s = by_dtype(a->dt, [&](auto t) -> pigan_status {
      HIP_TRY(launch_colsum_rows(in<decltype(t)>(a->g), a->M, a->N, p.db_slots, part, G, st));
      return PIGAN_OK;
    });
    if (s != PIGAN_OK) return s;
    HIP_TRY(launch_slot_sum(part, (int64_t)p.db_slots * a->N, p.db_slots, a->N, a->db, a->N, nullptr, G, st));
  }
  return PIGAN_OK;
}

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------
pigan_status check_norm(const pigan_norm* a) {
  if (!a) return fail(PIGAN_EINVAL, "null arguments");
  if (pigan_status st = check_dims(a->n_groups, a->dt, a->M, a->N)) return st;
  if (a->reserved) return fail(PIGAN_EINVAL, "reserved=%d must be 0", (int)a->reserved);
  const void* vecs[6] = {a->gamma, a->beta, a->mean, a->rstd, a->dgamma, a->dbeta};
  const char* names[6] = {"gamma", "beta", "mean", "rstd", "dgamma", "dbeta"};
  for (int i = 0; i < 6; ++i)
    if (pigan_status st = check_vec(vecs[i], names[i])) return st;
  if (a->M > 0 || a->x.p) return check_mat(a->x, "x", a->n_groups, a->M, a->N, esize(a->dt));
  return PIGAN_OK;
}

pigan_status check_norm_backward(const pigan_norm* a) {
  if (pigan_status st = check_norm(a)) return st;
  const size_t es = esize(a->dt);
  if (a->M == 0) return PIGAN_OK;   // dx has no elements, and may have no address
  if (!a->dx.p && !a->dgamma && !a->dbeta) return fail(PIGAN_EINVAL, "no output: dx, dgamma and dbeta are null");
  if (!a->mean || !a->rstd) return fail(PIGAN_EINVAL, "mean and rstd: null pointer");
  if (pigan_status st = check_mat(a->dy, "dy", a->n_groups, a->M, a->N, es)) return st;
  if (a->add.p)
    if (pigan_status st = check_mat(a->add, "add", a->n_groups, a->M, a->N, es)) return st;
  if (a->dx.p) {
    if (pigan_status st = check_mat(a->dx, "dx", a->n_groups, a->M, a->N, es)) return st;
  }
  return PIGAN_OK;
}

pigan_status check_norm_apart(const pigan_norm* a) {
  const size_t es = esize(a->dt);
  const int32_t G = a->n_groups;
  const int64_t cols = G * a->N * 4, rows = G * a->M * 4;
  const Region outs[] = {{"y", a->y, a->M, a->N, G, es}, {"mean", a->mean, rows}, {"rstd", a->rstd, rows}};
  const Region ins[] = {{"x", a->x, a->M, a->N, G, es}, {"gamma", a->gamma, cols}, {"beta", a->beta, cols}};
  return check_apart(outs, ins, [](int o, int i) { return o == 0 && i == 0; });
}

pigan_status check_norm_backward_apart(const pigan_norm* a, const void* ws, size_t need) {
  const size_t es = esize(a->dt);
  const int32_t G = a->n_groups;
  const int64_t cols = G * a->N * 4, rows = G * a->M * 4;
  const Region outs[] = {{"dx", a->dx, a->M, a->N, G, es}, {"dgamma", a->dgamma, cols}, {"dbeta", a->dbeta, cols},
                         {"the workspace", need ? ws : nullptr, (int64_t)need}};
  const Region ins[] = {{"dy", a->dy, a->M, a->N, G, es}, {"add", a->dx.p ? a->add : NO_MAT, a->M, a->N, G, es},
                        {"x", a->x, a->M, a->N, G, es}, {"gamma", a->gamma, cols}, {"mean", a->mean, rows},
                        {"rstd", a->rstd, rows}};
  return check_apart(outs, ins, [](int o, int i) { return o == 0 && i < 2; });
}

template <class T> NormArgs<T> norm_args(const pigan_norm* a) {
  NormArgs<T> n{};
  n.x = in<T>(a->x);
  n.gamma = a->gamma;
  n.beta = a->beta;
  n.mean = a->mean;
  n.rstd = a->rstd;
  n.M = a->M;
  n.N = a->N;
  n.eps = a->eps;
  return n;
}

size_t norm_ws(const pigan_norm* a) {
  return a->dgamma || a->dbeta ? (size_t)a->n_groups * norm_part_floats((int)esize(a->dt), a->M, a->N) * 4 : 0;
}

}  // namespace
}  // namespace pigan

using namespace pigan;

extern "C" {

size_t pigan_linear_forward_workspace(const pigan_linear* a) {
  size_t n = 0;
  guarded([&]() -> pigan_status {
    if (pigan_status st = check_linear(a)) return st;
    n = std::max<size_t>(plan_forward(a).total, 1);
    return PIGAN_OK;
  });
  return n;
}

pigan_status pigan_linear_forward(const pigan_linear* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> pigan_status {
    if (pigan_status st = check_forward(a)) return st;
    const ForwardPlan p = plan_forward(a);
    if (pigan_status st = check_ws(ws, ws_bytes, p.total)) return st;
    if (a->M == 0) return PIGAN_OK;
    if (pigan_status st = check_forward_apart(a, ws, p.total)) return st;
    return run_forward(a, p, (char*)ws, (hipStream_t)stream);
  });
}

size_t pigan_linear_backward_workspace(const pigan_linear* a) {
  size_t n = 0;
  guarded([&]() -> pigan_status {
    if (pigan_status st = check_linear(a)) return st;
    n = std::max<size_t>(plan_backward(a).total, 1);
    return PIGAN_OK;
  });
  return n;
}

pigan_status pigan_linear_backward(const pigan_linear* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> pigan_status {
    if (pigan_status st = check_backward(a)) return st;
    const BackwardPlan p = plan_backward(a);
    if (pigan_status st = check_ws(ws, ws_bytes, p.total)) return st;
    if (a->M > 0)
      if (pigan_status st = check_backward_apart(a, ws, p.total)) return st;
    return run_backward(a, p, (char*)ws, (hipStream_t)stream);
  });
}

pigan_status pigan_act_backward(const pigan_act_args* a, void* stream) {
  return guarded([&]() -> pigan_status {
    if (!a) return fail(PIGAN_EINVAL, "null arguments");
    if (pigan_status st = check_dims(a->n_groups, a->dt, a->M, a->N)) return st;
    if (pigan_status st = check_act(a->act)) return st;
    if (a->act == PIGAN_ACT_NONE) return fail(PIGAN_EINVAL, "act: no activation to differentiate");
    if (a->reserved) return fail(PIGAN_EINVAL, "reserved=%d must be 0", (int)a->reserved);
    if (a->M == 0) return PIGAN_OK;
    const size_t es = esize(a->dt);
    if (pigan_status st = check_mat(a->dy, "dy", a->n_groups, a->M, a->N, es)) return st;
    if (pigan_status st = check_mat(a->pre, "pre", a->n_groups, a->M, a->N, es)) return st;
    if (pigan_status st = check_mat(a->g, "g", a->n_groups, a->M, a->N, es)) return st;
    const Region outs[] = {{"g", a->g, a->M, a->N, a->n_groups, es}};
    const Region ins[] = {{"dy", a->dy, a->M, a->N, a->n_groups, es}, {"pre", a->pre, a->M, a->N, a->n_groups, es}};
    if (pigan_status st = check_apart(outs, ins, [](int, int) { return true; })) return st;
    const hipStream_t st = (hipStream_t)stream;
    ProfScope prof(st, "act_backward", 0.0, 3.0 * es * a->n_groups * (double)a->M * a->N);
    return by_dtype(a->dt, [&](auto t) -> pigan_status {
      typedef decltype(t) T;
      HIP_TRY(launch_act_bwd<T>(a->act, in<T>(a->dy), in<T>(a->pre), out<T>(a->g), a->M, a->N, a->n_groups, st));
      return PIGAN_OK;
    });
  });
}

pigan_status pigan_layer_norm_forward(const pigan_norm* a, void* stream) {
  return guarded([&]() -> pigan_status {
    if (pigan_status st = check_norm(a)) return st;
    if (!(a->eps > 0.0f) || !__builtin_isfinite(a->eps)) return fail(PIGAN_EINVAL, "eps=%g must be finite and > 0", a->eps);
    if (a->M == 0) return PIGAN_OK;
    if (pigan_status st = check_mat(a->y, "y", a->n_groups, a->M, a->N, esize(a->dt))) return st;
    if (pigan_status st = check_norm_apart(a)) return st;
    const hipStream_t st = (hipStream_t)stream;
    ProfScope prof(st, "layer_norm_fwd", 0.0, 2.0 * esize(a->dt) * a->n_groups * (double)a->M * a->N);
    return by_dtype(a->dt, [&](auto t) -> pigan_status {
      typedef decltype(t) T;
      NormArgs<T> n = norm_args<T>(a);
      n.out = out<T>(a->y);
      HIP_TRY(launch_norm_fwd(n, a->n_groups, st));
      return PIGAN_OK;
    });
  });
}

size_t pigan_layer_norm_backward_workspace(const pigan_norm* a) {
  size_t n = 0;
  guarded([&]() -> pigan_status {
    if (!a) return fail(PIGAN_EINVAL, "null arguments");
    if (pigan_status st = check_dims(a->n_groups, a->dt, a->M, a->N)) return st;
    n = std::max<size_t>(norm_ws(a), 1);
    return PIGAN_OK;
  });
  return n;
}

pigan_status pigan_layer_norm_backward(const pigan_norm* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> pigan_status {
    if (pigan_status st = check_norm_backward(a)) return st;
    if (pigan_status st = check_ws(ws, ws_bytes, norm_ws(a))) return st;
    if (a->M > 0)
      if (pigan_status st = check_norm_backward_apart(a, ws, norm_ws(a))) return st;
    const hipStream_t st = (hipStream_t)stream;
    ProfScope prof(st, "layer_norm_bwd", 0.0,
                   (2.0 + !!a->dx.p + !!a->add.p) * esize(a->dt) * a->n_groups * (double)a->M * a->N);
    return by_dtype(a->dt, [&](auto t) -> pigan_status {
      typedef decltype(t) T;
      NormArgs<T> n = norm_args<T>(a);
      n.dy = in<T>(a->dy);
      n.add = in<T>(a->add);
      n.out = out<T>(a->dx);
      n.dgamma = a->dgamma;
      n.dbeta = a->dbeta;
      n.part = (float*)ws;
      HIP_TRY(launch_norm_bwd(n, a->n_groups, st));
      return PIGAN_OK;
    });
  });
}

}  // extern "C"
