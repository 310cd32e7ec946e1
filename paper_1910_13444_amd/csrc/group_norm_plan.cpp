// How a call of group norm is cut, and its workspaces.
#include <algorithm>
#include <iterator>

#include "group_norm.h"

namespace pigan {

GnPlan gn_plan(bool backward, int fields, int elem_bytes, int64_t G, int64_t S, int64_t P, int64_t C, int64_t n) {
  GnPlan pl{};
  S = std::max<int64_t>(S, 1);
  const int64_t E = 16 / elem_bytes, cg = C / n;
  const bool whole_pieces = cg % E == 0;
  auto slab = [&](int64_t ng) {
    pl.ng = ng;
    pl.W = ng * cg;
    pl.chan_parts = 1;
    pl.slabs = cdiv(n, ng);
    pl.pw = (int32_t)std::min<int64_t>(cdiv(pl.W, E), 1 << 30);
  };
  pl.cg = cg;
  // Streamed stores leave no lines to be written back while the next kernel reads: of 512 MiB
  // the sums 50 for 73 us, the results 100 for 105; rows 116 for 131.  What the last-level
  // cache (256 MiB) holds beside its inputs is left there for the next layer (of 128 MiB
  // streaming would save 2 of 33 us here).
  pl.stream = (double)fields * elem_bytes * G * S * P * C > 192.0 * 1048576.0;
  pl.inv_n = 1.0 / ((double)cg * (double)P);
  auto finish = [&](int nth, int nv) {
    pl.nth = nth;
    pl.nv = nv;
    pl.rows = nth / pl.pw;
    pl.span = (int32_t)(whole_pieces && pl.ng > 1 ? cg / E : pl.ng > 1 ? cg : pl.pw);
    pl.ns = 1;
    pl.lanes = 64;
  };
  auto fit_lanes = [&](int64_t entries) {
    // as many lanes as entries, and no more groups in turns than need be
    while (pl.lanes > 1 && (pl.lanes / 2 >= entries || pl.lanes * pl.ng * pl.ns > pl.nth)) pl.lanes /= 2;
  };
  // blocks beside each other over a reverse pass's samples, four to a CU, and more where a
  // thread would have more than BWD_TERMS; few batches are one block's, as the sum of several
  // blocks' columns is a launch of its own (3.4 us)
  auto slots = [&](int64_t batches) {
    if (batches <= 6) return (int32_t)1;
    const int64_t each = std::max<int64_t>(1, 1024 / std::min<int64_t>(1024, G * pl.slabs));
    return (int32_t)std::min(batches, std::max(each, cdiv(batches, BWD_TERMS)));
  };
  const int64_t lanes = cg / E;
  if (P == 1 && whole_pieces && lanes <= 64 && (lanes & (lanes - 1)) == 0 && cdiv(n, 256 / lanes) <= 65535) {
    slab(std::min<int64_t>(n, 256 / lanes));
    finish(256, 4);
    pl.mode = GN_ROWS;
    pl.slots = slots(cdiv(S, pl.rows));
    return pl;
  }
  // One pass: slabs of 128 bytes of a point, 64 where those do not fit.  Where pieces are of
  // several groups, up to 512 threads with one piece come before more pieces (values in LDS,
  // not sums: 5674 x 7 x 624 in 12 groups 61 for 154 us), but neither 64 bytes (1472 x 92 x
  // 432 in 144 groups: 196 for 145 us) nor 1024 threads (253 us, one block to a CU).
  for (int64_t bytes : {128, 64}) {
    slab(std::min<int64_t>(n, std::max<int64_t>(1, cdiv(bytes, cg * elem_bytes))));
    const bool mixed = !whole_pieces && pl.ng > 1;
    const Shape* list = backward ? BWD_SHAPES : whole_pieces ? FWD_SHAPES : FWD_ODD;
    const size_t count = backward ? std::size(BWD_SHAPES) : whole_pieces ? std::size(FWD_SHAPES) : std::size(FWD_ODD);
    for (size_t i = 0; i < count; ++i) {
      const Shape f = list[i];
      if (f.nth < pl.pw || (int64_t)(f.nth / pl.pw) * f.nv < P) continue;
      // larger samples, or few, have ranges enough for blocks of their own
      if (backward && f.nth > 256 && (P * cdiv(C, E) > 1024 || G * S * pl.slabs < 128)) continue;
      const int64_t items = G * S * pl.slabs;
      if (items < 256 && (int64_t)f.nth * f.nv > 4096) break;   // few blocks with much to do: ranges of points
      finish(f.nth, f.nv);
      if (f.nv == 1 && P <= 256) {
        // short samples: wider slabs, then several samples of a block
        int64_t ng = pl.ng;
        while (ng < n && cdiv(std::min(n, 2 * ng) * cg, E) * P <= f.nth && (whole_pieces || mixed)) ng = std::min(n, 2 * ng);
        slab(ng);
        finish(f.nth, 1);
        pl.ns = (int32_t)std::max<int64_t>(1, std::min<int64_t>(pl.rows / P, S));
        if (pl.ns > 1) pl.rows = (int32_t)(pl.ns * P);
      }
      fit_lanes((pl.ns > 1 ? P : pl.rows) * (mixed ? cg : std::max<int64_t>(1, pl.pw / pl.ng)));
      pl.mode = GN_ONE;
      pl.slots = slots(cdiv(S, pl.ns));
      return pl;
    }
  }
  // ranges of points: 512 bytes of a point, for long runs
  const int64_t most = SPLIT_NTH * E;
  pl.mode = GN_SPLIT;
  if (cg > most) {
    pl.W = most;
    pl.ng = 1;
    pl.chan_parts = (int32_t)cdiv(cg, most);
    pl.slabs = n * pl.chan_parts;
    pl.pw = SPLIT_NTH;
  } else {
    slab(std::min<int64_t>(n, std::max<int64_t>(1, 32 * E / cg)));
  }
  finish(SPLIT_NTH, 1);
  while (pl.lanes > 1 && pl.lanes * pl.ng > SPLIT_NTH) pl.lanes /= 2;
  // Blocks that run at once, five or three to a CU, each with as much to do as the others;
  // where samples and slabs alone are more, four rounds of them.  Of 512, 1024 .. 8192 blocks:
  // 16 x 65,536 x 128 bf16, gelu 51 + 104 .. 48 + 142 us (1280: 50 + 101); backward 128 x 1024
  // x 256 bf16, silu 33 + 48 .. 44 + 57 (768: 32 + 45).
  const int64_t blocks = 256 * (backward ? 3 : 5), base = G * S * pl.slabs, least = cdiv(P, 4 * pl.rows);
  const int64_t each = base < blocks ? blocks / base : cdiv(4 * blocks, base);
  pl.splits = (int32_t)std::max<int64_t>(1, std::min(each, least));
  if (backward) pl.splits = (int32_t)std::max<int64_t>(pl.splits, cdiv(P, BWD_TERMS * pl.rows));
  pl.slots = (int32_t)std::min(S * pl.splits, std::max<int64_t>(1, blocks / std::min(blocks, G * pl.slabs)));
  return pl;
}

size_t gn_pairs_bytes(const GnPlan& pl, int64_t G, int64_t S, int64_t n) {
  return (size_t)(G * S * n) * (size_t)(pl.chan_parts * pl.splits) * sizeof(Pair);
}
size_t gn_forward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t n) {
  return pl.mode == GN_SPLIT ? gn_pairs_bytes(pl, G, S, n) + (size_t)(G * S * n) * 4 : 0;
}
size_t gn_backward_ws(const GnPlan& pl, int64_t G, int64_t S, int64_t C, int64_t n, bool cols) {
  const size_t sums = cols ? (size_t)(G * pl.slots * 2 * C) * 4 : 0;
  if (pl.mode != GN_SPLIT) return pl.slots > 1 ? sums : 0;
  return gn_pairs_bytes(pl, G, S, n) + sums;
}

}  // namespace pigan
