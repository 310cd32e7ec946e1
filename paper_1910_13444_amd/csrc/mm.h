// The tiled product of the linear layer on the 16-bit matrix cores of gfx950
// (see linear.h for the operands).
//
// A block of WM x WN waves forms a tile of C; a wave owns MT x NT fragments of
// 32 x 32.  Operands pass through LDS in stages of 64 values of k:
//   k along the row   a row of the stage is a 128-byte line of a row of A; its
//                     16-byte segment s sits at s ^ (row & 7), so the 32 rows
//                     of a fragment read spread over all banks;
//   k down the rows   a row of the stage holds the tile's columns of one k;
//                     segment s of row r sits at s ^ 4 (r & 3) (rows of eight
//                     segments: s ^ 4 (r / 2 & 1)), which puts the four rows of
//                     a transposing read in disjoint banks.
// With DMA the stages go straight to LDS (global_load_lds_dwordx4: lane l of a
// wave fills byte 16 l of 1 KB), NS - 1 of them ahead of the products; a last
// partial stage and unaligned operands go through registers, with zeros past
// the end of k.  Rows of a tile past the end of the matrix repeat the last
// row; their products are not stored.
//
// The matrix core is given (B, A), so a lane holds one row of C and runs of
// four columns; two lane exchanges make that eight consecutive columns, of
// which four lanes cover 32 consecutive ones, for the epilogue's accesses.
#pragma once
#include "act.h"
#include "linear.h"
#include "piece.h"
#include "tile.h"

namespace pigan {

enum MmKind { MM_FWD = 0, MM_DX = 1, MM_DW = 2 };

// segment swizzle of row r of a stage whose rows hold `side` columns of one k
__device__ __forceinline__ int mm_swizzle(int side, int r) { return side == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); }

// result columns of a fragment's 16 values after the exchanges: v[0..7] belong
// to row lane & 15, v[8..15] to that row + 16, both to columns mm_col() ..
__device__ __forceinline__ int mm_col(int lane) { return 16 * ((lane >> 4) & 1) + 8 * (lane >> 5); }

__device__ __forceinline__ void mm_exchange(float (&v)[16]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t a = __float_as_uint(v[8 * j + e]), b = __float_as_uint(v[8 * j + 4 + e]);
      swap32(a, b);
      v[8 * j + e] = __uint_as_float(a);
      v[8 * j + 4 + e] = __uint_as_float(b);
    }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[e]), __float_as_uint(v[8 + e]), false, false);
    v[e] = __uint_as_float(r[0]);
    v[8 + e] = __uint_as_float(r[1]);
  }
}

// epilogue of eight consecutive columns j.. of row i (i < I, j < J); `bias`
// holds their biases
template <int KIND, class TO>
__device__ __forceinline__ void mm_epilogue(const MmOut<TO>& o, int g, int64_t i, int64_t j, const float* bias,
                                            float* v) {
  const int64_t valid = o.J - j;
  if constexpr (KIND != MM_DW) {
    if constexpr (KIND == MM_FWD) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += bias[e];
      if (o.pre) store8(o.pre + g * o.gsp + i * o.ldp + j, valid, v);
      PIGAN_ACT_SWITCH(o.act, {
        _Pragma("unroll") for (int e = 0; e < 8; ++e) v[e] = act_value<ACT>(v[e]);
      })
    } else {
      if (o.pre) {
        float a[8];
        load8(o.pre + g * o.gsp + i * o.ldp + j, valid, a);
        PIGAN_ACT_SWITCH(o.act, {
          _Pragma("unroll") for (int e = 0; e < 8; ++e) v[e] *= act_slope<ACT>(a[e]);
        })
      }
    }
    if (o.add) {
      float r[8];
      load8(o.add + g * o.gsa + i * o.lda + j, valid, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
  }
  store8(o.out + g * o.gso + i * o.ldo + j, valid, v);
}

// all but N vector-memory operations and all LDS operations of this wave are
// done, then the block's barrier
template <int N>
__device__ __forceinline__ void stage_sync() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | ((N >> 4) << 14));   // vmcnt(N) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int WM, int WN, int MT, int NT, int NS>
struct MmShape {
  static constexpr int BM = 32 * MT * WM, BN = 32 * NT * WN, NTH = 64 * WM * WN;
  static constexpr int BK = 64;
  static constexpr int STAGE_A = BM * BK * 2, STAGE = (BM + BN) * BK * 2;
};

template <class T, class TO, int KIND, int WM, int WN, int MT, int NT, int NS, bool DMA, int OCC>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(OCC)))
k_mm(const MmArgs<T, TO> p) {
  typedef MmShape<WM, WN, MT, NT, NS> S;
  constexpr int BM = S::BM, BN = S::BN, NW = WM * WN, BK = S::BK, STAGE_A = S::STAGE_A;
  constexpr bool AK = KIND != MM_DW, BKC = KIND == MM_FWD;   // k along the row of A, of B
  constexpr int GA = BM / 8 / NW, GB = BN / 8 / NW, GPW = GA + GB;   // 1 KB groups per wave and stage
  static_assert(GA >= 1 && GB >= 1 && (NS - 2) * GPW <= 63, "whole groups");
  static_assert(NS == 2 || NS == 4, "stages");
  typedef typename Elem<T>::frag frag;
  // one object per stage: the compiler then knows which of them a load in
  // flight can touch, and waits for no other
  __shared__ __attribute__((aligned(1024))) char s0[S::STAGE];
  __shared__ __attribute__((aligned(1024))) char s1[S::STAGE];
  __shared__ __attribute__((aligned(1024))) char s2[NS > 2 ? S::STAGE : 16];
  __shared__ __attribute__((aligned(1024))) char s3[NS > 2 ? S::STAGE : 16];
  auto stage_at = [&](auto u) -> char* {
    constexpr int U = decltype(u)::value % NS;
    if constexpr (U == 0) return s0;
    else if constexpr (U == 1) return s1;
    else if constexpr (U == 2) return s2;
    else return s3;
  };

  const int g = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;

  // Tiles of one split are neighbours in the order in which an XCD walks them:
  // panels of four row tiles, column by column, share their rows in its L2.
  const int64_t ti = (p.o.I + BM - 1) / BM, tj = (p.o.J + BN - 1) / BN;
  const int64_t lb = xcd_remap(blockIdx.x, gridDim.x);
  const int split = (int)(lb / (ti * tj));
  int64_t t = lb % (ti * tj);
  const int64_t panel = t / (4 * tj), prow = ti - 4 * panel < 4 ? ti - 4 * panel : 4;
  t -= panel * 4 * tj;
  const int64_t i0 = (4 * panel + t % prow) * BM, j0 = t / prow * BN;

  // this split's stages of k (of every plane pair)
  const int64_t nk = (p.K + BK - 1) / BK;
  const int k_lo = (int)(nk * split / p.o.n_split);
  const int per_pair = (int)(nk * (split + 1) / p.o.n_split) - k_lo;
  const int stages = per_pair * p.pairs;

  f32x16 acc[MT][NT];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int b = 0; b < NT; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;
  float db[KIND == MM_DW ? MT : 1];
#pragma unroll
  for (int a = 0; a < (KIND == MM_DW ? MT : 1); ++a) db[a] = 0.0f;

  // ---- where this lane's 16 bytes of every group come from ----
  const T* pa = p.a.p + g * p.a.gs + (AK ? i0 * p.a.ld : i0);
  const T* pb = p.b.p + g * p.b.gs + (BKC ? j0 * p.b.ld : j0);
  // row of the stage and column segment of the lane in group q of an operand
  // with `side` rows (k along the row) or columns (k down the rows)
  auto place = [&](bool along, int side, int q, int& row, int& seg) __attribute__((always_inline)) {
    if (along) {
      row = q * 8 + (lane >> 3);
      seg = (lane & 7) ^ (row & 7);
    } else {
      const int spr = side / 8;               // segments per row
      row = (q * 64 + lane) / spr;
      seg = (lane % spr) ^ mm_swizzle(side, row);
    }
  };
  uint32_t off[GPW];   // byte offset from the stage's first element (DMA)
  if constexpr (DMA) {
#pragma unroll
    for (int n = 0; n < GPW; ++n) {
      const bool isA = n < GA;
      const bool along = isA ? AK : BKC;
      const int64_t ld = isA ? p.a.ld : p.b.ld, left = isA ? p.o.I - i0 : p.o.J - j0;
      int row, seg;
      place(along, isA ? BM : BN, wave + (isA ? n : n - GA) * NW, row, seg);
      int64_t o;
      if (along) o = (row < left ? row : left - 1) * ld + seg * 8;
      else o = row * ld + (seg * 8 < left ? seg * 8 : 0);
      off[n] = (uint32_t)(o * 2);
    }
  }
  // plane pairs in the order of growing products
  auto pair_planes = [&](int st, int& a, int& b, int64_t& k) __attribute__((always_inline)) {
    const int pr = p.pairs == 1 ? 5 : st / per_pair;
    k = (int64_t)(k_lo + (p.pairs == 1 ? st : st - pr * per_pair)) * BK;
    // pair:  0      1      2      3      4      5
    //        (0,2)  (1,1)  (2,0)  (0,1)  (1,0)  (0,0)
    a = pr == 0 ? 0 : pr == 1 ? 1 : pr == 2 ? 2 : pr == 4 ? 1 : 0;
    b = pr == 0 ? 2 : pr == 1 ? 1 : pr == 3 ? 1 : 0;
  };
  // a stage through registers: zeros past the end of k
  auto fetch = [&](piece_t (&r)[GPW], int st) __attribute__((always_inline)) {
    int qa, qb;
    int64_t k0;
    pair_planes(st, qa, qb, k0);
#pragma unroll
    for (int n = 0; n < GPW; ++n) {
      const bool isA = n < GA;
      const bool along = isA ? AK : BKC;
      const int64_t ld = isA ? p.a.ld : p.b.ld, left = isA ? p.o.I - i0 : p.o.J - j0;
      const T* base = isA ? pa + qa * p.a.plane : pb + qb * p.b.plane;
      int row, seg;
      place(along, isA ? BM : BN, wave + (isA ? n : n - GA) * NW, row, seg);
      if (along) {
        const int64_t k = k0 + seg * 8;
        r[n] = piece_load(base + (row < left ? row : left - 1) * ld + k, p.K - k);
      } else {
        const int64_t k = k0 + row;
        r[n] = piece_load(base + k * ld + seg * 8, k < p.K ? left - seg * 8 : 0);
      }
    }
  };
  auto put = [&](const piece_t (&r)[GPW], char* stage) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < GPW; ++n)
      *(piece_t*)(stage + (n < GA ? 0 : STAGE_A) + (wave + (n < GA ? n : n - GA) * NW) * 1024 + lane * 16) = r[n];
  };
  auto issue = [&](int st, char* stage) __attribute__((always_inline)) {
    int qa, qb;
    int64_t k0;
    pair_planes(st, qa, qb, k0);
    if (k0 + BK <= p.K) {
      const char* ba = (const char*)(pa + qa * p.a.plane + (AK ? k0 : k0 * p.a.ld));
      const char* bb = (const char*)(pb + qb * p.b.plane + (BKC ? k0 : k0 * p.b.ld));
#pragma unroll
      for (int n = 0; n < GPW; ++n)
        __builtin_amdgcn_global_load_lds((const void*)((n < GA ? ba : bb) + off[n]),
                                         (lds_ptr_t)(stage + (n < GA ? 0 : STAGE_A) +
                                                     (wave + (n < GA ? n : n - GA) * NW) * 1024), 16, 0, 0);
    } else {
      piece_t r[GPW];
      fetch(r, st);
      put(r, stage);
      wait_vmcnt<0>();   // also in a wave whose pieces are all past the end: the counts below stay upper bounds
    }
  };

  // ---- products of one stage ----
  const int grp = lane >> 4, t16 = lane & 15, rr = t16 >> 2, q4 = t16 & 3, kb = 8 * (lane >> 5);
  auto frag_at = [&](const char* base, bool along, int side, int c, int blk) __attribute__((always_inline)) -> frag {
    if (along) {
      const int row = blk + (lane & 31), seg = 2 * c + (lane >> 5);
      return *(const frag*)(base + row * 128 + ((seg ^ (row & 7)) << 4));
    }
    const int byte = (blk + 16 * (grp & 1) + 4 * q4) * 2, pitch = side * 2;
    const char* q = base + (c * 16 + kb + rr) * pitch + (((byte >> 4) ^ mm_swizzle(side, rr)) << 4) + (byte & 15);
    const u32x2 lo = lds_read_tr<T>(q), hi = lds_read_tr<T>(q + 4 * pitch);
    return __builtin_bit_cast(frag, (u32x4{lo.x, lo.y, hi.x, hi.y}));
  };
  // dw: the sums of A over k go by the blocks of a row of tiles in turn, the
  // chunks of a stage by the waves of a column in turn
  const int db_tiles = (int)tj, db_turn = (int)(j0 / BN);
  auto products = [&](const char* stage, int st) __attribute__((always_inline)) {
    // the first three plane pairs hold every plane of A once
    const bool sum_a = KIND == MM_DW && p.part_db && st < 3 * per_pair && st % db_tiles == db_turn;
#pragma unroll
    for (int c = 0; c < BK / 16; ++c) {
      frag fa[MT], fb[NT];
#pragma unroll
      for (int a = 0; a < MT; ++a) fa[a] = frag_at(stage, AK, BM, c, 32 * (wm * MT + a));
#pragma unroll
      for (int b = 0; b < NT; ++b) fb[b] = frag_at(stage + STAGE_A, BKC, BN, c, 32 * (wn * NT + b));
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) Elem<T>::mma(acc[a][b], fb[b], fa[a]);
      if constexpr (KIND == MM_DW) {
        if (sum_a && c % WN == wn) {
#pragma unroll
          for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int e = 0; e < 8; ++e) db[a] += Elem<T>::to_f(fa[a][e]);
        }
      }
    }
  };

  if constexpr (DMA) {
    auto first = [&](auto u) __attribute__((always_inline)) {
      if (u < stages) issue(u, stage_at(u));
    };
    first(std::integral_constant<int, 0>{});
    if constexpr (NS > 2) {
      first(std::integral_constant<int, 1>{});
      first(std::integral_constant<int, 2>{});
    }
    // stage st has arrived, and every wave is done with the stage that the next load replaces
    auto turn = [&](int st, auto u) __attribute__((always_inline)) {
      const int later = stages - 1 - st;
      if constexpr (NS > 2) {
        if (later >= 2) stage_sync<2 * GPW>();
        else if (later == 1) stage_sync<GPW>();
        else stage_sync<0>();
      } else {
        stage_sync<0>();
      }
      if (st + NS - 1 < stages) issue(st + NS - 1, stage_at(std::integral_constant<int, decltype(u)::value + NS - 1>{}));
      products(stage_at(u), st);
    };
    for (int st = 0; st < stages; st += NS) {
      turn(st, std::integral_constant<int, 0>{});
      if (st + 1 < stages) turn(st + 1, std::integral_constant<int, 1>{});
      if constexpr (NS > 2) {
        if (st + 2 < stages) turn(st + 2, std::integral_constant<int, 2>{});
        if (st + 3 < stages) turn(st + 3, std::integral_constant<int, 3>{});
      }
    }
  } else {
    piece_t r[GPW];
    if (stages > 0) {
      fetch(r, 0);
      put(r, s0);
    }
    auto turn = [&](int st, char* now, char* next) __attribute__((always_inline)) {
      const bool more = st + 1 < stages;
      if (more) fetch(r, st + 1);
      lds_sync();
      products(now, st);
      if (more) put(r, next);   // every wave is past the products that read it: the barrier above
    };
    for (int st = 0; st < stages; st += 2) {
      turn(st, s0, s1);
      if (st + 1 < stages) turn(st + 1, s1, s0);
    }
  }

  // ---- results ----
  const int64_t jc = j0 + 32 * wn * NT + mm_col(lane);
  float bias[KIND == MM_FWD ? NT : 1][8];
  if constexpr (KIND == MM_FWD) {
#pragma unroll
    for (int b = 0; b < NT; ++b)
      vec_load<8>(p.o.bias && !p.o.part ? p.o.bias + g * p.o.J : nullptr, jc + 32 * b, p.o.J, 0.0f, bias[b]);
  }
#pragma unroll
  for (int a = 0; a < MT; ++a) {
#pragma unroll
    for (int b = 0; b < NT; ++b) {
      float v[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) v[r] = acc[a][b][r];
      mm_exchange(v);
      const int64_t j = jc + 32 * b;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t i = i0 + 32 * (wm * MT + a) + 16 * h + (lane & 15);
        if (i < p.o.I && j < p.o.J) {
          if (p.o.part) store8(p.o.part + (((int64_t)g * p.o.n_split + split) * p.o.I + i) * p.o.J + j, p.o.J - j, v + 8 * h);
          else mm_epilogue<KIND>(p.o, g, i, j, bias[KIND == MM_FWD ? b : 0], v + 8 * h);
        }
      }
    }
  }
  if constexpr (KIND == MM_DW) {
    if (p.part_db) {
      // the waves' sums through LDS, in order
      float* sums = (float*)s0;   // [WN][BM]
      lds_sync();
#pragma unroll
      for (int a = 0; a < MT; ++a) {
        const float s = db[a] + __shfl_xor(db[a], 32);
        if (lane < 32) sums[wn * BM + 32 * (wm * MT + a) + lane] = s;
      }
      lds_sync();
      if (tid < BM && i0 + tid < p.o.I) {
        float s = sums[tid];
#pragma unroll
        for (int n = 1; n < WN; ++n) s += sums[n * BM + tid];
        p.part_db[(((int64_t)g * p.o.n_split + split) * tj + j0 / BN) * p.o.I + i0 + tid] = s;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// sums of split products
// ---------------------------------------------------------------------------
template <int KIND, class TO>
__global__ void __launch_bounds__(256) k_mm_join(const MmOut<TO> o) {
  const int g = blockIdx.z;
  const int64_t vpr = (o.J + 7) / 8, total = o.I * vpr;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t i = q / vpr, j = (q - i * vpr) * 8;
    float v[8], bias[8];
    double s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.0;
    const float* src = o.part + ((int64_t)g * o.n_split * o.I + i) * o.J + j;
    for (int n = 0; n < o.n_split; ++n) {
      load8(src + (int64_t)n * o.I * o.J, o.J - j, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += (double)v[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)s[e];
    vec_load<8>(KIND == MM_FWD && o.bias ? o.bias + g * o.J : nullptr, j, o.J, 0.0f, bias);
    mm_epilogue<KIND>(o, g, i, j, bias, v);
  }
}

template <int KIND, class TO>
hipError_t join_launch(const MmOut<TO>& o, int G, hipStream_t st) {
  const int64_t blocks = (o.I * ((o.J + 7) / 8) + 255) / 256;
  k_mm_join<KIND, TO><<<dim3((unsigned)(blocks < 8192 ? blocks : 8192), 1, G), 256, 0, st>>>(o);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// launch of a tile
// ---------------------------------------------------------------------------
template <class T, class TO, int KIND>
hipError_t mm_launch(const MmArgs<T, TO>& a, int tile, bool direct, int G, hipStream_t st) {
  const int64_t side = mm_tile_side(tile);
  const int64_t tiles = ((a.o.I + side - 1) / side) * ((a.o.J + side - 1) / side) * a.o.n_split;
  if (a.o.I < 1 || a.o.J < 1 || a.K < 1 || a.o.n_split < 1 || G < 1 || G > 65535 || tiles > 0x7fffffff ||
      (a.o.n_split > 1 && !a.o.part) || (a.pairs != 1 && a.pairs != 6) ||
      a.K > 0x7fffffff)
    return hipErrorInvalidValue;
  const dim3 grid((unsigned)tiles, 1, G);
  if (tile == MM_256) {
    if (direct) k_mm<T, TO, KIND, 2, 4, 4, 2, 2, true, 2><<<grid, 512, 0, st>>>(a);
    else k_mm<T, TO, KIND, 2, 4, 4, 2, 2, false, 2><<<grid, 512, 0, st>>>(a);
  } else if (tile == MM_128) {
    if (direct) k_mm<T, TO, KIND, 2, 2, 2, 2, 2, true, 2><<<grid, 256, 0, st>>>(a);
    else k_mm<T, TO, KIND, 2, 2, 2, 2, 2, false, 2><<<grid, 256, 0, st>>>(a);
  } else {
    if (direct) k_mm<T, TO, KIND, 2, 2, 1, 1, 4, true, 2><<<grid, 256, 0, st>>>(a);
    else k_mm<T, TO, KIND, 2, 2, 1, 1, 2, false, 2><<<grid, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace pigan
