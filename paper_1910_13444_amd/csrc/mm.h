// The tiled product of the linear layer on the 16-bit matrix cores of gfx950
// (see linear.h for the operands).
//
// A block of waves forms a tile of C; a wave owns MT x NT fragments of
// 32 x 32.  Operands pass through LDS in stages of 64 values of k:
//   k along the row   a row of the stage is a 128-byte line of a row of A; its
//                     16-byte segment s sits at s ^ (row / 2 & 7), so 16 rows'
//                     pieces of one k, read together, spread over all banks;
//   k down the rows   a row of the stage holds the tile's columns of one k;
//                     segment s of row r sits at s ^ 4 (r & 3) (rows of eight
//                     segments: s ^ 4 (r / 2 & 1)), which puts the four rows of
//                     a transposing read in disjoint banks.
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

// Eight consecutive columns of a row as they lie in memory.
template <class TO> struct Octet {
  piece_t q[8 / EPP<TO>];
  __device__ __forceinline__ void load(const TO* p, int64_t valid) {
#pragma unroll
    for (int i = 0; i < 8 / EPP<TO>; ++i) q[i] = piece_load(p + i * EPP<TO>, valid - i * EPP<TO>);
  }
  __device__ __forceinline__ void floats(float* f) const {
#pragma unroll
    for (int i = 0; i < 8 / EPP<TO>; ++i) piece_floats<TO>(q[i], f + i * EPP<TO>);
  }
};

// The epilogue of eight columns j.. of row i (i < I, j < J): `bias` holds the
// columns' biases, `pre` and `add` what it reads of those matrices.
template <int KIND, int ACT, class TO>
__device__ __forceinline__ void mm_epilogue(const MmOut<TO>& o, int g, int64_t i, int64_t j, int64_t valid,
                                            const Octet<TO>& pre, const Octet<TO>& add, const float* bias, float* v) {
  if constexpr (KIND == MM_FWD) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += bias[e];
    if (o.pre) store8(o.pre + g * o.gsp + i * o.ldp + j, valid, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_value<ACT, TO>(v[e]);
  } else if constexpr (KIND == MM_DX && ACT != PIGAN_ACT_NONE) {
    float a[8];
    pre.floats(a);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= act_slope<ACT, TO>(a[e]);
  }
  if constexpr (KIND != MM_DW)
    if (o.add) {
      float r[8];
      add.floats(r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
  store8(o.out + g * o.gso + i * o.ldo + j, valid, v);
}

// A wave's MT x NT fragments, from rows i0 and columns j0 on, to memory: as
// partial sums or through the epilogue (one branch on the activation for all of
// them: the accumulators stay in registers only if every loop unrolls).  What the
// epilogue reads is requested D - 1 fragments ahead, as many as the registers hold
// beside the accumulators: asked for one by one, each of 32 reads was waited for
// by itself, 30 us of the 60 that a 256 x 256 tile took at K = 1024.  The fragments
// of a row follow each other, so that the halves of a 128-byte line do (262,144 x
// 1024 x 1024 with a residual: 1.36 GB read and 0.56 written; column by column of
// fragments 1.57 and 0.67).  WHOLE: the columns come in whole eights.
template <int KIND, int ACT, bool PART, bool WHOLE, class TO, int MT, int NT>
__device__ __forceinline__ void mm_store(const MmOut<TO>& o, int g, int split, int64_t i0, int64_t j0,
                                         const f32x16 (&acc)[MT][NT]) {
  const int lane = threadIdx.x & 63;
  constexpr bool PRE = !PART && KIND == MM_DX && ACT != PIGAN_ACT_NONE, ADD = !PART && KIND != MM_DW;
  constexpr int NF = MT * NT;
  constexpr int WANT = !WHOLE ? 1 : sizeof(TO) == 4 ? 2 : PRE ? 4 : 6;
  constexpr int D = WANT < NF ? WANT : NF;
  Octet<TO> pre[PRE ? D : 1][2], add[ADD ? D : 1][2];
  // f(half, row, column, columns that are there) of fragment n
  auto each = [&](int n, auto f) __attribute__((always_inline)) {
    const int64_t j = j0 + 32 * (n % NT) + mm_col(lane);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t i = i0 + 32 * (n / NT) + 16 * h + (lane & 15);
      if (i < o.I && j < o.J) f(h, i, j, WHOLE ? (int64_t)8 : o.J - j);
    }
  };
  auto request = [&](int n) __attribute__((always_inline)) {
    each(n, [&](int h, int64_t i, int64_t j, int64_t valid) __attribute__((always_inline)) {
      if constexpr (PRE) pre[n % D][h].load(o.pre + g * o.gsp + i * o.ldp + j, valid);
      if constexpr (ADD)
        if (o.add) add[n % D][h].load(o.add + g * o.gsa + i * o.lda + j, valid);
    });
  };
  if constexpr (PRE || ADD)
#pragma unroll
    for (int n = 0; n < D - 1; ++n) request(n);
  float bias[KIND == MM_FWD ? NT : 1][8];
  if constexpr (KIND == MM_FWD && !PART)
#pragma unroll
    for (int b = 0; b < NT; ++b) {
      const int64_t j = j0 + 32 * b + mm_col(lane);
      vec_load<8>(o.bias && (!WHOLE || j < o.J) ? o.bias + g * o.J : nullptr, j, WHOLE ? j + 8 : o.J, 0.0f, bias[b]);
    }
#pragma unroll
  for (int n = 0; n < NF; ++n) {
    if constexpr (PRE || ADD)
      if (n + D - 1 < NF) request(n + D - 1);
    float v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = acc[n / NT][n % NT][r];
    mm_exchange(v);
    each(n, [&](int h, int64_t i, int64_t j, int64_t valid) __attribute__((always_inline)) {
      if constexpr (PART) store8(o.part + (((int64_t)g * o.n_split + split) * o.I + i) * o.J + j, valid, v + 8 * h);
      else mm_epilogue<KIND, ACT>(o, g, i, j, valid, pre[PRE ? n % D : 0][h], add[ADD ? n % D : 0][h], bias[KIND == MM_FWD ? n % NT : 0], v + 8 * h);
    });
  }
}

template <int KIND, bool WHOLE, class TO, int MT, int NT>
__device__ __forceinline__ void mm_results(const MmOut<TO>& o, int g, int split, int64_t i0, int64_t j0,
                                           const f32x16 (&acc)[MT][NT]) {
  if (o.part) {
    mm_store<KIND, PIGAN_ACT_NONE, true, WHOLE>(o, g, split, i0, j0, acc);
  } else if constexpr (KIND == MM_DW) {
    mm_store<KIND, PIGAN_ACT_NONE, false, WHOLE>(o, g, split, i0, j0, acc);
  } else {
    PIGAN_ACT_SWITCH(o.act, { mm_store<KIND, ACT, false, WHOLE>(o, g, split, i0, j0, acc); })
  }
}

// the first `valid` columns of an octet by itself
template <int KIND, class TO>
__device__ __forceinline__ void mm_finish(const MmOut<TO>& o, int g, int64_t i, int64_t j, int64_t valid,
                                          const float* bias, float* v) {
  PIGAN_ACT_SWITCH(KIND == MM_DW ? PIGAN_ACT_NONE : o.act, {
    Octet<TO> pre, add;
    if constexpr (KIND == MM_DX && ACT != PIGAN_ACT_NONE) pre.load(o.pre + g * o.gsp + i * o.ldp + j, valid);
    if constexpr (KIND != MM_DW)
      if (o.add) add.load(o.add + g * o.gsa + i * o.lda + j, valid);
    mm_epilogue<KIND, ACT>(o, g, i, j, valid, pre, add, bias, v);
  })
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

// One tile of C: group, first row and column, part of the contraction.
struct MmTilePos {
  int g, split, ti, tj;   // ti, tj: row and column of the tile
};

// Tile n of all.  Tiles of one split of a group are neighbours, in panels of four
// row tiles, column by column: an XCD, which walks a range of n, then shares
// their rows in its L2.
__device__ __forceinline__ MmTilePos mm_tile(uint32_t n, uint32_t rows, uint32_t cols, uint32_t n_split) {
  MmTilePos t;
  const uint32_t per = rows * cols, part = n / per;
  n -= part * per;
  t.g = (int)(part / n_split);
  t.split = (int)(part - t.g * n_split);
  const uint32_t panel = n / (4 * cols), prow = rows - 4 * panel < 4 ? rows - 4 * panel : 4;
  n -= panel * 4 * cols;
  t.tj = (int)(n / prow);
  t.ti = (int)(4 * panel + n - t.tj * prow);
  return t;
}

// a block's sum of column i0 + n of A (n < 0: none): db itself, or a slot of the split
template <class T, class TO>
__device__ __forceinline__ void mm_store_db(const MmArgs<T, TO>& p, int g, int split, int tj, int tiles, int64_t i0,
                                            int n, float sum) {
  if (n < 0 || i0 + n >= p.o.I) return;
  if (p.o.n_split > 1) p.part_db[(((int64_t)g * p.o.n_split + split) * tiles + tj) * p.o.I + i0 + n] = sum;
  else if (tj == 0) p.part_db[g * p.o.I + i0 + n] = sum;
}

// ---------------------------------------------------------------------------
// Operands of any alignment: stages pass through registers, one ahead of the
// products, with zeros past the end of k.  Rows of a tile past the end of the
// matrix repeat its last row; their products are not stored.  Bound by the waits
// for those registers (bf16 20,000 x 1032 x 1000 with rows 3 elements apart: 83 us
// where whole pieces take 70, 131,072 x 1024 x 1024 466 and 284).
// ---------------------------------------------------------------------------
template <class T, class TO, int KIND, int MT, int NT>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
k_mm_any(const MmArgs<T, TO> p) {
  constexpr int BM = 64 * MT, BN = 64 * NT, BK = 64, STAGE_A = BM * BK * 2, STAGE = STAGE_A + BN * BK * 2;
  constexpr bool AK = KIND != MM_DW, BKC = KIND == MM_FWD;   // k along the row of A, of B
  constexpr int GA = BM / 32, GPW = GA + BN / 32;            // 1 KB groups per wave and stage
  typedef typename Elem<T>::frag frag;
  __shared__ __attribute__((aligned(1024))) char s0[STAGE];
  __shared__ __attribute__((aligned(1024))) char s1[STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;

  const uint32_t rows = (uint32_t)((p.o.I + BM - 1) / BM), tj = (uint32_t)((p.o.J + BN - 1) / BN);
  const MmTilePos at = mm_tile((uint32_t)xcd_remap(blockIdx.x, gridDim.x), rows, tj, p.o.n_split);
  const int g = at.g, split = at.split;
  const int64_t i0 = (int64_t)at.ti * BM, j0 = (int64_t)at.tj * BN;

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
  float db[MT];
#pragma unroll
  for (int a = 0; a < MT; ++a) db[a] = 0.0f;

  const T* pa = p.a.p + g * p.a.gs + (AK ? i0 * p.a.ld : i0);
  const T* pb = p.b.p + g * p.b.gs + (BKC ? j0 * p.b.ld : j0);
  auto fetch = [&](piece_t (&r)[GPW], int st) __attribute__((always_inline)) {
    // plane pairs (0,2) (1,1) (2,0) (0,1) (1,0) (0,0), as in the aligned kernel
    const int pr = p.pairs == 1 ? 5 : st / per_pair;
    const int64_t k0 = (int64_t)(k_lo + (p.pairs == 1 ? st : st - pr * per_pair)) * BK;
    const int qa = (0x124 >> (2 * pr)) & 3, qb = (0x046 >> (2 * pr)) & 3;
#pragma unroll
    for (int n = 0; n < GPW; ++n) {
      const bool isA = n < GA;
      const bool along = isA ? AK : BKC;
      const int side = isA ? BM : BN, q = wave + (isA ? n : n - GA) * 4;
      const int64_t ld = isA ? p.a.ld : p.b.ld, left = isA ? p.o.I - i0 : p.o.J - j0;
      const T* base = isA ? pa + qa * p.a.plane : pb + qb * p.b.plane;
      if (along) {
        const int row = q * 8 + (lane >> 3);
        const int64_t k = k0 + ((lane & 7) ^ ((row >> 1) & 7)) * 8;
        r[n] = piece_load(base + (row < left ? row : left - 1) * ld + k, p.K - k);
      } else {
        const int spr = side / 8, row = (q * 64 + lane) / spr, seg = (lane % spr) ^ mm_swizzle(side, row);
        const int64_t k = k0 + row;
        r[n] = piece_load(base + k * ld + seg * 8, k < p.K ? left - seg * 8 : 0);
      }
    }
  };
  auto put = [&](const piece_t (&r)[GPW], char* stage) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < GPW; ++n)
      *(piece_t*)(stage + (n < GA ? 0 : STAGE_A) + (wave + (n < GA ? n : n - GA) * 4) * 1024 + lane * 16) = r[n];
  };
  const int grp = lane >> 4, t16 = lane & 15, rr = t16 >> 2, q4 = t16 & 3, kb = 8 * (lane >> 5);
  auto frag_at = [&](const char* base, bool along, int side, int c, int blk) __attribute__((always_inline)) -> frag {
    if (along)
      return *(const frag*)(base + (lane & 31) * 128 + (((2 * c + (lane >> 5)) ^ ((lane >> 1) & 7)) << 4) + blk * 4096);
    const int byte = (32 * blk + 16 * (grp & 1) + 4 * q4) * 2, pitch = side * 2;
    const char* q = base + (c * 16 + kb + rr) * pitch + (((byte >> 4) ^ mm_swizzle(side, rr)) << 4) + (byte & 15);
    const u32x2 lo = lds_read_tr<T>(q), hi = lds_read_tr<T>(q + 4 * pitch);
    return __builtin_bit_cast(frag, (u32x4{lo.x, lo.y, hi.x, hi.y}));
  };
  // db: as in the aligned kernel
  auto products = [&](const char* stage, int st) __attribute__((always_inline)) {
    const bool sum_a = KIND == MM_DW && p.part_db && st < 3 * per_pair &&
                       (p.o.n_split == 1 ? at.tj == 0 : (uint32_t)st % tj == (uint32_t)at.tj);
#pragma unroll
    for (int c = 0; c < BK / 16; ++c) {
      frag fa[MT], fb[NT];
#pragma unroll
      for (int a = 0; a < MT; ++a) fa[a] = frag_at(stage, AK, BM, c, MT * wm + a);
#pragma unroll
      for (int b = 0; b < NT; ++b) fb[b] = frag_at(stage + STAGE_A, BKC, BN, c, NT * wn + b);
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) Elem<T>::mma(acc[a][b], fb[b], fa[a]);
      if constexpr (KIND == MM_DW) {
        if (sum_a && (c & 1) == wn) {
#pragma unroll
          for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int e = 0; e < 8; ++e) db[a] += Elem<T>::to_f(fa[a][e]);
        }
      }
    }
  };

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
    if (more) put(r, next);   // its readers are past the barrier above
  };
  for (int st = 0; st < stages; st += 2) {
    turn(st, s0, s1);
    if (st + 1 < stages) turn(st + 1, s1, s0);
  }

  mm_results<KIND, false>(p.o, g, split, i0 + 32 * MT * wm, j0 + 32 * NT * wn, acc);
  if constexpr (KIND == MM_DW) {
    if (p.part_db) {
      // the waves' sums through LDS, in order
      float* sums = (float*)s0;   // [2][BM]
      lds_sync();
#pragma unroll
      for (int a = 0; a < MT; ++a) {
        const float s = db[a] + __shfl_xor(db[a], 32);
        if (lane < 32) sums[wn * BM + 32 * (MT * wm + a) + lane] = s;
      }
      lds_sync();
      mm_store_db(p, g, split, at.tj, (int)tj, i0, tid < BM ? tid : -1, sums[tid % BM] + sums[BM + tid % BM]);
    }
  }
}

// ---------------------------------------------------------------------------
// Aligned operands.  2 x WN waves form a tile of 64 MT x 32 NT WN, two stages of LDS.
// Fragments are read one chunk of 16 k ahead of their products, and the only wait
// of a stage stands before its last chunk, when the next stage has had three
// chunks' time to land and this stage's buffer has no reader left.
//   256 x 256  eight waves of 128 x 64, two per SIMD.  (Four waves of 128 x 128 read
//              a third less from LDS but leave the matrix cores idle at every wait
//              and in the epilogue: 8192^3 bf16 1170 against 1267 TFLOP/s before the
//              pieces' banks were spread, which made it 1354; 262,144 x 1024 x 1024
//              with a residual 786 against 703 us, then 674.)
//              Bound by the matrix cores' clock under load in the loop, by memory in
//              the epilogue: 131,072 x 1024 x 1024 dw 235 us, 1170 TFLOP/s; dx 330 us,
//              with relu's slope 414 (pre is read), with gelu's 420 to 480.
//   128 x 128  two blocks of four waves per CU, which fill each other's waits
//              (fp32 by six products, 1001 x 2000 x 513 dx and dw in one launch: 54 us)
//   64 x 64    four blocks per CU, for few tiles; for very few, one block of four
//              groups that share the contraction (1024 x 2000 x 1024 in 17 us, bound
//              by its eight stages one after the other)
// The loads are buffer loads: what is past the end of the matrix is out of the
// buffer's range and arrives as zeros.
// ---------------------------------------------------------------------------
// the buffer of `bytes` bytes from p on: the same in all lanes, whatever the
// compiler makes of the address
__device__ __forceinline__ u32x4 mm_buffer(const void* p, uint32_t bytes) {
  const uint64_t a = (uint64_t)p;
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)) & 0xffff,
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00027000};
}

// 16 bytes a lane from a buffer straight to 1 KB of LDS.  As an instruction that
// the compiler does not model: it cannot tell which object a transposing LDS read
// touches, and would have every one of them wait for every load in flight.  The
// load has no destination register; its arrival is waited for by stage_sync()
// alone, before the barrier behind which the stage is read.  M0 is a reserved
// register: nothing else in these kernels sets or reads it.
__device__ __forceinline__ void lds_load(const u32x4& buffer, uint32_t lds, uint32_t more, uint32_t lane_off,
                                         uint32_t off) {
  asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds"
               ::"s"(lds), "i"(more), "v"(lane_off), "s"(buffer), "s"(off) : "scc");
}

// bytes of a stage
template <int MT, int NT, int WN> constexpr int mm_stage() { return (64 * MT + 32 * NT * WN) * 64 * 2; }

// Block n of `blocks` of the product, with two stages of LDS for each of KG groups
// of 2 x WN waves: the groups share the contraction of the tile and meet in LDS, in
// order, before the epilogue.
template <class T, class TO, int KIND, int MT, int NT, int WN, bool WHOLE, int KG = 1>
__device__ __forceinline__ void mm_piped(const MmArgs<T, TO>& p, uint32_t n, uint32_t blocks, char* s0, char* s1) {
  static_assert(KG == 1 || MT * NT == 1, "groups: tiles of one fragment a wave");
  constexpr int BM = 64 * MT, BN = 32 * NT * WN, BK = 64, STAGE_A = BM * BK * 2, NW = 2 * WN, NTH = 64 * NW;
  constexpr bool AK = KIND != MM_DW, BKC = KIND == MM_FWD;
  constexpr int GA = BM / 8 / NW, GB = BN / 8 / NW;   // 1 KB groups per wave and stage
  static_assert(GA == GB, "one group of each operand at a time");
  typedef typename Elem<T>::frag frag;

  const int tid = KG == 1 ? (int)threadIdx.x : (int)threadIdx.x % NTH, lane = tid & 63;
  const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / NTH);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  if constexpr (KG > 1) {
    s0 += kg * mm_stage<MT, NT, WN>();
    s1 += kg * mm_stage<MT, NT, WN>();
  }

  const uint32_t rows = (uint32_t)((p.o.I + BM - 1) / BM), tj = (uint32_t)((p.o.J + BN - 1) / BN);
  const MmTilePos at = mm_tile((uint32_t)xcd_remap(n, blocks), rows, tj, p.o.n_split);
  const int64_t i0 = (int64_t)at.ti * BM, j0 = (int64_t)at.tj * BN;
  const uint32_t nk = (uint32_t)((p.K + BK - 1) / BK);
  int k_lo = (int)((uint64_t)nk * at.split / (uint32_t)p.o.n_split);
  int per_pair = (int)((uint64_t)nk * (at.split + 1) / (uint32_t)p.o.n_split) - k_lo;
  int turns = per_pair * p.pairs;
  if constexpr (KG > 1) {
    // this group's part; all of them take the turns of the longest one
    const int all = per_pair, lo = all * kg / KG;
    per_pair = all * (kg + 1) / KG - lo;
    k_lo += lo;
    turns = (all + KG - 1) / KG * p.pairs;
  }
  const int stages = per_pair * p.pairs;

  f32x16 acc[MT][NT];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int b = 0; b < NT; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;
  float db[MT];
#pragma unroll
  for (int a = 0; a < MT; ++a) db[a] = 0.0f;

  // ---- loads: lane offset within a group, uniform distance of groups ----
  const T* pa = p.a.p + at.g * p.a.gs + (AK ? i0 * p.a.ld : i0);
  const T* pb = p.b.p + at.g * p.b.gs + (BKC ? j0 * p.b.ld : j0);
  const int left_a = (int)(p.o.I - i0 < BM ? p.o.I - i0 : BM), left_b = (int)(p.o.J - j0 < BN ? p.o.J - j0 : BN);
  // a group is eight rows of an operand with k along the row, 512 / side rows of
  // one with k down the rows; a wave's groups are wave, wave + NW, ...
  constexpr uint32_t OUT = 0xffffffffu;   // never in range
  // k of the lane's piece (k along the row): a row's eight pieces are exchanged by
  // half its number, so that 16 rows' pieces of one k lie in different banks (by the
  // number itself, rows r and r + 8 share theirs)
  const int seg_k = ((lane & 7) ^ (4 * (wave & 1) + (lane >> 4))) * 8;
  auto lane_off = [&](bool along, int side, int64_t ld, int left) __attribute__((always_inline)) -> uint32_t {
    if (along) return (uint32_t)((8 * wave + (lane >> 3)) * ld * 2 + seg_k * 2);
    const int spr = side / 8, row = wave * (64 / spr) + lane / spr, seg = (lane % spr) ^ mm_swizzle(side, row);
    return seg * 8 < left ? (uint32_t)(row * ld * 2 + seg * 16) : OUT;
  };
  const uint32_t off_a = lane_off(AK, BM, p.a.ld, left_a), off_b = lane_off(BKC, BN, p.b.ld, left_b);
  const uint32_t step_a = (uint32_t)(NW * (AK ? 8 : 512 / BM) * p.a.ld * 2);
  const uint32_t step_b = (uint32_t)(NW * (BKC ? 8 : 512 / BN) * p.b.ld * 2);

  // the next stage to load: its first elements, its k, the stages left of its plane pair
  const int64_t adv_a = AK ? BK : BK * p.a.ld, adv_b = BKC ? BK : BK * p.b.ld;
  const int64_t k_first = (int64_t)k_lo * BK;
  const T *src_a = nullptr, *src_b = nullptr;
  int64_t k_left = 0;
  int pair = p.pairs == 1 ? 5 : 0, pair_left = 0;
  const uint32_t rows_a = (uint32_t)(left_a * p.a.ld * 2), rows_b = (uint32_t)(left_b * p.b.ld * 2);
  auto begin_pair = [&]() __attribute__((always_inline)) {
    // (0,2) (1,1) (2,0) (0,1) (1,0) (0,0): two bits each, from the lowest
    const int qa = (0x124 >> (2 * pair)) & 3, qb = (0x046 >> (2 * pair)) & 3;
    src_a = pa + qa * p.a.plane + (AK ? k_first : k_first * p.a.ld);
    src_b = pb + qb * p.b.plane + (BKC ? k_first : k_first * p.b.ld);
    k_left = p.K - k_first;
    pair_left = per_pair;
    ++pair;
  };
  // prepare() takes the next stage (past the last one: an empty buffer, so that
  // its loads only fill LDS with zeros), load() requests a group of each operand
  u32x4 ra, rb;
  uint32_t va = 0, vb = 0;
  int to_load = stages;
  auto prepare = [&]() __attribute__((always_inline)) {
    if (pair_left == 0 && to_load > 0) begin_pair();
    const int kl = to_load <= 0 ? 0 : (int)(k_left < BK ? k_left : BK);
    ra = mm_buffer(src_a, AK ? (kl ? rows_a : 0) : (uint32_t)(kl * p.a.ld * 2));
    rb = mm_buffer(src_b, BKC ? (kl ? rows_b : 0) : (uint32_t)(kl * p.b.ld * 2));
    const bool in_k = seg_k < kl;
    va = AK && !in_k ? OUT : off_a;
    vb = BKC && !in_k ? OUT : off_b;
    src_a += adv_a;
    src_b += adv_b;
    k_left -= BK;
    --pair_left;
    --to_load;
  };
  // where this wave's groups begin in either stage (LDS addresses in scalar registers)
  const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_ptr_t)s0) + wave * 1024;
  const uint32_t lds1 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_ptr_t)s1) + wave * 1024;
  auto load = [&](uint32_t lds, int q, int operand) __attribute__((always_inline)) {
    if (operand == 0) lds_load(ra, lds, q * NW * 1024, va, q * step_a);
    else lds_load(rb, lds, STAGE_A + q * NW * 1024, vb, q * step_b);
  };

  // ---- fragments ----
  // (each address is its stage plus ONE offset: through longer chains of pointer
  // arithmetic the compiler loses which stage is read)
  const int grp = lane >> 4, t16 = lane & 15, rr = t16 >> 2, q4 = t16 & 3, kb = 8 * (lane >> 5);
  auto frag_at = [&](const char* stage, int from, bool along, int side, int c, int blk)
      __attribute__((always_inline)) -> frag {
    if (along)
      return *(const frag*)(stage + (from + (lane & 31) * 128 + (((2 * c + (lane >> 5)) ^ ((lane >> 1) & 7)) << 4) + blk * 4096));
    const int byte = (32 * blk + 16 * (grp & 1) + 4 * q4) * 2, pitch = side * 2;
    const int off = from + (kb + rr) * pitch + (((byte >> 4) ^ mm_swizzle(side, rr)) << 4) + (byte & 15) + c * 16 * pitch;
    const u32x2 lo = lds_read_tr<T>(stage + off), hi = lds_read_tr<T>(stage + (off + 4 * pitch));
    return __builtin_bit_cast(frag, (u32x4{lo.x, lo.y, hi.x, hi.y}));
  };
  frag fa[2][MT], fb[2][NT];
  auto read1 = [&](int into, const char* stage, int c, int n) __attribute__((always_inline)) {
    if (n < MT) fa[into][n] = frag_at(stage, 0, AK, BM, c, MT * wm + n);
    if (n < NT) fb[into][n] = frag_at(stage, STAGE_A, BKC, BN, c, NT * wn + n);
  };
  // db: the first block of a row of tiles sums (with splits, which are joined
  // anyway, all blocks of the row take the stages in turn), the waves of a column
  // take the chunks in turn; the first three plane pairs hold every plane of A once
  auto sum_a = [&](int from, int c, uint32_t st) __attribute__((always_inline)) {
    if constexpr (KIND == MM_DW) {
      if (p.part_db && c % WN == wn && st < (uint32_t)(3 * per_pair) &&
          (p.o.n_split == 1 ? at.tj == 0 : st % tj == (uint32_t)at.tj)) {
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
          for (int e = 0; e < 8; ++e) db[a] += Elem<T>::to_f(fa[from][a][e]);
      }
    }
  };
  // the products of a chunk; the reads of the next chunk go out between the first
  // of them, a stage's loads between all of them
  auto chunk = [&](int from, const char* stage, int c, uint32_t into, auto loads) __attribute__((always_inline)) {
    constexpr int NP = MT * NT, RD = MT > NT ? MT : NT, PER = (2 * GA + NP - 1) / NP;
    constexpr bool LOADS = decltype(loads)::value;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      Elem<T>::mma(acc[n / NT][n % NT], fb[from][n % NT], fa[from][n / NT]);
      if (n < RD) read1(from ^ 1, stage, c, n);
      if constexpr (LOADS) {
#pragma unroll
        for (int q = n * PER; q < (n + 1) * PER; ++q)
          if (q < 2 * GA) load(into, q >> 1, q & 1);
      }
      if (n < RD || (LOADS && n * PER < 2 * GA)) __builtin_amdgcn_sched_barrier(0);
    }
  };
  // one stage; its first chunk is already in fragments 0
  auto turn = [&](int st, char* now, uint32_t lds_now, char* next) __attribute__((always_inline)) {
    prepare();
#pragma unroll
    for (int c = 0; c < 3; ++c) {
      chunk(c & 1, now, c + 1, 0, std::false_type{});
      sum_a(c & 1, c, st);
    }
    stage_sync<0>();
    chunk(1, next, 0, lds_now, std::true_type{});
    sum_a(1, 3, st);
  };
  prepare();
#pragma unroll
  for (int q = 0; q < 2 * GA; ++q) load(lds0, q >> 1, q & 1);
  prepare();
#pragma unroll
  for (int q = 0; q < 2 * GA; ++q) load(lds1, q >> 1, q & 1);
  stage_sync<2 * GA>();
#pragma unroll
  for (int q = 0; q < (MT > NT ? MT : NT); ++q) read1(0, s0, 0, q);
  for (int st = 0; st < turns; st += 2) {
    turn(st, s0, lds0, s1);
    if (st + 1 < turns) turn(st + 1, s1, lds1, s0);
  }
  stage_sync<0>();   // no load in flight when LDS is used again or given up

  if constexpr (KG > 1) {
    // a group's sums: [wave][16][64] in its first stage, those of A in its second
    float* mine = (float*)s0;
    if (kg > 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) mine[(wave * 16 + r) * 64 + lane] = acc[0][0][r];
      if constexpr (KIND == MM_DW) ((float*)s1)[tid] = db[0];
    }
    lds_sync();
    if (kg > 0) return;
#pragma unroll
    for (int q = 1; q < KG; ++q) {
      const float* from = (const float*)(s0 + q * mm_stage<MT, NT, WN>());
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[0][0][r] += from[(wave * 16 + r) * 64 + lane];
      if constexpr (KIND == MM_DW) db[0] += ((const float*)(s1 + q * mm_stage<MT, NT, WN>()))[tid];
    }
  }
  // element by element only where a wave's columns reach over the edge (dw has no
  // activation: both ways in one kernel)
  const int64_t iw = i0 + 32 * MT * wm, jw = j0 + 32 * NT * wn;
  if ((WHOLE && (KIND != MM_DW || p.o.J % 8 == 0)) || jw + 32 * NT <= p.o.J)
    mm_results<KIND, true>(p.o, at.g, at.split, iw, jw, acc);
  else
    mm_results<KIND, false>(p.o, at.g, at.split, iw, jw, acc);
  if constexpr (KIND == MM_DW) {
    if (p.part_db) {
      float* sums = (float*)s0;   // [WN][BM]
#pragma unroll
      for (int a = 0; a < MT; ++a) {
        const float s = db[a] + __shfl_xor(db[a], 32);
        if (lane < 32) sums[wn * BM + 32 * (MT * wm + a) + lane] = s;
      }
      lds_sync();
      float sum = sums[tid % BM];
#pragma unroll
      for (int n = 1; n < WN; ++n) sum += sums[n * BM + tid % BM];
      mm_store_db(p, at.g, at.split, at.tj, (int)tj, i0, tid < BM ? tid : -1, sum);
    }
  }
}

template <class T, class TO, int KIND, int MT, int NT, int WN, int OCC, bool WHOLE, int KG = 1>
__global__ void __launch_bounds__(128 * WN * KG) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
k_mm_piped(const MmArgs<T, TO> p) {
  __shared__ __attribute__((aligned(1024))) char s0[KG * mm_stage<MT, NT, WN>()];
  __shared__ __attribute__((aligned(1024))) char s1[KG * mm_stage<MT, NT, WN>()];
  mm_piped<T, TO, KIND, MT, NT, WN, WHOLE, KG>(p, blockIdx.x, gridDim.x, s0, s1);
}

// ---------------------------------------------------------------------------
// sums of split products
// ---------------------------------------------------------------------------
// the last db_blocks blocks (dw) add the slots of db: [G][slots][I]
template <int KIND, class TO>
__global__ void __launch_bounds__(256) k_mm_join(const MmOut<TO> o, const float* __restrict__ part_db, int slots,
                                                 float* __restrict__ db, int db_blocks) {
  const int g = blockIdx.z;
  const unsigned blocks = gridDim.x - db_blocks;
  if constexpr (KIND == MM_DW) {
    if (blockIdx.x >= blocks) {
      const int64_t i = (int64_t)(blockIdx.x - blocks) * 256 + threadIdx.x;
      if (i >= o.I) return;
      double s = 0.0;
#pragma unroll 8
      for (int n = 0; n < slots; ++n) s += (double)part_db[((int64_t)g * slots + n) * o.I + i];
      db[g * o.I + i] = (float)s;
      return;
    }
  }
  const int64_t vpr = (o.J + 7) / 8, total = o.I * vpr;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)blocks * 256) {
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
    mm_finish<KIND>(o, g, i, j, o.J - j, bias, v);
  }
}

template <int KIND, class TO>
hipError_t join_launch(const MmOut<TO>& o, int G, hipStream_t st, const float* part_db = nullptr, int slots = 0,
                       float* db = nullptr) {
  const int64_t blocks = (o.I * ((o.J + 7) / 8) + 255) / 256, more = db ? (o.I + 255) / 256 : 0;
  k_mm_join<KIND, TO><<<dim3((unsigned)((blocks < 8192 ? blocks : 8192) + more), 1, G), 256, 0, st>>>(o, part_db, slots, db,
                                                                                                      (int)more);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// launch of a tile
// ---------------------------------------------------------------------------
// blocks of a product, 0 where the kernels do not take it
template <class T, class TO, int KIND>
uint32_t mm_blocks(const MmArgs<T, TO>& a, int tile, bool direct, int G) {
  const int64_t side = mm_tile_side(tile);
  const int64_t rows = (a.o.I + side - 1) / side, cols = (a.o.J + side - 1) / side;
  // a launch's x dimension holds fewer than 2^32 threads
  const double threads = (double)rows * cols * a.o.n_split * G * mm_tile_threads(tile);
  if (a.o.I < 1 || a.o.J < 1 || a.K < 1 || a.o.n_split < 1 || G < 1 || G > 65535 ||
      threads > 4294967295.0 || a.o.n_split > (a.K + 63) / 64 || (a.o.n_split > 1 && !a.o.part) ||
      (a.pairs != 1 && a.pairs != 6) || a.K > 0x7fffffff || (!direct && (tile == MM_256 || tile == MM_64K)) ||
      (direct && !(mm_whole(a.a, KIND == MM_DW ? a.o.I : a.K, G) && mm_whole(a.b, KIND == MM_FWD ? a.K : a.o.J, G))))
    return 0;
  return (uint32_t)(rows * cols * a.o.n_split * G);
}

template <class T, class TO, int KIND, bool WHOLE>
void mm_direct(const MmArgs<T, TO>& a, int tile, uint32_t count, hipStream_t st) {
  if (tile == MM_256) k_mm_piped<T, TO, KIND, 4, 2, 4, 2, WHOLE><<<count, 512, 0, st>>>(a);
  else if (tile == MM_128) k_mm_piped<T, TO, KIND, 2, 2, 2, 2, WHOLE><<<count, 256, 0, st>>>(a);
  else if (tile == MM_64) k_mm_piped<T, TO, KIND, 1, 1, 2, 4, WHOLE><<<count, 256, 0, st>>>(a);
  else k_mm_piped<T, TO, KIND, 1, 1, 2, 4, WHOLE, 4><<<count, 1024, 0, st>>>(a);
}

template <class T, class TO, int KIND>
hipError_t mm_launch(const MmArgs<T, TO>& a, int tile, bool direct, int G, hipStream_t st) {
  const uint32_t count = mm_blocks<T, TO, KIND>(a, tile, direct, G);
  if (!count) return hipErrorInvalidValue;
  if (direct) {
    if (KIND == MM_DW || a.o.J % 8 == 0) mm_direct<T, TO, KIND, true>(a, tile, count, st);
    else if constexpr (KIND != MM_DW) mm_direct<T, TO, KIND, false>(a, tile, count, st);
  } else {
    if (tile == MM_128) k_mm_any<T, TO, KIND, 2, 2><<<count, 256, 0, st>>>(a);
    else k_mm_any<T, TO, KIND, 1, 1><<<count, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace pigan
