// Products of matrices of 8-bit numbers with a scale for each block of 128 numbers of the contraction:
//   C[m, n] = sum_b SA[m, b] SB[n, b] sum_{k in block b} A[m, k] B[n, k]          (B with a scale per row, or per 128 rows)
// The inner sum of a block starts from zero, is multiplied by its two scales and added in fp32.  B (the weights) is the instruction's first operand: a
// lane then holds four neighbouring columns of C for one row m, whose scale is one number of the lane.
// For a C of 16 bits the inner sum is one v_mfma_f32_16x16x128_f8f6f4, at twice the rate of 16-bit numbers: it cuts products off below 2^-13 of the
// largest of eight neighbours, a part of 1e-5 of the sum of |products| where C keeps 2^-8 or 2^-11 of itself.  For an fp32 C numbers go through
// fp16, where nothing is lost (mfma_wide).
//
// k_tiles_e4m3: for many rows, bound by the matrix cores.  k_rows_e4m3: for few rows, bound by the read of B.
#include "e4m3.h"
#include "tile.h"

namespace brsvd {

struct E4m3Args {
  Operand A, B;            // rows: m, n; pitch in bytes
  const float *SA, *SB;    // [m][blocks], [n or n / 128][blocks]
  int64_t k;
  int blocks, per_split;   // blocks of the contraction, and of a split
  void* C;                 // rows of ldc numbers of type dtype; with splits: [split][m][n] fp32
  int64_t ldc;
  int dtype, splits;
  int64_t tiles_n, tiles_m;
};

// Four neighbouring numbers of a row of C (of `left` that the row still has)
__device__ __forceinline__ void put_four(void* C, int64_t at, int64_t left, int dtype, floatx4 v) {
  if (dtype == BRSVD_DTYPE_F32) {
    float* o = (float*)C + at;
    if (left >= 4 && ((uintptr_t)o & 15) == 0) *(floatx4*)o = v;
    else
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (r < left) o[r] = v[r];
  } else {
    uint16_t h[4], *o = (uint16_t*)C + at;
#pragma unroll
    for (int r = 0; r < 4; ++r) h[r] = dtype == BRSVD_DTYPE_BF16 ? to16<Bf16>(v[r]) : to16<Fp16>(v[r]);
    if (left >= 4 && ((uintptr_t)o & 7) == 0) *(uint2*)o = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
    else
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (r < left) o[r] = h[r];
  }
}

// Whether an fp32 number is a power of two in the range of an 8-bit exponent
__device__ __forceinline__ bool is_power(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x807fffffu) == 0 && b - 1u < 0x7f7fffffu;
}

// 256 columns of C (B's rows, P) x 64 NQ rows (A's, Q): eight waves of 8 x NQ tiles.  A block of the contraction is a step of eight groups: two tile rows
// times half of the tile columns, NQ instructions.  Two tile rows are read from LDS two groups before they are multiplied; a half of A's fragments is
// replaced as soon as its last group is issued.  So a step needs no registers for the next one beside its own, and still no wave comes from
// the barrier (before the last two groups) with nothing to multiply.  The step after next is sent for in parts from the barrier on, see TileProduct,
// three a group: 8192 x 8192 x 8192 452 / 442 / 427 / 438 us with one / two / three / four on one card; 437 to 452 on others (2.43 to 2.58 Pflop/s, bound by the matrix cores and what
// feeds them: busy in 61 % of the cycles; a library product with one scale for all runs at 3.19).
// As long as a wave's scales of a step are powers of two, as those of the casts are, the instruction multiplies by them and adds to the sums; from the
// first step where they are not (and WIDE) the results of a group are scaled and added between the instructions of the next.
template <int NQ, bool PER_ROW, bool DIRECT, bool WIDE>
__global__ void __launch_bounds__(512, 2)
k_tiles_e4m3(const E4m3Args g) {
  constexpr int NP = 8, WP = 2, WQ = 4, BP = 16 * NP * WP, BQ = 16 * NQ * WQ, THREADS = 64 * WP * WQ, kHalf = (BP + BQ) * kStepBytes, QH = NQ / 2;
  constexpr int kPScales = PER_ROW ? BP : BP / kBlock;
  static_assert(16 * NP == kBlock && BQ + kPScales <= THREADS, "");
  __shared__ __attribute__((aligned(1024))) char lds[2 * kHalf];
  __shared__ __attribute__((aligned(16))) float scales[2][BQ + (PER_ROW ? BP : 4)];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_n, g.tiles_m, 8, &tp, &tq)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
  const int64_t p0 = tp * BP, q0 = tq * BQ;
  const int b0 = blockIdx.y * g.per_split, b1 = b0 + g.per_split < g.blocks ? b0 + g.per_split : g.blocks, whole = (int)(g.k / kBlock);
  const int steps = (b1 < whole ? b1 : whole) - b0;         // whole blocks; a last one that is not follows by itself
  Stager<E4m3, kRows, BP, THREADS, DIRECT> sp;
  Stager<E4m3, kRows, BQ, THREADS, DIRECT> sq;
  sp.init(g.B, p0, (int64_t)b0 * kBlock, tid);
  sq.init(g.A, q0, (int64_t)b0 * kBlock, tid);
  // Addresses that are needed once a step are worked out from the thread's index there: kept, they would cost registers that the tiles need.
  auto thread = [] {
    int x = threadIdx.x;
    asm volatile("" : "+v"(x));
    return x;
  };
  const float *sa0 = (const float*)scalar((int64_t)(g.SA + q0 * g.blocks + b0)), *sb0 = (const float*)scalar((int64_t)(g.SB + (PER_ROW ? p0 : p0 / kBlock) * g.blocks + b0));
  const int last_a = (int)(g.A.n - q0 < BQ ? g.A.n - q0 : BQ) - 1;
  const int last_b = (int)(PER_ROW ? (g.B.n - p0 < BP ? g.B.n - p0 : BP) : (g.B.n - p0 > kBlock ? 2 : 1)) - 1;
  // a step's scales, one a thread, straight into LDS; a wave's are all of A or all of B
  auto send_scales = [&](int t) {
    const int s = thread();
    const uint32_t to = lds_address(&scales[t & 1][64 * wave]);
    if (s < BQ) load4_to_lds(to, sa0 + (int64_t)((s < last_a ? s : last_a) * g.blocks + t));
    else if (s < BQ + kPScales) load4_to_lds(to, sb0 + (int64_t)((s - BQ < last_b ? s - BQ : last_b) * g.blocks + t));
  };
  constexpr int PARTS = decltype(sp)::kLoads + decltype(sq)::kLoads;
  auto send_part = [&](int t, int j) {
    char* to = lds + (t & 1) * kHalf;
    if (j < decltype(sp)::kLoads) sp.load_part(to, wave, j);
    else if (j < PARTS) sq.load_part(to + BP * kStepBytes, wave, j - decltype(sp)::kLoads);
  };
  auto fetch = [&] {
    sp.fetch();
    sq.fetch();
  };
  auto keep = [&](int t) {
    sp.store(lds + (t & 1) * kHalf, tid);
    sq.store(lds + (t & 1) * kHalf + BP * kStepBytes, tid);
  };
  auto send = [&](int t) {             // all of a step at once
    if (DIRECT) {
#pragma unroll
      for (int j = 0; j < PARTS; ++j) send_part(t, j);
      sp.next();
      sq.next();
    } else {
      fetch();
      keep(t);
    }
  };
  auto meet = [] {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  floatx4 acc[NP][NQ];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int q = 0; q < NQ; ++q) acc[p][q] = floatx4{0.f, 0.f, 0.f, 0.f};
  uint32_t bp = fragment_base<kRows, BP>(16 * wp * NP, lane), bq = fragment_base<kRows, BQ>(16 * wq * NQ, lane);
  int4v fp[2][2][2], fq[NQ][2];        // [pair & 1][row of the pair][half], [column][half]
  auto read_pair = [&](int t, int pair) {
    const char* tile = lds + (t & 1) * kHalf;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) fp[pair & 1][i][h] = fragment<kRows, BP>(tile, bp, 2 * pair + i, h);
  };
  auto read_half = [&](int t, int half) {
    const char* tile = lds + (t & 1) * kHalf + BP * kStepBytes;
#pragma unroll
    for (int i = 0; i < QH; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) fq[half * QH + i][h] = fragment<kRows, BQ>(tile, bq, half * QH + i, h);
  };
  if (steps > 0) {
    send_scales(0);
    send(0);
  }
  if (steps > 1) {
    send_scales(1);
    send(1);
  }
  meet();
  if (steps > 0) {
    read_pair(0, 0);
    read_half(0, 0);
  }
  // what a group does beside its products
  auto around = [&](int t, int G) {
    const int pair = G >> 1, half = G & 1;
    const bool more = t + 1 < steps, sends = t + 2 < steps;
    if (G == 0) read_half(t, 1);
    if (half == 0 && pair < 3) read_pair(t, pair + 1);
    if (G == 6) {
      meet();
      if (sends) send_scales(t + 2);
      if (more) read_pair(t + 1, 0);
      if (!DIRECT && sends) fetch();
    }
    if (G == 7 && more) read_half(t + 1, 0);
    if (DIRECT) {
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        if (G >= 6 && sends) send_part(t + 2, 3 * (G - 6) + j);
        if (G < 6 && 3 * G + 6 + j < PARTS && t > 0 && more) send_part(t + 1, 3 * G + 6 + j);
      }
      if (G == 5 && t > 0 && more) {
        sp.next();
        sq.next();
      }
    }
    if (!DIRECT && G == 7 && sends) keep(t + 2);
  };
  // the block that the contraction ends in, behind all others
  const bool ends = b1 > whole && g.k % kBlock != 0;
  auto stage_end = [&] {
    meet();
    const int64_t left = g.k - (int64_t)whole * kBlock;
    sp.load(lds, tid, wave, left);
    sq.load(lds + BP * kStepBytes, tid, wave, left);
    sp.store(lds, tid);
    sq.store(lds + BP * kStepBytes, tid);
    const int s = thread(), at = whole - b0;
    if (s < BQ) scales[0][s] = sa0[(int64_t)((s < last_a ? s : last_a) * g.blocks + at)];
    else if (s < BQ + kPScales) scales[0][s] = sb0[(int64_t)((s - BQ < last_b ? s - BQ : last_b) * g.blocks + at)];
    meet();
    read_half(0, 0);
    read_half(0, 1);
  };
  auto end = [&] {
    stage_end();
#pragma unroll
    for (int pair = 0; pair < 4; ++pair) {
      read_pair(0, pair);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        floatx4 sb = {1.f, 1.f, 1.f, 1.f};
        if (PER_ROW) sb = *(const floatx4*)&scales[0][BQ + 16 * (wp * NP + 2 * pair + i) + 4 * (lane >> 4)];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const float s = scales[0][16 * (wq * NQ + q) + (lane & 15)] * (PER_ROW ? 1.f : scales[0][BQ + wp]);
          floatx4 d;
          if (WIDE) d = mfma_wide(widen(fp[pair & 1][i][0], fp[pair & 1][i][1]), widen(fq[q][0], fq[q][1]));
          else d = mfma8(fp[pair & 1][i][0], fp[pair & 1][i][1], fq[q][0], fq[q][1], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[2 * pair + i][q][r] += d[r] * (s * sb[r]);
          settle(acc[2 * pair + i][q]);
        }
      }
    }
  };
  int t = 0;
  if constexpr (!WIDE) {
#pragma unroll 1
    for (; t < steps; ++t) {
      asm volatile("" : "+v"(bp), "+v"(bq));      // addresses are worked out from these where they are used, not kept
      // exponents of the step's scales: of the lane's row of each tile column, and of each tile row
      uint32_t ea = 0, eb[2] = {0u, 0u};
      bool powers = true;
      const float* s = scales[t & 1];
      const int l = thread() & 15;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float x = s[16 * (wq * NQ + q) + l];
        powers &= is_power(x);
        ea |= __float_as_uint(x) >> 23 << (8 * q);
      }
      if (PER_ROW) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const float x = s[BQ + 16 * (wp * NP + p) + l];
          powers &= is_power(x);
          eb[p / 4] |= __float_as_uint(x) >> 23 << (8 * (p & 3));
        }
      } else {
        const float x = s[BQ + wp];                // a wave's 128 rows of B are one block
        powers &= is_power(x);
        eb[0] = eb[1] = (__float_as_uint(x) >> 23) * 0x01010101u;
      }
      if (!__all(powers)) break;
#define BRSVD_SCALED(I, J)                                                                                                                            \
  {                                                                                                                                                   \
    constexpr int p = 2 * (G >> 1) + I, q = (G & 1) * QH + J;                                                                                         \
    acc[p][q] = mfma8_scaled<(p & 3), q>(fp[(G >> 1) & 1][I][0], fp[(G >> 1) & 1][I][1], fq[q][0], fq[q][1], acc[p][q], (int)eb[p / 4], (int)ea);     \
    settle(acc[p][q]);                                                                                                                                \
  }
#define BRSVD_GROUP(GROUP)                                                                                                                            \
  {                                                                                                                                                   \
    constexpr int G = GROUP;                                                                                                                          \
    around(t, G);                                                                                                                                     \
    BRSVD_SCALED(0, 0)                                                                                                                                \
    BRSVD_SCALED(1, 0)                                                                                                                                \
    if constexpr (QH == 2) {                                                                                                                          \
      BRSVD_SCALED(0, (QH - 1))                                                                                                                       \
      BRSVD_SCALED(1, (QH - 1))                                                                                                                       \
    }                                                                                                                                                 \
    __builtin_amdgcn_sched_barrier(0);                                                                                                                \
  }
      BRSVD_GROUP(0)
      BRSVD_GROUP(1)
      BRSVD_GROUP(2)
      BRSVD_GROUP(3)
      BRSVD_GROUP(4)
      BRSVD_GROUP(5)
      BRSVD_GROUP(6)
      BRSVD_GROUP(7)
#undef BRSVD_GROUP
#undef BRSVD_SCALED
    }
  }
#pragma unroll 1
  for (; t < steps; ++t) {
    asm volatile("" : "+v"(bp), "+v"(bq));
    floatx4 d[2][QH], sb[2], sb_last[2];
    float sa[NQ];
    Wide8 wp8[2], wq8[NQ];
    const int l = thread();
    const float w = PER_ROW ? 1.f : scales[t & 1][BQ + wp];
#pragma unroll
    for (int q = 0; q < NQ; ++q) sa[q] = scales[t & 1][16 * (wq * NQ + q) + (l & 15)] * w;
    // the result of the group before, of row i of its pair and column j of its half
    auto add = [&](int group, int i, int j) {
      const int p = 2 * (group >> 1) + i, q = (group & 1) * QH + j;
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[p][q][r] += d[i][j][r] * (PER_ROW ? sa[q] * sb_last[i][r] : sa[q]);
      settle(acc[p][q]);
    };
#pragma unroll
    for (int G = 0; G < 8; ++G) {
      const int pair = G >> 1, half = G & 1;
      if (PER_ROW && half == 0)
#pragma unroll
        for (int i = 0; i < 2; ++i) sb[i] = *(const floatx4*)&scales[t & 1][BQ + 16 * (wp * NP + 2 * pair + i) + (l & 48) / 4];
      around(t, G);
      if (WIDE) {
        if (pair == 0)
#pragma unroll
          for (int j = 0; j < QH; ++j) wq8[half * QH + j] = widen(fq[half * QH + j][0], fq[half * QH + j][1]);
        if (half == 0)
#pragma unroll
          for (int i = 0; i < 2; ++i) wp8[i] = widen(fp[pair & 1][i][0], fp[pair & 1][i][1]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < QH; ++j) {
          if (G > 0) add(G - 1, i, j);
          const int q = half * QH + j;
          if (WIDE) d[i][j] = mfma_wide(wp8[i], wq8[q]);
          else d[i][j] = mfma8(fp[pair & 1][i][0], fp[pair & 1][i][1], fq[q][0], fq[q][1], floatx4{0.f, 0.f, 0.f, 0.f});
        }
      if (PER_ROW && half == 0) sb_last[0] = sb[0], sb_last[1] = sb[1];
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < QH; ++j) add(7, i, j);
  }
  if (ends) end();
  if (g.dtype == BRSVD_DTYPE_F32) {
    char* C = (char*)g.C + (g.splits > 1 ? (int64_t)blockIdx.y * g.A.n * g.B.n * 4 : 0);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t m = q0 + 16 * (wq * NQ + q) + (lane & 15);
      if (m >= g.A.n) continue;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int64_t n = p0 + 16 * (wp * NP + p) + 4 * (lane >> 4);
        if (n < g.B.n) put_four(C, m * g.ldc + n, g.B.n - n, BRSVD_DTYPE_F32, acc[p][q]);
      }
    }
  } else {
    uint16_t* C = (uint16_t*)g.C + q0 * g.ldc + p0;
    meet();
    if (g.dtype == BRSVD_DTYPE_BF16) put_tile16<NQ>(acc, lds, C, g.ldc, g.A.n - q0, g.B.n - p0, [](float x, int) { return to16<Bf16>(x); });
    else put_tile16<NQ>(acc, lds, C, g.ldc, g.A.n - q0, g.B.n - p0, [](float x, int) { return to16<Fp16>(x); });
  }
}

// C (m x n, type dtype) = sum of the splits' parts, in their order
__global__ void __launch_bounds__(256)
k_join_splits(const float* __restrict__ part, int splits, int64_t m, int64_t n, void* __restrict__ C, int64_t ldc, int dtype, unsigned first_wg) {
  const int64_t quads = (n + 3) / 4, i = ((int64_t)first_wg + blockIdx.x) * 256 + threadIdx.x;
  if (i >= m * quads) return;
  const int64_t row = i / quads, col = (i - row * quads) * 4, at = row * n + col;
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (col + r < n) sum[r] += part[s * m * n + at + r];
  put_four(C, row * ldc + col, n - col, dtype, sum);
}

// Up to 16 MT rows of A.  The WAVES waves of a workgroup share 16 NT rows of B and take the blocks of the contraction in turn; their sums are added through
// LDS in wave order.  B goes from memory to the instruction's registers (a lane: 16 bytes at two places of a
// row's block), the U blocks that a wave takes next on their way; so does A, which all workgroups read and the caches hold.  DT >= 0: A comes in numbers of more
// bits, and a block of it is cast where it is used, in registers: four lanes hold a row's block, its largest number takes two exchanges.  Bound by the read
// of B: 24 x 20000 x 5000 29 us (100 MB, 3.4 TB/s); 1 x 4096 x 4096 6.4 us, of which a launch is four.
template <int MT, int NT, int U, int WAVES, int DT, bool WIDE>     // DT: type of A's numbers, -1: 8 bits with scales
__global__ void __launch_bounds__(64 * WAVES)
k_rows_e4m3(const E4m3Args g) {
  constexpr bool CAST = DT >= 0;
  constexpr int EB = DT == BRSVD_DTYPE_F32 ? 4 : DT >= 0 ? 2 : 1;
  __shared__ floatx4 parts[WAVES][MT * NT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16 * NT;
  const int row = lane & 15, piece = 16 * (lane >> 4);
  floatx4 acc[MT][NT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u) acc[t][u] = floatx4{0.f, 0.f, 0.f, 0.f};
  const char* rb[NT];
  const float* sb = g.SB + n0 / kBlock * g.blocks;        // 16 NT rows from a multiple of 16 NT on: one row of scales
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const int64_t n = n0 + 16 * u + row, in = n < g.B.n ? n : g.B.n - 1;
    rb[u] = g.B.base + in * g.B.ld + piece;
  }
  const char* ra[MT];
  const float* sa[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = 16 * t + row < g.A.n ? 16 * t + row : g.A.n - 1;
    ra[t] = g.A.base + m * g.A.ld + piece * EB;
    sa[t] = CAST ? nullptr : g.SA + m * g.blocks;
  }
  // what a lane has of a block: [piece at 0, piece at 64]
  struct Block {
    uint4 b[NT][2], a[MT][2 * EB];
    float sb, sa[MT];
  };
  auto fetch = [&](Block& x, int blk, bool whole, int64_t left) {       // left: numbers of the row from this lane's first piece on
    const int64_t at = (int64_t)blk * kBlock;
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) x.b[u][h] = piece_of<1>(rb[u] + at + 64 * h, whole ? 16 : left - 64 * h);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < EB; ++j) x.a[t][h * EB + j] = piece_of<EB>(ra[t] + (at + 64 * h) * EB + 16 * j, whole ? 16 : (left - 64 * h) * EB - 16 * j);
      if (!CAST) x.sa[t] = sa[t][blk];
    }
    x.sb = sb[blk];
  };
  auto multiply = [&](const Block& x) {
    Wide8 ew[NT];
    if (WIDE)
#pragma unroll
      for (int u = 0; u < NT; ++u) ew[u] = widen(__builtin_bit_cast(int4v, x.b[u][0]), __builtin_bit_cast(int4v, x.b[u][1]));
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      int4v f[2];
      float s;
      if constexpr (CAST) {
        float v[2][16], top = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < EB; ++j) {
            const uint4 p = x.a[t][h * EB + j];
            const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
            for (int i = 0; i < 16 / EB; ++i)
              v[h][16 / EB * j + i] = DT == BRSVD_DTYPE_F32 ? __uint_as_float(w[EB == 4 ? i : 0])
                                      : DT == BRSVD_DTYPE_BF16 ? from16<Bf16>((uint16_t)(w[i / 2] >> (16 * (i & 1)))) : from16<Fp16>((uint16_t)(w[i / 2] >> (16 * (i & 1))));
          }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, finite_abs(v[h][i]));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const int ex = block_exponent(top);
        const float inv = power_of_two(-ex);
        s = power_of_two(ex);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) f[h][i] = (int)pack_e4m3(v[h][4 * i] * inv, v[h][4 * i + 1] * inv, v[h][4 * i + 2] * inv, v[h][4 * i + 3] * inv);
      } else {
        f[0] = __builtin_bit_cast(int4v, x.a[t][0]);
        f[1] = __builtin_bit_cast(int4v, x.a[t][1]);
        s = x.sa[t];
      }
      s *= x.sb;
      Wide8 fw;
      if (WIDE) fw = widen(f[0], f[1]);
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        const floatx4 d = WIDE ? mfma_wide(ew[u], fw) : mfma8(__builtin_bit_cast(int4v, x.b[u][0]), __builtin_bit_cast(int4v, x.b[u][1]), f[0], f[1], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][u][r] += d[r] * s;
      }
    }
  };
  const int whole = (int)(g.k / kBlock);
  Block x[U];
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (wave + WAVES * i < whole) fetch(x[i], wave + WAVES * i, true, 0);
  for (int b = wave; b < whole; b += WAVES * U) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (b + WAVES * i < whole) multiply(x[i]);
      if (b + WAVES * (i + U) < whole) fetch(x[i], b + WAVES * (i + U), true, 0);
    }
  }
  if (whole < g.blocks && whole % WAVES == wave) {          // the contraction's end, after the wave's other blocks
    fetch(x[0], whole, false, g.k - (int64_t)whole * kBlock - piece);
    multiply(x[0]);
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u) parts[wave][t * NT + u][lane] = acc[t][u];
  __syncthreads();
  for (int i = wave; i < MT * NT; i += WAVES) {
    floatx4 sum = parts[0][i][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += parts[w][i][lane];
    const int64_t m = 16 * (i / NT) + row, n = n0 + 16 * (i % NT) + 4 * (lane >> 4);
    if (m < g.A.n && n < g.B.n) put_four(g.C, m * g.ldc + n, g.B.n - n, g.dtype, sum);
  }
}

static void join_splits(const float* part, int splits, int64_t m, int64_t n, void* C, int64_t ldc, int dtype, hipStream_t stream) {
  in_launches(ceil_div(m * ceil_div(n, 4), 256), 256, [&](unsigned first, dim3 grid) {
    hipLaunchKernelGGL(k_join_splits, grid, dim3(256), 0, stream, part, splits, m, n, C, ldc, dtype, first);
  });
}

// Rows up to which the read of B bounds the product.  Above 32 the tiles are ahead where B has rows for them: 60 x 20000 x 5000 47 us and 82, the
// other way round where it has not: 24 x 4096 x 4096 17.6 and 9.6, 24 x 20000 x 5000 43 and 41.
static bool few_rows(int64_t m, int64_t n) { return m <= 32 || (m <= 64 && n < 16 * 512); }
constexpr int64_t kCastRows = 16;     // rows up to which they are cast inside it

// How often the contraction is cut so that there are workgroups for every CU: only while a part keeps `least` blocks.
static int splits_for(int64_t workgroups, int blocks, int least) {
  int s = (int)(256 / workgroups);
  if (s > blocks / least) s = blocks / least;
  return s < 1 ? 1 : s > 16 ? 16 : s;
}
struct E4m3Plan {
  bool rows;               // k_rows_e4m3
  int splits, per_split;
  int64_t large;           // columns of C in tiles of 256 rows, in 256; the others in tiles of 128
};
static E4m3Plan e4m3_plan(int64_t m, int64_t n, int64_t k, bool per_row, int dtype) {
  E4m3Plan p;
  const int blocks = (int)ceil_div(k, kBlock);
  p.rows = few_rows(m, n) && !per_row;
  // A tile of 256 x 256 has no registers left for the fp16 numbers of an fp32 result.  Rounds of 256 workgroups: 1000 x 5000 from 3000 39 us in 256 x 128 and
  // 57 in 256 x 256 (160 tiles and 80, one round).
  const int64_t cols = ceil_div(n, 256);
  p.large = dtype == BRSVD_DTYPE_F32 || m <= 128 ? 0 : large_tiles(cols, ceil_div(m, 256), ceil_div(m, 128), blocks);
  p.splits = 1;
  if (!p.rows) p.splits = splits_for(p.large * ceil_div(m, 256) + (cols - p.large) * ceil_div(m, 128), blocks, 4);
  p.per_split = (int)ceil_div(blocks, p.splits);
  p.splits = (int)ceil_div(blocks, p.per_split);
  return p;
}
// Whether the launches of a plan may have their workgroups.  direct: rows of both operands at 16-byte addresses.
static bool e4m3_plan_fits(const E4m3Plan& p, int64_t m, int64_t n, bool direct, int dtype) {
  if (p.rows) return ceil_div(n, 32) <= launch_workgroups(256);          // as launch_rows where there are that many rows of B
  const int64_t cols = ceil_div(n, 256), large = direct && dtype != BRSVD_DTYPE_F32 ? p.large : 0;
  return tiles_fit(large, ceil_div(m, 256), 512) && tiles_fit(cols - large, ceil_div(m, 128), 512);
}
static uint64_t split_bytes(const E4m3Plan& p, int64_t m, int64_t n) { return p.splits > 1 ? (uint64_t)p.splits * m * n * 4 : 0; }

// NT: rows of A are read (and cast) once for 16 NT rows of B, as many as leave workgroups for every CU
template <int MT, int NT, int U, int WAVES, int DT, bool WIDE>
static void launch_rows(const E4m3Args& g, hipStream_t stream) {
  hipLaunchKernelGGL((k_rows_e4m3<MT, NT, U, WAVES, DT, WIDE>), dim3((unsigned)ceil_div(g.B.n, 16 * NT)), dim3(64 * WAVES), 0, stream, g);
}
template <int DT, bool WIDE>
static void launch_few(const E4m3Args& g, hipStream_t stream) {
  if (g.B.n >= 16 * 512) launch_rows<1, 2, 2, 4, DT, WIDE>(g, stream);
  else launch_rows<1, 1, 4, 8, DT, WIDE>(g, stream);
}
template <bool WIDE>
static void launch_more(const E4m3Args& g, hipStream_t stream) {
  if (g.A.n <= 32 && g.B.n >= 32 * 512) launch_rows<2, 2, 2, 4, -1, WIDE>(g, stream);
  else if (g.A.n <= 32) launch_rows<2, 1, 4, 8, -1, WIDE>(g, stream);
  else launch_rows<4, 1, 2, 8, -1, WIDE>(g, stream);
}
template <int NQ, bool PER_ROW, bool DIRECT, bool WIDE>
static void launch_tiles(E4m3Args g, hipStream_t stream) {
  g.tiles_n = ceil_div(g.B.n, 256);
  g.tiles_m = ceil_div(g.A.n, 64 * NQ);
  hipLaunchKernelGGL((k_tiles_e4m3<NQ, PER_ROW, DIRECT, WIDE>), dim3(tile_workgroups(g.tiles_n, g.tiles_m), (unsigned)g.splits), dim3(512), 0, stream, g);
}
template <bool PER_ROW, bool DIRECT>
static void launch_tiles(E4m3Args g, int64_t large, bool wide, hipStream_t stream) {
  if (wide) return launch_tiles<2, PER_ROW, DIRECT, true>(g, stream);
  if constexpr (DIRECT) {                       // nor for pieces on their way through them
    const int64_t n = g.B.n, first = 256 * large < n ? 256 * large : n;
    if (first > 0) {
      g.B.n = first;
      launch_tiles<4, PER_ROW, DIRECT, false>(g, stream);
      if (first == n) return;
      g.B.n = n - first;
      g.B.base += first * g.B.ld;
      g.SB += (PER_ROW ? first : first / kBlock) * g.blocks;
      g.C = (char*)g.C + first * (g.dtype == BRSVD_DTYPE_F32 ? 4 : 2);
    }
  }
  launch_tiles<2, PER_ROW, DIRECT, false>(g, stream);
}

// a_type: type of A's numbers, -1 for 8 bits with the scales SA
static int gemm_e4m3(const void* A, int64_t lda_bytes, int a_type, const float* SA, const uint8_t* B, int64_t ldb, const float* SB, bool per_row, int64_t m, int64_t n,
                     int64_t k, int dtype, void* C, int64_t ldc, const E4m3Plan& plan, float* part, hipStream_t stream) {
  E4m3Args g;
  g.A = Operand{(const char*)A, lda_bytes, m};
  g.B = Operand{(const char*)B, ldb, n};
  g.SA = SA;
  g.SB = SB;
  g.k = k;
  g.blocks = (int)ceil_div(k, kBlock);
  g.per_split = plan.per_split;
  g.splits = plan.splits;
  const bool split = plan.splits > 1;
  g.C = split ? part : C;
  g.ldc = split ? n : ldc;
  g.dtype = split ? BRSVD_DTYPE_F32 : dtype;
  if (plan.rows) {
    const bool wide = dtype == BRSVD_DTYPE_F32;
    if (m > kCastRows) wide ? launch_more<true>(g, stream) : launch_more<false>(g, stream);
    else if (a_type == BRSVD_DTYPE_F32) launch_few<BRSVD_DTYPE_F32, true>(g, stream);
    else if (a_type == BRSVD_DTYPE_BF16) launch_few<BRSVD_DTYPE_BF16, false>(g, stream);
    else if (a_type == BRSVD_DTYPE_F16) launch_few<BRSVD_DTYPE_F16, false>(g, stream);
    else wide ? launch_few<-1, true>(g, stream) : launch_few<-1, false>(g, stream);
  } else {
    const bool direct = aligned_pieces(A, lda_bytes) && aligned_pieces(B, ldb);
    const bool wide = dtype == BRSVD_DTYPE_F32;
    if (per_row && direct) launch_tiles<true, true>(g, plan.large, wide, stream);
    else if (per_row) launch_tiles<true, false>(g, plan.large, wide, stream);
    else if (direct) launch_tiles<false, true>(g, plan.large, wide, stream);
    else launch_tiles<false, false>(g, plan.large, wide, stream);
  }
  if (split) join_splits(part, plan.splits, m, n, C, ldc, dtype, stream);
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

static bool product_type(int dtype) { return dtype == BRSVD_DTYPE_F32 || dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16; }
static bool product_sizes(int64_t m, int64_t n, int64_t k) {
  return m >= 0 && n >= 0 && k >= 0 && k < kMaxPitch && m < (int64_t)1 << 31 && n < (int64_t)1 << 31 && ceil_div(m, 128) * ceil_div(n, 16) <= kMaxGrid;
}
// The cast of the activations for a product that takes them in 8 bits: rows, then their scales.
static uint64_t cast_pitch(int64_t k) { return (uint64_t)line_pitch(k); }
static uint64_t cast_bytes(int64_t m, int64_t k) { return ((uint64_t)m * cast_pitch(k) + 255) / 256 * 256 + ((uint64_t)m * ceil_div(k, kBlock) * 4 + 255) / 256 * 256; }

int quantize(const void* X, int64_t ldx, int64_t rows, int64_t cols, int dtype, int block_rows, uint8_t* Q, int64_t ldq, float* S, uint8_t* Qt, int64_t ldqt,
             float* St, hipStream_t stream);

}  // namespace brsvd

using namespace brsvd;

extern "C" uint64_t brsvd_gemm_e4m3_scratch_bytes(int64_t m, int64_t n, int64_t k, int32_t block_rows, int32_t dtype) {
  if (!product_sizes(m, n, k) || !product_type(dtype) || m == 0 || n == 0 || k == 0) return 0;
  return split_bytes(e4m3_plan(m, n, k, block_rows == 1, dtype), m, n);
}

extern "C" uint64_t brsvd_linear_e4m3_scratch_bytes(int64_t m, int64_t n, int64_t k, int32_t dtype) {
  if (!product_sizes(m, n, k) || !product_type(dtype) || m == 0 || n == 0 || k == 0) return 0;
  const E4m3Plan p = e4m3_plan(m, n, k, false, dtype);
  return split_bytes(p, m, n) + (m <= kCastRows ? 0 : cast_bytes(m, k));
}

extern "C" int brsvd_gemm_e4m3(const uint8_t* A, int64_t lda, const float* SA, const uint8_t* B, int64_t ldb, const float* SB, int32_t block_rows, int64_t m,
                               int64_t n, int64_t k, int32_t dtype, void* C, int64_t ldc, void* scratch, uint64_t scratch_bytes, void* stream) {
  if (!product_sizes(m, n, k) || !product_type(dtype) || (block_rows != 1 && block_rows != kBlock)) return BRSVD_ERR_ARG;
  if (m == 0 || n == 0) return BRSVD_OK;
  if (!C || ldc < n) return BRSVD_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  if (k == 0) {
    // an empty sum: the join of no parts
    join_splits(nullptr, 0, m, n, C, ldc, dtype, s);
    BRSVD_HIP_TRY(hipGetLastError());
    return BRSVD_OK;
  }
  if (!A || !B || !SA || !SB || lda < k || ldb < k || lda >= kMaxPitch || ldb >= kMaxPitch) return BRSVD_ERR_ARG;
  const E4m3Plan p = e4m3_plan(m, n, k, block_rows == 1, dtype);
  if (!e4m3_plan_fits(p, m, n, aligned_pieces(A, lda) && aligned_pieces(B, ldb), dtype)) return BRSVD_ERR_ARG;
  const uint64_t need = split_bytes(p, m, n);
  if (need && (!scratch || (uintptr_t)scratch % 256)) return BRSVD_ERR_ARG;
  if (scratch_bytes < need) return BRSVD_ERR_BUDGET;
  return gemm_e4m3(A, lda, -1, SA, B, ldb, SB, block_rows == 1, m, n, k, dtype, C, ldc, p, (float*)scratch, s);
}

extern "C" int brsvd_linear_e4m3(const void* X, int64_t ldx, int32_t dtype, const uint8_t* W, int64_t ldw, const float* SW, int64_t m, int64_t n, int64_t k,
                                 void* Y, int64_t ldy, void* scratch, uint64_t scratch_bytes, void* stream) {
  if (!product_sizes(m, n, k) || !product_type(dtype)) return BRSVD_ERR_ARG;
  if (m == 0 || n == 0 || k == 0) return brsvd_gemm_e4m3(nullptr, 0, nullptr, nullptr, 0, nullptr, kBlock, m, n, 0, dtype, Y, ldy, nullptr, 0, stream);
  const int eb = dtype == BRSVD_DTYPE_F32 ? 4 : 2;
  if (!X || !W || !SW || !Y || ldx < k || ldw < k || ldy < n || ldx >= kMaxPitch * 4 / eb || ldw >= kMaxPitch) return BRSVD_ERR_ARG;
  const E4m3Plan p = e4m3_plan(m, n, k, false, dtype);
  if (!e4m3_plan_fits(p, m, n, aligned_pieces(W, ldw), dtype)) return BRSVD_ERR_ARG;      // the cast of X lies at such addresses
  const uint64_t parts = split_bytes(p, m, n), need = parts + (m <= kCastRows ? 0 : cast_bytes(m, k));
  if (need && (!scratch || (uintptr_t)scratch % 256)) return BRSVD_ERR_ARG;
  if (scratch_bytes < need) return BRSVD_ERR_BUDGET;
  hipStream_t s = (hipStream_t)stream;
  if (m <= kCastRows) return gemm_e4m3(X, ldx * eb, dtype, nullptr, W, ldw, SW, false, m, n, k, dtype, Y, ldy, p, (float*)scratch, s);
  uint8_t* q = (uint8_t*)scratch;
  float* sq = (float*)(q + ((uint64_t)m * cast_pitch(k) + 255) / 256 * 256);
  BRSVD_TRY(quantize(X, ldx, m, k, dtype, 1, q, (int64_t)cast_pitch(k), sq, nullptr, 0, nullptr, s));
  return gemm_e4m3(q, (int64_t)cast_pitch(k), -1, sq, W, ldw, SW, false, m, n, k, dtype, Y, ldy, p, (float*)((char*)scratch + cast_bytes(m, k)), s);
}
