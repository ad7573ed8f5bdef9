// Products of matrices of 8-bit numbers with a scale for each block of 128 numbers of the contraction:
//   C[m, n] = sum_b SA[m, b] SB[n, b] sum_{k in block b} A[m, k] B[n, k]          (B with a scale per row, or per 128 rows)
// The inner sum of a block starts from zero, is multiplied by its two scales and added in fp32.  B (the weights) is the instruction's first operand: a
// lane then holds four neighbouring columns of C for one row m, whose scale is one number of the lane.
// For a C of 16 bits the inner sum is one v_mfma_f32_16x16x128_f8f6f4, at twice the rate of 16-bit numbers: it cuts products off below 2^-13 of the
// largest of eight neighbours, a part of 1e-5 of the sum of |products| where C keeps 2^-8 or 2^-11 of itself.  An fp32 C, and products of few
// rows, which wait for memory anyway, go through fp16, where nothing is lost (mfma_wide).
//
// k_tiles_e4m3: for many rows, bound by the matrix cores.  k_rows_e4m3: for up to 64 rows, bound by the read of B.
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

// NP x NQ tiles a wave, WP x WQ waves; P = B (columns of C), Q = A (rows of C).  Scales of a step come in beside its numbers.
template <int NP, int NQ, int WP, int WQ, bool PER_ROW, bool DIRECT, bool WIDE>
__global__ void __launch_bounds__(64 * WP * WQ, 2)
k_tiles_e4m3(const E4m3Args g) {
  constexpr int BP = 16 * NP * WP, BQ = 16 * NQ * WQ, THREADS = 64 * WP * WQ, kHalf = (BP + BQ) * kStepBytes;
  constexpr int kPScales = PER_ROW ? BP : BP / kBlock;
  static_assert(BP % kBlock == 0 && (16 * NP % kBlock == 0 || kBlock % (16 * NP) == 0) && BP + BQ <= THREADS * 2, "");
  __shared__ __attribute__((aligned(1024))) char lds[2 * kHalf];
  __shared__ float scales[2][BQ + kPScales];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_n, g.tiles_m, 4, &tp, &tq)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
  const int64_t p0 = tp * BP, q0 = tq * BQ;
  const int b0 = blockIdx.y * g.per_split, b1 = b0 + g.per_split < g.blocks ? b0 + g.per_split : g.blocks;
  Stager<E4m3, kRows, BP, THREADS, DIRECT> sp;
  Stager<E4m3, kRows, BQ, THREADS, DIRECT> sq;
  sp.init(g.B, p0, (int64_t)b0 * kBlock, tid);
  sq.init(g.A, q0, (int64_t)b0 * kBlock, tid);
  // which scale this thread fetches for each step, up to two of them
  const float* from[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = tid + i * THREADS;
    int64_t row = 0;
    if (s < BQ) row = q0 + s < g.A.n ? q0 + s : g.A.n - 1;
    else if (PER_ROW) row = p0 + s - BQ < g.B.n ? p0 + s - BQ : g.B.n - 1;
    else row = p0 / kBlock + s - BQ < (g.B.n - 1) / kBlock ? p0 / kBlock + s - BQ : (g.B.n - 1) / kBlock;
    from[i] = (s < BQ ? g.SA : g.SB) + row * g.blocks;
  }
  floatx4 acc[NP][NQ];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int q = 0; q < NQ; ++q) acc[p][q] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto fetch = [&](int b, float (&v)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (tid + i * THREADS < BQ + kPScales) v[i] = from[i][b];
  };
  auto keep = [&](int buffer, const float (&v)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (tid + i * THREADS < BQ + kPScales) scales[buffer][tid + i * THREADS] = v[i];
  };
  const uint32_t bb = fragment_base<kRows, BP>(16 * wp * NP, lane), ba = fragment_base<kRows, BQ>(16 * wq * NQ, lane);
  float v[2];
  fetch(b0, v);
  sp.load(lds, tid, wave, g.k - (int64_t)b0 * kBlock);
  sq.load(lds + BP * kStepBytes, tid, wave, g.k - (int64_t)b0 * kBlock);
  sp.store(lds, tid);
  sq.store(lds + BP * kStepBytes, tid);
  keep(0, v);
  loads_done();
  __syncthreads();
  for (int b = b0; b < b1; ++b) {
    const int buffer = (b - b0) & 1, cur = buffer * kHalf, nxt = kHalf - cur;
    if (b + 1 < b1) {
      const int64_t left = g.k - (int64_t)(b + 1) * kBlock;
      fetch(b + 1, v);
      sp.load(lds + nxt, tid, wave, left);
      sq.load(lds + nxt + BP * kStepBytes, tid, wave, left);
    }
    const char *tb = lds + cur, *ta = tb + BP * kStepBytes;
    int4v f0[NQ], f1[NQ];
    Wide8 fw[NQ];
    float sa[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      f0[q] = fragment<kRows, BQ>(ta, ba, q, 0);
      f1[q] = fragment<kRows, BQ>(ta, ba, q, 1);
      if (WIDE) fw[q] = widen(f0[q], f1[q]);
      sa[q] = scales[buffer][16 * (wq * NQ + q) + (lane & 15)];
      if (!PER_ROW && 16 * NP <= kBlock) sa[q] *= scales[buffer][BQ + wp * 16 * NP / kBlock];
    }
    // The fragments of the next tile row are on their way while this one is multiplied, and a sum is added once the products of the next tile row are
    // issued; the fences keep the compiler from fetching all rows at once, which it has no registers for.
    int4v e0 = fragment<kRows, BP>(tb, bb, 0, 0), e1 = fragment<kRows, BP>(tb, bb, 0, 1);
    floatx4 d[2][NQ], sb[2];
    sb[0] = sb[1] = floatx4{1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int p = 0; p <= NP; ++p) {
      if (p < NP) {
        const int4v c0 = e0, c1 = e1;
        if (p + 1 < NP) {
          e0 = fragment<kRows, BP>(tb, bb, p + 1, 0);
          e1 = fragment<kRows, BP>(tb, bb, p + 1, 1);
        }
        if (PER_ROW) sb[p & 1] = *(const floatx4*)&scales[buffer][BQ + 16 * (wp * NP + p) + 4 * (lane >> 4)];
        if (WIDE) {
          const Wide8 cw = widen(c0, c1);
#pragma unroll
          for (int q = 0; q < NQ; ++q) d[p & 1][q] = mfma_wide(cw, fw[q]);
        } else {
#pragma unroll
          for (int q = 0; q < NQ; ++q) d[p & 1][q] = mfma8(c0, c1, f0[q], f1[q], floatx4{0.f, 0.f, 0.f, 0.f});
        }
      }
      if (p > 0) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[p - 1][q][r] += d[(p - 1) & 1][q][r] * (PER_ROW ? sa[q] * sb[(p - 1) & 1][r] : sa[q]);
          settle(acc[p - 1][q]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (b + 1 < b1) {
      if (!DIRECT) {
        sp.store(lds + nxt, tid);
        sq.store(lds + nxt + BP * kStepBytes, tid);
      }
      keep(buffer ^ 1, v);
    }
    loads_done();
    __syncthreads();
  }
  char* C = (char*)g.C + (g.splits > 1 ? (int64_t)blockIdx.y * g.A.n * g.B.n * 4 : 0);
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int64_t m = q0 + 16 * (wq * NQ + q) + (lane & 15);
    if (m >= g.A.n) continue;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int64_t n = p0 + 16 * (wp * NP + p) + 4 * (lane >> 4);
      if (n < g.B.n) put_four(C, m * g.ldc + n, g.B.n - n, g.dtype, acc[p][q]);
    }
  }
}

// C (m x n, type dtype) = sum of the splits' parts, in their order
__global__ void __launch_bounds__(256)
k_join_splits(const float* __restrict__ part, int splits, int64_t m, int64_t n, void* __restrict__ C, int64_t ldc, int dtype) {
  const int64_t quads = (n + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= m * quads) return;
  const int64_t row = i / quads, col = (i - row * quads) * 4, at = row * n + col;
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (col + r < n) sum[r] += part[s * m * n + at + r];
  put_four(C, row * ldc + col, n - col, dtype, sum);
}

// Up to 16 MT rows of A.  A wave has 16 NT rows of B and every eighth block of the contraction: the waves of a workgroup share the rows of B and split the
// contraction, their sums are added through LDS in wave order.  B goes from memory to the instruction's registers (a lane: 16 bytes at two places of a
// row's block), the U blocks that a wave takes next at once; so does A, which all workgroups read and the caches hold.  DT >= 0: A comes in numbers of more
// bits, and a block of it is cast where it is used, in registers: four lanes hold a row's block, its largest number takes two exchanges.
template <int MT, int NT, int U, int DT>     // DT: type of A's numbers, -1: 8 bits with scales
__global__ void __launch_bounds__(512)
k_rows_e4m3(const E4m3Args g) {
  constexpr int WAVES = 8;
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
#pragma unroll
    for (int u = 0; u < NT; ++u) ew[u] = widen(__builtin_bit_cast(int4v, x.b[u][0]), __builtin_bit_cast(int4v, x.b[u][1]));
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      Wide8 fw;
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
        int4v f[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) f[h][i] = (int)pack_e4m3(v[h][4 * i] * inv, v[h][4 * i + 1] * inv, v[h][4 * i + 2] * inv, v[h][4 * i + 3] * inv);
        fw = widen(f[0], f[1]);
      } else {
        fw = widen(__builtin_bit_cast(int4v, x.a[t][0]), __builtin_bit_cast(int4v, x.a[t][1]));
        s = x.sa[t];
      }
      s *= x.sb;
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        const floatx4 d = mfma_wide(ew[u], fw);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][u][r] += d[r] * s;
      }
    }
  };
  const int whole = (int)(g.k / kBlock);
  for (int b = wave; b < whole; b += WAVES * U) {
    Block x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) fetch(x[i], b + WAVES * i < whole ? b + WAVES * i : b, true, 0);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (b + WAVES * i < whole) multiply(x[i]);
  }
  if (whole < g.blocks && whole % WAVES == wave) {          // the contraction's end, after the wave's other blocks
    Block x;
    fetch(x, whole, false, g.k - (int64_t)whole * kBlock - piece);
    multiply(x);
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

constexpr int64_t kFewRows = 64;      // rows up to which the read of B bounds the product
constexpr int64_t kCastRows = 16;     // rows up to which they are cast inside it

// How often the contraction is cut so that there are workgroups for every CU: only while a part keeps `least` blocks.
static int splits_for(int64_t workgroups, int blocks, int least) {
  int s = (int)(256 / workgroups);
  if (s > blocks / least) s = blocks / least;
  return s < 1 ? 1 : s > 16 ? 16 : s;
}
struct E4m3Plan {
  bool rows;               // k_rows_e4m3
  int nt, bq, splits, per_split;
};
static E4m3Plan e4m3_plan(int64_t m, int64_t n, int64_t k, bool per_row, int dtype) {
  E4m3Plan p;
  const int blocks = (int)ceil_div(k, kBlock);
  p.rows = m <= kFewRows && !per_row;
  p.nt = 1;
  p.bq = m > 128 && dtype != BRSVD_DTYPE_F32 ? 256 : 128;      // a tile of 256 x 256 has no registers left for numbers of 16 bits
  p.splits = 1;
  if (!p.rows) p.splits = splits_for(ceil_div(n, 256) * ceil_div(m, p.bq), blocks, 4);
  p.per_split = (int)ceil_div(blocks, p.splits);
  p.splits = (int)ceil_div(blocks, p.per_split);
  return p;
}
static uint64_t split_bytes(const E4m3Plan& p, int64_t m, int64_t n) { return p.splits > 1 ? (uint64_t)p.splits * m * n * 4 : 0; }

// NT: rows of A are read (and cast) once for 16 NT rows of B, as many as leave workgroups for every CU
template <int MT, int NT, int U, int DT>
static void launch_rows(const E4m3Args& g, hipStream_t stream) {
  hipLaunchKernelGGL((k_rows_e4m3<MT, NT, U, DT>), dim3((unsigned)ceil_div(g.B.n, 16 * NT)), dim3(512), 0, stream, g);
}
template <int DT>
static void launch_few(const E4m3Args& g, hipStream_t stream) {
  if (g.B.n >= 32 * 512) launch_rows<1, 4, 1, DT>(g, stream);
  else if (g.B.n >= 16 * 512) launch_rows<1, 2, 2, DT>(g, stream);
  else launch_rows<1, 1, 4, DT>(g, stream);
}
static void launch_more(const E4m3Args& g, hipStream_t stream) {
  if (g.A.n <= 32 && g.B.n >= 32 * 512) launch_rows<2, 2, 2, -1>(g, stream);
  else if (g.A.n <= 32) launch_rows<2, 1, 4, -1>(g, stream);
  else if (g.B.n >= 32 * 512) launch_rows<4, 2, 1, -1>(g, stream);
  else launch_rows<4, 1, 2, -1>(g, stream);
}
template <int NQ, bool PER_ROW, bool DIRECT, bool WIDE>
static void launch_tiles(const E4m3Args& g, hipStream_t stream) {
  hipLaunchKernelGGL((k_tiles_e4m3<8, NQ, 2, 4, PER_ROW, DIRECT, WIDE>), dim3(tile_workgroups(g.tiles_n, g.tiles_m), (unsigned)g.splits), dim3(512), 0, stream, g);
}
template <bool PER_ROW, bool DIRECT>
static void launch_tiles(const E4m3Args& g, int bq, bool wide, hipStream_t stream) {
  if (wide) launch_tiles<2, PER_ROW, DIRECT, true>(g, stream);
  else if constexpr (DIRECT) {
    if (bq == 256) launch_tiles<4, PER_ROW, DIRECT, false>(g, stream);
    else launch_tiles<2, PER_ROW, DIRECT, false>(g, stream);
  } else launch_tiles<2, PER_ROW, DIRECT, false>(g, stream);
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
  g.tiles_n = ceil_div(n, 256);
  g.tiles_m = ceil_div(m, plan.bq);
  if (plan.rows) {
    if (m > kCastRows) launch_more(g, stream);
    else if (a_type == BRSVD_DTYPE_F32) launch_few<BRSVD_DTYPE_F32>(g, stream);
    else if (a_type == BRSVD_DTYPE_BF16) launch_few<BRSVD_DTYPE_BF16>(g, stream);
    else if (a_type == BRSVD_DTYPE_F16) launch_few<BRSVD_DTYPE_F16>(g, stream);
    else launch_few<-1>(g, stream);
  } else {
    const bool direct = aligned_pieces(A, lda_bytes) && aligned_pieces(B, ldb);
    const bool wide = dtype == BRSVD_DTYPE_F32;
    if (!direct) g.tiles_m = ceil_div(m, 128);        // nor for pieces on their way through them
    if (per_row && direct) launch_tiles<true, true>(g, plan.bq, wide, stream);
    else if (per_row) launch_tiles<true, false>(g, plan.bq, wide, stream);
    else if (direct) launch_tiles<false, true>(g, plan.bq, wide, stream);
    else launch_tiles<false, false>(g, plan.bq, wide, stream);
  }
  if (split) hipLaunchKernelGGL(k_join_splits, dim3((unsigned)ceil_div(m * ceil_div(n, 4), 256)), dim3(256), 0, stream, part, plan.splits, m, n, C, ldc, dtype);
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

static bool product_type(int dtype) { return dtype == BRSVD_DTYPE_F32 || dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16; }
static bool product_sizes(int64_t m, int64_t n, int64_t k) {
  return m >= 0 && n >= 0 && k >= 0 && k < kMaxPitch && m < (int64_t)1 << 31 && n < (int64_t)1 << 31 && ceil_div(m, 128) * ceil_div(n, 16) <= kMaxGrid;
}
// The cast of the activations for a product that takes them in 8 bits: rows of whole 16 bytes, then their scales.
static uint64_t cast_pitch(int64_t k) { return (uint64_t)ceil_div(k, 16) * 16; }
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
    hipLaunchKernelGGL(k_join_splits, dim3((unsigned)ceil_div(m * ceil_div(n, 4), 256)), dim3(256), 0, s, (const float*)nullptr, 0, m, n, C, ldc, dtype);
    BRSVD_HIP_TRY(hipGetLastError());
    return BRSVD_OK;
  }
  if (!A || !B || !SA || !SB || lda < k || ldb < k || lda >= kMaxPitch || ldb >= kMaxPitch) return BRSVD_ERR_ARG;
  const E4m3Plan p = e4m3_plan(m, n, k, block_rows == 1, dtype);
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
  if (!X || !W || !SW || !Y || ldx < k || ldw < k || ldy < n || ldx * eb >= kMaxPitch * 4 || ldw >= kMaxPitch) return BRSVD_ERR_ARG;
  const E4m3Plan p = e4m3_plan(m, n, k, false, dtype);
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
