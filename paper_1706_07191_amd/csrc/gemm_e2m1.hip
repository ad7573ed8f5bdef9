// Products with a matrix W (n x k) in 4 bits with a scale for each 32 numbers of a row, and 16-bit activations:
//   Y = X W^T (X m x k),    dX = dY W (dY m x n)
// A number of W times its scale is a number of the activations' type (bf16 holds every one, fp16 those from 2^-23 to 49152), so the 16-bit matrix cores multiply
// exactly and add in fp32; Y is rounded once.  The conversion takes the scale with it: two numbers an instruction.  W is the instruction's first operand, a
// lane has four neighbouring columns of Y for one row of X.
//
// k_rows_e2m1: for few rows of X, bound by the read of W.  k_tiles_e2m1: for many, bound by the matrix cores; for Y, W's numbers are made where they are multiplied, for dX on
// their way into the tile that they are multiplied from.
#include "brsvd_steps.h"
#include "e2m1.h"

namespace brsvd {

constexpr int kChunk = 4 * kGroup;      // numbers of the contraction that a wave of k_rows_e2m1 takes at a time

struct E2m1Args {
  E2m1Operand W;
  Operand X;               // rows: m; pitch in bytes
  int64_t k;               // of the contraction
  int64_t per_split;
  void* C;                 // rows of ldc numbers of the activations' type; with splits: [split][m][cols] fp32
  int64_t ldc, cols;
  int splits;
  int64_t tiles_p, tiles_q, first;     // tiles along W and along X; column that the first tile begins with
};

// Up to 16 MT rows of X.  The eight waves of a workgroup share 16 NT rows of W and take chunks of 128 numbers of the contraction in turn; their sums are added
// through LDS in wave order.  A lane reads one group of a chunk, 16 bytes; lanes then exchange words, so that an instruction takes one
// group of all rows.  X, which all workgroups read and the caches hold, comes in pieces of 64 bytes of a row.  While a wave multiplies a chunk, those of the other seven are on their way.
// The scales of the workgroup's rows come first, whole rows of them, into LDS (where a contraction has more than there is room for, for as many chunks at a time): four bytes of 16
// rows for each chunk, as they are used, take as many lines as W itself.
// Bound by the pace of a wave's loads, the next chunk's being sent once the last one is multiplied: 1 x 4096 x 4096 5.0 us (8.9 MB; a launch is four), 1 x 20000 x 4096 10.8 us (43.5 MB,
// 4.0 TB/s), 24 x 20000 x 5000 19.5 us (58 MB fetched, 3.0 TB/s; 10.4 at a copy's rate): the 24 rows of X, which come from the caches with each 80 rows of W, are three fifths of what a wave
// loads, 12 bytes a clock and CU in all.  Scales read where they are used: 22.6 us; X kept in registers while W streams past: 27.
template <class El, int MT, int NT>
__global__ void __launch_bounds__(512)
k_rows_e2m1(const E2m1Args g) {
  struct __attribute__((packed, aligned(1))) Word { uint32_t x; };
  constexpr int WAVES = 8, kRoom = 24576, kChunks = kRoom / (64 * NT) - 1, kMine = 16 * NT / WAVES;      // bytes for scales; chunks whose scales they hold; rows of them that a wave brings
  constexpr int kParts = WAVES * MT * NT * 64 * 16;
  __shared__ __attribute__((aligned(16))) char lds[kParts > kRoom ? kParts : kRoom];
  uint32_t* scales = (uint32_t*)lds;
  auto parts = [&](int w, int i) -> floatx4& { return ((floatx4*)lds)[(w * MT * NT + i) * 64 + (threadIdx.x & 63)]; };
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 15, group = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16 * NT;
  floatx4 acc[MT][NT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u) acc[t][u] = floatx4{0.f, 0.f, 0.f, 0.f};
  const uint8_t* rw[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const int64_t n = n0 + 16 * u + row, in = n < g.W.n ? n : g.W.n - 1;
    rw[u] = g.W.base + in * g.W.ld + 16 * group;
  }
  const char* rx[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = 16 * t + row < g.X.n ? 16 * t + row : g.X.n - 1;
    rx[t] = g.X.base + m * g.X.ld + 16 * group;
  }
  struct Chunk { uint4 w[NT], x[MT][4]; };
  auto fetch = [&](Chunk& c, int at, bool whole, int64_t left) {       // left: numbers of the row from the chunk on
#pragma unroll
    for (int u = 0; u < NT; ++u) c.w[u] = group_of(rw[u] + (int64_t)at * 64, whole ? kGroup : left - kGroup * group, (int64_t)at * 64 + 16 * group);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const char* from = rx[t] + (int64_t)at * 256 + 64 * j;
        c.x[t][j] = whole ? piece_of<2>(from, 16) : piece_at_end((const uint8_t*)from, 2 * (left - kGroup * j - 8 * group), (int64_t)at * 256 + 64 * j + 16 * group);
      }
  };
  auto multiply = [&](const Chunk& c, const uint32_t* four, int pitch, uint32_t there, uint32_t missing) {       // four: scales of the chunk, of this lane's first row
    uint32_t four_of[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u) four_of[u] = four[16 * u * pitch];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const uint32_t s = (four_of[u] & there) | missing;
      uint32_t w[4] = {c.w[u].x, c.w[u].y, c.w[u].z, c.w[u].w};
      turn_groups(w);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int4v p = __builtin_bit_cast(int4v, eight_e2m1<El>(w[j], scale_e8m0(s >> (8 * j) & 255)));
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t][u] = mfma16<El>(p, __builtin_bit_cast(int4v, c.x[t][j]), acc[t][u]);
      }
      if (MT > 2) __builtin_amdgcn_sched_barrier(0);        // numbers of one tile at a time: the registers are taken
    }
  };
  // Four scales of row r of the workgroup's from chunk `at` on, behind those of the row's end any bytes; `last`: the array may end here
  auto four_scales = [&](int r, int at, bool last) {
    const int64_t n = n0 + r < g.W.n ? n0 + r : g.W.n - 1, left = last ? (g.W.n - n) * g.W.groups - 4 * (int64_t)at : 4;       // bytes that are there
    const uint8_t* from = g.W.scales + n * g.W.groups + 4 * (int64_t)at;
    if (left >= 4) return ((const Word*)from)->x;
    uint32_t x = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < left) x |= (uint32_t)from[j] << (8 * j);
    return x;
  };
  const int whole = (int)(g.k / kChunk), all = (int)((g.k + kChunk - 1) / kChunk);
  const bool last = (g.W.n - n0 - 16 * NT) * g.W.groups < 4;
  const uint32_t* four = scales;       // of this lane's first row, at chunk 0
  int pitch = 0;
  for (int first = 0; first < all; first += kChunks) {
    const int count = all - first < kChunks ? all - first : kChunks, end = first + count < whole ? first + count : whole;
    pitch = count | 1;                 // odd: rows in different banks
    if (first > 0) __syncthreads();
    for (int j = lane; j < count; j += 64) {
      uint32_t x[kMine];
      if (last) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) x[i] = four_scales(kMine * wave + i, first + j, true);
      } else {
#pragma unroll
        for (int i = 0; i < kMine; ++i) x[i] = four_scales(kMine * wave + i, first + j, false);
      }
#pragma unroll
      for (int i = 0; i < kMine; ++i) scales[(kMine * wave + i) * pitch + j] = x[i];
    }
    Chunk c;
    int at = first + wave;
    if (at < end) fetch(c, at, true, 0);
    meet_but<63>();              // what has been fetched may be on its way
    four = scales + row * pitch - first;
    for (; at < end; at += WAVES) {
      multiply(c, four + at, pitch, ~0u, 0);
      if (at + WAVES < end) fetch(c, at + WAVES, true, 0);
    }
  }
  if (whole < all && whole % WAVES == wave) {          // the contraction's end, after the wave's other chunks
    const int64_t left = g.k - (int64_t)whole * kChunk;
    const uint32_t there = left > 3 * kGroup ? ~0u : left > 2 * kGroup ? 0xffffffu : left > kGroup ? 0xffffu : 0xffu;      // scales of the row; other groups are zeros, times 1
    Chunk c;
    fetch(c, whole, false, left);
    multiply(c, four + whole, pitch, there, 0x7f7f7f7fu & ~there);
  }
  __syncthreads();               // the scales have been read
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u) parts(wave, t * NT + u) = acc[t][u];
  __syncthreads();
  for (int i = wave; i < MT * NT; i += WAVES) {
    floatx4 sum = parts(0, i);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += parts(w, i);
    const int64_t m = 16 * (i / NT) + row, n = n0 + 16 * (i % NT) + 4 * group;
    if (m < g.X.n && n < g.W.n) put_four(g.C, m * g.ldc + n, g.W.n - n, __is_same(El, Bf16) ? BRSVD_DTYPE_BF16 : BRSVD_DTYPE_F16, sum);
  }
}

// 256 columns of the result x 64 NQ rows.  O = kRows: Y, W's rows hold the contraction.  kCols: dX, the contraction runs down W's rows.  Bound by the matrix cores and what feeds
// them, busy for 61 and 51 % of the cycles: 4001 x 4096 x 6000 165 us and 194 back (two launches, 1.5 rounds of tiles), 8192 in all three 788 and 846 (1.40 and 1.30 Pflop/s;
// 16-bit weights in the library's product 681 and 777).
template <class El, int NQ, Order O>
__global__ void __launch_bounds__(512, 2)
k_tiles_e2m1(const E2m1Args g) {
  using T = E2m1Product<El, NQ, O>;
  static_assert(T::kLds >= T::BQ * 512, "put_tile16");
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_p, g.tiles_q * g.splits, 8, &tp, &tq)) return;
  const int split = (int)((unsigned)tq / (unsigned)g.tiles_q);
  tq -= split * g.tiles_q;
  const int64_t p0 = g.first + tp * T::BP, q0 = tq * T::BQ, k0 = split * g.per_split, k1 = k0 + g.per_split < g.k ? k0 + g.per_split : g.k;
  floatx4 acc[T::NP][NQ];
  T::run(acc, g.W, p0, g.X, q0, k0, k1, lds);
  if (g.splits > 1) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = wave % T::WP, wq = wave / T::WP;
    float* C = (float*)g.C + (int64_t)split * g.X.n * g.cols;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t m = q0 + 16 * (wq * NQ + q) + (lane & 15);
      if (m >= g.X.n) continue;
#pragma unroll
      for (int p = 0; p < T::NP; ++p) {
        const int64_t n = p0 + 16 * (wp * T::NP + p) + 4 * (lane >> 4);
        if (n < g.cols) put_four(C, m * g.cols + n, g.cols - n, BRSVD_DTYPE_F32, acc[p][q]);
      }
    }
  } else {
    put_tile16<NQ>(acc, lds, (uint16_t*)g.C + q0 * g.ldc + p0, g.ldc, g.X.n - q0, g.cols - p0, [](float x, int) { return to16<El>(x); });
  }
}

__global__ void __launch_bounds__(256)
k_align_rows(const char* __restrict__ from, int64_t ld, int64_t rows, int64_t bytes, char* __restrict__ to, int64_t pitch, unsigned first_wg) {
  const int64_t pieces = (bytes + 15) / 16, per = (pieces + 255) / 256, wg = (int64_t)first_wg + blockIdx.x, r = wg / per, c = (wg - r * per) * 256 + threadIdx.x;
  if (r < rows && c < pieces) *(uint4*)(to + r * pitch + 16 * c) = piece_of<1>(from + r * ld + 16 * c, bytes - 16 * c);
}
void align_rows(const void* from, int64_t ld, int64_t rows, int64_t bytes, void* to, int64_t pitch, hipStream_t stream) {
  in_launches(rows * ceil_div(ceil_div(bytes, 16), 256), 256, [&](unsigned first, dim3 grid) {
    hipLaunchKernelGGL(k_align_rows, grid, dim3(256), 0, stream, (const char*)from, ld, rows, bytes, (char*)to, pitch, first);
  });
}

static uint64_t whole256(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// Few rows of X: by the 16 rows of W in a wave (NT of them).  A round of 256 workgroups takes some time for what they read of W and of X, and all of them a start, which rounds share; with NT
// for which the workgroups fill rounds there is least to do.  In units of 0.08 us at 4096 columns: 16 x 12000 x 4096 10.2 us with three (250 workgroups), 14.1 with two (375), 16.3 with
// one (750); 16 x 20000 x 4096 12.7, 16.7, 19.6 and 24.8 with five, three, two and one; 1 x 20000 x 4096 10.8 and 12.6 with five and one.  Of 60 sizes the best is met or missed by 8 % at most.
static int rows_in_wave(int64_t m, int64_t n) {
  int best = 1;
  int64_t least = 0;
  for (int nt : {1, 2, 3, 5}) {
    const int64_t cost = ceil_div(ceil_div(n, 16 * nt), 256) * (16 + 10 * nt + 2 * m) + 10 * nt;
    if (nt == 1 || cost < least) least = cost, best = nt;
  }
  return best;
}
// 16-row tiles of X
static int row_tiles(int64_t m) { return (int)ceil_div(m, 16); }
struct E2m1Plan {
  bool rows;                    // k_rows_e2m1
  TilePlan tiles;
  uint64_t x, w, bytes;         // scratch: the parts at 0, X and W in aligned rows where they are laid out anew, all
};
// m rows of X, W n x k; aligned: rows of both begin at 16-byte addresses.
static E2m1Plan e2m1_plan(int64_t m, int64_t n, int64_t k, bool aligned, bool backward) {
  static constexpr int kForward[3] = {62, 82, 150}, kBackward[3] = {85, 110, 165};      // 1/100 us a step, see tile_plan
  const int64_t cols = backward ? k : n, in = backward ? n : k;
  E2m1Plan p;
  p.tiles = tile_plan(ceil_div(cols, 256), m, ceil_div(in, 64), 1, m * cols, backward ? kBackward : kForward);
  // Above 16 rows tiles are ahead where the contraction is long and W has few rows: 48 x 4096 x 10240 21 us, 31 in rows; the other way round 48 x 12000 x 4096 22 and 18.  Eight chunks of a
  // wave each take 0.35 us for 16 rows of W and 0.05 for a row of X.
  const int nt = rows_in_wave(m, n);
  const double rows_us = 3.5 + (double)(ceil_div(ceil_div(k, kChunk), 8) * ceil_div(ceil_div(n, 16 * nt), 256)) * (0.35 * nt + 0.05 * m);
  p.rows = !backward && (m <= 16 || (m <= 64 && rows_us <= p.tiles.us));
  if (p.rows) p.tiles.splits = 1;
  const bool laid = !p.rows && !aligned;
  p.x = p.tiles.splits > 1 ? whole256((uint64_t)p.tiles.splits * m * cols * 4) : 0;
  p.w = p.x + (laid ? whole256((uint64_t)m * line_pitch(2 * in)) : 0);
  p.bytes = p.w + (laid ? whole256((uint64_t)n * line_pitch((k + 1) / 2)) : 0);
  return p;
}

template <class El, int MT, int NT>
static void launch_rows(const E2m1Args& g, hipStream_t stream) {
  hipLaunchKernelGGL((k_rows_e2m1<El, MT, NT>), dim3((unsigned)ceil_div(g.W.n, 16 * NT)), dim3(512), 0, stream, g);
}
template <class El, int MT>
static void launch_rows(const E2m1Args& g, hipStream_t stream) {
  switch (rows_in_wave(g.X.n, g.W.n)) {
    case 1: return launch_rows<El, MT, 1>(g, stream);
    case 2: return launch_rows<El, MT, 2>(g, stream);
    case 3: return launch_rows<El, MT, 3>(g, stream);
    default: return launch_rows<El, MT, 5>(g, stream);
  }
}
template <class El, int NQ, Order O>
static void launch_tiles(E2m1Args g, hipStream_t stream) {
  g.tiles_q = ceil_div(g.X.n, 64 * NQ);
  hipLaunchKernelGGL((k_tiles_e2m1<El, NQ, O>), dim3(tile_workgroups(g.tiles_p, g.tiles_q * g.splits)), dim3(512), 0, stream, g);
}
template <class El, Order O>
static void launch_tiles(E2m1Args g, const TilePlan& t, hipStream_t stream) {
  g.first = 0;
  g.tiles_p = t.large;
  if (t.large > 0) launch_tiles<El, 4, O>(g, stream);
  g.first = 256 * t.large;
  g.tiles_p = t.tiles - t.large;
  if (g.tiles_p > 0) t.nq == 1 ? launch_tiles<El, 1, O>(g, stream) : launch_tiles<El, 2, O>(g, stream);
}

template <class El>
static int product_e2m1(E2m1Args g, const E2m1Plan& p, int64_t wrows, int64_t wbytes, bool backward, char* scratch, int dtype, hipStream_t stream) {
  void* C = g.C;
  const int64_t ldc = g.ldc;
  if (p.rows) {
    switch (row_tiles(g.X.n)) {
      case 1: launch_rows<El, 1>(g, stream); break;
      case 2: launch_rows<El, 2>(g, stream); break;
      case 3: launch_rows<El, 3>(g, stream); break;
      default: launch_rows<El, 4>(g, stream);
    }
  } else {
    if (!aligned_pieces(g.X.base, g.X.ld)) {
      const int64_t pitch = line_pitch(2 * g.k);
      align_rows(g.X.base, g.X.ld, g.X.n, 2 * g.k, scratch + p.x, pitch, stream);
      g.X.base = scratch + p.x;
      g.X.ld = pitch;
    }
    if (!aligned_pieces(g.W.base, g.W.ld)) {
      const int64_t pitch = line_pitch(wbytes);
      align_rows(g.W.base, g.W.ld, wrows, wbytes, scratch + p.w, pitch, stream);
      g.W.base = (const uint8_t*)scratch + p.w;
      g.W.ld = pitch;
    }
    g.splits = p.tiles.splits;
    g.per_split = p.tiles.per_split;
    if (g.splits > 1) g.C = scratch;
    backward ? launch_tiles<El, kCols>(g, p.tiles, stream) : launch_tiles<El, kRows>(g, p.tiles, stream);
    if (g.splits > 1) join_splits((const float*)scratch, g.splits, g.X.n, g.cols, C, ldc, dtype, stream);
  }
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

static bool half_type(int dtype) { return dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16; }
// A tile's rows are addressed with 32 bits, and launches have their workgroups.
static bool e2m1_sizes(int64_t m, int64_t n, int64_t k, bool backward) {
  if (m < 0 || n < 0 || k < 0 || m >= (int64_t)1 << 31 || n >= (int64_t)1 << 31 || k >= kMaxPitch / 2 || (backward && n >= kMaxPitch / 2)) return false;
  const int64_t cols = backward ? k : n;
  return tiles_fit(ceil_div(cols, 256), ceil_div(m, 64), 512) && ceil_div(n, 16) <= launch_workgroups(512) && m <= (int64_t)UINT32_MAX / ceil_div((backward ? n : k) + 1, 2048) &&
         n <= (int64_t)UINT32_MAX / ceil_div(k + 1, 8192);
}
static int check_e2m1(const void* X, int64_t ldx, int64_t in, int dtype, const uint8_t* W, int64_t ldw, const uint8_t* S, int64_t m, int64_t n, int64_t k, const void* Y,
                      int64_t ldy, int64_t out, bool backward) {
  if (!half_type(dtype) || !e2m1_sizes(m, n, k, backward)) return BRSVD_ERR_ARG;
  if (m == 0 || out == 0) return BRSVD_OK;
  if (!Y || ldy < out || ldy >= (int64_t)1 << 40) return BRSVD_ERR_ARG;
  if (in > 0 && (!X || !W || !S || ldx < in || ldx >= kMaxPitch / 2 || ldw < (k + 1) / 2 || ldw >= kMaxPitch / 2)) return BRSVD_ERR_ARG;
  return BRSVD_OK;
}

static int call_e2m1(const void* X, int64_t ldx, int64_t in, int dtype, const uint8_t* W, int64_t ldw, const uint8_t* S, int64_t m, int64_t n, int64_t k, void* Y,
                     int64_t ldy, int64_t out, bool backward, void* scratch, uint64_t scratch_bytes, hipStream_t s) {
  BRSVD_TRY(check_e2m1(X, ldx, in, dtype, W, ldw, S, m, n, k, Y, ldy, out, backward));
  if (m == 0 || out == 0) return BRSVD_OK;
  if (in == 0) {               // an empty sum
    join_splits(nullptr, 0, m, out, Y, ldy, dtype, s);
    BRSVD_HIP_TRY(hipGetLastError());
    return BRSVD_OK;
  }
  const bool aligned = aligned_pieces(X, 2 * ldx) && aligned_pieces(W, ldw);
  const E2m1Plan p = e2m1_plan(m, n, k, aligned, backward);
  if (p.bytes && (!scratch || (uintptr_t)scratch % 256)) return BRSVD_ERR_ARG;
  if (scratch_bytes < p.bytes) return BRSVD_ERR_BUDGET;
  E2m1Args g = {};
  g.W = E2m1Operand{W, ldw, out, S, ceil_div(k, kGroup)};
  g.X = Operand{(const char*)X, 2 * ldx, m};
  g.k = in;
  g.C = Y;
  g.ldc = ldy;
  g.cols = out;
  return dtype == BRSVD_DTYPE_BF16 ? product_e2m1<Bf16>(g, p, n, (k + 1) / 2, backward, (char*)scratch, dtype, s)
                                   : product_e2m1<Fp16>(g, p, n, (k + 1) / 2, backward, (char*)scratch, dtype, s);
}

}  // namespace brsvd

using namespace brsvd;

extern "C" uint64_t brsvd_linear_e2m1_scratch_bytes(int64_t m, int64_t n, int64_t k, int32_t aligned, int32_t backward) {
  if (!e2m1_sizes(m, n, k, backward != 0) || m == 0 || n == 0 || k == 0) return 0;
  return e2m1_plan(m, n, k, aligned != 0, backward != 0).bytes;
}

extern "C" int brsvd_linear_e2m1(const void* X, int64_t ldx, int32_t dtype, const uint8_t* W, int64_t ldw, const uint8_t* SW, int64_t m, int64_t n, int64_t k, void* Y,
                                 int64_t ldy, void* scratch, uint64_t scratch_bytes, void* stream) {
  return call_e2m1(X, ldx, k, dtype, W, ldw, SW, m, n, k, Y, ldy, n, false, scratch, scratch_bytes, (hipStream_t)stream);
}

extern "C" int brsvd_linear_e2m1_backward(const void* dY, int64_t lddy, int32_t dtype, const uint8_t* W, int64_t ldw, const uint8_t* SW, int64_t m, int64_t n, int64_t k,
                                          void* dX, int64_t lddx, void* scratch, uint64_t scratch_bytes, void* stream) {
  return call_e2m1(dY, lddy, n, dtype, W, ldw, SW, m, n, k, dX, lddx, k, true, scratch, scratch_bytes, (hipStream_t)stream);
}

extern "C" int brsvd_linear_e2m1_plan(int64_t m, int64_t n, int64_t k, int32_t backward, int32_t* out8) {
  if (!out8 || !e2m1_sizes(m, n, k, backward != 0) || m == 0 || n == 0 || k == 0) return BRSVD_ERR_ARG;
  const E2m1Plan p = e2m1_plan(m, n, k, true, backward != 0);
  p.rows ? describe_rows(row_tiles(m), rows_in_wave(m, n), out8) : describe_plan(p.tiles, out8);
  return BRSVD_OK;
}
