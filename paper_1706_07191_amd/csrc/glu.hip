// The first half of a gated feed-forward block and its gradients:
//   G = X Wg^T,  U = X Wu^T (X tokens x dim; Wg, Wu width x dim),   H = a(G) U          a: silu, gelu or gelu by tanh
//   dG = dH U a'(G),  dU = dH a(G),   dX = dG Wg + dU Wu,   dWg = dG^T X,  dWu = dU^T X
// Forward: one kernel.  A tile has 128 columns of G and the same of U, 64 of each in a wave, so that a lane holds both numbers of a product; sums are fp32 until H (and G, U
// where they are kept for the backward pass) is rounded.  Backward: dG and dU are formed once, in 16 bits, and multiplied: dX is one sum over both.
#include "brsvd_steps.h"
#include "tile.h"

namespace brsvd {

constexpr int kTileP = 256, kTileThreads = 512;

// ---- activations ----------------------------------------------------------------------------------------------------

struct Slope {
  float value, slope;
};
// a(g) = g p(g) and its derivative.  Exponentials and reciprocals are the hardware's, good to 2^-22, where results keep eleven bits at most.
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * x)); }
constexpr float kTanhA = 1.59576912f /* 2 sqrt(2 / pi) */, kTanhB = 0.044715f;
// Beyond 100 either way p is 0 or 1 in fp32, beyond 30 where its exponent is a square or a cube: g is taken as that there, so that powers stay finite and an infinity, which G may
// be once it is rounded, has its limit.  NaN stays NaN.
__device__ __forceinline__ float within(float g, float most) { return fabsf(g) > most ? copysignf(most, g) : g; }
__device__ __forceinline__ float above(float g) { return g < -100.f ? -100.f : g; }
__device__ __forceinline__ float activation(float g, int act) {
  if (act == BRSVD_ACT_SILU) return above(g) * logistic(g);
  if (act == BRSVD_ACT_GELU) return above(g) * (0.5f * erfcf(-0.707106781f * g));
  const float c = within(g, 30.f);
  return above(g) * logistic(kTanhA * (c + kTanhB * c * c * c));
}
__device__ __forceinline__ Slope activation_slope(float g, int act) {
  if (act == BRSVD_ACT_SILU) {
    const float p = logistic(g);
    return Slope{above(g) * p, p * (1.f + within(g, 100.f) * (1.f - p))};
  }
  const float c = within(g, 30.f);
  if (act == BRSVD_ACT_GELU) {
    const float p = 0.5f * erfcf(-0.707106781f * g);
    return Slope{above(g) * p, p + c * (0.398942280f * __builtin_amdgcn_exp2f(-0.721347520f * c * c))};
  }
  const float p = logistic(kTanhA * (c + kTanhB * c * c * c));
  return Slope{above(g) * p, p * (1.f + c * (1.f - p) * (kTanhA * (1.f + 3.f * kTanhB * c * c)))};
}

// ---- forward --------------------------------------------------------------------------------------------------------

struct PairOperand {
  const char *g, *u;
  int64_t ldg, ldu;     // bytes
  int64_t n;            // width
};

// Fills P's tile from rows of both matrices: 64 of Wg, 64 of Wu, the next 64 of Wg and of Wu.
struct PairStager {
  static constexpr int kLoads = 4;
  using Source = PairOperand;
  uint32_t off_g[2], off_u[2];
  const char *at_g, *at_u;      // of this step, the same in all lanes

  __device__ __forceinline__ void init(const PairOperand& op, int64_t first, int64_t k0, int tid) {
    const int64_t f0 = first / 2, left = op.n - f0;
    at_g = (const char*)scalar((int64_t)(op.g + f0 * op.ldg + 2 * k0));
    at_u = (const char*)scalar((int64_t)(op.u + f0 * op.ldu + 2 * k0));
    const int row = tid >> 3, src = 16 * ((tid ^ row) & 7);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = 64 * i + row < left ? 64 * i + row : left - 1;
      off_g[i] = (uint32_t)(r * op.ldg + src);
      off_u[i] = (uint32_t)(r * op.ldu + src);
    }
  }
  __device__ __forceinline__ bool plain(int64_t left) const { return left >= 64; }
  __device__ __forceinline__ void load_part(char* tile, int wave, int i) const {
    load_to_lds(lds_address(tile) + 16 * (i * kTileThreads + 64 * wave), (const char*)scalar((int64_t)(i & 1 ? at_u : at_g)), i & 1 ? off_u[i >> 1] : off_g[i >> 1]);
  }
  __device__ __forceinline__ void next() {
    at_g += kStepBytes;
    at_u += kStepBytes;
  }
  __device__ __forceinline__ void load(char* tile, int tid, int wave, int64_t left) {
    const int there = left >= 64 ? 16 : 2 * (int)left - 16 * ((tid ^ (tid >> 3)) & 7);
    if (there >= 16) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load_part(tile, wave, i);
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        *(uint4*)(tile + 16 * (i * kTileThreads + tid)) =
            there > 0 ? piece_of<2>(i & 1 ? at_u + off_u[i >> 1] : at_g + off_g[i >> 1], there) : make_uint4(0u, 0u, 0u, 0u);
    }
    next();
  }
  __device__ __forceinline__ void store(char*, int) {}
};

struct GluArgs {
  PairOperand W;
  Operand X;
  int64_t dim, per_split;
  int splits, act;
  uint16_t *H, *G, *U;       // G, U: null where they are not kept
  int64_t ldh, ldg, ldu;
  float* part;               // with splits: [split][token][2 width], G then U
  int64_t tiles_p, tiles_q, first;
};

// 128 columns x 64 NQ rows of 16-bit numbers to memory through LDS, a row's 128 as one piece: put_tile16 for tiles whose waves have four tile rows of the result.
template <int NQ, class Number>
__device__ __forceinline__ void put_pair16(char* lds, uint16_t* out, int64_t ldo, int64_t rows, int64_t cols, Number number) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wp = wave % 2, wq = wave / 2;
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      uint32_t h[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) h[r] = number(p, q, r);
      const int j = 16 * (wq * NQ + q) + (lane & 15), u = 4 * (4 * wp + p) + (lane >> 4);
      *(uint2*)(lds + j * 256 + 8 * (u ^ (4 * (lane & 7)))) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    }
  __syncthreads();
  const int piece = tid & 15;
  const int64_t left = cols - 8 * piece;
#pragma unroll
  for (int i = 0; i < 2 * NQ; ++i) {
    const int j = 32 * i + (tid >> 4);
    const uint4 v = *(const uint4*)(lds + j * 256 + 8 * ((2 * piece) ^ (4 * (j & 7))));
    if (j >= rows) continue;
    uint16_t* at = out + j * ldo + 8 * piece;
    if (left >= 8) *(Piece*)at = Piece{{v.x, v.y, v.z, v.w}};
    else {
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < left) at[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    }
  }
}

// Bound by the matrix cores, busy for 61 % of the cycles, and by a tile's start and end, 20 us of 115: 4001 x 12000 x 4096 with G and U kept 640 to 690 us (1.14 to 1.23 Pflop/s), of
// which the write of the results takes 55.  Stores are counted in order with the loads behind them, so that a next tile begun before this one's end would wait for them all the same.
template <class El, int NQ>
__global__ void __launch_bounds__(kTileThreads, 2)
k_glu_tiles(const GluArgs g) {
  using T = TileProduct<El, NQ, kRows, kRows, true, PairStager>;
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_p, g.tiles_q * g.splits, 8, &tp, &tq)) return;
  const int split = (int)((unsigned)tq / (unsigned)g.tiles_q);
  tq -= split * g.tiles_q;
  const int64_t f0 = g.first + 128 * tp, t0 = tq * T::BQ, k0 = split * g.per_split, k1 = k0 + g.per_split < g.dim ? k0 + g.per_split : g.dim;
  floatx4 acc[T::NP][NQ];
  T::run(acc, g.W, 2 * f0, g.X, t0, k0, k1, lds);
  if (g.splits > 1) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = wave % 2, wq = wave / 2;
    const int64_t width = g.W.n;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t t = t0 + 16 * (wq * NQ + q) + (lane & 15);
      if (t >= g.X.n) continue;
      const int64_t row = ((int64_t)split * g.X.n + t) * 2 * width;
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        const int64_t f = f0 + 64 * wp + 16 * (p & 3) + 4 * (lane >> 4);
        if (f < width) put_four(g.part, row + (p < 4 ? 0 : width) + f, width - f, BRSVD_DTYPE_F32, acc[p][q]);
      }
    }
    return;
  }
  const int64_t rows = g.X.n - t0, cols = g.W.n - f0;
  if (g.G) {
    put_pair16<NQ>(lds, g.G + t0 * g.ldg + f0, g.ldg, rows, cols, [&](int p, int q, int r) { return to16<El>(acc[p][q][r]); });
    __syncthreads();
    put_pair16<NQ>(lds, g.U + t0 * g.ldu + f0, g.ldu, rows, cols, [&](int p, int q, int r) { return to16<El>(acc[p + 4][q][r]); });
    __syncthreads();
  }
  put_pair16<NQ>(lds, g.H + t0 * g.ldh + f0, g.ldh, rows, cols, [&](int p, int q, int r) { return to16<El>(activation(acc[p][q][r], g.act) * acc[p + 4][q][r]); });
}

// The results of a contraction that was cut, a thread four neighbouring columns
template <class El>
__global__ void __launch_bounds__(256)
k_glu_join(const GluArgs g, Divisor quads) {
  const int64_t width = g.W.n, tokens = g.X.n;
  uint32_t c;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = divide((uint32_t)i, quads, &c), f = 4 * (int64_t)c;
  if (t >= tokens) return;
  const float* row = g.part + t * 2 * width + f;
  const floatx4 a = sum_of_parts(row, 2 * tokens * width, g.splits, width - f), b = sum_of_parts(row + width, 2 * tokens * width, g.splits, width - f);
  floatx4 h;
#pragma unroll
  for (int r = 0; r < 4; ++r) h[r] = activation(a[r], g.act) * b[r];
  constexpr int dtype = __is_same(El, Bf16) ? BRSVD_DTYPE_BF16 : BRSVD_DTYPE_F16;
  put_four(g.H, t * g.ldh + f, width - f, dtype, h);
  if (g.G) {
    put_four(g.G, t * g.ldg + f, width - f, dtype, a);
    put_four(g.U, t * g.ldu + f, width - f, dtype, b);
  }
}

// Up to 16 MT tokens: bound by the read of Wg and Wu.  A workgroup has 16 rows of both; its waves take chunks of 64 numbers of the contraction in turn, the U that come next
// on their way from memory to registers, and their sums are added through LDS in wave order.  Rows at any alignment.  One token, 12000 x 4096: 34 us (197 MB, 5.8 TB/s).
template <class El, int MT, int U, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
k_glu_rows(const GluArgs g) {
  __shared__ floatx4 parts[WAVES][2 * MT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 15, piece = 16 * (lane >> 4);
  const int64_t f0 = (int64_t)blockIdx.x * 16, n = f0 + row < g.W.n ? f0 + row : g.W.n - 1;
  const char *rw[2] = {g.W.g + n * g.W.ldg + piece, g.W.u + n * g.W.ldu + piece}, *rx[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = 16 * t + row < g.X.n ? 16 * t + row : g.X.n - 1;
    rx[t] = g.X.base + m * g.X.ld + piece;
  }
  floatx4 acc[MT][2];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t][0] = acc[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
  struct Chunk { uint4 w[2][2], x[MT][2]; };
  auto fetch = [&](Chunk& c, int at, bool whole, int64_t left) {            // left: bytes of the row from this lane's first piece on
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int u = 0; u < 2; ++u) c.w[u][h] = piece_of<2>(rw[u] + (int64_t)at * kStepBytes + 64 * h, whole ? 16 : left - 64 * h);
#pragma unroll
      for (int t = 0; t < MT; ++t) c.x[t][h] = piece_of<2>(rx[t] + (int64_t)at * kStepBytes + 64 * h, whole ? 16 : left - 64 * h);
    }
  };
  auto multiply = [&](const Chunk& c) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) acc[t][u] = mfma16<El>(__builtin_bit_cast(int4v, c.w[u][h]), __builtin_bit_cast(int4v, c.x[t][h]), acc[t][u]);
  };
  const int whole = (int)(g.dim / 64);
  Chunk c[U];
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (wave + WAVES * i < whole) fetch(c[i], wave + WAVES * i, true, 0);
  for (int b = wave; b < whole; b += WAVES * U) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (b + WAVES * i < whole) multiply(c[i]);
      if (b + WAVES * (i + U) < whole) fetch(c[i], b + WAVES * (i + U), true, 0);
    }
  }
  if (g.dim % 64 != 0 && whole % WAVES == wave) {          // the contraction's end, after the wave's other chunks
    fetch(c[0], whole, false, 2 * (g.dim - (int64_t)whole * 64) - piece);
    multiply(c[0]);
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < 2; ++u) parts[wave][2 * t + u][lane] = acc[t][u];
  __syncthreads();
  for (int t = wave; t < MT; t += WAVES) {
    floatx4 a = parts[0][2 * t][lane], b = parts[0][2 * t + 1][lane], h;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      a += parts[w][2 * t][lane];
      b += parts[w][2 * t + 1][lane];
    }
    const int64_t m = 16 * t + row, f = f0 + 4 * (lane >> 4), left = g.W.n - f;
    if (m >= g.X.n || left <= 0) continue;
    constexpr int dtype = __is_same(El, Bf16) ? BRSVD_DTYPE_BF16 : BRSVD_DTYPE_F16;
#pragma unroll
    for (int r = 0; r < 4; ++r) h[r] = activation(a[r], g.act) * b[r];
    put_four(g.H, m * g.ldh + f, left, dtype, h);
    if (g.G) {
      put_four(g.G, m * g.ldg + f, left, dtype, a);
      put_four(g.U, m * g.ldu + f, left, dtype, b);
    }
  }
}

// ---- backward -------------------------------------------------------------------------------------------------------

struct SlopeArgs {
  const char *G, *U, *dH;
  int64_t ldg, ldu, ldh;       // bytes
  int64_t tokens, width;
  Divisor pieces;
  int act;
  char* dG;                    // rows of dG and, `second` bytes behind, dU; zeros behind both
  int64_t second, pitch;       // bytes
  float* tops;                 // fp16: the largest |dG|, |dU| that each of kTops workgroups met
  float* down;                 // fp16: what the results are multiplied by
};
constexpr int kTops = 1024;

// Eight numbers of dG and of dU
template <class El>
__device__ __forceinline__ void slopes_of(const SlopeArgs& g, int64_t t, int64_t f, float (&a)[8], float (&b)[8]) {
  const int64_t left = 2 * (g.width - f);
  const uint4 x = piece_of<2>(g.G + t * g.ldg + 2 * f, left), y = piece_of<2>(g.U + t * g.ldu + 2 * f, left), z = piece_of<2>(g.dH + t * g.ldh + 2 * f, left);
  const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w}, zs[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int s = 16 * (i & 1);
    const Slope v = activation_slope(from16<El>((uint16_t)(xs[i / 2] >> s)), g.act);
    const float d = from16<El>((uint16_t)(zs[i / 2] >> s));
    a[i] = d * from16<El>((uint16_t)(ys[i / 2] >> s)) * v.slope;
    b[i] = d * v.value;
  }
}

__device__ __forceinline__ float max_of_workgroup(float x, float* red) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x = fmaxf(x, __shfl_xor(x, s));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// fp16: numbers of gradients may lie below its range.  dG and dU are multiplied by one power of two for which the largest is 2^14 to 2^15, and the results by its
// reciprocal: an entry is off by up to 2^-39 of the largest beside its rounding to eleven bits.  bf16 needs none.  999 x 5000 9 us, with the numbers still in the caches afterwards.
__global__ void __launch_bounds__(256)
k_glu_tops(const SlopeArgs g) {
  __shared__ float red[4];
  float top = 0.f;
  uint32_t c, dc;
  const uint32_t dt = divide(kTops * 256, g.pieces, &dc);
  for (int64_t t = divide(blockIdx.x * 256 + threadIdx.x, g.pieces, &c); t < g.tokens;) {
    float a[8], b[8];
    slopes_of<Fp16>(g, t, 8 * (int64_t)c, a, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float m = fabsf(a[j]), n = fabsf(b[j]);
      if (m <= 3.402823466e38f) top = fmaxf(top, m);
      if (n <= 3.402823466e38f) top = fmaxf(top, n);
    }
    t += dt;
    c += dc;
    if (c >= g.pieces.d) c -= g.pieces.d, ++t;
  }
  top = max_of_workgroup(top, red);
  if (threadIdx.x == 0) g.tops[blockIdx.x] = top;
}

// dG and dU, so that the activation's exponentials are taken once and not for every tile of the two products.  Bound by memory: 8192 x 16384 223 us (1.34 GB, 6.0 TB/s).
// They are rounded to 16 bits, as the matrix cores take them and as G, U and dH came: gradients are then off by two roundings for one, sqrt 2 in the mean (bf16 0.0024 from 64 bits for
// 0.0017, fp16 2.9e-4 for 2.1e-4).  Two numbers of 16 bits each would leave one rounding and double the products, 3200 of 3430 us at 8192 x 16384 x 4096.
template <class El>
__global__ void __launch_bounds__(256)
k_glu_slopes(const SlopeArgs g, int64_t first, int64_t rows) {
  __shared__ float red[4];
  float up = 1.f;
  if (__is_same(El, Fp16)) {
    const floatx4 v = *(const floatx4*)(g.tops + 4 * threadIdx.x);
    const float top = max_of_workgroup(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), red);
    int e = top > 0.f ? 14 - ((int)(__float_as_uint(top) >> 23) - 127) : 0;
    e = e > 120 ? 120 : e < -120 ? -120 : e;
    up = __uint_as_float((uint32_t)(e + 127) << 23);
    if (first == 0 && blockIdx.x == 0 && threadIdx.x == 0) *g.down = __uint_as_float((uint32_t)(127 - e) << 23);
  }
  uint32_t c;
  const int64_t t = divide(blockIdx.x * 256 + threadIdx.x, g.pieces, &c);
  if (t >= rows) return;
  float a[8], b[8];
  slopes_of<El>(g, first + t, 8 * (int64_t)c, a, b);
  uint32_t x[4], y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = to16<El>(a[2 * i] * up) | (uint32_t)to16<El>(a[2 * i + 1] * up) << 16;
    y[i] = to16<El>(b[2 * i] * up) | (uint32_t)to16<El>(b[2 * i + 1] * up) << 16;
  }
  const int64_t at = (first + t) * g.pitch + 16 * (int64_t)c;
  *(uint4*)(g.dG + at) = make_uint4(x[0], x[1], x[2], x[3]);
  *(uint4*)(g.dG + g.second + at) = make_uint4(y[0], y[1], y[2], y[3]);
}

// Two matrices with rows of one pitch, one below the other, as an operand whose rows the contraction runs down: `padded` numbers of it in each, whole steps, of which
// `rows` are there.
struct StackOperand {
  const char *top, *bottom;
  int64_t ld;                // bytes
  int64_t n;                 // columns
  int64_t rows, padded;
  int64_t end;               // of the part of the contraction that is multiplied
};
template <class El>
struct StackStager {
  using Source = StackOperand;
  using One = Stager<El, kCols, 256, 512, true>;
  static constexpr int kLoads = One::kLoads;
  One one;
  const char* bottom;
  int rows, padded, end, from;      // from: the number of the contraction that the next step begins with

  __device__ __forceinline__ void init(const StackOperand& op, int64_t first, int64_t k0, int tid) {
    rows = (int)op.rows;
    padded = (int)op.padded;
    end = (int)op.end;
    from = __builtin_amdgcn_readfirstlane((int)k0);
    bottom = (const char*)scalar((int64_t)(op.bottom + 2 * first));
    one.init(Operand{k0 < padded ? op.top : op.bottom, op.ld, op.n}, first, k0 < padded ? k0 : k0 - padded, tid);
  }
  // Rows that are there of the step with so much of the contraction left
  __device__ __forceinline__ int there(int64_t left) const {
    const int at = end - (int)left;
    return rows - (at < padded ? at : at - padded);
  }
  __device__ __forceinline__ void turn() {
    from += 64;
    if (from == padded) one.at = bottom;
  }
  __device__ __forceinline__ bool plain(int64_t left) const { return there(left) >= 64 && !one.ragged; }
  __device__ __forceinline__ void load_part(char* tile, int wave, int i) const { one.load_part(tile, wave, i); }
  __device__ __forceinline__ void next() {
    one.next();
    turn();
  }
  __device__ __forceinline__ void load(char* tile, int tid, int wave, int64_t left) {
    one.load(tile, tid, wave, there(left));
    turn();
  }
  __device__ __forceinline__ void store(char*, int) {}
};

struct GradArgs {
  StackOperand W;             // dX: P
  Operand X, D[2];            // dX: Q = D[0], rows of dG and dU;  dW: P = X, Q = dG or dU
  int64_t k, per_split;
  int splits;
  const float* down;          // null: 1
  uint16_t* out[2];
  int64_t ldo[2], rows, cols;
  float* part;                // with splits: [split][matrix][row][col]
  int64_t tiles_p, tiles_q, first;
};

template <class T, class El>
__device__ __forceinline__ void leave_gradient(const GradArgs& g, floatx4 (&acc)[T::NP][T::NQ], char* lds, int split, int which, int matrices, int64_t p0, int64_t q0) {
  constexpr int NQ = T::NQ;
  if (g.splits > 1) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = wave % T::WP, wq = wave / T::WP;
    float* part = g.part + ((int64_t)split * matrices + which) * g.rows * g.cols;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t r = q0 + 16 * (wq * NQ + q) + (lane & 15);
      if (r >= g.rows) continue;
#pragma unroll
      for (int p = 0; p < T::NP; ++p) {
        const int64_t c = p0 + 16 * (wp * T::NP + p) + 4 * (lane >> 4);
        if (c < g.cols) put_four(part, r * g.cols + c, g.cols - c, BRSVD_DTYPE_F32, acc[p][q]);
      }
    }
    return;
  }
  const float down = g.down ? *g.down : 1.f;
  put_tile16<NQ>(acc, lds, g.out[which] + q0 * g.ldo[which] + p0, g.ldo[which], g.rows - q0, g.cols - p0, [&](float x, int) { return to16<El>(x * down); });
}

// dX = dG Wg + dU Wu: the contraction runs through dG and dU, down the rows of Wg and of Wu.  Bound by the matrix cores, busy for 74 %: 8192 x 16384 x 4096 1561 us (1.41 Pflop/s).
template <class El, int NQ>
__global__ void __launch_bounds__(kTileThreads, 2)
k_glu_dx(const GradArgs g) {
  using T = TileProduct<El, NQ, kCols, kRows, true, StackStager<El>>;
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_p, g.tiles_q * g.splits, 8, &tp, &tq)) return;
  const int split = (int)((unsigned)tq / (unsigned)g.tiles_q);
  tq -= split * g.tiles_q;
  const int64_t p0 = g.first + tp * kTileP, q0 = tq * T::BQ, k0 = split * g.per_split, k1 = k0 + g.per_split < g.k ? k0 + g.per_split : g.k;
  StackOperand W = g.W;
  W.end = k1;
  floatx4 acc[T::NP][NQ];
  T::run(acc, W, p0, g.D[0], q0, k0, k1, lds);
  leave_gradient<T, El>(g, acc, lds, split, 0, 1, p0, q0);
}

// dWg and dWu, one launch: both operands hold the tokens in their rows.  Bound by the matrix cores, busy for 70 %: 8192 x 16384 x 4096 1632 us (1.35 Pflop/s).
template <class El, int NQ>
__global__ void __launch_bounds__(kTileThreads, 2)
k_glu_dw(const GradArgs g) {
  using T = TileProduct<El, NQ, kCols, kCols, true>;
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_p, 2 * g.tiles_q * g.splits, 8, &tp, &tq)) return;
  const int part = (int)((unsigned)tq / (unsigned)g.tiles_q), which = part & 1, split = part >> 1;
  tq -= part * g.tiles_q;
  const int64_t p0 = g.first + tp * kTileP, q0 = tq * T::BQ, k0 = split * g.per_split, k1 = k0 + g.per_split < g.k ? k0 + g.per_split : g.k;
  floatx4 acc[T::NP][NQ];
  T::run(acc, g.X, p0, g.D[which], q0, k0, k1, lds);
  leave_gradient<T, El>(g, acc, lds, split, which, 2, p0, q0);
}

// Sums of the parts of a contraction that was cut, in their order; a thread four neighbouring columns of `matrices` x rows
template <class El>
__global__ void __launch_bounds__(256)
k_glu_sum(const GradArgs g, int matrices, Divisor quads) {
  uint32_t c;
  const int64_t row = divide(blockIdx.x * 256 + threadIdx.x, quads, &c), col = 4 * (int64_t)c;
  if (row >= matrices * g.rows) return;
  const int which = row >= g.rows;
  floatx4 x = sum_of_parts(g.part + row * g.cols + col, matrices * g.rows * g.cols, g.splits, g.cols - col);
  if (g.down) x *= *g.down;
  put_four(g.out[which], (row - which * g.rows) * g.ldo[which] + col, g.cols - col, __is_same(El, Bf16) ? BRSVD_DTYPE_BF16 : BRSVD_DTYPE_F16, x);
}

// ---- plans ----------------------------------------------------------------------------------------------------------

static uint64_t whole256(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

static constexpr int kStep[3] = {60, 80, 147};        // 1/100 us a step, see tile_plan
// Tokens that go from memory to registers.  Above 32 the tiles are ahead unless they have little to do: 64 x 8000 x 4096 37 us in tiles and 49, 64 x 16000 x 4096 64 and 95, the other
// way round 64 x 8000 x 1000 17.6 and 12.7; at 32 both are alike (8000 x 4096 33 and 33) or these are behind (4096 x 4096 22 and 17).
static bool few_tokens(int64_t tokens, int64_t dim, int64_t width) { return tokens <= 32 || (tokens <= 64 && ceil_div(width, 16 * 256) * dim <= 3000); }

// 16-row tiles of X that a wave has of few tokens
static int token_tiles(int64_t tokens) { return tokens <= 16 ? 1 : tokens <= 32 ? 2 : 4; }

struct GluPlan {
  TilePlan forward, dx, dw;
  int64_t pitch_x, pitch_w, half;                                            // bytes; half: of a row of dG or dU
  uint64_t part, x, wg, wu, forward_bytes;                                    // offsets; x, wg, wu: rows laid out anew
  uint64_t tops, down, dg, part_dx, part_dw, bx, bwg, bwu, backward_bytes;
};
static GluPlan glu_plan(int64_t tokens, int64_t dim, int64_t width, bool aligned) {
  GluPlan p;
  p.forward = tile_plan(ceil_div(width, 128), tokens, ceil_div(dim, 64), 1, 2 * tokens * width, kStep);
  p.dx = tile_plan(ceil_div(dim, 256), tokens, 2 * ceil_div(width, 64), 1, tokens * dim, kStep);
  p.dw = tile_plan(ceil_div(dim, 256), width, ceil_div(tokens, 64), 2, 2 * width * dim, kStep);
  p.pitch_x = line_pitch(2 * dim);
  p.pitch_w = p.pitch_x;
  p.half = 128 * ceil_div(width, 64);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t here = at; at += whole256(bytes); return here; };
  if (!few_tokens(tokens, dim, width)) {
    p.part = take(p.forward.splits > 1 ? (uint64_t)p.forward.splits * tokens * width * 8 : 0);
    p.x = take(aligned ? 0 : (uint64_t)tokens * p.pitch_x);
    p.wg = take(aligned ? 0 : (uint64_t)width * p.pitch_w);
    p.wu = take(aligned ? 0 : (uint64_t)width * p.pitch_w);
  } else {
    p.part = p.x = p.wg = p.wu = 0;
  }
  p.forward_bytes = at;
  at = 0;
  p.tops = take(kTops * 4);
  p.down = take(4);
  p.dg = take((uint64_t)tokens * 2 * p.half);
  p.part_dx = take(p.dx.splits > 1 ? (uint64_t)p.dx.splits * tokens * dim * 4 : 0);
  p.part_dw = take(p.dw.splits > 1 ? (uint64_t)p.dw.splits * width * dim * 8 : 0);
  p.bx = take(aligned ? 0 : (uint64_t)tokens * p.pitch_x);
  p.bwg = take(aligned ? 0 : (uint64_t)width * p.pitch_w);
  p.bwu = take(aligned ? 0 : (uint64_t)width * p.pitch_w);
  p.backward_bytes = at;
  return p;
}

static bool half_type(int dtype) { return dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16; }
// Tiles' rows are addressed with 32 bits, and launches have their workgroups: of tiles, of rows laid out anew, of sums of parts.
static bool glu_sizes(int64_t tokens, int64_t dim, int64_t width) {
  if (tokens < 0 || dim < 0 || width < 0 || tokens >= (int64_t)1 << 30 || dim >= kMaxPitch / 2 || width >= kMaxPitch / 2) return false;
  return tiles_fit(ceil_div(width, 128), ceil_div(tokens, 64), kTileThreads) && tiles_fit(ceil_div(dim, 256), ceil_div(tokens, 64), kTileThreads) &&
         tiles_fit(ceil_div(dim, 256), 2 * ceil_div(width, 64), kTileThreads) && tokens <= (int64_t)UINT32_MAX / ceil_div(dim + 1, 2048);
}

struct GluCall {
  const void *X, *Wg, *Wu;
  int64_t ldx, ldwg, ldwu, tokens, dim, width;
  int dtype, act;
};
// Whether all rows begin at 16-byte addresses, those of Wg and Wu as far from each other
static bool rows_aligned(const GluCall& c) {
  return aligned_pieces(c.X, 2 * c.ldx) && aligned_pieces(c.Wg, 2 * c.ldwg) && aligned_pieces(c.Wu, 2 * c.ldwu) && c.ldwg == c.ldwu;
}

static Operand laid_out(const void* base, int64_t ld, int64_t n, int64_t cols, bool as_it_is, char* to, int64_t pitch, hipStream_t stream) {
  if (as_it_is) return Operand{(const char*)base, 2 * ld, n};
  align_rows(base, 2 * ld, n, 2 * cols, to, pitch, stream);
  return Operand{to, pitch, n};
}

template <class El>
static int glu_forward(const GluCall& c, const GluPlan& p, bool aligned, char* ws, GluArgs g, hipStream_t stream) {
  g.dim = c.dim;
  g.act = c.act;
  if (few_tokens(c.tokens, c.dim, c.width)) {
    g.W = PairOperand{(const char*)c.Wg, (const char*)c.Wu, 2 * c.ldwg, 2 * c.ldwu, c.width};
    g.X = Operand{(const char*)c.X, 2 * c.ldx, c.tokens};
    const dim3 grid((unsigned)ceil_div(c.width, 16));
    const int mt = token_tiles(c.tokens);
    if (mt == 1) hipLaunchKernelGGL((k_glu_rows<El, 1, 4, 8>), grid, dim3(512), 0, stream, g);
    else if (mt == 2) hipLaunchKernelGGL((k_glu_rows<El, 2, 2, 8>), grid, dim3(512), 0, stream, g);
    else hipLaunchKernelGGL((k_glu_rows<El, 4, 2, 8>), grid, dim3(512), 0, stream, g);
  } else {
    g.X = laid_out(c.X, c.ldx, c.tokens, c.dim, aligned, ws + p.x, p.pitch_x, stream);
    const Operand a = laid_out(c.Wg, c.ldwg, c.width, c.dim, aligned, ws + p.wg, p.pitch_w, stream), b = laid_out(c.Wu, c.ldwu, c.width, c.dim, aligned, ws + p.wu, p.pitch_w, stream);
    g.W = PairOperand{a.base, b.base, a.ld, b.ld, c.width};
    g.splits = p.forward.splits;
    g.per_split = p.forward.per_split;
    g.part = (float*)(ws + p.part);
    auto launch = [&](int64_t tiles, int nq) {
      g.tiles_p = tiles;
      g.tiles_q = ceil_div(c.tokens, 64 * nq);
      const dim3 grid(tile_workgroups(g.tiles_p, g.tiles_q * g.splits));
      if (nq == 4) hipLaunchKernelGGL((k_glu_tiles<El, 4>), grid, dim3(kTileThreads), 0, stream, g);
      else if (nq == 2) hipLaunchKernelGGL((k_glu_tiles<El, 2>), grid, dim3(kTileThreads), 0, stream, g);
      else hipLaunchKernelGGL((k_glu_tiles<El, 1>), grid, dim3(kTileThreads), 0, stream, g);
    };
    if (p.forward.large > 0) launch(p.forward.large, 4);
    g.first = 128 * p.forward.large;
    if (p.forward.large < p.forward.tiles) launch(p.forward.tiles - p.forward.large, p.forward.nq);
    if (g.splits > 1) {
      const int64_t quads = ceil_div(c.width, 4);
      hipLaunchKernelGGL(k_glu_join<El>, dim3((unsigned)ceil_div(c.tokens * quads, 256)), dim3(256), 0, stream, g, divisor((uint32_t)quads));
    }
  }
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

template <class El, class Launch>
static void gradient(GradArgs g, const TilePlan& t, int matrices, Launch launch, hipStream_t stream) {
  g.splits = t.splits;
  g.per_split = t.per_split;
  g.first = 0;
  if (t.large > 0) launch(g, t.large, 4);
  g.first = 256 * t.large;
  if (t.large < t.tiles) launch(g, t.tiles - t.large, t.nq);
  if (g.splits > 1) {
    const int64_t quads = ceil_div(g.cols, 4);
    hipLaunchKernelGGL(k_glu_sum<El>, dim3((unsigned)ceil_div(matrices * g.rows * quads, 256)), dim3(256), 0, stream, g, matrices, divisor((uint32_t)quads));
  }
}

template <class El>
static int glu_backward(const GluCall& c, const GluPlan& p, bool aligned, char* ws, SlopeArgs s, void* dX, int64_t lddx, void* dWg, int64_t lddwg, void* dWu, int64_t lddwu,
                        hipStream_t stream) {
  constexpr bool scaled = __is_same(El, Fp16);
  s.tokens = c.tokens;
  s.width = c.width;
  s.pieces = divisor((uint32_t)(p.half / 16));
  s.act = c.act;
  s.dG = ws + p.dg;
  s.second = p.half;
  s.pitch = 2 * p.half;
  s.tops = (float*)(ws + p.tops);
  s.down = (float*)(ws + p.down);
  if (scaled) hipLaunchKernelGGL(k_glu_tops, dim3(kTops), dim3(256), 0, stream, s);
  by_rows(c.tokens, s.pieces.d, 256, [&](int64_t first, int64_t rows, dim3 grid) { hipLaunchKernelGGL(k_glu_slopes<El>, grid, dim3(256), 0, stream, s, first, rows); });
  GradArgs g = {};
  g.down = scaled ? s.down : nullptr;
  // rows that the contraction runs across are read in whole pieces
  const bool across = aligned && c.dim % 8 == 0;
  const int64_t cols = ceil_div(c.dim, 8) * 8;
  if (dX) {
    const Operand a = laid_out(c.Wg, c.ldwg, c.width, c.dim, across, ws + p.bwg, p.pitch_w, stream);
    const Operand b = laid_out(c.Wu, c.ldwu, c.width, c.dim, across, ws + p.bwu, p.pitch_w, stream);
    g.W = StackOperand{a.base, b.base, a.ld, cols, c.width, p.half / 2, 0};
    g.D[0] = Operand{s.dG, s.pitch, c.tokens};
    g.k = p.half;
    g.out[0] = (uint16_t*)dX;
    g.ldo[0] = lddx;
    g.rows = c.tokens;
    g.cols = c.dim;
    g.part = (float*)(ws + p.part_dx);
    gradient<El>(g, p.dx, 1, [&](GradArgs g, int64_t tiles, int nq) {
      g.tiles_p = tiles;
      g.tiles_q = ceil_div(g.rows, 64 * nq);
      const dim3 grid(tile_workgroups(g.tiles_p, g.tiles_q * g.splits));
      if (nq == 4) hipLaunchKernelGGL((k_glu_dx<El, 4>), grid, dim3(kTileThreads), 0, stream, g);
      else if (nq == 2) hipLaunchKernelGGL((k_glu_dx<El, 2>), grid, dim3(kTileThreads), 0, stream, g);
      else hipLaunchKernelGGL((k_glu_dx<El, 1>), grid, dim3(kTileThreads), 0, stream, g);
    }, stream);
  }
  if (dWg) {
    g.X = laid_out(c.X, c.ldx, c.tokens, c.dim, across, ws + p.bx, p.pitch_x, stream);
    g.X.n = cols;
    g.D[0] = Operand{s.dG, s.pitch, ceil_div(c.width, 8) * 8};
    g.D[1] = Operand{s.dG + s.second, s.pitch, ceil_div(c.width, 8) * 8};
    g.k = c.tokens;
    g.out[0] = (uint16_t*)dWg;
    g.out[1] = (uint16_t*)dWu;
    g.ldo[0] = lddwg;
    g.ldo[1] = lddwu;
    g.rows = c.width;
    g.cols = c.dim;
    g.part = (float*)(ws + p.part_dw);
    gradient<El>(g, p.dw, 2, [&](GradArgs g, int64_t tiles, int nq) {
      g.tiles_p = tiles;
      g.tiles_q = ceil_div(g.rows, 64 * nq);
      const dim3 grid(tile_workgroups(g.tiles_p, 2 * g.tiles_q * g.splits));
      if (nq == 4) hipLaunchKernelGGL((k_glu_dw<El, 4>), grid, dim3(kTileThreads), 0, stream, g);
      else if (nq == 2) hipLaunchKernelGGL((k_glu_dw<El, 2>), grid, dim3(kTileThreads), 0, stream, g);
      else hipLaunchKernelGGL((k_glu_dw<El, 1>), grid, dim3(kTileThreads), 0, stream, g);
    }, stream);
  }
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

// Refusals that both calls share
static int check_glu(const GluCall& c) {
  if (!half_type(c.dtype) || c.act < BRSVD_ACT_SILU || c.act > BRSVD_ACT_GELU_TANH || !glu_sizes(c.tokens, c.dim, c.width)) return BRSVD_ERR_ARG;
  if (c.dim == 0 || c.tokens == 0 || c.width == 0) return BRSVD_OK;
  if (!c.X || !c.Wg || !c.Wu || c.ldx < c.dim || c.ldwg < c.dim || c.ldwu < c.dim) return BRSVD_ERR_ARG;
  return c.ldx >= kMaxPitch / 2 || c.ldwg >= kMaxPitch / 2 || c.ldwu >= kMaxPitch / 2 ? BRSVD_ERR_ARG : BRSVD_OK;
}
static int check_workspace(const void* ws, uint64_t have, uint64_t need) {
  if (need && (!ws || (uintptr_t)ws % 256)) return BRSVD_ERR_ARG;
  return have < need ? BRSVD_ERR_BUDGET : BRSVD_OK;
}
static bool pitch_fits(int64_t ld, int64_t least) { return ld >= least && ld < (int64_t)1 << 40; }

}  // namespace brsvd

using namespace brsvd;

extern "C" uint64_t brsvd_glu_workspace_bytes(int64_t tokens, int64_t dim, int64_t width, int32_t aligned, int32_t backward) {
  if (!glu_sizes(tokens, dim, width) || tokens == 0 || dim == 0 || width == 0) return 0;
  const GluPlan p = glu_plan(tokens, dim, width, aligned && (!backward || dim % 8 == 0));
  return backward ? p.backward_bytes : p.forward_bytes;
}

extern "C" int brsvd_glu_forward(const void* X, int64_t ldx, const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu, int64_t tokens, int64_t dim, int64_t width,
                                 int32_t dtype, int32_t act, void* H, int64_t ldh, void* G, int64_t ldg, void* U, int64_t ldu, void* workspace, uint64_t workspace_bytes,
                                 void* stream) {
  const GluCall c{X, Wg, Wu, ldx, ldwg, ldwu, tokens, dim, width, dtype, act};
  BRSVD_TRY(check_glu(c));
  if (tokens == 0 || width == 0) return BRSVD_OK;
  if (!H || !pitch_fits(ldh, width) || !G != !U || (G && (!pitch_fits(ldg, width) || !pitch_fits(ldu, width)))) return BRSVD_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  if (dim == 0) {              // sums of nothing
    join_splits(nullptr, 0, tokens, width, H, ldh, dtype, s);
    if (G) join_splits(nullptr, 0, tokens, width, G, ldg, dtype, s), join_splits(nullptr, 0, tokens, width, U, ldu, dtype, s);
    BRSVD_HIP_TRY(hipGetLastError());
    return BRSVD_OK;
  }
  const bool aligned = rows_aligned(c);
  const GluPlan p = glu_plan(tokens, dim, width, aligned);
  BRSVD_TRY(check_workspace(workspace, workspace_bytes, p.forward_bytes));
  GluArgs g = {};
  g.H = (uint16_t*)H;
  g.G = (uint16_t*)G;
  g.U = (uint16_t*)U;
  g.ldh = ldh;
  g.ldg = ldg;
  g.ldu = ldu;
  return dtype == BRSVD_DTYPE_BF16 ? glu_forward<Bf16>(c, p, aligned, (char*)workspace, g, s) : glu_forward<Fp16>(c, p, aligned, (char*)workspace, g, s);
}

extern "C" int brsvd_glu_backward(const void* X, int64_t ldx, const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu, const void* G, int64_t ldg, const void* U,
                                  int64_t ldu, const void* dH, int64_t lddh, int64_t tokens, int64_t dim, int64_t width, int32_t dtype, int32_t act, void* dX, int64_t lddx,
                                  void* dWg, int64_t lddwg, void* dWu, int64_t lddwu, void* workspace, uint64_t workspace_bytes, void* stream) {
  const GluCall c{X, Wg, Wu, ldx, ldwg, ldwu, tokens, dim, width, dtype, act};
  BRSVD_TRY(check_glu(c));
  if (!dWg != !dWu || (dX && !pitch_fits(lddx, dim)) || (dWg && (!pitch_fits(lddwg, dim) || !pitch_fits(lddwu, dim)))) return BRSVD_ERR_ARG;
  if (!dX && !dWg && tokens > 0 && dim > 0 && width > 0) return BRSVD_ERR_ARG;       // without elements any may be NULL
  if (dim == 0) return BRSVD_OK;
  hipStream_t s = (hipStream_t)stream;
  if (tokens == 0 || width == 0) {      // sums of nothing
    if (!(dX && tokens > 0) && !(dWg && width > 0)) return BRSVD_OK;
    if (dX && tokens > 0) join_splits(nullptr, 0, tokens, dim, dX, lddx, dtype, s);
    if (dWg && width > 0) join_splits(nullptr, 0, width, dim, dWg, lddwg, dtype, s), join_splits(nullptr, 0, width, dim, dWu, lddwu, dtype, s);
    BRSVD_HIP_TRY(hipGetLastError());
    return BRSVD_OK;
  }
  if (!G || !U || !dH || !pitch_fits(ldg, width) || !pitch_fits(ldu, width) || !pitch_fits(lddh, width)) return BRSVD_ERR_ARG;
  const bool aligned = rows_aligned(c);
  const GluPlan p = glu_plan(tokens, dim, width, aligned && dim % 8 == 0);
  BRSVD_TRY(check_workspace(workspace, workspace_bytes, p.backward_bytes));
  SlopeArgs a = {};
  a.G = (const char*)G;
  a.U = (const char*)U;
  a.dH = (const char*)dH;
  a.ldg = 2 * ldg;
  a.ldu = 2 * ldu;
  a.ldh = 2 * lddh;
  char* ws = (char*)workspace;
  return dtype == BRSVD_DTYPE_BF16 ? glu_backward<Bf16>(c, p, aligned, ws, a, dX, lddx, dWg, lddwg, dWu, lddwu, s)
                                   : glu_backward<Fp16>(c, p, aligned, ws, a, dX, lddx, dWg, lddwg, dWu, lddwu, s);
}

extern "C" int brsvd_glu_plan(int32_t which, int64_t tokens, int64_t dim, int64_t width, int32_t* out8) {
  if (!out8 || which < 0 || which > 2 || !glu_sizes(tokens, dim, width) || tokens == 0 || dim == 0 || width == 0) return BRSVD_ERR_ARG;
  const GluPlan p = glu_plan(tokens, dim, width, true);
  if (which == 0 && few_tokens(tokens, dim, width)) describe_rows(token_tiles(tokens), 1, out8);
  else describe_plan(which == 0 ? p.forward : which == 1 ? p.dx : p.dw, out8);
  return BRSVD_OK;
}
