// Losses of a model's output matrix over a large vocabulary, and their gradients, without the tokens x vocabulary logits.
//   z = H W^T (H tokens x dim, W vocab x dim),  p_t = softmax(z_t / tau),  lse_t = log sum_v exp(z_tv / tau)
//   cross entropy  loss_t = lse_t - z_{t, y_t}                          (tau = 1)
//   distillation   loss_t = tau^2 sum_j q_tj (log q_tj - z_{t, id_tj} / tau + lse_t),  q_t = softmax(a_t / tau) over the teacher's listed logits
//   gradient       G = g_t tau (p_t - target_t),  dH = G W,  dW = G^T H
// Forward: a workgroup forms a 256 (vocabulary) x 256 (tokens) tile of z in registers and leaves, for every token, its largest entry and the sum of
// exponentials relative to it; the parts are joined per token.  Backward: for a piece of the vocabulary at a time G is formed again from z and
// lse, in 16 bits, and multiplied: dH is added up over the pieces in fp32, dW of a piece is finished at once.
//
// Tokens that do not count (label outside the vocabulary, nothing listed) are left out of the backward pass from the start: the rows that count are copied
// next to each other.  What stands in the others, NaN or infinities too, then reaches nothing, and half a batch of prompts costs half.
#include "tile.h"

namespace brsvd {

// Tiles of eight waves, 256 of the vocabulary (or of dim) x 256 tokens; x 128 or 64 where there are few tokens, so that a tile's columns are not mostly
// empty.
template <class El, Order OP, Order OQ, bool DIRECT, int BQ> using Tiles = TileProduct<El, BQ / 64, OP, OQ, DIRECT>;
constexpr int kTileP = 256, kTileThreads = 512;
// The logits, both operands with dim in their rows: up to 64 tokens without LDS, four waves.
template <class El, bool DIRECT, int BQ> struct Logits : Tiles<El, kRows, kRows, DIRECT, BQ> {};
template <class El, bool DIRECT> struct Logits<El, DIRECT, 64> : RowsProduct<El, 2, 4, 4, 2> {};
template <class El, bool DIRECT> struct Logits<El, DIRECT, 32> : RowsProduct<El, 2, 2, 4, 4> {};
template <class El, bool DIRECT> struct Logits<El, DIRECT, 16> : RowsProduct<El, 2, 1, 4, 4> {};
// How many tiles along the other side (others) have 256 tokens, the rest 128 or fewer.  256 x 256 has no registers left for pieces on their way through
// them.  130 tokens over 32000 words of width 2000, one round of 250 tiles or of 125: 41 us and 53.
static int64_t large_token_tiles(int64_t tokens, bool direct, int64_t others, int64_t contraction) {
  return tokens <= 128 || !direct ? 0 : large_tiles(others, ceil_div(tokens, 256), ceil_div(tokens, 128), ceil_div(contraction, 64));
}
static int small_tile(int64_t tokens) { return tokens <= 64 ? 64 : 128; }
// The logits of `words` words: the first `large` in tiles of 256 words x 256 tokens, the others in tiles of `rows` words x `bl` tokens.
struct LogitTiles {
  int64_t large;
  int bl, rows;
  int64_t first, count;      // tiles along the vocabulary: large ones, all
};
static LogitTiles logit_tiles(int64_t tokens, bool direct, int64_t words, int64_t dim) {
  LogitTiles t;
  t.first = large_token_tiles(tokens, direct, ceil_div(words, kTileP), dim);
  t.large = kTileP * t.first < words ? kTileP * t.first : words;
  t.bl = tokens <= 16 ? 16 : tokens <= 32 ? 32 : small_tile(tokens);
  t.rows = t.bl <= 64 ? 128 : kTileP;
  t.count = t.first + ceil_div(words - t.large, t.rows);
  return t;
}

// What the backward pass knows on the device: how many tokens count, and the power of two that G is multiplied by so that its numbers of 16 bits hold what
// matters: 2^e max |g_t| is 2^14 to 2^15, which |p - target| <= 1 keeps inside fp16, and for the token with that factor a probability of 2^-28 is still a normal
// number.  One power serves all tokens, as dW adds them up: in fp16 an entry is off by 2^-39 max |g_t| where it is small, whatever its own token's factor.
struct HeadMeta {
  int count;
  float up, down;      // 2^e, 2^-e
  int pad;
};

struct HeadArgs {
  Operand W, H;            // kRows, over dim
  int64_t dim;
  float scale;             // 1 / tau
  int64_t tiles_v, tiles_t;
  const int64_t* label;    // null: distillation
  float2* part;            // forward: [vocabulary tile][token], largest and sum
  float* zlabel;           // forward: the label's logit
  const HeadMeta* meta;    // backward
  const float *lse, *coef; // backward, of the tokens that count
  const int* label_c;
  int64_t first;           // row of W that the first tile begins with
  int64_t v0;              // backward: the piece's first row
  uint16_t* G;             // backward: [token][pitch]
  int64_t pitch;
};

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
// What is taken off before exponentials: the largest, but nothing where that is infinite, so that a row of -inf sums to 0 and one with a +inf to infinity.
__device__ __forceinline__ float reference(float top) { return fabsf(top) == INFINITY ? 0.f : top; }

// What a tile of logits leaves: the label's logit, and for every token the largest and the sum.  Exponentials are powers of two of x log2(e); what is
// kept of a row is in units of log 2, too.
template <class T>
__device__ __forceinline__ void leave_tile(const HeadArgs& g, floatx4 (&acc)[T::NP][T::NQ], int64_t tv, int64_t tt, float2* red) {
  constexpr int NP = T::NP, NQ = T::NQ, WP = T::WP, BQ = T::BQ;
  const int64_t v0 = g.first + tv * T::BP, t0 = tt * BQ;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wp = wave % WP, wq = wave / WP;
  const int64_t vwave = v0 + 16 * wp * NP, vlane = vwave + 4 * (lane >> 4);
  const float scale = g.scale * kLog2e;
  if (vwave + 16 * NP > g.W.n) {        // words beyond the last one
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (vlane + 16 * p + r >= g.W.n)
#pragma unroll
          for (int q = 0; q < NQ; ++q) acc[p][q][r] = -INFINITY;
  }
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[p][q][r]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32)) * scale;
    // The largest entry's exponent, less its rounded value, is up to 2^-24 of it: an exponential stands that up to 2^30.  Beyond, all exponents are taken down so
    // that the largest is 2^28 (three roundings: off by 48 at most).  What that adds to log2 of the sum is within the rounding of the largest.
    float ref = reference(top), s = scale;
    if (fabsf(ref) > 0x1p30f) {
      s = scale * (0x1p28f / fabsf(ref));
      ref = copysignf(0x1p28f, ref);
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(fmaf(acc[p][q][r], s, -ref));
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lane < 16) red[wp * BQ + 16 * (wq * NQ + q) + lane] = make_float2(top, sum);
  }
  if (g.label) {
    int64_t at[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t t = t0 + 16 * (wq * NQ + q) + (lane & 15);
      at[q] = g.label[t < g.H.n ? t : g.H.n - 1] - vlane;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t t = t0 + 16 * (wq * NQ + q) + (lane & 15);
      const bool mine = at[q] >= 0 && at[q] < 16 * NP && (at[q] & 15) < 4 && at[q] + vlane < g.W.n && t < g.H.n;
      if (__any(mine)) {
        float z = 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (at[q] == 16 * p + r) z = acc[p][q][r];
        if (mine) g.zlabel[t] = z;
      }
    }
  }
  __syncthreads();
  for (int col = threadIdx.x; col < BQ; col += T::kThreads) {
    if (t0 + col >= g.H.n) continue;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WP; ++w) top = fmaxf(top, red[w * BQ + col].x);
    const float ref = reference(top);
#pragma unroll
    for (int w = 0; w < WP; ++w) sum += red[w * BQ + col].y * __builtin_amdgcn_exp2f(red[w * BQ + col].x - ref);
    g.part[tv * g.H.n + t0 + col] = make_float2(top, sum);
  }
}

// A workgroup takes every gridDim-th tile.  Without pieces in registers the next tile's first steps are on their way while this one's exponentials are
// worked out.  Bound by the matrix cores where there are many tokens: 8192 x 100000 over 4096 4.6 to 5.1 ms (1.3 to 1.45 Pflop/s); at width 272 a tile's steps take
// 7 us and its 65536 exponentials 4, 300 us for 4096 x 100000.  By the read of W for few: 7 x 32000 x 1000 13 us (64 MB, 4.9 TB/s).
template <class El, bool DIRECT, int BQ>
__global__ void __launch_bounds__((Logits<El, DIRECT, BQ>::kThreads), 2)
k_head_lse(const HeadArgs g) {
  using T = Logits<El, DIRECT, BQ>;
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  __shared__ float2 red[T::WP * BQ];
  floatx4 acc[T::NP][T::NQ];
  int64_t tv, tt;
  unsigned b = blockIdx.x;
  if (!tile_of_workgroup(b, g.tiles_v, g.tiles_t, 8, &tv, &tt)) return;
  if constexpr (T::kThreads == kTileThreads && DIRECT) {
    T tile;
    tile.begin(g.W, g.first + tv * T::BP, g.H, tt * BQ, 0, g.dim, lds);
    while (true) {
      tile.multiply(acc);
      int64_t nv = 0, nt = 0;
      b += gridDim.x;
      const bool more = tile_of_workgroup(b, g.tiles_v, g.tiles_t, 8, &nv, &nt);
      if (more) tile.begin(g.W, g.first + nv * T::BP, g.H, nt * BQ, 0, g.dim, lds);
      leave_tile<T>(g, acc, tv, tt, red);
      if (!more) break;
      tv = nv;
      tt = nt;
    }
  } else {
    do {
      T::run(acc, g.W, g.first + tv * T::BP, g.H, tt * BQ, 0, g.dim, lds);
      leave_tile<T>(g, acc, tv, tt, red);
      __syncthreads();
      b += gridDim.x;
    } while (tile_of_workgroup(b, g.tiles_v, g.tiles_t, 8, &tv, &tt));
  }
}

// lse of 16 tokens a workgroup from their parts, in a fixed order, and with labels the loss.  4 to 9 us, a launch: only another could join workgroups that
// end at different times.
__global__ void __launch_bounds__(256)
k_head_join(const float2* __restrict__ part, int64_t tiles, int64_t tokens, const int64_t* __restrict__ label, int64_t vocab, const float* __restrict__ zlabel,
            float* __restrict__ lse, float* __restrict__ loss, unsigned first_wg) {
  __shared__ float2 red[16][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t t = ((int64_t)first_wg + blockIdx.x) * 16 + c;
  float top = -INFINITY, sum = 0.f;
  auto add = [&](float2 v) {
    const float to = fmaxf(top, v.x), ref = reference(to);
    sum = sum * __builtin_amdgcn_exp2f(top - ref) + v.y * __builtin_amdgcn_exp2f(v.x - ref);
    top = to;
  };
  if (t < tokens) {
    int64_t i = r;
    for (; i + 48 < tiles; i += 64) {
      float2 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = part[(i + 16 * j) * tokens + t];
#pragma unroll
      for (int j = 0; j < 4; ++j) add(v[j]);
    }
    for (; i < tiles; i += 16) add(part[i * tokens + t]);
  }
  red[r][c] = make_float2(top, sum);
  __syncthreads();
  if (r != 0 || t >= tokens) return;
  float all = -INFINITY;
  for (int i = 0; i < 16; ++i) all = fmaxf(all, red[i][c].x);
  const float ref = reference(all);
  sum = 0.f;
  for (int i = 0; i < 16; ++i) sum += red[i][c].y * __builtin_amdgcn_exp2f(red[i][c].x - ref);
  const float l = (all + log2f(sum)) * kLn2;
  lse[t] = l;
  if (label) loss[t] = label[t] >= 0 && label[t] < vocab ? l - zlabel[t] : 0.f;
}

// ---- the teacher's side of a distillation -------------------------------------------------------------------------

// Eight numbers of 16 bits, of which `valid` are there
template <class El>
__device__ __forceinline__ void eight16(const char* src, int64_t valid, float (&x)[8]) {
  const uint4 v = piece_of<2>(src, 2 * valid);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = from16<El>((uint16_t)(w[i / 2] >> (16 * (i & 1))));
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x += __shfl_xor(x, s);
  return x;
}

struct Teacher {
  const int64_t* ids;
  const float* logits;
  int top;
  float scale;          // 1 / tau
};
__device__ __forceinline__ bool is_listed(int64_t id, float a, int64_t vocab) { return id >= 0 && id < vocab && a > -INFINITY; }
// Largest listed logit of token t, and the sum of exponentials of (logit - largest) / tau, in every lane of the wave.  Taken off before the division: a mask of the
// lowest fp32 number over a tau below one would be -inf.
__device__ __forceinline__ float2 teacher_norm(const Teacher& te, int64_t t, int64_t vocab, int lane) {
  float top = -INFINITY, sum = 0.f;
  for (int j = lane; j < te.top; j += 64) {
    const float a = te.logits[t * te.top + j];
    if (is_listed(te.ids[t * te.top + j], a, vocab)) top = fmaxf(top, a);
  }
  top = wave_max(top);
  for (int j = lane; j < te.top; j += 64) {
    const float a = te.logits[t * te.top + j];
    if (is_listed(te.ids[t * te.top + j], a, vocab)) sum += __builtin_amdgcn_exp2f((a - top) * te.scale * kLog2e);
  }
  return make_float2(top, wave_sum(sum));
}

// One token a workgroup: the student's logits of the listed words (dot products in fp32, four at a time a wave), then the loss.  Bound by the rows of W that
// it reads, tokens x top of them: 4096 tokens x 64 words of width 2048 149 us (1.07 GB, 7.2 TB/s, much of it from the caches).
template <class El>
__global__ void __launch_bounds__(256)
k_distill_loss(const Operand W, const Operand H, int64_t dim, const Teacher te, const float* __restrict__ lse, float* __restrict__ z, float* __restrict__ loss,
               unsigned first_wg) {
  __shared__ float part[4];
  const int64_t t = first_wg + blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float2 norm = teacher_norm(te, t, W.n, lane);
  const float l = lse[t], logsum = logf(norm.y);
  float sum = 0.f;
  for (int j0 = 4 * wave; j0 < te.top; j0 += 16) {
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    const char* row[4];
    bool in[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + i < te.top ? j0 + i : te.top - 1;
      const int64_t id = te.ids[t * te.top + j];
      in[i] = j0 + i < te.top && is_listed(id, te.logits[t * te.top + j], W.n);
      row[i] = W.base + (in[i] ? id : 0) * W.ld;
    }
    for (int64_t k = 8 * lane; k < dim; k += 512) {
      float h[8], w[8];
      eight16<El>(H.base + t * H.ld + 2 * k, dim - k, h);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        eight16<El>(row[i] + 2 * k, dim - k, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[i] += h[e] * w[e];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      acc[i] = wave_sum(acc[i]);
      if (j0 + i >= te.top) continue;
      const int64_t at = t * te.top + j0 + i;
      if (in[i]) {
        const float logq = (te.logits[at] - norm.x) * te.scale - logsum, q = __builtin_amdgcn_exp2f(logq * kLog2e);
        if (q != 0.f) sum += q * (logq - acc[i] * te.scale + l);          // q log q is 0 for q = 0, where log q may be -inf
      }
      if (lane == 0) z[at] = in[i] ? acc[i] : 0.f;
    }
  }
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  // tau times tau, one after the other: tau^2 may leave fp32 where the loss does not
  if (threadIdx.x == 0) loss[t] = norm.y == 0.f ? 0.f : (part[0] + part[1] + part[2] + part[3]) / te.scale / te.scale;
}

// q of every listed word (0 for the others), added up over the token's entries with the same word, and whether the token has any.  A wave a token.
__global__ void __launch_bounds__(256)
k_distill_targets(const Teacher te, int64_t tokens, int64_t vocab, float* __restrict__ q, int* __restrict__ counts, unsigned first_wg) {
  const int64_t t = ((int64_t)first_wg + blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (t >= tokens) return;
  const float2 norm = teacher_norm(te, t, vocab, lane);
  const float inv = norm.y == 0.f ? 0.f : 1.f / norm.y;
  for (int j0 = 0; j0 < te.top; j0 += 64) {
    const int64_t mine = j0 + lane < te.top ? te.ids[t * te.top + j0 + lane] : -1;
    float sum = 0.f;
    for (int i0 = 0; i0 < te.top; i0 += 64) {
      const int64_t at = t * te.top + (i0 + lane < te.top ? i0 + lane : 0);
      const float a = te.logits[at];
      const int64_t id = i0 + lane < te.top && is_listed(te.ids[at], a, vocab) ? te.ids[at] : -1;
      const float x = id >= 0 ? __builtin_amdgcn_exp2f((a - norm.x) * te.scale * kLog2e) * inv : 0.f;
      const int last = te.top - i0 < 64 ? te.top - i0 : 64;
      for (int i = 0; i < last; ++i) {
        const int other = __builtin_amdgcn_readlane((int)id, i);           // words are below 2^30
        const float y = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), i));
        if (other == (int)mine) sum += y;
      }
    }
    if (j0 + lane < te.top) q[t * te.top + j0 + lane] = mine >= 0 && mine < vocab ? sum : 0.f;
  }
  if (lane == 0) counts[t] = norm.y != 0.f;
}

// The listed words of a piece in G: exp(z / tau - lse) - q.  A thread an entry; entries with the same word write the same number.
template <class El>
__global__ void __launch_bounds__(256)
k_distill_scatter(const Teacher te, const float* __restrict__ q, const float* __restrict__ z, const HeadMeta* __restrict__ meta, const int* __restrict__ index,
                  const float* __restrict__ lse, const float* __restrict__ coef, int64_t v0, int64_t rows, int64_t vocab, uint16_t* __restrict__ G, int64_t pitch,
                  unsigned first_wg) {
  const int64_t i = ((int64_t)first_wg + blockIdx.x) * 256 + threadIdx.x, c = i / te.top;
  if (c >= meta->count) return;
  const int64_t t = index[c], at = t * te.top + (i - c * te.top), id = te.ids[at];
  if (id < v0 || id >= v0 + rows || !is_listed(id, te.logits[at], vocab)) return;
  G[c * pitch + id - v0] = to16<El>(coef[c] * (__builtin_amdgcn_exp2f((z[at] * te.scale - lse[c]) * kLog2e) - q[at]));
}

// ---- backward -----------------------------------------------------------------------------------------------------

// Which tokens count, in order, and the scale of G.  One workgroup: a running count over blocks of 1024 tokens.
__global__ void __launch_bounds__(1024)
k_head_prepare(const int64_t* __restrict__ label, int64_t vocab, const int* __restrict__ counts, int64_t tokens, const float* __restrict__ grad, int64_t grad_stride,
               float factor, HeadMeta* __restrict__ meta, int* __restrict__ index, float* __restrict__ coef) {
  __shared__ int wave_count[16];
  __shared__ float wave_top[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t before = 0;
  float top = 0.f;
  for (int64_t t0 = 0; t0 < tokens; t0 += 1024) {
    const int64_t t = t0 + threadIdx.x;
    const bool in = t < tokens && (label ? label[t] >= 0 && label[t] < vocab : counts[t] != 0);
    const unsigned long long mask = __ballot(in);
    if (lane == 0) wave_count[wave] = __popcll(mask);
    __syncthreads();
    int64_t at = before + __popcll(mask & ((1ull << lane) - 1));
    for (int w = 0; w < 16; ++w) {
      if (w < wave) at += wave_count[w];
      before += wave_count[w];
    }
    if (in) {
      const float s = grad[t * grad_stride] * factor;
      index[at] = (int)t;
      coef[at] = s;
      if (fabsf(s) <= 3.402823466e38f) top = fmaxf(top, fabsf(s));
    }
    __syncthreads();
  }
  top = wave_max(top);
  if (lane == 0) wave_top[wave] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 0; w < 16; ++w) top = fmaxf(top, wave_top[w]);
    int e = top > 0.f ? 14 - ((int)(__float_as_uint(top) >> 23) - 127) : 0;
    e = e > 120 ? 120 : e < -120 ? -120 : e;
    meta->count = (int)before;
    meta->up = __uint_as_float((uint32_t)(e + 127) << 23);
    meta->down = __uint_as_float((uint32_t)(127 - e) << 23);
  }
}

// The rows of H that count next to each other (pitch in bytes, a multiple of 16, what lies beyond dim is never read), with their lse, factor and label;
// and zeros into the rows of dH (may be null) that do not.
__global__ void __launch_bounds__(256)
k_head_gather(const Operand H, int64_t dim, int64_t vocab, const HeadMeta* __restrict__ meta, const int* __restrict__ index, const float* __restrict__ lse,
              const int64_t* __restrict__ label, const int* __restrict__ counts, char* __restrict__ Hc, int64_t pitch, float* __restrict__ lse_c,
              float* __restrict__ coef, int* __restrict__ label_c, uint16_t* __restrict__ dH, int64_t lddh, unsigned first_wg) {
  const int64_t c = first_wg + blockIdx.x;
  if (dH && !(label ? label[c] >= 0 && label[c] < vocab : counts[c] != 0))
    for (int64_t d = threadIdx.x; d < dim; d += 256) dH[c * lddh + d] = 0;
  if (c >= meta->count) return;
  const int64_t t = index[c];
  for (int64_t k = 8 * (int64_t)threadIdx.x; k < dim; k += 2048) *(uint4*)(Hc + c * pitch + 2 * k) = piece_of<2>(H.base + t * H.ld + 2 * k, 2 * (dim - k));
  if (threadIdx.x == 0) {
    lse_c[c] = lse[t];
    coef[c] *= meta->up;
    label_c[c] = label ? (int)label[t] : -1;
  }
}

// A piece of G: the logits again, then the gradient with respect to them.  Bound as the forward pass is: 8192 x 100000 over 4096 5.1 ms in seven pieces.  To keep the
// logits instead would take 1.6 GB there, and a read and a write of them.
template <class El, bool DIRECT, int BQ>
__global__ void __launch_bounds__((Logits<El, DIRECT, BQ>::kThreads), 2)
k_head_grad(const HeadArgs g) {
  using T = Logits<El, DIRECT, BQ>;
  constexpr int NP = T::NP, NQ = T::NQ, WP = T::WP;
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  int64_t tv, tt;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_v, g.tiles_t, 8, &tv, &tt)) return;
  const int64_t count = g.meta->count, p0 = g.first + tv * T::BP, t0 = tt * BQ;
  if (t0 >= count) return;
  Operand H = g.H;
  H.n = count;
  floatx4 acc[NP][NQ];
  T::run(acc, g.W, p0, H, t0, 0, g.dim, lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wp = wave % WP, wq = wave / WP;
  const int vlane = (int)p0 + 16 * wp * NP + 4 * (lane >> 4), rows = (int)g.W.n;
  const float scale = g.scale * kLog2e;
  float l[NQ], s[NQ];
  int at[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int64_t c = t0 + 16 * (wq * NQ + q) + (lane & 15), in = c < count ? c : count - 1;
    l[q] = g.lse[in] * kLog2e;
    s[q] = g.coef[in];
    at[q] = g.label_c[in] - (int)g.v0 - vlane;
  }
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int64_t c = t0 + 16 * (wq * NQ + q) + (lane & 15);
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[p][q][r] = __builtin_amdgcn_exp2f(fmaf(acc[p][q][r], scale, -l[q]));
    if (__any(at[q] >= 0 && at[q] < 16 * NP)) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (at[q] == 16 * p + r) acc[p][q][r] -= 1.f;
    }
    if constexpr (T::kThreads != kTileThreads) {
      if (c >= count) continue;
      uint16_t* row = g.G + c * g.pitch;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        uint16_t h[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = to16<El>(s[q] * acc[p][q][r]);
        // the pitch is a multiple of eight: what is written beyond the piece's last row stays inside the token's row of G
        if (vlane + 16 * p < rows) *(uint2*)(row + vlane + 16 * p) = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
      }
    }
  }
  if constexpr (T::kThreads == kTileThreads)
    put_tile16<NQ>(acc, lds, g.G + t0 * g.pitch + p0, g.pitch, count - t0, g.pitch - p0, [&](float x, int q) { return to16<El>(s[q] * x); });
}

struct HeadProduct {
  Operand P, Q;            // P: the side along which the result is contiguous
  int64_t k;               // of the contraction; < 0: the tokens that count
  int64_t per_split;       // of the contraction
  const HeadMeta* meta;
  int64_t tiles_p, tiles_q;
  float* sum;              // dH: [split][token][dim], added to if `more`
  bool more;
  uint16_t* out;           // dW
  int64_t first;           // dW: the word that the first tile begins with
  int64_t words, width;    // dW: its rows and columns
  int64_t ldo;
};

// dH (+)= G W of a piece.  The splits of the contraction keep sums of their own, which the last kernel adds up: no part waits for another.
// Bound by the matrix cores: 8192 x 4096 over 100000 5.0 ms (1.34 Pflop/s).
template <class El, bool DIRECT, int BQ>
__global__ void __launch_bounds__(kTileThreads, 2)
k_head_dh(const HeadProduct g) {
  using T = Tiles<El, kCols, kRows, DIRECT, BQ>;
  constexpr int NP = T::NP, NQ = T::NQ, WP = T::WP;
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_p, g.tiles_q, 8, &tp, &tq)) return;
  Operand Q = g.Q;
  Q.n = g.meta->count;
  const int64_t p0 = tp * kTileP, q0 = tq * BQ, k0 = blockIdx.y * g.per_split, k1 = k0 + g.per_split < g.k ? k0 + g.per_split : g.k;
  if (q0 >= Q.n || k0 >= k1) return;
  floatx4 acc[NP][NQ];
  T::run(acc, g.P, p0, Q, q0, k0, k1, lds);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = wave % WP, wq = wave / WP;
  float* sum = g.sum + (int64_t)blockIdx.y * g.Q.n * g.P.n;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int64_t c = q0 + 16 * (wq * NQ + q) + (lane & 15);
    if (c >= Q.n) continue;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int64_t d = p0 + 16 * (wp * NP + p) + 4 * (lane >> 4);
      float* at = sum + c * g.P.n + d;
      if (d + 4 <= g.P.n && g.P.n % 4 == 0) {
        floatx4 v = acc[p][q];
        if (g.more) v += *(const floatx4*)at;
        *(floatx4*)at = v;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (d + r < g.P.n) at[r] = acc[p][q][r] + (g.more ? at[r] : 0.f);
      }
    }
  }
}

// dW = G^T H of a piece: both operands hold the tokens in their rows.  100000 x 4096 over 8192 5.2 ms (1.30 Pflop/s); with few tokens bound by the writing of dW and
// the reading of G, which a round of tiles does at the same time: 50001 x 1000 over 999 128 us.
template <class El, int BQ>
__global__ void __launch_bounds__(kTileThreads, 2)
k_head_dw(const HeadProduct g) {
  using T = Tiles<El, kCols, kCols, true, BQ>;
  __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
  int64_t tp, tq;
  if (!tile_of_workgroup(blockIdx.x, g.tiles_p, g.tiles_q, 8, &tp, &tq)) return;
  const int64_t p0 = tp * kTileP, q0 = g.first + tq * BQ;
  floatx4 acc[T::NP][T::NQ];
  T::run(acc, g.P, p0, g.Q, q0, 0, g.meta->count, lds);
  const float down = g.meta->down;
  put_tile16<T::NQ>(acc, lds, g.out + q0 * g.ldo + p0, g.ldo, g.words - q0, g.width - p0, [&](float x, int) { return to16<El>(x * down); });
}

// A matrix of zeros
__global__ void __launch_bounds__(256)
k_head_zero(uint16_t* __restrict__ dW, int64_t ld, int64_t dim, unsigned first_wg) {
  for (int64_t d = threadIdx.x; d < dim; d += 256) dW[((int64_t)first_wg + blockIdx.x) * ld + d] = 0;
}
// The rows of dH that count: the sum of the splits' parts in their order.  A thread a number of a row, eight parts at a time on their way.
template <class El>
__global__ void __launch_bounds__(256)
k_head_finish(const float* __restrict__ sum, int splits, int64_t tokens, int64_t dim, const HeadMeta* __restrict__ meta, const int* __restrict__ index,
              uint16_t* __restrict__ dH, int64_t ld, unsigned first_wg) {
  const int64_t per = (dim + 255) / 256, wg = first_wg + blockIdx.x, c = wg / per, d = (wg - c * per) * 256 + threadIdx.x;
  if (c >= meta->count || d >= dim) return;
  const float* from = sum + c * dim + d;
  float x = 0.f;
  int s = 0;
  for (; s + 8 <= splits; s += 8) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = from[(s + i) * tokens * dim];
#pragma unroll
    for (int i = 0; i < 8; ++i) x += v[i];
  }
  for (; s < splits; ++s) x += from[s * tokens * dim];
  dH[index[c] * ld + d] = to16<El>(x * meta->down);
}

// ---- plans ---------------------------------------------------------------------------------------------------------

static uint64_t whole256(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// Rows of W that a backward pass takes at a time: so many that G takes no more than 256 MiB (what the chip's last cache holds), pieces of equal size.
constexpr int64_t kGradEntries = (int64_t)1 << 27, kMaxPiece = kMaxPitch / 4;
static int64_t piece_rows(int64_t tokens, int64_t vocab, int64_t piece) {
  int64_t most = piece > 0 ? piece : kGradEntries / (tokens > 1 ? tokens : 1);
  if (most > kMaxPiece) most = kMaxPiece;
  most = most / kTileP * kTileP;
  if (most < kTileP) most = kTileP;
  const int64_t pieces = ceil_div(vocab, most);
  return ceil_div(ceil_div(vocab, pieces), kTileP) * kTileP;
}

struct HeadPlan {
  int64_t piece, per_split, pitch_h;      // pitch_h: bytes
  int splits;
  uint64_t part, zlabel;                  // forward
  uint64_t meta, index, coef, lse, label, counts, q, hc, grad, sum, backward_bytes, forward_bytes;     // offsets, backward
};
static HeadPlan head_plan(int64_t tokens, int64_t vocab, int64_t dim, int64_t piece, int top) {
  HeadPlan p;
  p.piece = piece_rows(tokens, vocab, piece);
  p.pitch_h = line_pitch(2 * dim);
  // dH has few tiles where there are few tokens: then the piece's rows are cut, too
  const int64_t tiles = ceil_div(dim, kTileP) * ceil_div(tokens, tokens <= 64 ? 64 : tokens <= 128 ? 128 : 256);
  int64_t s = 256 / tiles;
  if (s > ceil_div(p.piece, 256)) s = ceil_div(p.piece, 256);
  if (s < 1) s = 1;
  p.per_split = ceil_div(ceil_div(p.piece, s), 64) * 64;
  p.splits = (int)ceil_div(p.piece, p.per_split);
  p.part = 0;
  p.zlabel = whole256((uint64_t)logit_tiles(tokens, true, vocab, dim).count * tokens * 8);
  p.forward_bytes = p.zlabel + whole256((uint64_t)tokens * 4);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t here = at; at += whole256(bytes); return here; };
  p.meta = take(sizeof(HeadMeta));
  p.index = take((uint64_t)tokens * 4);
  p.coef = take((uint64_t)tokens * 4);
  p.lse = take((uint64_t)tokens * 4);
  p.label = take((uint64_t)tokens * 4);
  p.counts = take((uint64_t)tokens * 4);
  p.q = take((uint64_t)tokens * top * 4);
  p.hc = take((uint64_t)tokens * p.pitch_h);
  p.grad = take((uint64_t)tokens * p.piece * 2);
  p.sum = take((uint64_t)p.splits * tokens * dim * 4);
  p.backward_bytes = at;
  return p;
}

// Tiles that launches may not have, with 128 tokens each (64 where there are no more; 256 in some): the logits of a piece, dH, dW of a piece.
static bool head_tiles_fit(int64_t tokens, int64_t vocab, int64_t dim, int64_t piece) {
  const int64_t rows = piece_rows(tokens, vocab, piece), tiles_t = ceil_div(tokens, 128), tiles_d = ceil_div(dim, kTileP);
  return tiles_fit(ceil_div(rows, kTileP), tiles_t, kTileThreads) && tiles_fit(tiles_d, tiles_t, kTileThreads) && tiles_fit(tiles_d, ceil_div(rows, 128), kTileThreads);
}
static bool head_sizes(int64_t tokens, int64_t vocab, int64_t dim, int64_t piece, int64_t top) {
  return tokens >= 0 && vocab >= 1 && dim >= 1 && piece >= 0 && top >= 0 && dim < kMaxPitch / 2 && tokens < (int64_t)1 << 30 && vocab < (int64_t)1 << 30 &&
         ceil_div(vocab, kTileP) * ceil_div(tokens, 16) <= kMaxGrid && tokens <= kMaxGrid / ceil_div(dim, 256) && (top == 0 || tokens <= kMaxGrid / top) &&
         head_tiles_fit(tokens, vocab, dim, piece);
}
static bool half_type(int dtype) { return dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16; }

#define BRSVD_LOGITS(KERNEL, El, DIRECT, bl, grid, stream, args)                                                  \
  do {                                                                                                           \
    const dim3 few(Logits<El, true, 16>::kThreads);                                                              \
    if (bl == 256 && DIRECT) hipLaunchKernelGGL((KERNEL<El, true, 256>), grid, dim3(kTileThreads), 0, stream, args); \
    else if (bl >= 128) hipLaunchKernelGGL((KERNEL<El, DIRECT, 128>), grid, dim3(kTileThreads), 0, stream, args); \
    else if (bl == 64) hipLaunchKernelGGL((KERNEL<El, true, 64>), grid, few, 0, stream, args);                    \
    else if (bl == 32) hipLaunchKernelGGL((KERNEL<El, true, 32>), grid, few, 0, stream, args);                    \
    else hipLaunchKernelGGL((KERNEL<El, true, 16>), grid, few, 0, stream, args);                                  \
  } while (0)
#define BRSVD_BY_TILE(KERNEL, El, DIRECT, grid, stream, args)                                                    \
  do {                                                                                                           \
    if (bq == 256 && DIRECT) hipLaunchKernelGGL((KERNEL<El, true, 256>), grid, dim3(kTileThreads), 0, stream, args); \
    else if (bq >= 128) hipLaunchKernelGGL((KERNEL<El, DIRECT, 128>), grid, dim3(kTileThreads), 0, stream, args); \
    else hipLaunchKernelGGL((KERNEL<El, DIRECT, 64>), grid, dim3(kTileThreads), 0, stream, args);                 \
  } while (0)

struct HeadCall {
  const void *H, *W;
  int64_t ldh, ldw, tokens, vocab, dim;
  int dtype;
  const int64_t* label;
  Teacher teacher;
  float scale;
};

static Operand rows_of(const void* base, int64_t ld, int64_t n) { return Operand{(const char*)base, 2 * ld, n}; }

template <class El>
static int head_forward(const HeadCall& c, const HeadPlan& plan, char* ws, float* loss, float* lse, float* z, hipStream_t stream) {
  HeadArgs g = {};
  g.W = rows_of(c.W, c.ldw, c.vocab);
  g.H = rows_of(c.H, c.ldh, c.tokens);
  g.dim = c.dim;
  g.scale = c.scale;
  const bool direct = aligned_pieces(c.W, 2 * c.ldw) && aligned_pieces(c.H, 2 * c.ldh);
  const LogitTiles tiles = logit_tiles(c.tokens, direct, c.vocab, c.dim);
  g.label = c.label;
  g.part = (float2*)(ws + plan.part);
  g.zlabel = (float*)(ws + plan.zlabel);
  auto launch = [&](int64_t tiles_v, int bl) {
    g.tiles_v = tiles_v;
    g.tiles_t = ceil_div(c.tokens, bl);
    unsigned workgroups = tile_workgroups(g.tiles_v, g.tiles_t);
    if (bl >= 128 && workgroups > 256) workgroups = 256;        // as many as run at once
    const dim3 grid(workgroups);
    if (direct) BRSVD_LOGITS(k_head_lse, El, true, bl, grid, stream, g);
    else BRSVD_LOGITS(k_head_lse, El, false, bl, grid, stream, g);
  };
  if (tiles.first > 0) launch(tiles.first, 256);
  if (tiles.first < tiles.count) {
    g.first = tiles.large;
    g.part += tiles.first * c.tokens;
    launch(tiles.count - tiles.first, tiles.bl);
  }
  in_launches(ceil_div(c.tokens, 16), 256, [&](unsigned first, dim3 grid) {
    hipLaunchKernelGGL(k_head_join, grid, dim3(256), 0, stream, (const float2*)(ws + plan.part), tiles.count, c.tokens, c.label, c.vocab, g.zlabel, lse, loss, first);
  });
  if (!c.label)
    in_launches(c.tokens, 256, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL(k_distill_loss<El>, grid, dim3(256), 0, stream, g.W, g.H, c.dim, c.teacher, lse, z, loss, first);
    });
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

template <class El>
static int head_backward(const HeadCall& c, const HeadPlan& plan, char* ws, const float* lse, const float* z, const float* grad, int64_t grad_stride, void* dH,
                         int64_t lddh, void* dW, int64_t lddw, hipStream_t stream) {
  HeadMeta* meta = (HeadMeta*)(ws + plan.meta);
  int *index = (int*)(ws + plan.index), *label_c = (int*)(ws + plan.label), *counts = (int*)(ws + plan.counts);
  float *coef = (float*)(ws + plan.coef), *lse_c = (float*)(ws + plan.lse), *q = (float*)(ws + plan.q), *sum = (float*)(ws + plan.sum);
  char* hc = ws + plan.hc;
  uint16_t* G = (uint16_t*)(ws + plan.grad);
  const Operand H = rows_of(c.H, c.ldh, c.tokens);
  if (!c.label)
    in_launches(ceil_div(c.tokens, 4), 256, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL(k_distill_targets, grid, dim3(256), 0, stream, c.teacher, c.tokens, c.vocab, q, counts, first);
    });
  hipLaunchKernelGGL(k_head_prepare, dim3(1), dim3(1024), 0, stream, c.label, c.vocab, counts, c.tokens, grad, grad_stride, 1.f / c.scale, meta, index, coef);
  in_launches(c.tokens, 256, [&](unsigned first, dim3 grid) {
    hipLaunchKernelGGL(k_head_gather, grid, dim3(256), 0, stream, H, c.dim, c.vocab, meta, index, lse, c.label, counts, hc, plan.pitch_h, lse_c, coef, label_c,
                       (uint16_t*)dH, lddh, first);
  });
  const bool direct = aligned_pieces(c.W, 2 * c.ldw);
  const int bq = large_token_tiles(c.tokens, direct, ceil_div(c.dim, kTileP) * plan.splits, plan.per_split) > 0 ? 256 : small_tile(c.tokens);
  const int64_t tiles_t = ceil_div(c.tokens, bq);
  for (int64_t v0 = 0; v0 < c.vocab; v0 += plan.piece) {
    const int64_t rows = c.vocab - v0 < plan.piece ? c.vocab - v0 : plan.piece;
    HeadArgs g = {};
    g.W = rows_of((const uint16_t*)c.W + v0 * c.ldw, c.ldw, rows);
    g.H = Operand{hc, plan.pitch_h, c.tokens};
    g.dim = c.dim;
    g.scale = c.scale;
    g.meta = meta;
    g.lse = lse_c;
    g.coef = coef;
    g.label_c = label_c;
    g.v0 = v0;
    g.G = G;
    g.pitch = plan.piece;
    const LogitTiles tiles = logit_tiles(c.tokens, direct, rows, c.dim);
    auto launch = [&](int64_t tiles_v, int bl) {
      g.tiles_v = tiles_v;
      g.tiles_t = ceil_div(c.tokens, bl);
      const dim3 grid(tile_workgroups(g.tiles_v, g.tiles_t));
      if (direct) BRSVD_LOGITS(k_head_grad, El, true, bl, grid, stream, g);
      else BRSVD_LOGITS(k_head_grad, El, false, bl, grid, stream, g);
    };
    if (tiles.first > 0) launch(tiles.first, 256);
    if (tiles.first < tiles.count) {
      g.first = tiles.large;
      launch(tiles.count - tiles.first, tiles.bl);
    }
    if (!c.label)
      in_launches(ceil_div(c.tokens * c.teacher.top, 256), 256, [&](unsigned first, dim3 grid) {
        hipLaunchKernelGGL(k_distill_scatter<El>, grid, dim3(256), 0, stream, c.teacher, q, z, meta, index, lse_c, coef, v0, rows, c.vocab, G, plan.piece, first);
      });
    if (dH) {
      HeadProduct h = {};
      h.P = Operand{g.W.base, g.W.ld, c.dim};
      h.Q = Operand{(const char*)G, 2 * plan.piece, c.tokens};
      h.k = rows;
      h.per_split = plan.per_split;
      h.meta = meta;
      h.tiles_p = ceil_div(c.dim, kTileP);
      h.tiles_q = tiles_t;
      h.sum = sum;
      h.more = v0 > 0;
      const dim3 hg(tile_workgroups(h.tiles_p, h.tiles_q), (unsigned)plan.splits);
      if (direct) BRSVD_BY_TILE(k_head_dh, El, true, hg, stream, h);
      else BRSVD_BY_TILE(k_head_dh, El, false, hg, stream, h);
    }
    if (dW) {
      HeadProduct w = {};
      // rows of both end behind whole pieces: what a piece holds beyond the last column goes into sums that are not stored
      w.P = Operand{hc, plan.pitch_h, ceil_div(c.dim, 8) * 8};
      w.Q = Operand{(const char*)G, 2 * plan.piece, ceil_div(rows, 8) * 8};
      w.words = rows;
      w.width = c.dim;
      w.meta = meta;
      w.tiles_p = ceil_div(c.dim, kTileP);
      w.out = (uint16_t*)dW + v0 * lddw;
      w.ldo = lddw;
      const int64_t all = ceil_div(rows, 256), large = large_tiles(all, w.tiles_p, 2 * w.tiles_p, ceil_div(c.tokens, 64));
      w.tiles_q = large;
      if (large > 0) hipLaunchKernelGGL((k_head_dw<El, 256>), dim3(tile_workgroups(w.tiles_p, w.tiles_q)), dim3(kTileThreads), 0, stream, w);
      if (large < all) {
        w.first = 256 * large;
        w.tiles_q = ceil_div(rows - w.first, 128);
        hipLaunchKernelGGL((k_head_dw<El, 128>), dim3(tile_workgroups(w.tiles_p, w.tiles_q)), dim3(kTileThreads), 0, stream, w);
      }
    }
  }
  // a last piece that is shorter than the others may leave splits without rows: their parts hold what the pieces before gave
  const int64_t first = c.vocab < plan.piece ? c.vocab : plan.piece;
  const int splits = (int)ceil_div(first, plan.per_split);
  if (dH)
    in_launches(c.tokens * ceil_div(c.dim, 256), 256, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL(k_head_finish<El>, grid, dim3(256), 0, stream, sum, splits, c.tokens, c.dim, meta, index, (uint16_t*)dH, lddh, first);
    });
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

// Refusals that all calls share
static int check_head(const HeadCall& c, int64_t piece) {
  if (!half_type(c.dtype) || !head_sizes(c.tokens, c.vocab, c.dim, piece, c.teacher.top)) return BRSVD_ERR_ARG;
  if (!c.label && !(c.scale > 0.f && c.scale <= 3.402823466e38f)) return BRSVD_ERR_ARG;
  if (c.tokens > 0 && (!c.H || c.ldh < c.dim || c.ldh >= kMaxPitch / 2)) return BRSVD_ERR_ARG;
  if (!c.W || c.ldw < c.dim || c.ldw >= kMaxPitch / 2) return BRSVD_ERR_ARG;
  return BRSVD_OK;
}
static int check_workspace(const void* ws, uint64_t have, uint64_t need) {
  if (!ws || (uintptr_t)ws % 256) return BRSVD_ERR_ARG;
  return have < need ? BRSVD_ERR_BUDGET : BRSVD_OK;
}

}  // namespace brsvd

using namespace brsvd;

extern "C" uint64_t brsvd_head_workspace_bytes(int64_t tokens, int64_t vocab, int64_t dim, int64_t piece, int32_t top, int32_t backward) {
  if (!head_sizes(tokens, vocab, dim, piece, top) || tokens == 0) return 0;
  const HeadPlan p = head_plan(tokens, vocab, dim, piece, top);
  return backward ? p.backward_bytes : p.forward_bytes;
}

extern "C" int brsvd_xent_forward(const void* H, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels, int64_t tokens, int64_t vocab, int64_t dim,
                                  int32_t dtype, float* loss, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  const HeadCall c{H, W, ldh, ldw, tokens, vocab, dim, dtype, labels, Teacher{}, 1.f};
  if (tokens > 0 && (!labels || !loss || !lse)) return BRSVD_ERR_ARG;
  if (!half_type(dtype) || !head_sizes(tokens, vocab, dim, 0, 0)) return BRSVD_ERR_ARG;
  if (tokens == 0) return BRSVD_OK;
  BRSVD_TRY(check_head(c, 0));
  const HeadPlan p = head_plan(tokens, vocab, dim, 0, 0);
  BRSVD_TRY(check_workspace(workspace, workspace_bytes, p.forward_bytes));
  hipStream_t s = (hipStream_t)stream;
  return dtype == BRSVD_DTYPE_BF16 ? head_forward<Bf16>(c, p, (char*)workspace, loss, lse, nullptr, s) : head_forward<Fp16>(c, p, (char*)workspace, loss, lse, nullptr, s);
}

extern "C" int brsvd_distill_forward(const void* H, int64_t ldh, const void* W, int64_t ldw, const int64_t* ids, const float* logits, int32_t top, float temperature,
                                     int64_t tokens, int64_t vocab, int64_t dim, int32_t dtype, float* loss, float* lse, float* z, void* workspace,
                                     uint64_t workspace_bytes, void* stream) {
  const HeadCall c{H, W, ldh, ldw, tokens, vocab, dim, dtype, nullptr, Teacher{ids, logits, top, 1.f / temperature}, 1.f / temperature};
  if (top < 1 || !(temperature > 0.f) || (tokens > 0 && (!ids || !logits || !loss || !lse || !z))) return BRSVD_ERR_ARG;
  if (!half_type(dtype) || !head_sizes(tokens, vocab, dim, 0, top)) return BRSVD_ERR_ARG;
  if (tokens == 0) return BRSVD_OK;
  BRSVD_TRY(check_head(c, 0));
  const HeadPlan p = head_plan(tokens, vocab, dim, 0, top);
  BRSVD_TRY(check_workspace(workspace, workspace_bytes, p.forward_bytes));
  hipStream_t s = (hipStream_t)stream;
  return dtype == BRSVD_DTYPE_BF16 ? head_forward<Bf16>(c, p, (char*)workspace, loss, lse, z, s) : head_forward<Fp16>(c, p, (char*)workspace, loss, lse, z, s);
}

// Backward of either loss; with no tokens dW is zero
static int head_backward_call(const HeadCall& c, int64_t piece, const float* lse, const float* z, const float* grad, int64_t grad_stride, void* dH, int64_t lddh,
                              void* dW, int64_t lddw, void* workspace, uint64_t workspace_bytes, hipStream_t s) {
  if ((c.tokens > 0 && !dH && !dW) || grad_stride < 0) return BRSVD_ERR_ARG;      // of no tokens dH has no elements and may be NULL
  BRSVD_TRY(check_head(c, piece));
  if ((dH && lddh < c.dim) || (dW && lddw < c.dim)) return BRSVD_ERR_ARG;
  if (c.tokens == 0) {
    if (!dW) return BRSVD_OK;
    in_launches(c.vocab, 256, [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(k_head_zero, grid, dim3(256), 0, s, (uint16_t*)dW, lddw, c.dim, first); });
    BRSVD_HIP_TRY(hipGetLastError());
    return BRSVD_OK;
  }
  if (!lse || !grad) return BRSVD_ERR_ARG;
  const HeadPlan p = head_plan(c.tokens, c.vocab, c.dim, piece, c.teacher.top);
  BRSVD_TRY(check_workspace(workspace, workspace_bytes, p.backward_bytes));
  char* ws = (char*)workspace;
  return c.dtype == BRSVD_DTYPE_BF16 ? head_backward<Bf16>(c, p, ws, lse, z, grad, grad_stride, dH, lddh, dW, lddw, s)
                                     : head_backward<Fp16>(c, p, ws, lse, z, grad, grad_stride, dH, lddh, dW, lddw, s);
}

extern "C" int brsvd_xent_backward(const void* H, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels, const float* lse, const float* grad,
                                   int64_t grad_stride, int64_t tokens, int64_t vocab, int64_t dim, int64_t piece, int32_t dtype, void* dH, int64_t lddh, void* dW,
                                   int64_t lddw, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (tokens > 0 && !labels) return BRSVD_ERR_ARG;
  static const int64_t none = -1;      // of a call without tokens, never read
  const HeadCall c{H, W, ldh, ldw, tokens, vocab, dim, dtype, labels ? labels : &none, Teacher{}, 1.f};
  return head_backward_call(c, piece, lse, nullptr, grad, grad_stride, dH, lddh, dW, lddw, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" int brsvd_distill_backward(const void* H, int64_t ldh, const void* W, int64_t ldw, const int64_t* ids, const float* logits, int32_t top, float temperature,
                                      const float* lse, const float* z, const float* grad, int64_t grad_stride, int64_t tokens, int64_t vocab, int64_t dim,
                                      int64_t piece, int32_t dtype, void* dH, int64_t lddh, void* dW, int64_t lddw, void* workspace, uint64_t workspace_bytes,
                                      void* stream) {
  if (top < 1 || !(temperature > 0.f) || (tokens > 0 && (!ids || !logits || !z))) return BRSVD_ERR_ARG;
  const HeadCall c{H, W, ldh, ldw, tokens, vocab, dim, dtype, nullptr, Teacher{ids, logits, top, 1.f / temperature}, 1.f / temperature};
  return head_backward_call(c, piece, lse, z, grad, grad_stride, dH, lddh, dW, lddw, workspace, workspace_bytes, (hipStream_t)stream);
}
