// Casting a matrix into 8 bits with a scale for each block, and back.
//   s_b = 2^e, the least e with max |x| <= 448 * 2^e over the block;  q = e4m3(x / s_b)
// A block is 128 numbers of one row, or 128 rows of them (128 x 128).  The transpose is cast too where it is wanted (its blocks run down the
// columns), from one read.
#include "e4m3.h"
#include "tile.h"

namespace brsvd {

// How a workgroup of 256 threads lies over a 128 x 128 part: a thread has 16 bytes (kWide numbers) of each of kRows rows that follow each other, so
// that 16 (fp32: 32) lanes read a row's 128 numbers as one piece of memory, and the kRows numbers of a column in a thread are neighbours in the
// transpose.
template <int DT> struct Part {
  static constexpr int kBytes = DT == BRSVD_DTYPE_F32 ? 4 : 2, kWide = 16 / kBytes, kLanes = kBlock / kWide, kRows = kBlock / (256 / kLanes);
};

// The numbers of 16 bytes from `src` on, of which `valid` are there.
template <int DT>
__device__ __forceinline__ void numbers(const char* src, int valid, float (&x)[Part<DT>::kWide]) {
  constexpr int EB = Part<DT>::kBytes;
  const uint4 v = piece_of<EB>(src, valid * EB);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < Part<DT>::kWide; ++i)
    x[i] = EB == 4 ? __uint_as_float(w[EB == 4 ? i : 0])
                   : DT == BRSVD_DTYPE_BF16 ? from16<Bf16>((uint16_t)(w[i / 2] >> (16 * (i & 1)))) : from16<Fp16>((uint16_t)(w[i / 2] >> (16 * (i & 1))));
}

// N bytes to memory at any address, of which `valid` are wanted
template <int N>
__device__ __forceinline__ void put_bytes(void* dst, int valid, const uint32_t (&v)[N / 4]) {
  struct __attribute__((packed, aligned(1))) Bytes { uint32_t x[N / 4]; };
  if (valid >= N) {
    Bytes b;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) b.x[i] = v[i];
    *(Bytes*)dst = b;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < valid) ((uint8_t*)dst)[i] = (uint8_t)(v[i / 4] >> (8 * (i & 3)));
  }
}

// Largest of 16 neighbouring lanes, in all of them (rotations inside a row of 16: no LDS)
__device__ __forceinline__ float max16(float x) {
#define BRSVD_ROTATED_MAX(N) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, true)))
  BRSVD_ROTATED_MAX(8);
  BRSVD_ROTATED_MAX(4);
  BRSVD_ROTATED_MAX(2);
  BRSVD_ROTATED_MAX(1);
#undef BRSVD_ROTATED_MAX
  return x;
}

// Magnitudes in a word of memory as it is, one number or two: keys that order as they do, and below all of them what is not finite.  A largest key costs three
// instructions for two numbers of 16 bits, their floats twice that each.
template <int DT> struct Keys {
  typedef short Two __attribute__((ext_vector_type(2)));
  static constexpr uint32_t kFrom = DT == BRSVD_DTYPE_F32 ? 0x00800000u : DT == BRSVD_DTYPE_BF16 ? 0x0080u : 0x0400u;    // of zero
  static constexpr uint32_t kNone = DT == BRSVD_DTYPE_F32 ? kFrom : kFrom << 16 | kFrom;
  static __device__ __forceinline__ uint32_t of(uint32_t w) {
    if (DT == BRSVD_DTYPE_F32) return (w & 0x7fffffffu) + kFrom;
    const Two from = {(short)kFrom, (short)kFrom};
    return __builtin_bit_cast(uint32_t, (Two)(__builtin_bit_cast(Two, w & 0x7fff7fffu) + from));
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    if (DT == BRSVD_DTYPE_F32) return (uint32_t)max((int32_t)a, (int32_t)b);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Two, a), __builtin_bit_cast(Two, b)));
  }
  // the magnitude of a word's number i
  static __device__ __forceinline__ float magnitude(uint32_t key, int i) {
    if (DT == BRSVD_DTYPE_F32) return __uint_as_float(key - kFrom);
    const uint16_t h = (uint16_t)((uint16_t)(key >> (16 * i)) - kFrom);
    return DT == BRSVD_DTYPE_BF16 ? from16<Bf16>(h) : from16<Fp16>(h);
  }
  // of a word's numbers
  static __device__ __forceinline__ float largest(uint32_t key) {
    return DT == BRSVD_DTYPE_F32 ? magnitude(key, 0) : fmaxf(magnitude(key, 0), magnitude(key, 1));
  }
  // of 16 neighbouring lanes, in all of them
  static __device__ __forceinline__ uint32_t largest16(uint32_t x) {
#define BRSVD_ROTATED_KEYS(N) x = larger(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, true))
    BRSVD_ROTATED_KEYS(8);
    BRSVD_ROTATED_KEYS(4);
    BRSVD_ROTATED_KEYS(2);
    BRSVD_ROTATED_KEYS(1);
#undef BRSVD_ROTATED_KEYS
    return x;
  }
};
template <int DT>
__device__ __forceinline__ float number_of(const uint32_t (&w)[4], int j) {
  if (DT == BRSVD_DTYPE_F32) return __uint_as_float(w[j & 3]);
  const uint16_t h = (uint16_t)(w[j / 2 & 3] >> (16 * (j & 1)));
  return DT == BRSVD_DTYPE_BF16 ? from16<Bf16>(h) : from16<Fp16>(h);
}

// One workgroup per 128 x 128 part.  Bound by memory: what it reads and writes once.  Numbers stay as they came in registers, so that all workgroups of a
// matrix of some 4000 x 6000 run at once: 4001 x 6000 bf16 by rows with its transpose 24 us (96 MB, 3.9 TB/s), 27 with floats.  The transpose goes through LDS in words of a thread's kRows
// numbers of a column, word g of column c at g ^ (c / kWide): the lanes that write, and those that read, then lie in different banks.
template <int DT, bool SQUARE, bool STRAIGHT, bool TRANSPOSED>
__global__ void __launch_bounds__(256)
k_quantize(const char* __restrict__ X, int64_t ldx, int64_t rows, int64_t cols, uint8_t* __restrict__ Q, int64_t ldq, float* __restrict__ S,
           uint8_t* __restrict__ Qt, int64_t ldqt, float* __restrict__ St, unsigned first_wg) {
  using P = Part<DT>;
  using K = Keys<DT>;
  constexpr int W = P::kWide, R = P::kRows, L = P::kLanes, GROUPS = kBlock / R;
  __shared__ uint32_t top[4][4 * L];
  __shared__ __attribute__((aligned(16))) uint8_t turned[TRANSPOSED ? kBlock * kBlock : 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid % L, c = cg * W, g = tid / L;
  const int64_t ncb = (cols + kBlock - 1) / kBlock, nrb = (rows + kBlock - 1) / kBlock;
  const unsigned wg = first_wg + blockIdx.x;
  const int64_t rb = wg / (unsigned)ncb, cb = wg % (unsigned)ncb, row0 = rb * kBlock, col0 = cb * kBlock;
  const int width = (int)(cols - col0 - c < W ? (cols - col0 - c > 0 ? cols - col0 - c : 0) : W);
  uint32_t x[R][4];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t row = row0 + g * R + i;
    const uint4 v = piece_of<P::kBytes>(X + row * ldx + (col0 + c) * P::kBytes, row < rows ? width * P::kBytes : 0);
    x[i][0] = v.x; x[i][1] = v.y; x[i][2] = v.z; x[i][3] = v.w;
  }
  // the numbers' floats are worked out again where they are used: kept, they would double the registers
  auto again = [&] {
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(x[i][j]));
  };
  auto row_key = [&](int i) { return K::larger(K::larger(K::of(x[i][0]), K::of(x[i][1])), K::larger(K::of(x[i][2]), K::of(x[i][3]))); };
  float f_square = 1.f;
  if (SQUARE) {
    uint32_t all = K::kNone;
#pragma unroll
    for (int i = 0; i < R; ++i) all = K::larger(all, row_key(i));
    all = K::largest16(all);
    all = K::larger(all, __shfl_xor(all, 16));
    all = K::larger(all, __shfl_xor(all, 32));
    if (lane == 0) top[wave][0] = all;
    __syncthreads();
    const int e = block_exponent(K::largest(K::larger(K::larger(top[0][0], top[1][0]), K::larger(top[2][0], top[3][0]))));
    f_square = power_of_two(-e);
    if (tid == 0 && STRAIGHT) S[rb * ncb + cb] = power_of_two(e);
    if (tid == 0 && TRANSPOSED) St[cb * nrb + rb] = power_of_two(e);
  }
  if (STRAIGHT) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t row = row0 + g * R + i;
      float f = f_square;
      if (!SQUARE) {
        uint32_t t = K::larger(K::kNone, K::largest16(row_key(i)));
        if (L == 32) t = K::larger(t, __shfl_xor(t, 16));
        const int e = block_exponent(K::largest(t));
        f = power_of_two(-e);
        if (row < rows && cg == 0) S[row * ncb + cb] = power_of_two(e);
      }
      uint32_t v[W / 4];
#pragma unroll
      for (int j = 0; j < W; j += 4)
        v[j / 4] = pack_e4m3(number_of<DT>(x[i], j) * f, number_of<DT>(x[i], j + 1) * f, number_of<DT>(x[i], j + 2) * f, number_of<DT>(x[i], j + 3) * f);
      if (row < rows) put_bytes<W>(Q + row * ldq + col0 + c, width, v);
    }
  }
  if (TRANSPOSED) {
    float f[W];
    again();
    if (!SQUARE) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t t = K::kNone;
#pragma unroll
        for (int i = 0; i < R; ++i) t = K::larger(t, K::of(x[i][j]));
        if (L == 16) t = K::larger(t, __shfl_xor(t, 16));
        t = K::larger(t, __shfl_xor(t, 32));
        if (lane < L) top[wave][4 * cg + j] = t;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const int w = 4 * cg + j * 4 / W;
        const int e = block_exponent(K::magnitude(K::larger(K::larger(top[0][w], top[1][w]), K::larger(top[2][w], top[3][w])), j % (W / 4)));
        f[j] = power_of_two(-e);
        if (g == 0 && j < width) St[(col0 + c + j) * nrb + rb] = power_of_two(e);
      }
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) f[j] = f_square;
    }
#pragma unroll
    for (int j = 0; j < W; ++j) {
      uint32_t v[R / 4];
#pragma unroll
      for (int i = 0; i < R; i += 4)
        v[i / 4] = pack_e4m3(number_of<DT>(x[i], j) * f[j], number_of<DT>(x[i + 1], j) * f[j], number_of<DT>(x[i + 2], j) * f[j], number_of<DT>(x[i + 3], j) * f[j]);
      uint8_t* at = turned + (c + j) * kBlock + R * (g ^ (cg & (GROUPS - 1)));
      if (R == 16) *(uint4*)at = make_uint4(v[0], v[1], v[R / 4 - 2], v[R / 4 - 1]);
      else *(uint2*)at = make_uint2(v[0], v[1]);
    }
    __syncthreads();
    // eight threads a column, 16 bytes each
    const int part = tid & 7;
    const int height = (int)(rows - row0 - 16 * part < 16 ? rows - row0 - 16 * part : 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int cc = (tid >> 3) + 32 * i, mix = cc / W & (GROUPS - 1);
      if (col0 + cc >= cols || height <= 0) continue;
      const uint8_t* at = turned + cc * kBlock;
      uint32_t v[4];
      if (R == 16) {
        const uint4 w = *(const uint4*)(at + 16 * (part ^ mix));
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
      } else {
        const uint2 lo = *(const uint2*)(at + 8 * ((2 * part) ^ mix)), hi = *(const uint2*)(at + 8 * ((2 * part + 1) ^ mix));
        v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
      }
      put_bytes<16>(Qt + (col0 + cc) * ldqt + row0 + 16 * part, height, v);
    }
  }
}

// Blocks of a row by themselves: 16 (fp32: 32) lanes a block, the blocks of a row one after the other, SETS of them a thread at once: enough reads on their
// way for the memory, which is the bound.  8192 x 8192 bf16 37 us (201 MB, 5.4 TB/s); small parts, so that small matrices reach all CUs.
template <int DT>
__global__ void __launch_bounds__(256)
k_quantize_rows(const char* __restrict__ X, int64_t ldx, int64_t rows, int64_t cols, uint8_t* __restrict__ Q, int64_t ldq, float* __restrict__ S, unsigned first_wg) {
  using P = Part<DT>;
  constexpr int W = P::kWide, L = P::kLanes, SETS = 4;
  const int cg = threadIdx.x % L;
  const unsigned ncb = (unsigned)((cols + kBlock - 1) / kBlock);
  const int64_t first = ((int64_t)first_wg + blockIdx.x) * (256 / L * SETS) + threadIdx.x / L, blocks = rows * ncb;
  float x[SETS][W];
  int64_t row[SETS], col[SETS];
  int width[SETS];
#pragma unroll
  for (int i = 0; i < SETS; ++i) {
    const int64_t b = first + i * (256 / L);
    row[i] = b / ncb;
    col[i] = (b - row[i] * ncb) * kBlock + cg * W;
    const int64_t left = b < blocks ? cols - col[i] : 0;
    width[i] = (int)(left < W ? (left > 0 ? left : 0) : W);
    numbers<DT>(X + row[i] * ldx + col[i] * P::kBytes, width[i], x[i]);
  }
#pragma unroll
  for (int i = 0; i < SETS; ++i) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) t = fmaxf(t, finite_abs(x[i][j]));
    t = max16(t);
    if (L == 32) t = fmaxf(t, __shfl_xor(t, 16));
    const int e = block_exponent(t);
    const float f = power_of_two(-e);
    uint32_t v[W / 4];
#pragma unroll
    for (int j = 0; j < W; j += 4) v[j / 4] = pack_e4m3(x[i][j] * f, x[i][j + 1] * f, x[i][j + 2] * f, x[i][j + 3] * f);
    put_bytes<W>(Q + row[i] * ldq + col[i], width[i], v);
    const int64_t b = first + i * (256 / L);
    if (cg == 0 && b < blocks) S[b] = power_of_two(e);
  }
}

// 128 x 128 blocks by themselves: a wave reads 1 KiB of a row at a time, 2 (16-bit: 4) blocks next to each other, the waves share the 128 rows.  Bound by
// memory: 20000 x 20000 fp32 455 us (2.0 GB, 4.4 TB/s).
template <int DT>
__global__ void __launch_bounds__(DT == BRSVD_DTYPE_F32 ? 512 : 1024)
k_quantize_square(const char* __restrict__ X, int64_t ldx, int64_t rows, int64_t cols, uint8_t* __restrict__ Q, int64_t ldq, float* __restrict__ S, unsigned first_wg) {
  using P = Part<DT>;
  constexpr int W = P::kWide, L = P::kLanes, BLOCKS = 64 / L, WAVES = DT == BRSVD_DTYPE_F32 ? 8 : 16, R = kBlock / WAVES;
  __shared__ float top[WAVES][BLOCKS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = lane / L;
  const unsigned wg = first_wg + blockIdx.x, ncb = (unsigned)((cols + kBlock - 1) / kBlock), across = (ncb + BLOCKS - 1) / BLOCKS, rb = wg / across, cb = (wg % across) * BLOCKS;
  const int64_t row0 = (int64_t)rb * kBlock + wave * R, col = (int64_t)cb * kBlock + lane * W;
  const int width = (int)(cols - col < W ? (cols - col > 0 ? cols - col : 0) : W);
  float x[R][W], t = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) numbers<DT>(X + (row0 + i) * ldx + col * P::kBytes, row0 + i < rows ? width : 0, x[i]);
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < W; ++j) t = fmaxf(t, finite_abs(x[i][j]));
  t = max16(t);
  if (L == 32) t = fmaxf(t, __shfl_xor(t, 16));
  if (lane % L == 0) top[wave][mine] = t;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) t = fmaxf(t, top[w][mine]);
  const int e = block_exponent(t);
  const float f = power_of_two(-e);
  if (wave == 0 && lane % L == 0 && cb + mine < ncb) S[(int64_t)rb * ncb + cb + mine] = power_of_two(e);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    uint32_t v[W / 4];
#pragma unroll
    for (int j = 0; j < W; j += 4) v[j / 4] = pack_e4m3(x[i][j] * f, x[i][j + 1] * f, x[i][j + 2] * f, x[i][j + 3] * f);
    if (row0 + i < rows) put_bytes<W>(Q + (row0 + i) * ldq + col, width, v);
  }
}

// X = Q * S: a thread writes 16 bytes of X at a time, neighbouring lanes neighbouring pieces, four rows.  Bound by memory: 20000 x 20000 fp32 357 us (2.0 GB,
// 5.6 TB/s).
template <int DT>
__global__ void __launch_bounds__(256)
k_dequantize(const uint8_t* __restrict__ Q, int64_t ldq, const float* __restrict__ S, int64_t rows, int64_t cols, int block_rows, char* __restrict__ X, int64_t ldx,
             unsigned first_wg) {
  using P = Part<DT>;
  constexpr int W = P::kWide, R = 4, STEP = 256 / P::kLanes;
  const int c = (int)(threadIdx.x % P::kLanes) * W, r = threadIdx.x / P::kLanes;
  const unsigned wg = first_wg + blockIdx.x;
  const int64_t ncb = (cols + kBlock - 1) / kBlock, rb = wg / (unsigned)ncb, cb = wg % (unsigned)ncb, col = cb * kBlock + c, row0 = rb * (STEP * R) + r;
  const int width = (int)(cols - col < W ? cols - col : W);
  if (width <= 0) return;
  uint32_t w[R][W / 4];
  float f[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t row = row0 + STEP * i;
    if (row >= rows) continue;
    const uint8_t* src = Q + row * ldq + col;
    f[i] = S[(block_rows == 1 ? row : row / kBlock) * ncb + cb];
    struct __attribute__((packed, aligned(1))) Bytes { uint32_t x[W / 4]; };
    if (width == W) {
      const Bytes v = *(const Bytes*)src;
#pragma unroll
      for (int j = 0; j < W / 4; ++j) w[i][j] = v.x[j];
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        if (j % 4 == 0) w[i][j / 4] = 0;
        if (j < width) w[i][j / 4] |= (uint32_t)src[j] << (8 * (j & 3));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t row = row0 + STEP * i;
    if (row >= rows) continue;
    float x[W];
#pragma unroll
    for (int j = 0; j < W / 4; ++j) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i][j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i][j], true);
      x[4 * j] = lo[0] * f[i];
      x[4 * j + 1] = lo[1] * f[i];
      x[4 * j + 2] = hi[0] * f[i];
      x[4 * j + 3] = hi[1] * f[i];
    }
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (DT == BRSVD_DTYPE_F32) v[j] = __float_as_uint(x[W == 4 ? j : 0]);
      else if (DT == BRSVD_DTYPE_BF16) v[j] = to16<Bf16>(x[W == 8 ? 2 * j : 0]) | (uint32_t)to16<Bf16>(x[W == 8 ? 2 * j + 1 : 0]) << 16;
      else v[j] = to16<Fp16>(x[W == 8 ? 2 * j : 0]) | (uint32_t)to16<Fp16>(x[W == 8 ? 2 * j + 1 : 0]) << 16;
    }
    put_bytes<16>(X + row * ldx + col * P::kBytes, width * P::kBytes, v);
  }
}

template <int DT, bool SQUARE>
static void launch_quantize(const char* X, int64_t ldx, int64_t rows, int64_t cols, uint8_t* Q, int64_t ldq, float* S, uint8_t* Qt, int64_t ldqt, float* St,
                            hipStream_t stream) {
  const int64_t parts = ceil_div(cols, kBlock) * ceil_div(rows, kBlock);
  const int64_t pitch = ldx * (DT == BRSVD_DTYPE_F32 ? 4 : 2);
  if (!SQUARE && !Qt) {
    in_launches(ceil_div(rows * ceil_div(cols, kBlock), 256 / Part<DT>::kLanes * 4), 256, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL(k_quantize_rows<DT>, grid, dim3(256), 0, stream, X, pitch, rows, cols, Q, ldq, S, first);
    });
  } else if (Q && Qt) {
    in_launches(parts, 256, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL((k_quantize<DT, SQUARE, true, true>), grid, dim3(256), 0, stream, X, pitch, rows, cols, Q, ldq, S, Qt, ldqt, St, first);
    });
  } else if (Q) {
    const int threads = DT == BRSVD_DTYPE_F32 ? 512 : 1024;
    in_launches(ceil_div(ceil_div(cols, kBlock), 64 / Part<DT>::kLanes) * ceil_div(rows, kBlock), threads, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL(k_quantize_square<DT>, grid, dim3(threads), 0, stream, X, pitch, rows, cols, Q, ldq, S, first);
    });
  } else {
    in_launches(parts, 256, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL((k_quantize<DT, SQUARE, false, true>), grid, dim3(256), 0, stream, X, pitch, rows, cols, Q, ldq, S, Qt, ldqt, St, first);
    });
  }
}

int quantize(const void* X, int64_t ldx, int64_t rows, int64_t cols, int dtype, int block_rows, uint8_t* Q, int64_t ldq, float* S, uint8_t* Qt, int64_t ldqt,
             float* St, hipStream_t stream) {
  const char* x = (const char*)X;
  const bool square = block_rows == kBlock;
#define BRSVD_QUANTIZE(DT)                                                                    \
  (square ? launch_quantize<DT, true>(x, ldx, rows, cols, Q, ldq, S, Qt, ldqt, St, stream)    \
          : launch_quantize<DT, false>(x, ldx, rows, cols, Q, ldq, S, Qt, ldqt, St, stream))
  if (dtype == BRSVD_DTYPE_F32) BRSVD_QUANTIZE(BRSVD_DTYPE_F32);
  else if (dtype == BRSVD_DTYPE_BF16) BRSVD_QUANTIZE(BRSVD_DTYPE_BF16);
  else BRSVD_QUANTIZE(BRSVD_DTYPE_F16);
#undef BRSVD_QUANTIZE
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

static bool model_type(int dtype) { return dtype == BRSVD_DTYPE_F32 || dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16; }

}  // namespace brsvd

using namespace brsvd;

extern "C" int brsvd_quantize_e4m3(const void* X, int64_t ldx, int64_t rows, int64_t cols, int32_t dtype, int32_t block_rows, uint8_t* Q, int64_t ldq,
                                   float* S, uint8_t* Qt, int64_t ldqt, float* St, void* stream) {
  if (rows < 0 || cols < 0 || !model_type(dtype) || (block_rows != 1 && block_rows != kBlock)) return BRSVD_ERR_ARG;
  if (rows == 0 || cols == 0) return BRSVD_OK;
  if (!X || (!Q && !Qt) || ldx < cols || (Q && (!S || ldq < cols)) || (Qt && (!St || ldqt < rows)) || ldx > INT64_MAX / 4 || cols > kMaxGrid * kBlock ||
      rows > (kMaxGrid << 2) / ceil_div(cols, kBlock))
    return BRSVD_ERR_ARG;
  return quantize(X, ldx, rows, cols, dtype, block_rows, Q, ldq, S, Qt, ldqt, St, (hipStream_t)stream);
}

extern "C" int brsvd_dequantize_e4m3(const uint8_t* Q, int64_t ldq, const float* S, int64_t rows, int64_t cols, int32_t block_rows, int32_t dtype, void* X,
                                     int64_t ldx, void* stream) {
  if (rows < 0 || cols < 0 || !model_type(dtype) || (block_rows != 1 && block_rows != kBlock)) return BRSVD_ERR_ARG;
  if (rows == 0 || cols == 0) return BRSVD_OK;
  if (!Q || !S || !X || ldq < cols || ldx < cols || ldx > INT64_MAX / 4 || cols > kMaxGrid * kBlock ||
      rows > (kMaxGrid << 2) / ceil_div(cols, kBlock))
    return BRSVD_ERR_ARG;
  const int64_t pitch = ldx * (dtype == BRSVD_DTYPE_F32 ? 4 : 2);
  in_launches(ceil_div(cols, kBlock) * ceil_div(rows, dtype == BRSVD_DTYPE_F32 ? 32 : 64), 256, [&](unsigned first, dim3 grid) {
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, Q, ldq, S, rows, cols, block_rows, (char*)X, pitch, first); };
    if (dtype == BRSVD_DTYPE_F32) launch(k_dequantize<BRSVD_DTYPE_F32>);
    else if (dtype == BRSVD_DTYPE_BF16) launch(k_dequantize<BRSVD_DTYPE_BF16>);
    else launch(k_dequantize<BRSVD_DTYPE_F16>);
  });
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}
