// Casting a matrix into 8 bits with a scale for each block, and back.
//   s_b = 2^e, the least e with max |x| <= 448 * 2^e over the block;  q = e4m3(x / s_b)
// A block is 128 numbers of one row, or 128 rows of them (128 x 128).  The transpose is cast too where it is wanted (its blocks run down the
// columns), from one read.
#include "e4m3.h"
#include "tile.h"

namespace brsvd {

// Eight numbers of a row from `src` on, of which `valid` are there.
template <int DT>
__device__ __forceinline__ void eight(const char* src, int valid, float (&x)[8]) {
  constexpr int EB = DT == BRSVD_DTYPE_F32 ? 4 : 2;
  if (valid >= 8) {
    uint32_t w[2 * EB];
#pragma unroll
    for (int i = 0; i < EB / 2; ++i) {
      const Piece v = *(const Piece*)(src + 16 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = v.x[j];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = DT == BRSVD_DTYPE_F32 ? __uint_as_float(w[EB == 4 ? i : 0])
             : DT == BRSVD_DTYPE_BF16 ? from16<Bf16>((uint16_t)(w[i / 2] >> (16 * (i & 1)))) : from16<Fp16>((uint16_t)(w[i / 2] >> (16 * (i & 1))));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = i >= valid ? 0.f : DT == BRSVD_DTYPE_F32 ? ((const float*)src)[i]
             : DT == BRSVD_DTYPE_BF16 ? from16<Bf16>(((const uint16_t*)src)[i]) : from16<Fp16>(((const uint16_t*)src)[i]);
  }
}

// Up to eight bytes to a row of numbers of 8 bits
__device__ __forceinline__ void put_eight(uint8_t* dst, int valid, uint2 v) {
  if (valid >= 8 && ((uintptr_t)dst & 7) == 0) *(uint2*)dst = v;
  else
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) dst[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
}

// One workgroup per 128 x 128 part: lane group of 16 per row, eight numbers a lane, 16 rows of the workgroup at a time.  Bound by memory: what it reads and
// writes once.
template <int DT, bool SQUARE, bool STRAIGHT, bool TRANSPOSED>
__global__ void __launch_bounds__(256)
k_quantize(const char* __restrict__ X, int64_t ldx, int64_t rows, int64_t cols, uint8_t* __restrict__ Q, int64_t ldq, float* __restrict__ S,
           uint8_t* __restrict__ Qt, int64_t ldqt, float* __restrict__ St) {
  constexpr int EB = DT == BRSVD_DTYPE_F32 ? 4 : 2;
  __shared__ float top[4][kBlock];
  __shared__ __attribute__((aligned(16))) uint8_t turned[TRANSPOSED ? kBlock : 1][kBlock + 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = (tid & 15) * 8, r = tid >> 4;
  const int64_t ncb = (cols + kBlock - 1) / kBlock, nrb = (rows + kBlock - 1) / kBlock;
  const int64_t rb = blockIdx.x / (unsigned)ncb, cb = blockIdx.x % (unsigned)ncb, row0 = rb * kBlock, col0 = cb * kBlock;
  const int width = (int)(cols - col0 - c < 8 ? (cols - col0 - c > 0 ? cols - col0 - c : 0) : 8);
  float x[8][8], rowtop[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + r + 16 * i;
    eight<DT>(X + row * ldx + (col0 + c) * EB, row < rows ? width : 0, x[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) t = fmaxf(t, finite_abs(x[i][j]));
#pragma unroll
    for (int s = 1; s < 16; s <<= 1) t = fmaxf(t, __shfl_xor(t, s));
    rowtop[i] = t;
  }
  int e_square = 0;
  if (SQUARE) {
    float t = rowtop[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) t = fmaxf(t, rowtop[i]);
    t = fmaxf(t, __shfl_xor(t, 16));
    t = fmaxf(t, __shfl_xor(t, 32));
    if (lane == 0) top[wave][0] = t;
    __syncthreads();
    e_square = block_exponent(fmaxf(fmaxf(top[0][0], top[1][0]), fmaxf(top[2][0], top[3][0])));
    if (tid == 0 && STRAIGHT) S[rb * ncb + cb] = power_of_two(e_square);
    if (tid == 0 && TRANSPOSED) St[cb * nrb + rb] = power_of_two(e_square);
  }
  if (STRAIGHT) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + r + 16 * i;
      const int e = SQUARE ? e_square : block_exponent(rowtop[i]);
      const float f = power_of_two(-e);
      const uint2 v = make_uint2(pack_e4m3(x[i][0] * f, x[i][1] * f, x[i][2] * f, x[i][3] * f), pack_e4m3(x[i][4] * f, x[i][5] * f, x[i][6] * f, x[i][7] * f));
      if (row < rows) {
        put_eight(Q + row * ldq + col0 + c, width, v);
        if (!SQUARE && (tid & 15) == 0) S[row * ncb + cb] = power_of_two(e);
      }
    }
  }
  if (TRANSPOSED) {
    float f[8];
    if (!SQUARE) {
      float t[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        t[j] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t[j] = fmaxf(t[j], finite_abs(x[i][j]));
        t[j] = fmaxf(t[j], __shfl_xor(t[j], 16));
        t[j] = fmaxf(t[j], __shfl_xor(t[j], 32));
        if (lane < 16) top[wave][c + j] = t[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = block_exponent(fmaxf(fmaxf(top[0][c + j], top[1][c + j]), fmaxf(top[2][c + j], top[3][c + j])));
        f[j] = power_of_two(-e);
        if (r == 0 && j < width) St[(col0 + c + j) * nrb + rb] = power_of_two(e);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = power_of_two(-e_square);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        const uint32_t v = pack_e4m3(x[i][j] * f[j], x[i][j + 1] * f[j + 1], x[i][j + 2] * f[j + 2], x[i][j + 3] * f[j + 3]);
#pragma unroll
        for (int b = 0; b < 4; ++b) turned[c + j + b][r + 16 * i] = (uint8_t)(v >> (8 * b));
      }
    }
    __syncthreads();
    const int height = (int)(rows - row0 - c < 8 ? (rows - row0 - c > 0 ? rows - row0 - c : 0) : 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t col = col0 + r + 16 * i;
      if (col < cols) put_eight(Qt + col * ldqt + row0 + c, height, *(const uint2*)&turned[r + 16 * i][c]);
    }
  }
}

// X = Q * S, a lane takes eight numbers of a row.
template <int DT>
__global__ void __launch_bounds__(256)
k_dequantize(const uint8_t* __restrict__ Q, int64_t ldq, const float* __restrict__ S, int64_t rows, int64_t cols, int block_rows, char* __restrict__ X, int64_t ldx) {
  const int c = (threadIdx.x & 15) * 8, r = threadIdx.x >> 4;
  const int64_t ncb = (cols + kBlock - 1) / kBlock, rb = blockIdx.x / (unsigned)ncb, cb = blockIdx.x % (unsigned)ncb, col = cb * kBlock + c;
  const int width = (int)(cols - col < 8 ? cols - col : 8);
  if (width <= 0) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = rb * kBlock + r + 16 * i;
    if (row >= rows) return;
    const uint8_t* src = Q + row * ldq + col;
    const float f = S[(block_rows == 1 ? row : row / kBlock) * ncb + cb];
    uint32_t w[2] = {0u, 0u};
    if (width == 8) {
      struct __attribute__((packed, aligned(1))) Two { uint32_t x[2]; };
      const Two v = *(const Two*)src;
      w[0] = v.x[0];
      w[1] = v.x[1];
    } else {
      for (int j = 0; j < width; ++j) w[j / 4] |= (uint32_t)src[j] << (8 * (j & 3));
    }
    float x[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
      x[4 * j] = lo[0] * f;
      x[4 * j + 1] = lo[1] * f;
      x[4 * j + 2] = hi[0] * f;
      x[4 * j + 3] = hi[1] * f;
    }
    if (DT == BRSVD_DTYPE_F32) {
      float* out = (float*)(X + row * ldx) + col;
      if (width == 8 && ((uintptr_t)out & 15) == 0) {
        ((floatx4*)out)[0] = floatx4{x[0], x[1], x[2], x[3]};
        ((floatx4*)out)[1] = floatx4{x[4], x[5], x[6], x[7]};
      } else
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < width) out[j] = x[j];
    } else {
      uint16_t* out = (uint16_t*)(X + row * ldx) + col;
      uint16_t h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = DT == BRSVD_DTYPE_BF16 ? to16<Bf16>(x[j]) : to16<Fp16>(x[j]);
      if (width == 8 && ((uintptr_t)out & 15) == 0)
        *(uint4*)out = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < width) out[j] = h[j];
    }
  }
}

template <int DT, bool SQUARE>
static void launch_quantize(const char* X, int64_t ldx, int64_t rows, int64_t cols, uint8_t* Q, int64_t ldq, float* S, uint8_t* Qt, int64_t ldqt, float* St,
                            hipStream_t stream) {
  const dim3 grid((unsigned)(ceil_div(cols, kBlock) * ceil_div(rows, kBlock)));
  const int64_t pitch = ldx * (DT == BRSVD_DTYPE_F32 ? 4 : 2);
  if (Q && Qt) hipLaunchKernelGGL((k_quantize<DT, SQUARE, true, true>), grid, dim3(256), 0, stream, X, pitch, rows, cols, Q, ldq, S, Qt, ldqt, St);
  else if (Q) hipLaunchKernelGGL((k_quantize<DT, SQUARE, true, false>), grid, dim3(256), 0, stream, X, pitch, rows, cols, Q, ldq, S, Qt, ldqt, St);
  else hipLaunchKernelGGL((k_quantize<DT, SQUARE, false, true>), grid, dim3(256), 0, stream, X, pitch, rows, cols, Q, ldq, S, Qt, ldqt, St);
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
  if (!X || (!Q && !Qt) || ldx < cols || (Q && (!S || ldq < cols)) || (Qt && (!St || ldqt < rows)) || ceil_div(rows, kBlock) * ceil_div(cols, kBlock) > kMaxGrid) return BRSVD_ERR_ARG;
  return quantize(X, ldx, rows, cols, dtype, block_rows, Q, ldq, S, Qt, ldqt, St, (hipStream_t)stream);
}

extern "C" int brsvd_dequantize_e4m3(const uint8_t* Q, int64_t ldq, const float* S, int64_t rows, int64_t cols, int32_t block_rows, int32_t dtype, void* X,
                                     int64_t ldx, void* stream) {
  if (rows < 0 || cols < 0 || !model_type(dtype) || (block_rows != 1 && block_rows != kBlock)) return BRSVD_ERR_ARG;
  if (rows == 0 || cols == 0) return BRSVD_OK;
  if (!Q || !S || !X || ldq < cols || ldx < cols || ceil_div(rows, kBlock) * ceil_div(cols, kBlock) > kMaxGrid) return BRSVD_ERR_ARG;
  const dim3 grid((unsigned)(ceil_div(cols, kBlock) * ceil_div(rows, kBlock)));
  const int64_t pitch = ldx * (dtype == BRSVD_DTYPE_F32 ? 4 : 2);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == BRSVD_DTYPE_F32) hipLaunchKernelGGL(k_dequantize<BRSVD_DTYPE_F32>, grid, dim3(256), 0, s, Q, ldq, S, rows, cols, block_rows, (char*)X, pitch);
  else if (dtype == BRSVD_DTYPE_BF16) hipLaunchKernelGGL(k_dequantize<BRSVD_DTYPE_BF16>, grid, dim3(256), 0, s, Q, ldq, S, rows, cols, block_rows, (char*)X, pitch);
  else hipLaunchKernelGGL(k_dequantize<BRSVD_DTYPE_F16>, grid, dim3(256), 0, s, Q, ldq, S, rows, cols, block_rows, (char*)X, pitch);
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}
