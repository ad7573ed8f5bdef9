// Casting a matrix into 4 bits with a scale for each 32 neighbouring numbers of a row, and back.
//   s = 2^e, the least e >= -126 with max |x| <= 6 * 2^e over the group;  q = e2m1(x / s), to the nearest, ties to an even code
// A power of two as the scale rounds nothing: a number is rounded once.  Numbers of 4 bits know neither infinity nor NaN: a group with one gets the scale NaN.
#include "e2m1.h"

namespace brsvd {

// Numbers that a thread takes of a group, 16 bytes of them, and lanes of a group
template <int DT> struct Share {
  static constexpr int kBytes = DT == BRSVD_DTYPE_F32 ? 4 : 2, kWide = 16 / kBytes, kLanes = kGroup / kWide;
};

// Largest key of the lanes that share a group, in all of them: exchanges inside four lanes, then with the four beside them.
template <int LANES>
__device__ __forceinline__ uint32_t max_of_group(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));        // lanes 1 0 3 2
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));        // lanes 2 3 0 1
  if (LANES == 8) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));     // lane 7 - i of eight
  return x;
}

// A thread has 16 bytes of a group, so that lanes read next to each other, and U such pieces on their way; the group's largest number goes between four or eight lanes in registers.
// Bound by memory: 20000 x 20000 fp32 373 us (1.81 GB, 4.9 TB/s).
template <int DT, int U>
__global__ void __launch_bounds__(256)
k_quantize_e2m1(const char* __restrict__ X, int64_t ldx_bytes, int64_t rows, int64_t cols, Divisor groups, uint8_t* __restrict__ Q, int64_t ldq, uint8_t* __restrict__ S) {
  using P = Share<DT>;
  constexpr int W = P::kWide, L = P::kLanes, PER = 256 / L;
  const int tid = threadIdx.x, part = tid % L;
  const uint32_t all = (uint32_t)rows * groups.d;
  uint4 v[U];
  uint32_t row[U], at[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t g = (blockIdx.x * U + i) * PER + tid / L;
    row[i] = divide(g, groups, &at[i]);
    const int64_t c = (int64_t)at[i] * kGroup + part * W, left = g < all ? cols - c : 0;
    v[i] = piece_of<P::kBytes>(X + (int64_t)row[i] * ldx_bytes + c * P::kBytes, left * P::kBytes);
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
    float x[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const uint16_t h = (uint16_t)(w[j * P::kBytes / 4] >> (16 * (j & 1)));
      x[j] = DT == BRSVD_DTYPE_F32 ? __uint_as_float(w[j & 3]) : DT == BRSVD_DTYPE_BF16 ? from16<Bf16>(h) : from16<Fp16>(h);
    }
    // magnitudes order as their bits do, infinities and NaN above all numbers
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    top = max_of_group<L>(top);
    const bool numbers = top < 0x7f800000u;
    const int e = numbers ? group_exponent(__uint_as_float(top)) : 128;
    const float scale = numbers ? __uint_as_float((uint32_t)(e + 127) << 23) : 1.f;
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[0], x[1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[2], x[3], scale, 1);
    if constexpr (W == 8) {
      q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[4], x[5], scale, 2);
      q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[6], x[7], scale, 3);
    }
    if (!numbers) q = 0;
    const uint32_t g = (blockIdx.x * U + i) * PER + tid / L;
    if (g >= all) continue;
    const int64_t c = (int64_t)at[i] * kGroup + part * W, left = cols - c;
    if (part == 0) S[(int64_t)row[i] * groups.d + at[i]] = (uint8_t)(e + 127);
    uint8_t* to = Q + (int64_t)row[i] * ldq + c / 2;
    const int bytes = (int)(left >= W ? W / 2 : left > 0 ? (left + 1) / 2 : 0);
    if (bytes == W / 2) {
      if (W == 8) {
        struct __attribute__((packed, aligned(1))) Four { uint32_t x; };
        *(Four*)to = Four{q};
      } else {
        struct __attribute__((packed, aligned(1))) Two { uint16_t x; };
        *(Two*)to = Two{(uint16_t)q};
      }
    } else {
#pragma unroll
      for (int b = 0; b < W / 2; ++b)
        if (b < bytes) to[b] = (uint8_t)(q >> (8 * b));
    }
  }
}

// A thread writes 16 bytes, and has U such pieces on their way.  Bound by memory: 20000 x 20000 to fp32 300 us (1.81 GB, 6.0 TB/s).
template <int DT, int U>
__global__ void __launch_bounds__(256)
k_dequantize_e2m1(const uint8_t* __restrict__ Q, int64_t ldq, const uint8_t* __restrict__ S, int64_t rows, int64_t cols, Divisor pieces, int64_t groups,
                  char* __restrict__ X, int64_t ldx_bytes) {
  using P = Share<DT>;
  constexpr int W = P::kWide;
  const uint32_t all = (uint32_t)rows * pieces.d;
  uint32_t q[U], s[U], row[U], at[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t g = (blockIdx.x * U + i) * 256 + threadIdx.x;
    row[i] = divide(g, pieces, &at[i]);
    q[i] = s[i] = 0;
    if (g >= all) continue;
    const int64_t c = (int64_t)at[i] * W, left = cols - c;
    const uint8_t* from = Q + (int64_t)row[i] * ldq + c / 2;
    if (left >= W) {
      if (W == 8) {
        struct __attribute__((packed, aligned(1))) Four { uint32_t x; };
        q[i] = ((const Four*)from)->x;
      } else {
        struct __attribute__((packed, aligned(1))) Two { uint16_t x; };
        q[i] = ((const Two*)from)->x;
      }
    } else {
#pragma unroll
      for (int b = 0; b < W / 2; ++b)
        if (2 * b < left) q[i] |= (uint32_t)from[b] << (8 * b);
    }
    s[i] = S[(int64_t)row[i] * groups + c / kGroup];
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t g = (blockIdx.x * U + i) * 256 + threadIdx.x;
    if (g >= all) continue;
    const int64_t c = (int64_t)at[i] * W, left = cols - c;
    const float scale = scale_e8m0(s[i]);
    uint32_t v[4];
    if constexpr (DT == BRSVD_DTYPE_F32) {
      const floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], scale, 1);
      v[0] = __float_as_uint(a[0]); v[1] = __float_as_uint(a[1]); v[2] = __float_as_uint(b[0]); v[3] = __float_as_uint(b[1]);
    } else {
      using El = typename std::conditional<DT == BRSVD_DTYPE_BF16, Bf16, Fp16>::type;
      const uint4 x = eight_e2m1<El>(q[i], scale);
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    }
    char* to = X + (int64_t)row[i] * ldx_bytes + c * P::kBytes;
    if (left >= W) *(Piece*)to = Piece{{v[0], v[1], v[2], v[3]}};
    else
#pragma unroll
      for (int j = 0; j < W; ++j)
        if (j < left) {
          if (DT == BRSVD_DTYPE_F32) ((uint32_t*)to)[j] = v[j & 3];
          else ((uint16_t*)to)[j] = (uint16_t)(v[j / 2 & 3] >> (16 * (j & 1)));
        }
  }
}

static int bytes_of(int dtype) { return dtype == BRSVD_DTYPE_F32 ? 4 : dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16 ? 2 : 0; }

// Sizes of a matrix in 4 bits: a row has at most 2^31 units of work, and bytes are numbers of 64 bits
static bool sizes_e2m1(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows < (int64_t)1 << 40 && cols <= (int64_t)1 << 33; }
static bool pitch_fits(int64_t ld) { return ld < (int64_t)1 << 40; }

}  // namespace brsvd

using namespace brsvd;

extern "C" int brsvd_quantize_e2m1(const void* X, int64_t ldx, int64_t rows, int64_t cols, int32_t dtype, uint8_t* Q, int64_t ldq, uint8_t* S, void* stream) {
  const int eb = bytes_of(dtype);
  if (!eb || !sizes_e2m1(rows, cols)) return BRSVD_ERR_ARG;
  if (rows == 0 || cols == 0) return BRSVD_OK;
  if (!X || !Q || !S || ldx < cols || ldq < (cols + 1) / 2 || !pitch_fits(ldx) || !pitch_fits(ldq)) return BRSVD_ERR_ARG;
  const int64_t groups = ceil_div(cols, kGroup);
  const Divisor by = divisor((uint32_t)groups);
  hipStream_t s = (hipStream_t)stream;
  constexpr int U = 4;
  by_rows(rows, groups, U * (eb == 4 ? 32 : 64), [&](int64_t r, int64_t n, dim3 grid) {
    const char* x = (const char*)X + r * ldx * eb;
    uint8_t *q = Q + r * ldq, *sc = S + r * groups;
    if (dtype == BRSVD_DTYPE_F32) hipLaunchKernelGGL((k_quantize_e2m1<BRSVD_DTYPE_F32, U>), grid, dim3(256), 0, s, x, ldx * eb, n, cols, by, q, ldq, sc);
    else if (dtype == BRSVD_DTYPE_BF16) hipLaunchKernelGGL((k_quantize_e2m1<BRSVD_DTYPE_BF16, U>), grid, dim3(256), 0, s, x, ldx * eb, n, cols, by, q, ldq, sc);
    else hipLaunchKernelGGL((k_quantize_e2m1<BRSVD_DTYPE_F16, U>), grid, dim3(256), 0, s, x, ldx * eb, n, cols, by, q, ldq, sc);
  });
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

extern "C" int brsvd_dequantize_e2m1(const uint8_t* Q, int64_t ldq, const uint8_t* S, int64_t rows, int64_t cols, int32_t dtype, void* X, int64_t ldx, void* stream) {
  const int eb = bytes_of(dtype);
  if (!eb || !sizes_e2m1(rows, cols)) return BRSVD_ERR_ARG;
  if (rows == 0 || cols == 0) return BRSVD_OK;
  if (!Q || !S || !X || ldx < cols || ldq < (cols + 1) / 2 || !pitch_fits(ldx) || !pitch_fits(ldq)) return BRSVD_ERR_ARG;
  const int64_t pieces = ceil_div(cols, 16 / eb), groups = ceil_div(cols, kGroup);
  const Divisor by = divisor((uint32_t)pieces);
  hipStream_t s = (hipStream_t)stream;
  constexpr int U = 4;
  by_rows(rows, pieces, U * 256, [&](int64_t r, int64_t n, dim3 grid) {
    const uint8_t *q = Q + r * ldq, *sc = S + r * groups;
    char* x = (char*)X + r * ldx * eb;
    if (dtype == BRSVD_DTYPE_F32) hipLaunchKernelGGL((k_dequantize_e2m1<BRSVD_DTYPE_F32, U>), grid, dim3(256), 0, s, q, ldq, sc, n, cols, by, groups, x, ldx * eb);
    else if (dtype == BRSVD_DTYPE_BF16) hipLaunchKernelGGL((k_dequantize_e2m1<BRSVD_DTYPE_BF16, U>), grid, dim3(256), 0, s, q, ldq, sc, n, cols, by, groups, x, ldx * eb);
    else hipLaunchKernelGGL((k_dequantize_e2m1<BRSVD_DTYPE_F16, U>), grid, dim3(256), 0, s, q, ldq, sc, n, cols, by, groups, x, ldx * eb);
  });
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}
