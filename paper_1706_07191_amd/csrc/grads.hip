// The norm over many tensors, and the tensors clipped by it:
//   norm = |scale| sqrt(sum of x^2 over all numbers of all tensors),    y = x scale min(1, max_norm / norm)
// Squares and their sums are fp64: neither a number of 1e30 nor one of 1e-30 is lost, and no order of a long sum shows.  A workgroup takes a piece of at most kPiece
// numbers of one tensor; the pieces' sums are added in their order.
//
// The tensors' addresses and sizes are arguments of the launches, as many tensors at a time as those hold: nothing is copied to the device, and a captured launch keeps them.
#include <algorithm>
#include <new>

#include "tile.h"

namespace brsvd {

constexpr int kTensors = 64;                  // of a launch
constexpr int64_t kPiece = 1 << 15;           // numbers of a workgroup

// Tensors of a launch, and which pieces are theirs: those of tensor i are first[i] to first[i + 1].
struct TensorList {
  const char* x[kTensors];
  char* y[kTensors];
  int64_t cols[kTensors];      // numbers of a row
  int64_t ldx[kTensors], ldy[kTensors];      // numbers
  int32_t rows_per[kTensors];  // rows of a piece; 0: a row has several pieces
  int32_t rows[kTensors];      // rows, where pieces have several
  uint32_t first[kTensors + 1];
  uint8_t tx[kTensors], ty[kTensors];
  int count;
};

static int bytes_of(int dtype) { return dtype == BRSVD_DTYPE_F32 ? 4 : dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16 ? 2 : 0; }

// Eight numbers of type dtype from `src`, `valid` of them there, the others zero
__device__ __forceinline__ void eight_numbers(const char* src, int64_t valid, int dtype, float (&x)[8]) {
  if (dtype == BRSVD_DTYPE_F32) {
    const uint4 a = piece_of<4>(src, 4 * valid), b = piece_of<4>(src + 16, 4 * valid - 16);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
  } else {
    const uint4 a = piece_of<2>(src, 2 * valid);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint16_t h = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
      x[i] = dtype == BRSVD_DTYPE_BF16 ? from16<Bf16>(h) : from16<Fp16>(h);
    }
  }
}

// Which tensor a piece is of: the last one that begins at or before it
__device__ __forceinline__ int tensor_of(const TensorList& l, uint32_t piece) {
  int at = 0;
#pragma unroll
  for (int step = kTensors / 2; step > 0; step >>= 1)
    if (at + step < l.count && l.first[at + step] <= piece) at += step;
  return __builtin_amdgcn_readfirstlane(at);
}

// Calls take(row, column, numbers of the row from there on, at most eight) for all eights of a piece; threads take neighbouring ones.
template <class Take>
__device__ __forceinline__ void eights_of(const TensorList& l, int i, uint32_t piece, Take take) {
  const uint32_t p = piece - l.first[i];
  const int64_t cols = l.cols[i];
  if (l.rows_per[i] == 0) {
    const uint32_t per = (uint32_t)((cols + kPiece - 1) / kPiece), row = p / per;
    const int64_t c0 = (int64_t)(p - row * per) * kPiece, left = cols - c0 < kPiece ? cols - c0 : kPiece;
    for (int c = 8 * threadIdx.x; c < left; c += 8 * 256) take((int64_t)row, c0 + c, left - c);
  } else {
    const uint32_t eights = (uint32_t)((cols + 7) / 8), r0 = p * l.rows_per[i], rows = l.rows[i] - r0 < (uint32_t)l.rows_per[i] ? l.rows[i] - r0 : l.rows_per[i];
    for (uint32_t e = threadIdx.x; e < rows * eights; e += 256) {
      const uint32_t r = e / eights, c = 8 * (e - r * eights);
      take((int64_t)(r0 + r), (int64_t)c, cols - c);
    }
  }
}

__device__ __forceinline__ double sum_of_workgroup(double x, double* red) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x += __shfl_xor(x, s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = 0.0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) sum += red[w];
  return sum;
}

__global__ void __launch_bounds__(256)
k_grad_squares(const TensorList l, double* __restrict__ sums) {
  __shared__ double red[4];
  const int i = tensor_of(l, blockIdx.x);
  const int dtype = l.tx[i], eb = dtype == BRSVD_DTYPE_F32 ? 4 : 2;
  double sum = 0.0;
  eights_of(l, i, blockIdx.x, [&](int64_t r, int64_t c, int64_t left) {
    float x[8];
    eight_numbers(l.x[i] + (r * l.ldx[i] + c) * eb, left, dtype, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fma((double)x[j], (double)x[j], sum);
  });
  sum = sum_of_workgroup(sum, red);
  if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(1024)
k_grad_norm(const double* __restrict__ sums, int64_t n, double scale, float* __restrict__ norm) {
  __shared__ double red[16];
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) sum += sums[i];
  sum = sum_of_workgroup(sum, red);
  if (threadIdx.x == 0) *norm = (float)(sqrt(sum) * scale);
}

__global__ void __launch_bounds__(256)
k_grad_clip(const TensorList l, const float* __restrict__ norm, double scale, double max_norm) {
  const int i = tensor_of(l, blockIdx.x);
  const double n = *norm;
  // a norm that is no finite number says nothing about how long the gradients are: they are scaled alone
  const double f = n > max_norm && n <= 3.402823466e38 ? scale * (max_norm / n) : scale;
  if (f == 1.0 && l.x[i] == l.y[i]) return;
  // in two factors, so that neither leaves fp32's range where the product does not
  const double a = fabs(f) < 0x1p-100 ? f * 0x1p100 : fabs(f) > 0x1p100 ? f * 0x1p-100 : f;
  const float f1 = (float)a, f2 = fabs(f) < 0x1p-100 ? 0x1p-100f : fabs(f) > 0x1p100 ? 0x1p100f : 1.f;
  const int tx = l.tx[i], ty = l.ty[i], ex = tx == BRSVD_DTYPE_F32 ? 4 : 2, ey = ty == BRSVD_DTYPE_F32 ? 4 : 2;
  eights_of(l, i, blockIdx.x, [&](int64_t r, int64_t c, int64_t left) {
    float x[8];
    eight_numbers(l.x[i] + (r * l.ldx[i] + c) * ex, left, tx, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = x[j] * f1 * f2;
    char* to = l.y[i] + (r * l.ldy[i] + c) * ey;
    if (ty == BRSVD_DTYPE_F32) {
      if (left >= 8) {
        *(Piece*)to = Piece{{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}};
        *(Piece*)(to + 16) = Piece{{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])}};
      } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (j < left) ((float*)to)[j] = x[j];
      }
    } else {
      uint16_t h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = ty == BRSVD_DTYPE_BF16 ? to16<Bf16>(x[j]) : to16<Fp16>(x[j]);
      if (left >= 8) {
        *(Piece*)to = Piece{{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16}};
      } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (j < left) ((uint16_t*)to)[j] = h[j];
      }
    }
  });
}

// A tensor as kernels take it: rows next to each other are one long row.
struct Shape {
  int64_t rows, cols;
  int rows_per;
  int64_t pieces;
};
static Shape shape_of(const brsvd_tensor& x, const brsvd_tensor* y) {
  Shape s{x.rows, x.cols, 0, 0};
  if (x.rows == 0 || x.cols == 0) return s;
  if (x.rows == 1 || (x.ld == x.cols && (!y || y->ld == y->cols))) s.cols = x.rows * x.cols, s.rows = 1;
  if (s.rows > 1 && s.cols < kPiece) {
    s.rows_per = (int)(kPiece / s.cols);
    s.pieces = ceil_div(s.rows, s.rows_per);
  } else {
    s.pieces = s.rows * ceil_div(s.cols, kPiece);
  }
  return s;
}
constexpr int64_t kMaxNumbers = (int64_t)1 << 44, kMaxPieces = (int64_t)1 << 24;
// Number of pieces of all tensors, -1 where one is refused
static int64_t check_list(const brsvd_tensor* x, const brsvd_tensor* y, int64_t count) {
  if (count < 0 || (count > 0 && !x)) return -1;
  int64_t pieces = 0;
  for (int64_t i = 0; i < count; ++i) {
    for (int k = 0; k < (y ? 2 : 1); ++k) {
      const brsvd_tensor& t = k ? y[i] : x[i];
      if (!bytes_of((int)t.dtype) || t.dtype != (int)t.dtype || t.rows < 0 || t.cols < 0 || t.rows != x[i].rows || t.cols != x[i].cols) return -1;
      if (t.rows == 0 || t.cols == 0) continue;
      if (!t.data || t.cols > kMaxNumbers || t.rows > kMaxNumbers / t.cols || t.rows > INT32_MAX) return -1;
      if (t.rows > 1 && (t.ld < t.cols || t.ld > kMaxNumbers / t.rows)) return -1;
    }
    pieces += shape_of(x[i], y ? y + i : nullptr).pieces;
    if (pieces > kMaxPieces) return -1;
  }
  return pieces;
}
// Whether numbers of one tensor are another's too: an address of `out` twice, or that of another tensor; and one that is its own tensor's has to be laid out like it.
static int check_places(const brsvd_tensor* x, const brsvd_tensor* y, int64_t count) {
  if (count == 0) return BRSVD_OK;
  const void** places = new (std::nothrow) const void*[count];
  if (!places) return BRSVD_ERR_ALLOC;
  int64_t n = 0;
  bool good = true;
  for (int64_t i = 0; i < count; ++i)
    if (x[i].rows > 0 && x[i].cols > 0) {
      places[n++] = y[i].data;
      good &= y[i].data != x[i].data || (y[i].dtype == x[i].dtype && (x[i].rows == 1 || y[i].ld == x[i].ld));
    }
  if (!std::is_sorted(places, places + n)) std::sort(places, places + n);
  for (int64_t i = 1; i < n; ++i) good &= places[i] != places[i - 1];
  for (int64_t i = 0; i < count && good; ++i)
    if (x[i].rows > 0 && x[i].cols > 0 && x[i].data != y[i].data) good &= !std::binary_search(places, places + n, (const void*)x[i].data);
  delete[] places;
  return good ? BRSVD_OK : BRSVD_ERR_ARG;
}
// launch(list, workgroups) for as many tensors at a time as a list holds
template <class Launch>
static void in_lists(const brsvd_tensor* x, const brsvd_tensor* y, int64_t count, Launch launch) {
  TensorList l;
  l.count = 0;
  uint32_t pieces = 0;
  auto flush = [&] {
    if (pieces == 0) return;
    l.first[l.count] = pieces;
    launch(l, pieces);
    l.count = 0;
    pieces = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const Shape s = shape_of(x[i], y ? y + i : nullptr);
    if (s.pieces == 0) continue;
    const int c = l.count++;
    l.x[c] = (const char*)x[i].data;
    l.ldx[c] = x[i].ld;
    l.tx[c] = (uint8_t)x[i].dtype;
    l.y[c] = y ? (char*)y[i].data : nullptr;
    l.ldy[c] = y ? y[i].ld : 0;
    l.ty[c] = y ? (uint8_t)y[i].dtype : 0;
    l.cols[c] = s.cols;
    l.rows[c] = (int32_t)s.rows;
    l.rows_per[c] = s.rows_per;
    l.first[c] = pieces;
    pieces += (uint32_t)s.pieces;
    if (l.count == kTensors) flush();
  }
  flush();
}

}  // namespace brsvd

using namespace brsvd;

extern "C" uint64_t brsvd_grad_norm_workspace_bytes(const brsvd_tensor* tensors, int64_t count) {
  const int64_t pieces = check_list(tensors, nullptr, count);
  return pieces < 0 ? 0 : (uint64_t)(pieces + 32) / 32 * 256;
}

extern "C" int brsvd_grad_norm(const brsvd_tensor* tensors, int64_t count, float scale, float* norm, void* workspace, uint64_t workspace_bytes, void* stream) {
  const int64_t pieces = check_list(tensors, nullptr, count);
  if (pieces < 0 || !norm || !(fabsf(scale) <= 3.402823466e38f)) return BRSVD_ERR_ARG;
  if (!workspace || (uintptr_t)workspace % 256) return BRSVD_ERR_ARG;
  if (workspace_bytes < (uint64_t)(pieces + 32) / 32 * 256) return BRSVD_ERR_BUDGET;
  hipStream_t s = (hipStream_t)stream;
  double* sums = (double*)workspace;
  in_lists(tensors, nullptr, count, [&](const TensorList& l, unsigned grid) {
    hipLaunchKernelGGL(k_grad_squares, dim3(grid), dim3(256), 0, s, l, sums);
    sums += grid;
  });
  hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(1024), 0, s, (const double*)workspace, pieces, fabs((double)scale), norm);
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

extern "C" int brsvd_grad_clip(const brsvd_tensor* tensors, const brsvd_tensor* out, int64_t count, float scale, float max_norm, const float* norm, void* stream) {
  const int64_t pieces = count > 0 && !out ? -1 : check_list(tensors, out, count);
  if (pieces < 0 || !norm || !(fabsf(scale) <= 3.402823466e38f) || !(max_norm >= 0.f)) return BRSVD_ERR_ARG;
  BRSVD_TRY(check_places(tensors, out, count));
  if (pieces == 0) return BRSVD_OK;
  hipStream_t s = (hipStream_t)stream;
  in_lists(tensors, out, count, [&](const TensorList& l, unsigned grid) {
    hipLaunchKernelGGL(k_grad_clip, dim3(grid), dim3(256), 0, s, l, norm, (double)scale, (double)max_norm);
  });
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}
