// The norm over many tensors, and the tensors clipped by it:
//   norm = |scale| sqrt(sum of x^2 over all numbers of all tensors),    y = x scale min(1, max_norm / norm)
// Squares and their sums are fp64: neither a number of 1e30 nor one of 1e-30 is lost, and no order of a long sum shows.  A workgroup takes a piece of one
// tensor; the pieces' sums are added in their order.
//
// The tensors' addresses and sizes are arguments of the launches, as many tensors at a time as those hold: nothing is copied to the device, and a captured launch keeps them.
#include <algorithm>
#include <new>

#include "tile.h"

namespace brsvd {

// Places in a launch's list.  What arguments a launch can have, 4 KB, is what there is: so a tensor without gaps takes one of 29 bytes, and one with strided rows two.
constexpr int kPlaces = 128;
// Numbers of a piece: so many that there are some 2000 pieces, within these bounds.  10 tensors of 155 000 numbers: squares 4.3 us in pieces of 2^12, 8.0 in pieces of 2^15.
// 106 million bf16 numbers of 57 tensors into fp32: pieces of 2^15 140 us, 2^14 131, 2^13 125, as the last round of workgroups is a smaller part; the norm's sums
// are added by one workgroup, which has 16 us to do for 2^13 and 10 for 2^14.
constexpr int kLeastPiece = 12, kNormPiece = 14, kClipPiece = 13;      // as powers of 2

// Tensors of a launch, and which pieces are theirs: those of the tensor at place i are first[i] up to the next tensor's.
struct TensorList {
  const char* x[kPlaces];
  char* y[kPlaces];
  int64_t cols[kPlaces];       // numbers of a row
  uint32_t first[kPlaces];
  uint8_t types[kPlaces];      // x's, y's << 2; kStrided: the place behind a tensor that has several rows
  int32_t count, piece;
  // of such a place: x and y are the rows' distances in numbers, cols is rows_per << 32 | rows.  rows_per: rows of a piece, 0 where a row has several pieces
};
constexpr uint8_t kStrided = 0xff;
static_assert(sizeof(TensorList) <= 3840 && BRSVD_DTYPE_F32 < 4 && BRSVD_DTYPE_BF16 < 4 && BRSVD_DTYPE_F16 < 4, "");

static int bytes_of(int dtype) { return dtype == BRSVD_DTYPE_F32 ? 4 : dtype == BRSVD_DTYPE_BF16 || dtype == BRSVD_DTYPE_F16 ? 2 : 0; }

// W numbers of a type as they lie in memory
template <int DT, int W> struct Some {
  static constexpr int kNumber = DT == BRSVD_DTYPE_F32 ? 4 : 2, kWords = W * kNumber / 4;
  struct __attribute__((packed, aligned(1))) Words { uint32_t x[kWords]; };
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const char* src, int64_t valid) {       // valid of them are there, the others zero
    if (valid >= W) {
      const Words v = *(const Words*)src;
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = v.x[i];
    } else {
      const uint4 v = piece_of<kNumber>(src, kNumber * valid);
      const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = x[i];
    }
  }
  __device__ __forceinline__ float number(int i) const {
    if (kNumber == 4) return __uint_as_float(w[i % kWords]);
    const uint16_t h = (uint16_t)(w[(i >> 1) % kWords] >> (16 * (i & 1)));
    return DT == BRSVD_DTYPE_BF16 ? from16<Bf16>(h) : from16<Fp16>(h);
  }
  static __device__ __forceinline__ void put(char* to, int64_t left, const float (&x)[W]) {
    uint32_t v[kWords];
    if (kNumber == 4) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) v[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i)
        v[i] = DT == BRSVD_DTYPE_BF16 ? to16<Bf16>(x[2 * i % W]) | (uint32_t)to16<Bf16>(x[(2 * i + 1) % W]) << 16
                                      : to16<Fp16>(x[2 * i % W]) | (uint32_t)to16<Fp16>(x[(2 * i + 1) % W]) << 16;
    }
    if (left >= W) {
      Words o;
#pragma unroll
      for (int i = 0; i < kWords; ++i) o.x[i] = v[i];
      *(Words*)to = o;
    } else {
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        if (j < left) {
          if (kNumber == 4) ((uint32_t*)to)[j] = v[j % kWords];
          else ((uint16_t*)to)[j] = (uint16_t)(v[j / 2] >> (16 * (j & 1)));
        }
    }
  }
};

// The tensor that a piece is of, and its first piece
struct Mine {
  int at;
  bool strided;
  uint32_t first;
};
__device__ __forceinline__ Mine tensor_of(const TensorList& l, uint32_t piece) {
  const int lane = threadIdx.x & 63;
  int at = -1;
#pragma unroll
  for (int h = 0; h < kPlaces; h += 64) at += __popcll(__ballot(h + lane < l.count && l.first[h + lane] <= piece));      // a place of rows begins with its tensor
  at = __builtin_amdgcn_readfirstlane(at);
  const bool strided = l.types[at] == kStrided;
  return {at - (strided ? 1 : 0), strided, l.first[at]};
}

// Calls take(W numbers, row, column, numbers of the row from there on) for all of a piece; threads take neighbouring ones, 64 bytes a thread on their way.
template <int DT, int W, class Take>
__device__ __forceinline__ void all_of(const TensorList& l, Mine mine, Take take) {
  constexpr int EB = Some<DT, W>::kNumber, U = 64 / (W * EB), kStep = 256 * W;
  const int i = mine.at;
  const uint32_t p = blockIdx.x - mine.first;
  const int64_t cols = l.cols[i], ld = mine.strided ? (int64_t)l.x[i + 1] : 0, shape = mine.strided ? l.cols[i + 1] : 0;
  const uint32_t rows_per = (uint32_t)(shape >> 32), all_rows = (uint32_t)shape;
  Some<DT, W> x[U];
  if (rows_per == 0) {
    uint32_t row = 0, part = p;
    if (mine.strided) {
      const uint32_t per = (uint32_t)((cols + l.piece - 1) / l.piece);
      row = p / per;
      part = p - row * per;
    }
    const int64_t c0 = (int64_t)part * l.piece, there = cols - c0 < l.piece ? cols - c0 : l.piece;
    const char* from = l.x[i] + (row * ld + c0) * EB;
    const int left = (int)there;
    for (int c = W * threadIdx.x; c < left; c += kStep * U) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c + kStep * u < left) x[u].load(from + (int64_t)(c + kStep * u) * EB, left - c - kStep * u);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c + kStep * u < left) take(x[u], (int64_t)row, c0 + c + kStep * u, (int64_t)(left - c - kStep * u));
    }
  } else {
    const uint32_t some = (uint32_t)((cols + W - 1) / W), r0 = p * rows_per, rows = all_rows - r0 < rows_per ? all_rows - r0 : rows_per;
    for (uint32_t e = threadIdx.x; e < rows * some; e += 256) {
      const uint32_t r = e / some, c = W * (e - r * some);
      x[0].load(l.x[i] + ((int64_t)(r0 + r) * ld + c) * EB, cols - c);
      take(x[0], (int64_t)(r0 + r), (int64_t)c, cols - c);
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

template <int DT>
__device__ __forceinline__ double squares_of(const TensorList& l, Mine mine) {
  constexpr int W = DT == BRSVD_DTYPE_F32 ? 4 : 8;
  double sum[2] = {0.0, 0.0};
  all_of<DT, W>(l, mine, [&](const Some<DT, W>& x, int64_t, int64_t, int64_t) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const double v = x.number(j);
      sum[j & 1] = fma(v, v, sum[j & 1]);
    }
  });
  return sum[0] + sum[1];
}
// Bound by memory: 128 tensors of 241 million bf16 numbers in all 79 us (482 MB, 6.1 TB/s).
__global__ void __launch_bounds__(256)
k_grad_squares(const TensorList l, double* __restrict__ sums) {
  __shared__ double red[4];
  const Mine mine = tensor_of(l, blockIdx.x);
  const int dtype = l.types[mine.at] & 3;
  double sum = dtype == BRSVD_DTYPE_F32 ? squares_of<BRSVD_DTYPE_F32>(l, mine) : dtype == BRSVD_DTYPE_BF16 ? squares_of<BRSVD_DTYPE_BF16>(l, mine)
                                                                                                           : squares_of<BRSVD_DTYPE_F16>(l, mine);
  sum = sum_of_workgroup(sum, red);
  if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(1024)
k_grad_norm(const double* __restrict__ sums, int64_t n, double scale, float* __restrict__ norm) {
  __shared__ double red[16];
  double sum = 0.0;
  int64_t i = threadIdx.x;
  for (; i + 7 * 1024 < n; i += 8 * 1024) {
    double x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = sums[i + 1024 * j];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += x[j];
  }
  for (; i < n; i += 1024) sum += sums[i];
  sum = sum_of_workgroup(sum, red);
  if (threadIdx.x == 0) *norm = (float)(sqrt(sum) * scale);
}

template <int DT, int DY>
__device__ __forceinline__ void clip_piece(const TensorList& l, Mine mine, float f1, float f2) {
  constexpr int W = DT == BRSVD_DTYPE_F32 || DY == BRSVD_DTYPE_F32 ? 4 : 8;        // 16 bytes of the wider type: lanes write next to each other
  char* y0 = l.y[mine.at];
  const int64_t ld = mine.strided ? (int64_t)l.y[mine.at + 1] : 0;
  all_of<DT, W>(l, mine, [&](const Some<DT, W>& x, int64_t r, int64_t c, int64_t left) {
    float y[W];
#pragma unroll
    for (int j = 0; j < W; ++j) y[j] = x.number(j) * f1 * f2;
    Some<DY, W>::put(y0 + (r * ld + c) * Some<DY, W>::kNumber, left, y);
  });
}
template <int DT>
__device__ __forceinline__ void clip_into(const TensorList& l, Mine mine, float f1, float f2) {
  const int ty = l.types[mine.at] >> 2;
  if (ty == BRSVD_DTYPE_F32) clip_piece<DT, BRSVD_DTYPE_F32>(l, mine, f1, f2);
  else if (ty == BRSVD_DTYPE_BF16) clip_piece<DT, BRSVD_DTYPE_BF16>(l, mine, f1, f2);
  else clip_piece<DT, BRSVD_DTYPE_F16>(l, mine, f1, f2);
}
// Bound by memory: the same tensors into fp32 249 us (1.45 GB, 5.8 TB/s).  In place and with nothing to do it reads nothing.
__global__ void __launch_bounds__(256)
k_grad_clip(const TensorList l, const float* __restrict__ norm, double scale, double max_norm) {
  const Mine mine = tensor_of(l, blockIdx.x);
  const int tx = l.types[mine.at] & 3;
  const double n = *norm;
  // a norm that is no finite number says nothing about how long the gradients are: they are scaled alone
  const double f = n > max_norm && n <= 3.402823466e38 ? scale * (max_norm / n) : scale;
  if (f == 1.0 && l.x[mine.at] == l.y[mine.at]) return;
  // In two factors, so that neither leaves fp32's range where the product does not.  The second is a power of two.  The first is rounded to 24 bits as a normal number where
  // a result is one: f below 2^-275 leaves fewer than three bits of the largest x.
  const double size = fabs(f), f2 = size < 0x1p-200 ? 0x1p-149 : size < 0x1p-100 ? 0x1p-100 : size > 0x1p100 ? 0x1p100 : 1.0;
  const float a = (float)(f / f2), b = (float)f2;
  if (tx == BRSVD_DTYPE_F32) clip_into<BRSVD_DTYPE_F32>(l, mine, a, b);
  else if (tx == BRSVD_DTYPE_BF16) clip_into<BRSVD_DTYPE_BF16>(l, mine, a, b);
  else clip_into<BRSVD_DTYPE_F16>(l, mine, a, b);
}

// A tensor as kernels take it: rows next to each other are one long row.
struct Shape {
  int64_t rows, cols;
  int rows_per;
  int64_t pieces;
};
static Shape shape_of(const brsvd_tensor& x, const brsvd_tensor* y, int log_piece) {
  const int64_t piece = (int64_t)1 << log_piece;
  Shape s{x.rows, x.cols, 0, 0};
  if (x.rows == 0 || x.cols == 0) return s;
  if (x.rows == 1 || (x.ld == x.cols && (!y || y->ld == y->cols))) s.cols = x.rows * x.cols, s.rows = 1;
  if (s.rows > 1 && s.cols < piece) {
    s.rows_per = (int)(piece / s.cols);
    s.pieces = ceil_div(s.rows, s.rows_per);
  } else {
    s.pieces = s.rows * ((s.cols + piece - 1) >> log_piece);
  }
  return s;
}
constexpr int64_t kMaxNumbers = (int64_t)1 << 44, kMaxPieces = ((int64_t)1 << 24) - 1;      // of a launch, 256 threads each
// A list's pieces of up to `most` numbers, of more where there are too many for a launch.  pieces < 0: a tensor is refused
struct Pieces {
  int log_piece;
  int64_t pieces;
};
static Pieces check_list(const brsvd_tensor* x, const brsvd_tensor* y, int64_t count, int most) {
  const Pieces refused{0, -1};
  if (count < 0 || (count > 0 && !x)) return refused;
  int64_t numbers = 0;
  for (int64_t i = 0; i < count; ++i) {
    for (int k = 0; k < (y ? 2 : 1); ++k) {
      const brsvd_tensor& t = k ? y[i] : x[i];
      if (t.dtype != (int)t.dtype || !bytes_of((int)t.dtype) || t.rows < 0 || t.cols < 0 || t.rows != x[i].rows || t.cols != x[i].cols) return refused;
      if (t.rows == 0 || t.cols == 0) continue;
      int64_t all = 0;
      if (!t.data || t.rows > INT32_MAX || __builtin_mul_overflow(t.rows, t.cols, &all) || all > kMaxNumbers) return refused;
      if (t.rows > 1 && (t.ld < t.cols || __builtin_mul_overflow(t.rows, t.ld, &all) || all > kMaxNumbers)) return refused;
    }
    numbers += x[i].rows * x[i].cols;
    if (numbers > kMaxNumbers) return refused;
  }
  Pieces p{kLeastPiece, 0};
  while ((p.log_piece < most && numbers >> p.log_piece > 2048) || numbers >> p.log_piece > 1 << 22) ++p.log_piece;
  for (int64_t i = 0; i < count; ++i) {
    p.pieces += shape_of(x[i], y ? y + i : nullptr, p.log_piece).pieces;
    if (p.pieces > kMaxPieces) return refused;
  }
  return p;
}
// Where a tensor's numbers lie: `rows` times `width` bytes from `lo` on, `ld` bytes apart
struct Place {
  uintptr_t lo, hi;
  int64_t width, ld;         // ld = 0: one row
  bool written;
};
static Place place_of(const brsvd_tensor& t, bool written) {
  const int64_t eb = bytes_of((int)t.dtype);
  const bool one = t.rows == 1 || t.ld == t.cols;
  const uintptr_t lo = (uintptr_t)t.data;
  return Place{lo, lo + (uintptr_t)(((t.rows - 1) * (one ? t.cols : t.ld) + t.cols) * eb), (one ? t.rows * t.cols : t.cols) * eb, one ? 0 : t.ld * eb, written};
}
// Of places of which b begins in a's extent: whether they share no number, as columns of one matrix do not
static bool apart(const Place& a, const Place& b) {
  const int64_t ld = a.ld ? a.ld : b.ld;
  if (ld == 0 || (a.ld && b.ld && a.ld != b.ld)) return false;
  const int64_t d = (int64_t)((b.lo - a.lo) % (uintptr_t)ld);
  return d >= a.width && d + b.width <= ld;
}
// Whether a number that one tensor is written to is another's too, whichever of its list, or part of the norm, which all workgroups read; a tensor may be written to its own place.
static int check_places(const brsvd_tensor* x, const brsvd_tensor* y, int64_t count, const float* norm) {
  if (count == 0) return BRSVD_OK;
  Place* places = new (std::nothrow) Place[2 * count + 1];
  if (!places) return BRSVD_ERR_ALLOC;
  int64_t n = 0;
  bool good = true;
  for (int list = 0; list < 2; ++list) {
    const int64_t first = n;
    for (int64_t i = 0; i < count; ++i) {
      if (x[i].rows == 0 || x[i].cols == 0) continue;
      if (list == 0) {
        places[n++] = place_of(y[i], true);
        good &= y[i].data != x[i].data || (y[i].dtype == x[i].dtype && (x[i].rows == 1 || y[i].ld == x[i].ld));
      } else if (y[i].data != x[i].data) {
        places[n++] = place_of(x[i], false);
      }
    }
    if (list == 1) places[n++] = Place{(uintptr_t)norm, (uintptr_t)norm + sizeof(float), sizeof(float), 0, false};
    auto before = [](const Place& a, const Place& b) { return a.lo < b.lo; };
    if (!std::is_sorted(places + first, places + n, before)) std::sort(places + first, places + n, before);
    if (list == 1) std::inplace_merge(places, places + first, places + n, before);
  }
  for (int64_t i = 0; i < n; ++i)
    for (int64_t j = i + 1; j < n && places[j].lo < places[i].hi && good; ++j) good = (!places[i].written && !places[j].written) || apart(places[i], places[j]);
  delete[] places;
  return good ? BRSVD_OK : BRSVD_ERR_ARG;
}
// launch(list, workgroups) for as many tensors at a time as a list holds
template <class Launch>
static void in_lists(const brsvd_tensor* x, const brsvd_tensor* y, int64_t count, int log_piece, Launch launch) {
  TensorList l;
  l.count = 0;
  l.piece = 1 << log_piece;
  uint32_t pieces = 0;
  auto flush = [&] {
    if (pieces == 0) return;
    launch(l, pieces);
    l.count = 0;
    pieces = 0;
  };
  auto put = [&](const void* a, void* b, int64_t cols, int types) {
    const int c = l.count++;
    l.x[c] = (const char*)a;
    l.y[c] = (char*)b;
    l.cols[c] = cols;
    l.first[c] = pieces;
    l.types[c] = (uint8_t)types;
  };
  for (int64_t i = 0; i < count; ++i) {
    const Shape s = shape_of(x[i], y ? y + i : nullptr, log_piece);
    if (s.pieces == 0) continue;
    if (l.count + (s.rows > 1 ? 2 : 1) > kPlaces) flush();
    put(x[i].data, y ? y[i].data : nullptr, s.cols, (int)x[i].dtype | (y ? (int)y[i].dtype << 2 : 0));
    if (s.rows > 1) put((const void*)x[i].ld, y ? (void*)y[i].ld : nullptr, (int64_t)s.rows_per << 32 | s.rows, kStrided);
    pieces += (uint32_t)s.pieces;
  }
  flush();
}

}  // namespace brsvd

using namespace brsvd;

extern "C" uint64_t brsvd_grad_norm_workspace_bytes(const brsvd_tensor* tensors, int64_t count) {
  const int64_t pieces = check_list(tensors, nullptr, count, kNormPiece).pieces;
  return pieces < 0 ? 0 : (uint64_t)(pieces + 32) / 32 * 256;
}

extern "C" int brsvd_grad_norm(const brsvd_tensor* tensors, int64_t count, float scale, float* norm, void* workspace, uint64_t workspace_bytes, void* stream) {
  const Pieces p = check_list(tensors, nullptr, count, kNormPiece);
  if (p.pieces < 0 || !norm || !(fabsf(scale) <= 3.402823466e38f)) return BRSVD_ERR_ARG;
  if (!workspace || (uintptr_t)workspace % 256) return BRSVD_ERR_ARG;
  if (workspace_bytes < (uint64_t)(p.pieces + 32) / 32 * 256) return BRSVD_ERR_BUDGET;
  hipStream_t s = (hipStream_t)stream;
  double* sums = (double*)workspace;
  in_lists(tensors, nullptr, count, p.log_piece, [&](const TensorList& l, unsigned grid) {
    hipLaunchKernelGGL(k_grad_squares, dim3(grid), dim3(256), 0, s, l, sums);
    sums += grid;
  });
  hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(1024), 0, s, (const double*)workspace, p.pieces, fabs((double)scale), norm);
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}

extern "C" int brsvd_grad_clip(const brsvd_tensor* tensors, const brsvd_tensor* out, int64_t count, float scale, float max_norm, const float* norm, void* stream) {
  const Pieces p = count > 0 && !out ? Pieces{0, -1} : check_list(tensors, out, count, kClipPiece);
  if (p.pieces < 0 || !norm || !(fabsf(scale) <= 3.402823466e38f) || !(max_norm >= 0.f)) return BRSVD_ERR_ARG;
  BRSVD_TRY(check_places(tensors, out, count, norm));
  if (p.pieces == 0) return BRSVD_OK;
  hipStream_t s = (hipStream_t)stream;
  in_lists(tensors, out, count, p.log_piece, [&](const TensorList& l, unsigned grid) {
    hipLaunchKernelGGL(k_grad_clip, dim3(grid), dim3(256), 0, s, l, norm, (double)scale, (double)max_norm);
  });
  BRSVD_HIP_TRY(hipGetLastError());
  return BRSVD_OK;
}
