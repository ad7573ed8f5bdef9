// Numbers of 4 bits (e2m1: two bits of exponent, one of fraction: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives), two in a byte, the first in its lower half,
// with a scale of 8 bits (e8m0: 2^(byte - 127), 255 for NaN) for each 32 neighbouring numbers of a row.
#pragma once
#include "tile.h"

namespace brsvd {

constexpr int kGroup = 32;       // numbers of a row that share a scale

// The least e >= -126 with top <= 6 * 2^e, 0 for top = 0; top >= 0 is finite.  6 = 1.5 * 2^2, so it is read off the bits.
__device__ __forceinline__ int group_exponent(float top) {
  const uint32_t b = __float_as_uint(top);
  const int e = (int)(b >> 23) - 129 + ((b & 0x7fffffu) > 0x400000u);
  return top > 0.f ? (e < -126 ? -126 : e) : 0;
}
// What the conversions take as a scale: they read its eight bits of exponent alone, 0 as 2^-127 and 255 as NaN (measured over all bytes and numbers).
__device__ __forceinline__ float scale_e8m0(uint32_t byte) { return __uint_as_float(byte << 23); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// The two numbers of byte B of w times the scale, rounded to the type (bf16 holds all of them from 2^-127 to 6 * 2^125)
template <class El, int B>
__device__ __forceinline__ uint32_t two_e2m1(uint32_t w, float scale) {
  if constexpr (__is_same(El, Bf16)) return __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
  else return __builtin_bit_cast(uint32_t, (f16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, B));
}
// Eight numbers
template <class El>
__device__ __forceinline__ uint4 eight_e2m1(uint32_t w, float scale) {
  return make_uint4(two_e2m1<El, 0>(w, scale), two_e2m1<El, 1>(w, scale), two_e2m1<El, 2>(w, scale), two_e2m1<El, 3>(w, scale));
}

// 16 bytes from `src`, the numbers of a group, of which the first `valid` are there; the others are zero.
__device__ __forceinline__ uint4 group_of(const uint8_t* src, int64_t valid) {
  if (valid >= kGroup) {
    const Piece v = *(const Piece*)src;
    return make_uint4(v.x[0], v.x[1], v.x[2], v.x[3]);
  }
  uint4 v = piece_of<1>((const char*)src, valid > 0 ? (valid + 1) / 2 : 0);
  if (valid > 0 && (valid & 1)) {            // the upper half of the last byte is no number of the row
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((int)valid / 8 == i) w[i] &= ~(0xfu << (4 * ((int)valid & 7)));
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}

// A matrix in 4 bits as an operand of a tile product
struct E2m1Operand {
  const uint8_t* base;
  int64_t ld;                // bytes from one stored row to the next
  int64_t n;                 // rows (kRows) or columns (kCols) of the output that it spans
  const uint8_t* scales;     // [row][groups]
  int64_t groups;
};

// Fills P's tile from a matrix in 4 bits: a thread has a group of a step, makes 32 numbers of 16 bits of it and writes them where Stager puts them.
//   kRows: the step's 64 numbers of a row are two groups, of two threads.    kCols: 64 rows of 256 columns, eight groups of a row.
template <class El, Order O>
struct E2m1Stager {
  static constexpr bool kAhead = true;
  static constexpr int kLoads = 0;   // straight into LDS
  using Source = E2m1Operand;
  struct Pieces {
    uint4 w;
    uint32_t s;
  };
  Pieces ahead;
  const uint8_t *at, *scale_at;      // of the next step, the same in all lanes
  uint32_t off, scale_off;
  int64_t step, scale_step;
  int32_t valid;                     // kCols: the group's columns that are there

  __device__ __forceinline__ void init(const E2m1Operand& op, int64_t first, int64_t k0, int tid) {
    const int64_t left = op.n - first;
    if (O == kRows) {
      const int64_t row = tid >> 1, r = row < left ? row : left - 1;
      at = op.base + first * op.ld + k0 / 2;
      scale_at = op.scales + first * op.groups + k0 / kGroup;
      step = 32;
      scale_step = 2;
      off = (uint32_t)(r * op.ld + 16 * (tid & 1));
      scale_off = (uint32_t)(r * op.groups + (tid & 1));
    } else {
      const int row = tid >> 3, c = tid & 7;
      at = op.base + k0 * op.ld + first / 2;
      scale_at = op.scales + k0 * op.groups + first / kGroup;
      step = 64 * op.ld;
      scale_step = 64 * op.groups;
      valid = (int32_t)(left - kGroup * c < kGroup ? left - kGroup * c : kGroup);
      off = (uint32_t)(row * op.ld + 16 * c);
      scale_off = (uint32_t)(row * op.groups + c);
    }
    at = (const uint8_t*)scalar((int64_t)at);
    scale_at = (const uint8_t*)scalar((int64_t)scale_at);
    step = scalar(step);
    scale_step = scalar(scale_step);
  }
  __device__ __forceinline__ bool plain(int64_t) const { return true; }
  // left: numbers of the contraction from the step on
  __device__ __forceinline__ void fetch(Pieces& x, int64_t left) {
    const int there = O == kRows ? (int)(left < 64 ? left : 64) - kGroup * (threadIdx.x & 1) : (int)threadIdx.x >> 3 < left ? valid : 0;
    if (there >= kGroup) {
      const Piece v = *(const Piece*)(at + off);
      x.w = make_uint4(v.x[0], v.x[1], v.x[2], v.x[3]);
      x.s = scale_at[scale_off];
    } else {
      x.w = group_of(at + off, there);
      x.s = there > 0 ? scale_at[scale_off] : 127;
    }
    at += step;
    scale_at += scale_step;
  }
  // Behind the workgroup's barrier, for which all loads have come: the compiler's own wait for these is here, before others are sent for.
  __device__ __forceinline__ void arrived() { asm volatile("" : "+v"(ahead.w.x), "+v"(ahead.w.y), "+v"(ahead.w.z), "+v"(ahead.w.w), "+v"(ahead.s)); }
  // Eight of the numbers
  __device__ __forceinline__ void store_part(char* tile, const Pieces& x, int i) const {
    const int tid = threadIdx.x;
    const uint32_t w = i == 0 ? x.w.x : i == 1 ? x.w.y : i == 2 ? x.w.z : x.w.w;
    uint32_t to;
    if (O == kRows) {
      const int row = tid >> 1;
      to = row * kStepBytes + 16 * ((4 * (tid & 1) + i) ^ (row & 7));
    } else {
      const int row = tid >> 3, src = 4 * (tid & 7) + i;
      to = row * 512 + 16 * (((src >> 1) ^ (Stager<El, kCols, 256, 512, true>::mix(row) & 15)) * 2 + (src & 1));
    }
    *(uint4*)(tile + to) = eight_e2m1<El>(w, scale_e8m0(x.s));
  }
};

}  // namespace brsvd
