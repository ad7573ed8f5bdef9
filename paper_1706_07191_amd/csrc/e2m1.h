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

// Lane l of a wave has word i of group l / 16 of row l % 16 in w[i]; afterwards word l / 16 of group i.  What an instruction multiplies next to each other is
// then next to each other in the row, as 16-bit operands that are read 16 bytes a lane have it.
__device__ __forceinline__ void turn_groups(uint32_t (&w)[4]) {
  typedef uint32_t Two __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Two v = __builtin_amdgcn_permlane32_swap(w[i], w[i + 2], false, false);      // the upper half of one with the lower half of the other
    w[i] = v[0];
    w[i + 2] = v[1];
  }
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const Two v = __builtin_amdgcn_permlane16_swap(w[i], w[i + 1], false, false);      // odd sixteens of one with even sixteens of the other
    w[i] = v[0];
    w[i + 1] = v[1];
  }
}

// A matrix in 4 bits as an operand of a tile product
struct E2m1Operand {
  const uint8_t* base;
  int64_t ld;                // bytes from one stored row to the next
  int64_t n;                 // rows (kRows) or columns (kCols) of the output that it spans
  const uint8_t* scales;     // [row][groups]
  int64_t groups;
};

// 1 byte per lane into LDS, a word each, at `dst` (the same in all lanes) + 4 lane, from `off` bytes behind an address that all lanes share.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load1_to_lds(uint32_t dst, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %2, %1" ::"s"(__builtin_amdgcn_readfirstlane(dst)), "s"(base), "v"(off) : "memory", "m0");
}
#pragma clang diagnostic pop

// A tile product like TileProduct's (its order of slots, fragments and sums) whose P is a matrix in 4 bits.  A step takes 256 x 64 numbers of it, two groups of 256 rows
// (kRows) or eight groups of 64 rows (kCols), a group a thread.  Pieces of 16 bytes and their scales go straight into a ring in LDS, NB + 1 steps ahead; behind the
// workgroup's barrier in step t each thread makes 32 numbers of 16 bits of its own group of step t + 2 and writes them, where Stager would put them, into the buffer that has
// just been read.  So all loads are counted in the order they were sent, and the barrier waits only for those of the step that comes next; Q's tiles are NB deep.
// W's rows begin at 16-byte addresses.
template <class El, int NQ_, Order O>
struct E2m1Product {
  static constexpr int NP = 8, NQ = NQ_, WP = 2, WQ = 4;
  static constexpr int BP = 16 * NP * WP, BQ = 16 * NQ * WQ, kThreads = 64 * WP * WQ;
  static constexpr int NB = NQ == 4 ? 2 : NQ == 2 ? 3 : 4;
  static constexpr int kP = BP * kStepBytes, kQ = BQ * kStepBytes, kRing = kThreads * 20;
  static constexpr int kLds = 2 * kP + NB * kQ + NB * kRing;
  using StageQ = Stager<El, kRows, BQ, kThreads, true>;
  static constexpr int PARTS = StageQ::kLoads;

  StageQ sq;
  char* lds;
  int64_t k;                         // of the contraction
  const uint8_t *at, *scale_at;      // of the next step, the same in all lanes
  uint32_t off, scale_off;
  int64_t step, scale_step;
  int32_t valid;                     // kCols: the group's columns that are there
  bool ragged;                       // kCols: the columns end inside the tile's last group

  struct Group {
    uint4 w;
    uint32_t s;
  };
  __device__ __forceinline__ int steps() const { return (int)((k + 63) / 64); }
  __device__ __forceinline__ char* p_tile(int t) const { return lds + (t & 1) * kP; }
  __device__ __forceinline__ char* q_tile(int slot) const { return lds + 2 * kP + slot * kQ; }
  __device__ __forceinline__ char* ring(int slot) const { return lds + 2 * kP + NB * kQ + slot * kRing; }
  // Whether all of a step's pieces are there in whole: a row's last piece may lie on memory behind the matrix in its last row only
  __device__ __forceinline__ bool plain(int t) const {
    const int64_t left = k - (int64_t)t * 64;
    return left >= 64 && !(O == kCols && ragged && left <= 64);
  }
  __device__ __forceinline__ void init(const E2m1Operand& op, int64_t first, int64_t k0) {
    const int tid = threadIdx.x;
    const int64_t left = op.n - first;
    if (O == kRows) {
      const int64_t row = tid >> 1, r = row < left ? row : left - 1;
      at = op.base + first * op.ld + k0 / 2;
      scale_at = op.scales + first * op.groups + k0 / kGroup;
      step = 32;
      scale_step = 2;
      off = (uint32_t)(r * op.ld + 16 * (tid & 1));
      scale_off = (uint32_t)(r * op.groups + (tid & 1));
      ragged = false;
      valid = kGroup;
    } else {
      const int row = tid >> 3, c = kGroup * (tid & 7) < left ? tid & 7 : 0;      // a group beyond the end: some other one, nothing of it is stored
      at = op.base + k0 * op.ld + first / 2;
      scale_at = op.scales + k0 * op.groups + first / kGroup;
      step = 64 * op.ld;
      scale_step = 64 * op.groups;
      ragged = left < BP && left % kGroup != 0;
      valid = (int32_t)(left - kGroup * c < kGroup ? left - kGroup * c : kGroup);
      off = (uint32_t)(row * op.ld + 16 * c);
      scale_off = (uint32_t)(row * op.groups + c);
    }
    at = (const uint8_t*)scalar((int64_t)at);
    scale_at = (const uint8_t*)scalar((int64_t)scale_at);
    step = scalar(step);
    scale_step = scalar(scale_step);
  }
  // This thread's group of step t, which is the next
  __device__ __forceinline__ Group fetch(int t) {
    const int64_t left = k - (int64_t)t * 64;
    const int there = O == kRows ? (int)(left < 64 ? left : 64) - kGroup * (threadIdx.x & 1) : (int)threadIdx.x >> 3 < left ? valid : 0;
    Group x;
    x.w = group_of(at + off, there);
    x.s = there > 0 ? scale_at[scale_off] : 127;
    at += step;
    scale_at += scale_step;
    return x;
  }
  __device__ __forceinline__ void send_group(int t, char* to) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (plain(t)) {
      load_to_lds(lds_address(to) + 1024 * wave, (const char*)scalar((int64_t)at), off);
      load1_to_lds(lds_address(to) + kThreads * 16 + 256 * wave, (const void*)scalar((int64_t)scale_at), scale_off);
      at += step;
      scale_at += scale_step;
    } else {
      const Group x = fetch(t);
      *(uint4*)(to + 16 * tid) = x.w;
      *(uint32_t*)(to + kThreads * 16 + 4 * tid) = x.s;
    }
  }
  __device__ __forceinline__ Group group_in(const char* from) const {
    const int tid = threadIdx.x;
    return Group{*(const uint4*)(from + 16 * tid), *(const uint32_t*)(from + kThreads * 16 + 4 * tid)};
  }
  // Eight of a group's numbers to where fragments of them are read
  __device__ __forceinline__ void make_part(char* tile, const Group& x, int i) const {
    const int tid = threadIdx.x;
    const uint32_t w = i == 0 ? x.w.x : i == 1 ? x.w.y : i == 2 ? x.w.z : x.w.w;
    uint32_t to;
    if (O == kRows) {
      const int row = tid >> 1;
      to = row * kStepBytes + 16 * ((4 * (tid & 1) + i) ^ (row & 7));
    } else {
      const int row = tid >> 3, src = 4 * (tid & 7) + i;
      to = row * (2 * BP) + 16 * (((src >> 1) ^ (Stager<El, kCols, BP, kThreads, true>::mix(row) & 15)) * 2 + (src & 1));
    }
    *(uint4*)(tile + to) = eight_e2m1<El>(w, scale_e8m0(x.s));
  }
  // The workgroup's barrier.  ahead: steps whose loads may still be on their way, sent in full, and the groups of the one before them.
  template <int AHEAD>
  static __device__ __forceinline__ void meet() {
    __builtin_amdgcn_sched_barrier(0);
    if (AHEAD >= 0) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD < 0 ? 0 : AHEAD) * (PARTS + 2) + 2) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void send_q(int t, char* to) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    sq.load(to, threadIdx.x, wave, k - (int64_t)t * 64);
  }

  static __device__ __forceinline__ void run(floatx4 (&acc)[NP][NQ], const E2m1Operand& P, int64_t p0, const Operand& Q, int64_t q0, int64_t k0, int64_t k1, char* lds_) {
    E2m1Product x;
    x.lds = lds_;
    x.k = scalar(k1 - k0);
    x.init(P, p0, k0);
    x.sq.init(Q, q0, k0, threadIdx.x);
    x.multiply(acc);
  }
  __device__ __forceinline__ void multiply(floatx4 (&acc)[NP][NQ]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP, steps = this->steps();
    constexpr int SLOTS = 2 * NP, MEET = SLOTS - 4;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int q = 0; q < NQ; ++q) acc[p][q] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (steps == 0) return;
    {
      // the first two steps' groups through registers, all else behind them
      Group x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (steps > t) x[t] = fetch(t);
#pragma unroll
      for (int t = 0; t < NB; ++t)
        if (steps > t) send_q(t, q_tile(t));
#pragma unroll
      for (int t = 2; t < NB + 2; ++t)
        if (steps > t) send_group(t, ring(t % NB));
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (steps > t)
#pragma unroll
          for (int i = 0; i < 4; ++i) make_part(p_tile(t), x[t], i);
    }
    int4v fp[8], fq[2][NQ];
    uint32_t bp = fragment_base<O, BP>(16 * wp * NP, lane), bq = fragment_base<kRows, BQ>(16 * wq * NQ, lane);
    auto read_p = [&](const char* tile, int slot) { fp[slot & 7] = fragment<O, BP>(tile, bp, slot & 7, slot >> 3); };
    auto read_q = [&](const char* tile, int kk, int q) { fq[kk][q] = fragment<kRows, BQ>(tile, bq, q, kk); };
    meet<-1>();
#pragma unroll
    for (int i = 0; i < 4; ++i) read_p(p_tile(0), i);
#pragma unroll
    for (int q = 0; q < NQ; ++q) read_q(q_tile(0), 0, q);
    int slot = 0, rslot = 2 % NB;        // t % NB, (t + 2) % NB
    Group x = {};
    for (int t = 0; t < steps; ++t) {
      slot = __builtin_amdgcn_readfirstlane(slot);
      rslot = __builtin_amdgcn_readfirstlane(rslot);
      const int next = slot == NB - 1 ? 0 : slot + 1;
      char *pc = p_tile(t), *qc = q_tile(slot);
      const char *pn = p_tile(t + 1), *qn = q_tile(next);
      const bool more = t + 1 < steps, sends = t + NB < steps, makes = t + 2 < steps, groups = t + NB + 2 < steps;
      bool parts = false;
      asm volatile("" : "+v"(bp), "+v"(bq));      // addresses are worked out from these where they are used, not kept
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        if (s < 4) {
          read_p(pc, s + 4);
          if (s < NQ) read_q(qc, 1, s);
        } else if (s < 6) {
          read_p(pc, 2 * s);
          read_p(pc, 2 * s + 1);
        } else if (s < 10) {
          read_p(pc, s + 6);
        } else if (s == MEET) {
          if (t + 1 + NB < steps && plain(t + 1 + NB)) meet<NB - 2>();
          else meet<-1>();
          if (makes) x = group_in(ring(rslot));
          parts = sends && plain(t + NB);
          if (sends && !parts) send_q(t + NB, qc);
        }
        if (s >= MEET) {
          if (parts && s - MEET < PARTS) sq.load_part(qc, wave, s - MEET);
          if (parts && s == MEET + PARTS - 1) sq.next();
          if (more) {
            read_p(pn, s - MEET);
            if (s - MEET < NQ) read_q(qn, 0, s - MEET);
          }
          if (makes) {
            if (s == MEET + 1) make_part(pc, x, 0);
            if (s == MEET + 2) make_part(pc, x, 1), make_part(pc, x, 2);
            if (s == MEET + 3) make_part(pc, x, 3);
          }
          if (s == SLOTS - 1 && groups) send_group(t + NB + 2, ring(rslot));
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          acc[s & 7][q] = mfma16<El>(fp[s & 7], fq[s >> 3][q], acc[s & 7][q]);
          settle(acc[s & 7][q]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      slot = next;
      rslot = rslot == NB - 1 ? 0 : rslot + 1;
    }
    meet<-1>();
  }
};

}  // namespace brsvd
