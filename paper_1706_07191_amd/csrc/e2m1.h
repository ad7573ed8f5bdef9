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

// The two numbers of byte B of w times the scale, rounded to the type: bf16 holds all of them, from 2^-128 to 1.5 * 2^127, fp16 those from 2^-23 to 49152; from 2^128 and 2^16 on
// they are infinite
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

// 16 bytes from `src`, of which the first `have` are there and the others zero; `before` bytes of the row are in front of them.  One load, of the row's last 16 bytes: put together
// number by number, each waiting for the one before, the end of a contraction took as long as ten of its steps.
__device__ __forceinline__ uint4 piece_at_end(const uint8_t* src, int64_t have, int64_t before) {
  if (have <= 0) return make_uint4(0u, 0u, 0u, 0u);
  if (have < 16 && before + have < 16) return piece_of<1>((const char*)src, have);
  const int back = have < 16 ? 16 - (int)have : 0;
  const Piece v = *(const Piece*)(src - back);
  uint64_t lo = v.x[0] | (uint64_t)v.x[1] << 32, hi = v.x[2] | (uint64_t)v.x[3] << 32;
  const int s = 8 * back;
  if (s >= 64) lo = hi >> (s - 64), hi = 0;
  else if (s > 0) lo = lo >> s | hi << (64 - s), hi >>= s;
  return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

// 16 bytes from `src`, the numbers of a group, of which the first `valid` are there; the others are zero.  `before`: the row's bytes in front of them
__device__ __forceinline__ uint4 group_of(const uint8_t* src, int64_t valid, int64_t before) {
  if (valid >= kGroup) {
    const Piece v = *(const Piece*)src;
    return make_uint4(v.x[0], v.x[1], v.x[2], v.x[3]);
  }
  uint4 v = piece_at_end(src, valid > 0 ? (valid + 1) / 2 : 0, before);
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

// What brings a matrix in 4 bits into LDS for tile products.  A step takes 64 numbers of the contraction: of 256 rows two groups each (kRows), or of 64 rows eight groups each
// (kCols); a group a thread.  Its 16 bytes and its scale, a word, go straight into a slot of a ring.  Rows begin at 16-byte addresses.
template <Order O>
struct E2m1Feed {
  static constexpr int kThreads = 512, kSlot = kThreads * 20, kLoads = 2;      // bytes; loads of a wave for a step
  int64_t k;                         // of the contraction
  const uint8_t *at, *scale_at;      // of the next step, the same in all lanes
  uint32_t off, scale_off;
  int64_t step, scale_step;
  int32_t valid;                     // kCols: the group's columns that are there
  int32_t front;                     // bytes of the row that are in front of the first step's group at least
  bool ragged;                       // kCols: the columns end inside the tile's last group

  struct Group {
    uint4 w;
    uint32_t s;
  };
  __device__ __forceinline__ void init(const E2m1Operand& op, int64_t first, int64_t k0, int64_t k1) {
    const int tid = threadIdx.x;
    const int64_t left = op.n - first;
    k = scalar(k1 - k0);
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
      front = 16 * (tid & 1);
    } else {
      const int row = tid >> 3, c = kGroup * (tid & 7) < left ? tid & 7 : 0;      // a group beyond the end: some other one, nothing of it is stored
      at = op.base + k0 * op.ld + first / 2;
      scale_at = op.scales + k0 * op.groups + first / kGroup;
      step = 64 * op.ld;
      scale_step = 64 * op.groups;
      ragged = left < 256 && left % kGroup != 0;
      valid = (int32_t)(left - kGroup * c < kGroup ? left - kGroup * c : kGroup);
      front = 16 * c;
      off = (uint32_t)(row * op.ld + 16 * c);
      scale_off = (uint32_t)(row * op.groups + c);
    }
    at = (const uint8_t*)scalar((int64_t)at);
    scale_at = (const uint8_t*)scalar((int64_t)scale_at);
    step = scalar(step);
    scale_step = scalar(scale_step);
  }
  __device__ __forceinline__ int steps() const { return (int)((k + 63) / 64); }
  // Whether all of a step's pieces are there in whole: a row's last piece may lie on memory behind the matrix in its last row only
  __device__ __forceinline__ bool plain(int t) const {
    const int64_t left = k - (int64_t)t * 64;
    return left >= 64 && !(O == kCols && ragged && left <= 64);
  }
  // This thread's group of step t, which is the next
  __device__ __forceinline__ Group fetch(int t) {
    const int64_t left = k - (int64_t)t * 64;
    const int there = O == kRows ? (int)(left < 64 ? left : 64) - kGroup * (threadIdx.x & 1) : (int)threadIdx.x >> 3 < left ? valid : 0;
    Group x;
    x.w = group_of(at + off, there, front + (O == kRows ? (int64_t)t * 32 : 0));
    x.s = there > 0 ? scale_at[scale_off] : 127;
    at += step;
    scale_at += scale_step;
    return x;
  }
  __device__ __forceinline__ void send(int t, char* to) {
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
  static __device__ __forceinline__ Group mine(const char* slot) {
    const int tid = threadIdx.x;
    return Group{*(const uint4*)(slot + 16 * tid), *(const uint32_t*)(slot + kThreads * 16 + 4 * tid)};
  }
};

// The workgroup's barrier; up to LOADS of a wave's loads may still be on their way.
template <int LOADS>
__device__ __forceinline__ void meet_but() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Tile products like TileProduct's (its slots, its fragments of Q, its sums) whose P is a matrix in 4 bits.  E2m1Product<.., kRows>: fragments of P are made where they are
// multiplied.  Of a row's 64 numbers in a step lane group g has the 16 from 32 (g & 1) + 16 (g >> 1) on, one read of eight bytes for both halves of the step, and one
// scale; Q's fragments are read in the same order.  That reads 14 KiB from LDS a wave and step, where fragments of 16 bits are 24, and
// leaves room for NB steps in LDS: the barrier waits for the step that comes next only.
template <class El, int NQ_, Order O> struct E2m1Product;
template <class El, int NQ_>
struct E2m1Product<El, NQ_, kRows> {
  static constexpr int NP = 8, NQ = NQ_, WP = 2, WQ = 4;
  static constexpr int BP = 16 * NP * WP, BQ = 16 * NQ * WQ, kThreads = 64 * WP * WQ;
  using Feed = E2m1Feed<kRows>;
  using StageQ = Stager<El, kRows, BQ, kThreads, true>;
  static constexpr int NB = NQ == 4 ? 3 : NQ == 2 ? 4 : 6, kQ = BQ * kStepBytes, kPart = kQ + Feed::kSlot, LOADS = StageQ::kLoads + Feed::kLoads;
  static constexpr int kLds = NB * kPart > BQ * 512 ? NB * kPart : BQ * 512;        // put_tile16 takes BQ rows of 512 bytes

  static __device__ __forceinline__ void run(floatx4 (&acc)[NP][NQ], const E2m1Operand& P, int64_t p0, const Operand& Q, int64_t q0, int64_t k0, int64_t k1, char* lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
    constexpr int SLOTS = 2 * NP, MEET = SLOTS - 4;
    Feed feed;
    StageQ sq;
    feed.init(P, p0, k0, k1);
    sq.init(Q, q0, k0, tid);
    const int steps = feed.steps();
    auto left = [&](int t) { return feed.k - (int64_t)t * 64; };
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int q = 0; q < NQ; ++q) acc[p][q] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < NB; ++t)
      if (steps > t) {
        sq.load(lds + t * kPart, tid, wave, left(t));
        feed.send(t, lds + t * kPart + kQ);
      }
    uint2 w[NP];
    uint32_t s[NP];
    int4v fq[2][NQ];
    const int row = lane & 15, g = lane >> 4;
    uint32_t bp = 32 * (16 * wp * NP + row) + 16 * (g & 1) + 8 * (g >> 1), bs = kThreads * 16 + 8 * (16 * wp * NP + row) + 4 * (g & 1);
    uint32_t bq = (16 * wq * NQ + row) * kStepBytes + 16 * ((4 * (g & 1) + 2 * (g >> 1)) ^ (row & 7));
    auto read_p = [&](const char* part, int p) {
      w[p] = *(const uint2*)(part + kQ + bp + 512 * p);
      s[p] = *(const uint32_t*)(part + kQ + bs + 128 * p);
    };
    auto read_q = [&](const char* part, int kk, int q) { fq[kk][q] = *(const int4v*)(part + (bq ^ (16 * kk)) + q * 16 * kStepBytes); };
    if (steps >= NB && feed.plain(NB - 1)) meet_but<(NB - 1) * LOADS>();
    else meet_but<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i) read_p(lds, i);
#pragma unroll
    for (int q = 0; q < NQ; ++q) read_q(lds, 0, q);
    int slot = 0;                // t % NB
    for (int t = 0; t < steps; ++t) {
      slot = __builtin_amdgcn_readfirstlane(slot);
      const int next = slot == NB - 1 ? 0 : slot + 1;
      char* cur = lds + slot * kPart;
      const char* nxt = lds + next * kPart;
      const bool more = t + 1 < steps, sends = t + NB < steps;
      bool parts = false;
      asm volatile("" : "+v"(bp), "+v"(bq), "+v"(bs));      // addresses are worked out from these where they are used, not kept
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) {
        if (i < 4) {
          read_p(cur, i + 4);
          if (i < NQ) read_q(cur, 1, i);
        } else if (i == MEET) {
          if (t + NB - 1 < steps && feed.plain(t + NB - 1)) meet_but<(NB - 2) * LOADS>();
          else meet_but<0>();
          parts = sends && feed.plain(t + NB);
          if (sends && !parts) {
            sq.load(cur, tid, wave, left(t + NB));
            feed.send(t + NB, cur + kQ);
          }
        }
        if (i >= MEET) {
          if (parts && i - MEET < StageQ::kLoads) sq.load_part(cur, wave, i - MEET);
          if (parts && i == SLOTS - 1) {
            sq.next();
            feed.send(t + NB, cur + kQ);
          }
          if (more) {
            read_p(nxt, i - MEET);
            if (i - MEET < NQ) read_q(nxt, 0, i - MEET);
          }
        }
        const int p = i & 7, kk = i >> 3;
        // raw numbers of tile rows 0 to 3 are replaced from MEET on, their last use is before
        const int4v f = __builtin_bit_cast(int4v, eight_e2m1<El>(kk ? w[p].y : w[p].x, scale_e8m0(s[p])));
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          acc[p][q] = mfma16<El>(f, fq[kk][q], acc[p][q]);
          settle(acc[p][q]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      slot = next;
    }
    meet_but<0>();
  }
};

// E2m1Product<.., kCols>: the contraction runs down W's rows, a fragment has numbers of eight of them, with scales of their own.  So behind the workgroup's barrier in
// step t each thread makes 32 numbers of 16 bits of its group of step t + 2 and writes them where Stager would put them, into the buffer that has just been read; the groups
// come NB + 2 steps ahead, Q's tiles NB.
template <class El, int NQ_>
struct E2m1Product<El, NQ_, kCols> {
  static constexpr int NP = 8, NQ = NQ_, WP = 2, WQ = 4;
  static constexpr int BP = 16 * NP * WP, BQ = 16 * NQ * WQ, kThreads = 64 * WP * WQ;
  using Feed = E2m1Feed<kCols>;
  using Group = Feed::Group;
  using StageQ = Stager<El, kRows, BQ, kThreads, true>;
  static constexpr int NB = NQ == 4 ? 2 : NQ == 2 ? 3 : 4;
  static constexpr int kP = BP * kStepBytes, kQ = BQ * kStepBytes, kLds = 2 * kP + NB * kQ + NB * Feed::kSlot, LOADS = StageQ::kLoads + Feed::kLoads;

  // Eight of a group's numbers to where fragments of them are read.  Threads of a row write its eight groups, in turns so that they meet no bank twice: `x` comes turned by
  // half the group's number.
  static __device__ __forceinline__ Group turned(Group x) {
    const int r = threadIdx.x >> 1;
    const uint32_t a = r & 1 ? x.w.y : x.w.x, b = r & 1 ? x.w.z : x.w.y, c = r & 1 ? x.w.w : x.w.z, d = r & 1 ? x.w.x : x.w.w;
    return Group{r & 2 ? make_uint4(c, d, a, b) : make_uint4(a, b, c, d), x.s};
  }
  static __device__ __forceinline__ void make_part(char* tile, const Group& x, int i) {
    const int tid = threadIdx.x, row = tid >> 3, src = 4 * (tid & 7) + ((i + (tid >> 1)) & 3);
    const uint32_t w = i == 0 ? x.w.x : i == 1 ? x.w.y : i == 2 ? x.w.z : x.w.w;
    *(uint4*)(tile + row * (2 * BP) + 16 * (((src >> 1) ^ (Stager<El, kCols, BP, kThreads, true>::mix(row) & 15)) * 2 + (src & 1))) = eight_e2m1<El>(w, scale_e8m0(x.s));
  }

  static __device__ __forceinline__ void run(floatx4 (&acc)[NP][NQ], const E2m1Operand& P, int64_t p0, const Operand& Q, int64_t q0, int64_t k0, int64_t k1, char* lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
    constexpr int SLOTS = 2 * NP, MEET = SLOTS - 4;
    Feed feed;
    StageQ sq;
    feed.init(P, p0, k0, k1);
    sq.init(Q, q0, k0, tid);
    const int steps = feed.steps();
    auto left = [&](int t) { return feed.k - (int64_t)t * 64; };
    auto p_tile = [&](int t) { return lds + (t & 1) * kP; };
    auto q_tile = [&](int slot) { return lds + 2 * kP + slot * kQ; };
    auto ring = [&](int slot) { return lds + 2 * kP + NB * kQ + slot * Feed::kSlot; };
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int q = 0; q < NQ; ++q) acc[p][q] = floatx4{0.f, 0.f, 0.f, 0.f};
    {
      // the first two steps' groups through registers, all else behind them
      Group x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (steps > t) x[t] = feed.fetch(t);
#pragma unroll
      for (int t = 0; t < NB; ++t)
        if (steps > t) sq.load(q_tile(t), tid, wave, left(t));
#pragma unroll
      for (int t = 2; t < NB + 2; ++t)
        if (steps > t) feed.send(t, ring(t % NB));
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (steps > t) {
          x[t] = turned(x[t]);
#pragma unroll
          for (int i = 0; i < 4; ++i) make_part(p_tile(t), x[t], i);
        }
    }
    int4v fp[8], fq[2][NQ];
    uint32_t bp = fragment_base<kCols, BP>(16 * wp * NP, lane), bq = fragment_base<kRows, BQ>(16 * wq * NQ, lane);
    auto read_p = [&](const char* tile, int slot) { fp[slot & 7] = fragment<kCols, BP>(tile, bp, slot & 7, slot >> 3); };
    auto read_q = [&](const char* tile, int kk, int q) { fq[kk][q] = fragment<kRows, BQ>(tile, bq, q, kk); };
    meet_but<0>();
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
          // all loads but those sent since the ones for Q's next tile: its groups, and the steps after it
          if (t + 1 + NB < steps && feed.plain(t + 1 + NB)) meet_but<(NB - 2) * LOADS + Feed::kLoads>();
          else meet_but<0>();
          if (makes) x = Feed::mine(ring(rslot));
          parts = sends && feed.plain(t + NB);
          if (sends && !parts) sq.load(qc, tid, wave, left(t + NB));
        }
        if (s >= MEET) {
          if (parts && s - MEET < StageQ::kLoads) sq.load_part(qc, wave, s - MEET);
          if (parts && s == MEET + StageQ::kLoads - 1) sq.next();
          if (more) {
            read_p(pn, s - MEET);
            if (s - MEET < NQ) read_q(qn, 0, s - MEET);
          }
          if (makes) {
            if (s == MEET + 1) x = turned(x), make_part(pc, x, 0);
            if (s == MEET + 2) make_part(pc, x, 1), make_part(pc, x, 2);
            if (s == MEET + 3) make_part(pc, x, 3);
          }
          if (s == SLOTS - 1 && groups) feed.send(t + NB + 2, ring(rslot));
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
    meet_but<0>();
  }
};

}  // namespace brsvd
