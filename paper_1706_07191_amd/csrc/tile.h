// Tile products on the 16-bit and 8-bit matrix cores (gfx950), shared by the 8-bit products and the losses over a vocabulary.
//
// A workgroup of WP x WQ waves works out D (BP x BQ) = P Q^T over a contraction of K numbers; a wave has NP x NQ tiles of 16 x 16.  In the
// instruction's result a lane holds four consecutive rows (of P) of one column (of Q), so P is the side along which the output is
// contiguous in memory: it is stored four numbers at a time.
//
// A step of the contraction takes 128 bytes of every row of P and Q (64 numbers of 16 bits, 128 of 8) into LDS, straight from memory
// (global_load_lds, 16 bytes a lane) into one of two buffers (three, TileProduct) while another is multiplied; one barrier a step.  An operand is
//   kRows: its rows hold the contraction, [rows][K].  A tile is [rows][128 bytes] in LDS, the 16-byte pieces of row r at piece ^ (r & 7): the 16
//          rows that a fragment is read from then lie in different banks.
//   kCols: the contraction runs down its rows, [K][cols] (16-bit numbers).  A tile is [64][cols]; fragments come out transposed
//          (ds_read_b64_tr_b16), pieces of 32 bytes are exchanged by a function of the row for the same reason.
// Rows and columns beyond the operand's end are read from inside it and dropped at the store; numbers of the contraction beyond K are zero on
// both sides: a piece that straddles an end is put together number by number.  DIRECT = false: for operands whose rows do not begin at 16-byte
// addresses; all pieces pass through registers.
#pragma once
#include "common.h"

namespace brsvd {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

// Element types of the operands.
struct Bf16 { static constexpr int kBytes = 2; };
struct Fp16 { static constexpr int kBytes = 2; };
struct E4m3 { static constexpr int kBytes = 1; };

constexpr int kStepBytes = 128;          // of the contraction per step
constexpr int64_t kMaxGrid = (int64_t)1 << 30;   // tiles or pieces of work of a call, which kernels count in 32 bits
enum Order { kRows = 0, kCols = 1 };

// One operand as a kernel gets it.
struct Operand {
  const char* base;
  int64_t ld;       // bytes from one stored row to the next
  int64_t n;        // rows (kRows) or columns (kCols) of the output that it spans
};

// Whether the pieces of 16 bytes that an operand's rows are read in lie at 16-byte addresses.
inline bool aligned_pieces(const void* base, int64_t ld_bytes) { return (uintptr_t)base % 16 == 0 && ld_bytes % 16 == 0; }
// Bytes between rows of an operand that a call lays out itself: a step takes 128 bytes of every row, one line of the caches and not parts of two.  8-bit products
// of 4096 x 6000 over 4001 116 us, in rows of 4016 bytes 131; short rows are only made whole pieces, lines would be much of them.
inline int64_t line_pitch(int64_t bytes) { return bytes < 1024 ? (bytes + 15) / 16 * 16 : (bytes + 127) / 128 * 128; }
// Bytes between rows up to which a tile's pieces are addressed with 32 bits.
constexpr int64_t kMaxPitch = (int64_t)1 << 22;

struct __attribute__((packed, aligned(1))) Piece { uint32_t x[4]; };

// 16 bytes per lane into LDS at `dst` (the same in all lanes) + 16 lane, from `off` bytes (below 2^31) behind an address that all lanes share.  Written
// out so that the compiler does not hold back reads of the other buffer until it is done; the wait before the barrier that hands the
// buffer over is written out, too.  m0 is among the registers that the compiler keeps for itself, and it warns of one that is named: here it has to know.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(uint32_t dst, const char* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1" ::"s"(__builtin_amdgcn_readfirstlane(dst)), "s"(base), "v"(off) : "memory", "m0");
}
// 4 bytes per lane, to `dst` + 4 lane.
__device__ __forceinline__ void load4_to_lds(uint32_t dst, const void* src) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(dst), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop
// The same value in scalar registers, for one that all lanes share.
__device__ __forceinline__ int64_t scalar(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const lds_char*)p; }

// 16 bytes from `src`, of which the first `valid` are there; the others are zero.
template <int EB>
__device__ __forceinline__ uint4 piece_of(const char* src, int64_t valid) {
  if (valid >= 16) {
    const Piece v = *(const Piece*)src;
    return make_uint4(v.x[0], v.x[1], v.x[2], v.x[3]);
  }
  uint64_t lo = 0, hi = 0;
#pragma unroll 1
  for (int at = 0; at < (int)valid; at += EB) {
    const uint64_t e = EB == 1 ? (uint64_t) * (const uint8_t*)(src + at) : EB == 2 ? (uint64_t) * (const uint16_t*)(src + at) : (uint64_t) * (const uint32_t*)(src + at);
    if (at < 8) lo |= e << (8 * at);
    else hi |= e << (8 * at - 64);
  }
  return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

// The part of a workgroup that fills the LDS tile of one operand: N rows (columns) of the output, THREADS threads.
template <class El, Order O, int N, int THREADS, bool DIRECT>
struct Stager {
  static constexpr int kPieces = N * (kStepBytes / 16), kLoads = kPieces / THREADS;
  static constexpr int kPerRow = O == kRows ? kStepBytes / 16 : N * 2 / 16;      // pieces per row of the tile in LDS
  static constexpr int kStepK = kStepBytes / El::kBytes;
  static_assert(kPieces % THREADS == 0 && (O == kRows || El::kBytes == 2), "");
  uint32_t off[kLoads];      // from `at`
  const char* at;            // of this step, the same in all lanes
  int64_t step;
  int32_t valid[O == kRows ? 1 : kLoads];   // kCols: bytes of the piece inside the columns
  bool ragged = false;                       // kCols: the columns end inside one of the tile's pieces
  uint4 reg[DIRECT ? 1 : kLoads];

  // first: the output row (column) that the tile begins with; k0: the number of the contraction that it begins with
  __device__ __forceinline__ void init(const Operand& op, int64_t first, int64_t k0, int tid) {
    const int64_t left = op.n - first;
    if (O == kRows) {
      at = op.base + first * op.ld + k0 * El::kBytes;
      step = kStepBytes;
    } else {
      at = op.base + k0 * op.ld + first * 2;
      step = (int64_t)kStepK * op.ld;
      ragged = left < N && left % 8 != 0;
    }
    at = (const char*)scalar((int64_t)at);
    step = scalar(step);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = i * THREADS + tid, row = slot / kPerRow, pc = slot % kPerRow;
      if (O == kRows) {
        const int src = pc ^ (row & 7);
        const int64_t r = row < left ? row : left - 1;
        off[i] = (uint32_t)(r * op.ld + 16 * src);
      } else {
        const int src = ((pc >> 1) ^ (mix(row) & (kPerRow / 2 - 1))) * 2 + (pc & 1);
        const int64_t c = 8 * src < left ? 8 * src : 0;      // a piece beyond the end: some other one, nothing of it is stored
        off[i] = (uint32_t)((int64_t)row * op.ld + 2 * c);
        valid[i] = (int32_t)(left - c >= 8 ? 16 : 2 * (left - c));
      }
    }
  }
  // rows of a kCols tile whose pieces of one column would lie in the same banks, told apart: a fragment is read from rows 8 g + i, g, i < 4
  static __device__ __forceinline__ int mix(int row) { return (row & 3) | ((row >> 3) & 3) << 2; }

  // left: numbers of the contraction from this step on
  __device__ __forceinline__ bool plain(int64_t left) const { return DIRECT && left >= kStepK && !ragged; }
  // one of the kLoads parts of a plain step; the step is over with next()
  __device__ __forceinline__ void load_part(char* tile, int wave, int i) const { load_to_lds(lds_address(tile) + 16 * (i * THREADS + 64 * wave), (const char*)scalar((int64_t)at), off[i]); }
  __device__ __forceinline__ void next() { at += step; }
  // a whole step into registers
  __device__ __forceinline__ void fetch() {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if (!DIRECT) reg[i] = piece_of<El::kBytes>(at + off[i], 16);
    next();
  }
  __device__ __forceinline__ void load(char* tile, int tid, int wave, int64_t left) {
    const int near = (int)(left < kStepK ? left : kStepK);
    if (plain(left)) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load_part(tile, wave, i);
    } else if (O == kRows) {
      // the step that the contraction ends in: all of a thread's pieces are whole, or none
      const int there = near * El::kBytes - 16 * ((tid ^ (tid >> 3)) & 7);
      if (DIRECT && there >= 16) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_part(tile, wave, i);
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const uint4 v = there > 0 ? piece_of<El::kBytes>(at + off[i], there) : make_uint4(0u, 0u, 0u, 0u);
          if (DIRECT) *(uint4*)(tile + 16 * (i * THREADS + tid)) = v;
          else reg[i] = v;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int there = i * (THREADS / kPerRow) + tid / kPerRow < near ? valid[O == kRows ? 0 : i] : 0;
        if (!DIRECT) reg[i] = piece_of<El::kBytes>(at + off[i], there);
        else if (there >= 16) load_part(tile, wave, i);
        else *(uint4*)(tile + 16 * (i * THREADS + tid)) = there > 0 ? piece_of<El::kBytes>(at + off[i], there) : make_uint4(0u, 0u, 0u, 0u);
      }
    }
    at += step;
  }
  __device__ __forceinline__ void store(char* tile, int tid) {
    if (!DIRECT)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) *(uint4*)(tile + 16 * (i * THREADS + tid)) = reg[i];
  }
};

// Where a lane reads fragments of 16 rows (columns) of a tile, 16 bytes of the half step kk (kStepBytes / 2 of the contraction): `first` (a multiple of
// 128 rows, or of 16 N of them) is the wave's first row.  Tile row f of the wave is at this plus 16 f rows (kRows), or with f exchanged into it (kCols).
template <Order O, int N>
__device__ __forceinline__ uint32_t fragment_base(int first, int lane) {
  const int g = lane >> 4, i = lane & 15;
  if (O == kRows) return (first + i) * kStepBytes + ((g ^ (i & 7)) * 16);
  const int mix = ((i >> 2) | g << 2) & (N / 16 - 1);
  return (8 * g + (i >> 2)) * (N * 2) + (i & 3) * 8 + ((first >> 4) ^ mix) * 32;
}
template <Order O, int N>
__device__ __forceinline__ int4v fragment(const char* tile, uint32_t base, int f, int kk) {
  if (O == kRows) return *(const int4v*)(tile + (base ^ (kk * 64)) + f * 16 * kStepBytes);
  const char* at = tile + (base ^ (f * 32)) + kk * 32 * (N * 2);
  typedef __attribute__((address_space(3))) short4v lds_short4;
  const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)at);
  const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(at + 4 * N * 2));
  const short8v both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(int4v, both);
}

// Has a sum worked out here: left alone, the compiler moves what only the next step needs behind everything else, out of the order that the reads from
// LDS go by, and keeps all operands in registers until then.
__device__ __forceinline__ void settle(floatx4& x) { asm volatile("" : "+v"(x)); }

template <class El>
__device__ __forceinline__ floatx4 mfma16(int4v p, int4v q, floatx4 c) {
  if constexpr (__is_same(El, Bf16)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
}
// 128 numbers of 8 bits; any order of them that both sides share will do
__device__ __forceinline__ floatx4 mfma8(int4v p0, int4v p1, int4v q0, int4v q1, floatx4 c) {
  const int8v p = {p0[0], p0[1], p0[2], p0[3], p1[0], p1[1], p1[2], p1[3]}, q = {q0[0], q0[1], q0[2], q0[3], q1[0], q1[1], q1[2], q1[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, c, 0, 0, 0, 0, 0, 0);
}

// The same with a power of two for each row of P and of Q, added to c: byte PB of sp and QB of sq are exponents (bias 127) for the row of the lane.
template <int PB, int QB>
__device__ __forceinline__ floatx4 mfma8_scaled(int4v p0, int4v p1, int4v q0, int4v q1, floatx4 c, int sp, int sq) {
  const int8v p = {p0[0], p0[1], p0[2], p0[3], p1[0], p1[1], p1[2], p1[3]}, q = {q0[0], q0[1], q0[2], q0[3], q1[0], q1[1], q1[2], q1[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, c, 0, 0, PB, sp, QB, sq);
}
// The same through fp16, which holds every e4m3 number: products exact, sums in fp32.  mfma8 keeps less: of eight neighbouring products the instruction
// cuts off what is below 2^-13 of the largest (measured; sums of different eights keep 24 bits).
struct Wide8 { f16x8 x[4]; };
__device__ __forceinline__ Wide8 widen(int4v p0, int4v p1) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  Wide8 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int a = i < 2 ? p0[2 * i] : p1[2 * i - 4], b = i < 2 ? p0[2 * i + 1] : p1[2 * i - 3];
    const f16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), v1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
    const f16x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), v3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
    w.x[i] = f16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
  }
  return w;
}
__device__ __forceinline__ floatx4 mfma_wide(const Wide8& p, const Wide8& q) {
  floatx4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(p.x[i], q.x[i], c, 0, 0, 0);
  return c;
}

// A tile product of 16-bit numbers.  A step is 2 NP slots, one for each tile row of a wave and half of the step; a slot is NQ instructions.
// What a slot multiplies was read from LDS at least four slots before.  All of a step is read by slot 9 of 16: at slot 12 the
// workgroup meets once, the next step's numbers, under way for a whole step, are there, the step two (three) ahead is sent for into the buffer that has just been read,
// and the first fragments of the next step are read while the last four slots multiply.  So no wave comes from the barrier with nothing to multiply.
// Bound by the matrix cores: a tile of 256 x 256 takes 1.46 us a step (1.47 Pflop/s on 256 CUs); 1.66 where fragments are read behind the barrier, 1.90 where
// a step is sent for at once, too (4096 x 65536 logits, widths from 256 to 2048).
template <class El, int NQ_, Order OP, Order OQ, bool DIRECT>
struct TileProduct {
  static constexpr int NP = 8, NQ = NQ_, WP = 2, WQ = 4;
  static constexpr int BP = 16 * NP * WP, BQ = 16 * NQ * WQ, kThreads = 64 * WP * WQ;
  static constexpr int kStepK = kStepBytes / El::kBytes;
  // Steps in LDS: the one that is multiplied and those on their way, two where there is room: a step of a smaller tile is over before memory has answered.
  // Loss of 500 tokens, 8000 words of width 4000: 59 us, with one 69; 100, 32000, 2000: 38 and 44.
  static constexpr int NB = DIRECT && NQ <= 2 ? 3 : 2, kPart = (BP + BQ) * kStepBytes, kLds = NB * kPart;

  static constexpr int PARTS = Stager<El, OP, BP, kThreads, DIRECT>::kLoads + Stager<El, OQ, BQ, kThreads, DIRECT>::kLoads;
  Stager<El, OP, BP, kThreads, DIRECT> sp;
  Stager<El, OQ, BQ, kThreads, DIRECT> sq;
  char* lds;
  int64_t k;         // of the contraction

  // The workgroup's barrier; `late`: but for the last PARTS loads, all have come.
  static __device__ __forceinline__ void meet(bool late = false) {
    __builtin_amdgcn_sched_barrier(0);
    if (late) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PARTS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ int steps() const { return (int)((k + kStepK - 1) / kStepK); }
  __device__ __forceinline__ bool plain(int t) const {
    const int64_t left = k - (int64_t)t * kStepK;
    return sp.plain(left) && sq.plain(left);
  }
  __device__ __forceinline__ void send(int t, char* to, int wave) {
    const int64_t left = k - (int64_t)t * kStepK;
    sp.load(to, threadIdx.x, wave, left);
    sq.load(to + BP * kStepBytes, threadIdx.x, wave, left);
  }
  __device__ __forceinline__ void keep(char* to) {
    sp.store(to, threadIdx.x);
    sq.store(to + BP * kStepBytes, threadIdx.x);
  }
  // Sends for the first NB steps of a tile.  LDS has to be free.
  __device__ __forceinline__ void begin(const Operand& P, int64_t p0, const Operand& Q, int64_t q0, int64_t k0, int64_t k1, char* lds_) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lds = lds_;
    k = scalar(k1 - k0);
    sp.init(P, p0, k0, threadIdx.x);
    sq.init(Q, q0, k0, threadIdx.x);
    if (steps() == 0) return;
    send(0, lds, wave);
    keep(lds);
#pragma unroll
    for (int t = 1; t < NB; ++t)
      if (steps() > t) send(t, lds + t * kPart, wave);
  }
  // The tile that was begun; LDS is free afterwards.
  __device__ __forceinline__ void multiply(floatx4 (&acc)[NP][NQ]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP, steps = this->steps();
    constexpr int SLOTS = 2 * NP, MEET = SLOTS - 4;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int q = 0; q < NQ; ++q) acc[p][q] = floatx4{0.f, 0.f, 0.f, 0.f};
    int4v fp[8], fq[2][NQ];
    uint32_t bp = fragment_base<OP, BP>(16 * wp * NP, lane), bq = fragment_base<OQ, BQ>(16 * wq * NQ, lane);
    auto read_p = [&](const char* tile, int slot) { fp[slot & 7] = fragment<OP, BP>(tile, bp, slot & 7, slot >> 3); };
    auto read_q = [&](const char* tile, int kk, int q) { fq[kk][q] = fragment<OQ, BQ>(tile + BP * kStepBytes, bq, q, kk); };
    // the parts of a plain step, one a slot: sent all at once they would queue up before the memory unit, and the waves behind them
    auto send_part = [&](char* to, int j) {
      if (j < decltype(sp)::kLoads) sp.load_part(to, wave, j);
      else if (j < PARTS) sq.load_part(to + BP * kStepBytes, wave, j - decltype(sp)::kLoads);
    };
    bool parts = false;          // the step after this one is being sent for in parts
    if (steps == 0) return;
    meet();
    if (!DIRECT && steps > 1) keep(lds + kPart);        // the pieces of step 1 have left their registers before those of step 2 come
#pragma unroll
    for (int i = 0; i < 4; ++i) read_p(lds, i);
#pragma unroll
    for (int q = 0; q < NQ; ++q) read_q(lds, 0, q);
    int slot = 0;                // t % NB
    for (int t = 0; t < steps; ++t) {
      // of the step before, this one and the next in LDS
      slot = __builtin_amdgcn_readfirstlane(NB == 2 ? t & 1 : slot);
      const int at = slot * kPart, nat = slot == NB - 1 ? 0 : at + kPart, pat = slot == 0 ? (NB - 1) * kPart : at - kPart;
      const char *cur = lds + at, *nxt = lds + nat;
      const bool more = t + 1 < steps, sends = t + NB < steps;
      asm volatile("" : "+v"(bp), "+v"(bq));      // addresses are worked out from these where they are used, not kept
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        if (s < 4) {
          read_p(cur, s + 4);
          if (s < NQ) read_q(cur, 1, s);
        } else if (s < 6) {
          read_p(cur, 2 * s);
          read_p(cur, 2 * s + 1);
        } else if (s < 10) {
          read_p(cur, s + 6);
        } else if (s == MEET) {
          meet(NB > 2 && plain(t + 2));
          parts = sends && plain(t + NB);
          if (sends && !parts) send(t + NB, lds + at, wave);
        }
        if (parts) {
          if (s >= MEET) send_part(lds + at, s - MEET);
          else if (s < PARTS - 4) send_part(lds + pat, s + 4);
          if (s == PARTS - 5) {
            sp.next();
            sq.next();
            parts = false;
          }
        }
        if (s >= MEET && more) {
          read_p(nxt, s - MEET);
          if (s - MEET < NQ) read_q(nxt, 0, s - MEET);
        }
        if (!DIRECT && s == SLOTS - 1 && sends) keep(lds + at);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          acc[s & 7][q] = mfma16<El>(fp[s & 7], fq[s >> 3][q], acc[s & 7][q]);
          settle(acc[s & 7][q]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      slot = slot == NB - 1 ? 0 : slot + 1;
    }
    meet();
  }

  static __device__ __forceinline__ void run(floatx4 (&acc)[NP][NQ], const Operand& P, int64_t p0, const Operand& Q, int64_t q0, int64_t k0, int64_t k1, char* lds) {
    TileProduct x;
    x.begin(P, p0, Q, q0, k0, k1, lds);
    x.multiply(acc);
  }
};

// The same for up to 64 rows of Q, where the read of P is what it takes: no LDS, a wave has 16 NP rows of P and all rows of Q, and both go from memory (Q
// from the caches) to the instruction's registers, U steps ahead.  Rows at any alignment.
template <class El, int NP_, int NQ_, int WP_, int U>
struct RowsProduct {
  static constexpr int NP = NP_, NQ = NQ_, WP = WP_, WQ = 1;
  static constexpr int BP = 16 * NP * WP, BQ = 16 * NQ, kThreads = 64 * WP;
  static constexpr int kLds = 16;                                // none
  struct Step { uint4 p[NP][2], q[NQ][2]; };

  static __device__ __forceinline__ void run(floatx4 (&acc)[NP][NQ], const Operand& P, int64_t p0, const Operand& Q, int64_t q0, int64_t k0, int64_t k1, char*) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, piece = 16 * (lane >> 4);
    const char *rp[NP], *rq[NQ];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int64_t r = p0 + 16 * (wave * NP + p) + row;
      rp[p] = P.base + (r < P.n ? r : P.n - 1) * P.ld + 2 * k0 + piece;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t r = q0 + 16 * q + row;
      rq[q] = Q.base + (r < Q.n ? r : Q.n - 1) * Q.ld + 2 * k0 + piece;
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int q = 0; q < NQ; ++q) acc[p][q] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int64_t bytes = 2 * (k1 - k0);
    const int whole = (int)(bytes / kStepBytes);
    auto fetch = [&](Step& x, int t, bool all, int64_t left) {            // left: bytes of the row from this lane's first piece on
      const int64_t at = (int64_t)t * kStepBytes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int p = 0; p < NP; ++p) x.p[p][h] = piece_of<2>(rp[p] + at + 64 * h, all ? 16 : left - 64 * h);
#pragma unroll
        for (int q = 0; q < NQ; ++q) x.q[q][h] = piece_of<2>(rq[q] + at + 64 * h, all ? 16 : left - 64 * h);
      }
    };
    auto multiply = [&](const Step& x) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const floatx4 d = mfma16<El>(__builtin_bit_cast(int4v, x.p[p][0]), __builtin_bit_cast(int4v, x.q[q][0]), acc[p][q]);
          acc[p][q] = mfma16<El>(__builtin_bit_cast(int4v, x.p[p][1]), __builtin_bit_cast(int4v, x.q[q][1]), d);
        }
    };
    Step x[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (i < whole) fetch(x[i], i, true, 0);
    for (int t = 0; t < whole; t += U) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (t + i < whole) multiply(x[i]);
        if (t + i + U < whole) fetch(x[i], t + i + U, true, 0);
      }
    }
    if (bytes > (int64_t)whole * kStepBytes) {
      fetch(x[0], whole, false, bytes - (int64_t)whole * kStepBytes - piece);
      multiply(x[0]);
    }
  }
};

// 16-bit numbers from fp32, to the nearest
template <class El> __device__ __forceinline__ uint16_t to16(float x) {
  if constexpr (__is_same(El, Bf16)) { const __bf16 h = (__bf16)x; return __builtin_bit_cast(uint16_t, h); }
  else { const _Float16 h = (_Float16)x; return __builtin_bit_cast(uint16_t, h); }
}
template <class El> __device__ __forceinline__ float from16(uint16_t x) {
  if constexpr (__is_same(El, Bf16)) return __builtin_bit_cast(float, (uint32_t)x << 16);
  else return (float)__builtin_bit_cast(_Float16, x);
}

// A workgroup's tile D (of sums, a wave has 8 x NQ tiles of it) to memory as 16-bit numbers: row j of `out` (pitch ldo numbers) gets column j of D, of which
// `rows` and `cols` are there.  A lane's four numbers of a row go through LDS, so that a row's 256 leave as one piece of memory, 16 bytes a lane at any
// alignment: stored from where they are, 32 bytes of a row at a time, an 8192 x 8192 result took 33 us.  Eight bytes u of row j lie at
// u ^ 4 (j & 15): 16 rows in different banks.  LDS has to be free.  `number(x, q)` makes the 16 bits of a sum of the wave's tile column q.
template <int NQ, class Number>
__device__ __forceinline__ void put_tile16(const floatx4 (&acc)[8][NQ], char* lds, uint16_t* out, int64_t ldo, int64_t rows, int64_t cols, Number number) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wp = wave % 2, wq = wave / 2;
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      uint32_t h[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) h[r] = number(acc[p][q][r], q);
      const int j = 16 * (wq * NQ + q) + (lane & 15), u = 4 * (8 * wp + p) + (lane >> 4);
      *(uint2*)(lds + j * 512 + 8 * (u ^ (4 * (lane & 15)))) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    }
  __syncthreads();
  const int piece = tid & 31;
  const int64_t left = cols - 8 * piece;
#pragma unroll
  for (int i = 0; i < 4 * NQ; ++i) {
    const int j = 16 * i + (tid >> 5);
    const uint4 v = *(const uint4*)(lds + j * 512 + 8 * ((2 * piece) ^ (4 * (j & 15))));
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

// Tiles of a np x nq grid (np along P) to workgroups: workgroups b, b + 8, b + 16 ... share an XCD and its L2, so each XCD gets a run of tiles, and a run
// goes through `band` rows of the grid at a time.  Returns false for workgroups beyond the grid (the grid is rounded up to eight).
__device__ __forceinline__ bool tile_of_workgroup(unsigned b, int64_t np_, int64_t nq_, unsigned band, int64_t* tp, int64_t* tq) {
  const unsigned np = (unsigned)np_, nq = (unsigned)nq_, all = np * nq, per = (all + 7) / 8, i = (b & 7) * per + (b >> 3);
  if ((b >> 3) >= per || i >= all) return false;
  const unsigned group = i / (band * nq), first = group * band, height = np - first < band ? np - first : band, in = i - group * band * nq;
  *tp = __builtin_amdgcn_readfirstlane(first + in % height);
  *tq = __builtin_amdgcn_readfirstlane(in / height);
  return true;
}
inline unsigned tile_workgroups(int64_t np, int64_t nq) { return (unsigned)(8 * ((np * nq + 7) / 8)); }
// Whether a launch may have that many tiles
inline bool tiles_fit(int64_t np, int64_t nq, int threads) { return nq == 0 || (np <= kMaxGrid / nq && tile_workgroups(np, nq) <= launch_workgroups(threads)); }

// A product's tiles on 256 CUs: np of them along one side, each a column of q256 tiles of 256 x 256 or of q128 of half the size (seven tenths of the time).  The
// first so many of the np go in large ones (what it returns): all, none, or those of the full rounds, so that only the last round is of small ones.  A tile
// takes as long as its steps and three more, the second launch is taken to cost four steps.  8 bits: 4096 x 6000 over 4001 130 us and 142 without,
// 4001 x 6000 over 4096 93 and 104; loss and gradients of 999 tokens, 50001 words of width 1000 525 and 539.  With five steps (width 272) and 24 full rounds
// the cut cost 1 %, so it is not made there.
inline int64_t large_tiles(int64_t np, int64_t q256, int64_t q128, int64_t steps) {
  auto rounds = [](int64_t tiles) { return (tiles + 255) / 256; };
  const int64_t large = 10 * rounds(np * q256), small = 7 * rounds(np * q128), full = np * q256 / 256 * 256 / q256;
  if (full > 0 && full < np) {
    const int64_t best = large < small ? large : small;
    if ((best - 10 * rounds(full * q256) - 7 * rounds((np - full) * q128)) * (steps + 3) > 40) return full;
  }
  return small < large ? 0 : np;
}

}  // namespace brsvd
