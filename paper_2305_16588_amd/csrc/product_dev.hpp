// Products of matrices by tiles: what the gated projections, their gradients and the products of rows in 8-bit integers share.
#pragma once

#include "rows_dev.hpp"

#include <type_traits>

namespace lgp {
namespace layer {
namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));

// D[32, 32] += A[32, K] B[K, 32] with K of two chunks of 16 bytes, of which lane l holds chunk l / 32 of A row l % 32 and of B column l % 32; D as in layer_dev.hpp.
// few: D[16, 16] += A[16, K] B[K, 16] with K of four chunks, of which lane l holds chunk l / 16 of A row l % 16 and of B column l % 16; of D it holds column l % 16,
// register r being row 4 (l / 16) + r.
__device__ __forceinline__ floatx4 few_mfma(vec8<f16> a, vec8<f16> b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 few_mfma(vec8<bf16> a, vec8<bf16> b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <typename T> struct Unit {
  typedef vec8<T> chunk;
  typedef floatx16 sums;
  typedef float sum;
  typedef floatx4 few_sums;
  static constexpr int kSize = 2;
  static __device__ __forceinline__ sums mfma(chunk a, chunk b, sums c) { return Elem<T>::mfma(a, b, c); }
  static __device__ __forceinline__ few_sums few(chunk a, chunk b, few_sums c) { return few_mfma(a, b, c); }
};
template <> struct Unit<int8_t> {
  typedef intx4 chunk;
  typedef intx16 sums;
  typedef int sum;
  typedef intx4 few_sums;
  static constexpr int kSize = 1;
  static __device__ __forceinline__ few_sums few(chunk a, chunk b, few_sums c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ sums mfma(chunk a, chunk b, sums c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};

__device__ __align__(16) const uint32_t kNothing[4] = {};       // what is read where there is nothing to read

// 16 bytes of each lane, from an address of its own; else as copy16.
__device__ __forceinline__ void copy16_from(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}
// 4 bytes of each lane, as copy16.
__device__ __forceinline__ void copy4(const void* from, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(from) : "memory");
}
template <int N> __device__ __forceinline__ void loads_left() { __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14); }      // all but the last N are done
__device__ __forceinline__ void together() {       // everyone's reads of LDS are done, and so are the loads that each has waited for
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One side of a product.  Along: a row of the tile is a row of memory, and the sum runs along it.  Across: the sum runs over rows of memory, whose columns
// are the tile's rows.  `second` is the matrix of the other half: of the tile's rows (along, gated) or of the sum (across, from `half` on).
struct Operand {
  const char *first, *second;
  int64_t row_bytes;
  int32_t rows;                      // of memory, in each matrix; at least one
  int32_t chunks;                    // of 16 bytes in a row; at least one
  int32_t half;                      // across: where the second matrix begins in the sum (a multiple of a stage), or more than there is
  const int32_t* pos;                // across: rows with a negative entry count as zeros; NULL: none
  const int32_t* order;              // rows are order[0], order[1] ... of memory; NULL: 0, 1 ...
};
typedef const __attribute__((address_space(4))) int32_t* Fixed;        // read by the scalar unit: nothing writes it while the kernel runs
__device__ __forceinline__ Fixed fixed(const int32_t* p) { return (Fixed)(uintptr_t)p; }
__device__ __forceinline__ int turned(int row) { return int(__brev(uint32_t(row)) >> 28); }        // a row's low four bits in reverse
// The order of 32 rows of A that leaves a lane 16 consecutive rows of D.
__device__ __forceinline__ int in_order(int m) { return (m & ~31) + 16 * (m >> 2 & 1) + 4 * (m >> 3 & 3) + (m & 3); }

template <int N> using Int = std::integral_constant<int, N>;
template <int N, int I = 0, typename F> __device__ __forceinline__ void each(F f) {       // f(0) ... f(N - 1), with constants
  if constexpr (I < N) {
    f(Int<I>());
    each<N, I + 1>(f);
  }
}

// BM x BN of a product by WM x WN waves, each 32 MI x 32 NJ of it.  A stage is CH chunks of the sum: while one is multiplied, STAGES - 1 are on their way to LDS, past the
// registers.  Every copy is issued whatever there is to copy -- what lies beyond an end is another valid row whose results are not used, or zeros where it
// is part of a sum -- so a wave knows how many of its loads are under way.
//
// The 32 rows of a block of A lie in LDS in an order (or are read in one) that leaves a lane 16 consecutive rows of D: register r of lane l is row 16 (l / 32) + r, so
// results are written 32 bytes at a time.
template <typename T, int BM_, int BN_, int WM_, int WN_, int CH_, int STAGES_, bool GATED, bool A_ACROSS, bool B_ACROSS> struct Tiles {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, CH = CH_, STAGES = STAGES_;
  static constexpr int kThreads = 64 * WM * WN, MI = BM / 32 / WM, NJ = BN / 32 / WN;
  static constexpr int kStage = CH * 16 / Unit<T>::kSize;       // places of the sum
  static constexpr int NA = BM * CH / kThreads, NB = BN * CH / kThreads;       // copies of a thread
  static_assert(BM * CH % kThreads == 0 && BN * CH % kThreads == 0 && (!GATED || MI % 2 == 0), "whole copies");
  typedef typename Unit<T>::chunk chunk;
  typedef typename Unit<T>::sums sums;
  struct Shared {
    alignas(16) char a[STAGES][BM * CH * 16];
    alignas(16) char b[STAGES][BN * CH * 16];
    int32_t listed[A_ACROSS ? 8 : 1][64];         // A's rows of a stage, where there is a list
  };

  // A thread's places in the tile of one side, and what it copies there.
  template <int ROWS, int N, bool ACROSS, bool PAIR, bool ORDER> struct Side {
    uint32_t offset[N];
    static constexpr int kWide = ROWS / 8;           // across: chunks of a row in LDS

    __device__ __forceinline__ Side(const Operand& o, int32_t row0, int tid) {       // along: o begins at the tile's first row
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int place = tid + j * kThreads;
        if constexpr (ACROSS) {
          const int r = place / kWide, c = row0 / 8 + ((place % kWide) ^ (turned(r) & (kWide - 1)));
          offset[j] = uint32_t(r) * uint32_t(o.row_bytes) + (c < o.chunks ? c : 0) * 16;
        } else {
          const int r = place / CH, c = (place % CH) ^ (turned(r) & (CH - 1));
          int at = PAIR ? r % (ROWS / 2) : r;
          if (ORDER) at = in_order(at);
          at = at < o.rows ? at : o.rows - 1;
          if (!PAIR && o.order) offset[j] = uint32_t(o.order[at]) * uint32_t(o.row_bytes / 16) + c;       // in units of 16 bytes
          else offset[j] = uint32_t(at) * uint32_t(o.row_bytes) + c * 16;
        }
      }
    }
    // at: the stage's first place of the sum; listed: its rows, where there is a list.
    __device__ __forceinline__ void copy(const Operand& o, int32_t at, char* to, const int32_t* listed, int tid) const {
      const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(to) + (tid & ~63) * 16);
      if constexpr (ACROSS) {
        const bool later = at >= o.half;
        const int32_t row = later ? at - o.half : at;
        const char* from = (later ? o.second : o.first) + (o.order ? 0 : int64_t(row) * o.row_bytes);
        if (row + kStage <= o.rows && !o.pos && !o.order) {
#pragma unroll
          for (int j = 0; j < N; ++j) copy16(in_all_lanes(from), offset[j], lds + j * kThreads * 16);
        } else {
          constexpr int kEach = 64 / kWide > 0 ? 64 / kWide : 1;       // rows of a wave
          const void* lane_from[N];          // all places first: each is known when a list or the positions are read
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int r = (tid + j * kThreads) / kWide, r0 = __builtin_amdgcn_readfirstlane(r);
            const char* place = from + offset[j];
            bool there = row + r < o.rows;
            if (o.order) {
              place = from + int64_t(listed[there ? r : 0]) * o.row_bytes + (offset[j] - uint32_t(r) * uint32_t(o.row_bytes));
            } else if (o.pos) {
#pragma unroll
              for (int e = 0; e < kEach; ++e) {
                const int32_t t = row + r0 + e < o.rows ? row + r0 + e : o.rows - 1;
                if (fixed(o.pos)[t] < 0) there = there && r != r0 + e;
              }
            }
            lane_from[j] = there ? static_cast<const void*>(place) : kNothing;
          }
#pragma unroll
          for (int j = 0; j < N; ++j) copy16_from(lane_from[j], lds + j * kThreads * 16);
        }
      } else {
        const int32_t c0 = at / (16 / Unit<T>::kSize);
        const bool whole = c0 + CH <= o.chunks;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const char* from = o.first;
          if (PAIR && __builtin_amdgcn_readfirstlane((tid + j * kThreads) / CH) >= ROWS / 2) from = o.second;
          from += int64_t(c0) * 16;
          if (!PAIR && o.order) {
            const int place = tid + j * kThreads, c = (place % CH) ^ (turned(place / CH) & (CH - 1));
            copy16_from(c0 + c < o.chunks ? static_cast<const void*>(from + (uint64_t(offset[j]) << 4)) : kNothing, lds + j * kThreads * 16);
          } else if (whole) {
            copy16(in_all_lanes(from), offset[j], lds + j * kThreads * 16);
          } else {
            const int place = tid + j * kThreads, c = (place % CH) ^ (turned(place / CH) & (CH - 1));
            copy16_from(c0 + c < o.chunks ? static_cast<const void*>(from + offset[j]) : kNothing, lds + j * kThreads * 16);
          }
        }
        static_assert(!PAIR || (ROWS / 2) % (64 / CH) == 0, "a wave's rows are of one matrix");
      }
    }
  };

  // Where a lane finds the chunk of its row (along) or column (across) of a block of 32 in step kk of a stage.
  template <int ROWS, bool ACROSS, bool ORDER> struct Place {
    int at;
    __device__ __forceinline__ explicit Place(int lane) {
      if constexpr (ACROSS) {
        // sixteen lanes read four rows of 16 columns, which the LDS hands out transposed: lanes of the upper half the later eight rows
        const int i = lane & 15, r = 8 * (lane >> 5) + (i >> 2), p = 4 * (lane >> 4 & 1) + (i & 3), c = ORDER ? 16 * (p & 1) + 4 * (p >> 1) : 4 * p;
        at = r * ROWS + (((c >> 3) ^ (turned(r) & (ROWS / 8 - 1))) << 3) + (c & 7);
      } else {
        const int r = lane & 31;
        at = r * CH + ((lane >> 5) ^ (turned(r) & (CH - 1)));
      }
    }
    __device__ __forceinline__ chunk read(const char* tile, int row0, int kk) const {
      if constexpr (ACROSS) {
        typedef __attribute__((address_space(3))) shortx4* place;
        union { shortx4 s[2]; chunk v; } u;
        const short* rows = reinterpret_cast<const short*>(tile) + kk * 16 * ROWS;
        const int here = at ^ row0;
        u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(rows + here));
        u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(rows + 4 * ROWS + (here ^ 16)));       // the turn of a row four further on
        return u.v;
      } else {
        return *reinterpret_cast<const chunk*>(tile + ((at ^ (2 * kk)) + row0 * CH) * 16);
      }
    }
  };

  // First row of a wave's block i of A, in the tile.
  static __device__ __forceinline__ int block_of(int wm, int i) {
    if constexpr (GATED) return (i < MI / 2 ? 0 : BM / 2) + (wm * (MI / 2) + i % (MI / 2)) * 32;
    else return (wm * MI + i) * 32;
  }

  // acc += over places [begin, end) of the sum; begin is a multiple of a stage.
  static __device__ __forceinline__ void run(Shared& s, Operand a, Operand b, int32_t a_row, int32_t b_row, int32_t begin, int32_t end,
                                             sums (&acc)[MI][NJ]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM;
    if constexpr (!A_ACROSS) a.first += a_row * a.row_bytes, a.second += a_row * a.row_bytes, a.rows -= a_row;
    if constexpr (!B_ACROSS) {
      if (b.order) b.order += b_row;
      else b.first += b_row * b.row_bytes;
      b.rows -= b_row;
    }
    const Side<BM, NA, A_ACROSS, GATED, true> from_a(a, a_row, tid);
    const Side<BN, NB, B_ACROSS, false, false> from_b(b, b_row, tid);
    const Place<BM, A_ACROSS, true> at_a(lane);
    const Place<BN, B_ACROSS, false> at_b(lane);
    const int32_t n = (end - begin + kStage - 1) / kStage;
    // A list's part for a stage comes with the stage two before it.
    auto list = [&](int32_t k) {
      if (wave == 0 && k < n)
        copy4(a.order + begin + k * kStage, min(lane, end - 1 - begin - k * kStage) * 4, __builtin_amdgcn_readfirstlane(lds_address(s.listed[A_ACROSS ? k % 8 : 0])));
    };
    auto fetch = [&](int32_t k) {
      const int to = k % STAGES;
      if (A_ACROSS && a.order) list(k + 2);
      from_a.copy(a, begin + k * kStage, s.a[to], s.listed[A_ACROSS ? k % 8 : 0], tid);
      from_b.copy(b, begin + k * kStage, s.b[to], nullptr, tid);
    };
    chunk x[2][MI], y[2][NJ];
    auto read = [&](int32_t k, int kk) {
      const char *ta = s.a[k % STAGES], *tb = s.b[k % STAGES];
#pragma unroll
      for (int i = 0; i < MI; ++i) x[kk & 1][i] = at_a.read(ta, block_of(wm, i), kk);
#pragma unroll
      for (int j = 0; j < NJ; ++j) y[kk & 1][j] = at_b.read(tb, (wn * NJ + j) * 32, kk);
    };
    if (n <= 0) return;
    if (A_ACROSS && a.order) {
#pragma unroll
      for (int k = 0; k < STAGES; ++k) list(k);
      loads_done();
      together();
    }
#pragma unroll
    for (int k = 0; k < STAGES; ++k)
      if (k < n) fetch(k);
    if (n >= STAGES) loads_left<(STAGES - 1) * (NA + NB)>();
    else loads_done();
    together();
    read(0, 0);
    for (int32_t k = 0; k < n; ++k) {
      each<CH / 2>([&](auto step) {
        constexpr int kk = decltype(step)::value;
        if (kk + 1 < CH / 2) {
          read(k, kk + 1);
        } else if (k + 1 < n) {        // all of this stage is in registers
          if (n - k >= STAGES) loads_left<(STAGES - 2) * (NA + NB)>();
          else loads_done();
          together();
          read(k + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);       // the next operands are on their way before these are multiplied, not just before they are wanted
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = Unit<T>::mfma(x[kk & 1][i], y[kk & 1][j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
        if (kk + 1 == CH / 2 && k + STAGES < n) fetch(k + STAGES);
      });
    }
  }
};

// Narrow rows: the weights stay in registers.  With sums of up to KS steps of two chunks a wave has 64 rows of A (32 of each of a pair), which it loads once; the rows of B
// pass by, 32 after 32, a few slots of them on their way to LDS, and each wave multiplies them with its own rows.  A SIMD has two waves: while one multiplies, the other
// works on what came of its last 32 rows (out.step) -- the later four waves are half a turn behind.  With 32 steps there are registers for one wave, which does both in
// turn.
//
// A wave waits for all but its last copies of SLOTS - 2 slots: what is newer than the copies of the slot that it wants are at least those of the next ones, which are issued
// after a slot's work, so the wait does not depend on how many results were written.  Where there is a list, its part for a slot comes with the rows of
// the slot that many before it.
template <typename T, int KS_, int WAVES_, bool PAIR> struct Narrow {
  static constexpr int KS = KS_, WAVES = WAVES_, kThreads = 64 * WAVES, kPerCu = KS < 16 && WAVES == 4 ? 2 : 1;       // workgroups
  static constexpr int CH = 2 * KS, kRows = KS > 16 ? 32 : 64, SLOTS = 4, NC = kRows * CH / kThreads;
  static constexpr int kRing = 4;                // blocks of 32 rows that the loop takes at once
  static_assert(kRows * CH % kThreads == 0, "whole copies");
  typedef typename Unit<T>::chunk chunk;
  typedef typename Unit<T>::sums sums;
  struct Shared {
    alignas(16) char rows[SLOTS][kRows * CH * 16];
    int32_t listed[2 * SLOTS][64];               // of each slot
  };

  // Rows [begin, end) of B (of its order) with rows a_row ... of A: a wave has 32 of each of a pair, or 64, from `own` on.  out.start<q>(row, listed) is told of the 32 rows that are
  // multiplied next, q counting up to kRing, and where they are listed; out.step<q, r>(acc) is given register r of what came of them, as the q that they had; out.next(row, listed)
  // is told afterwards which rows' results come next.  Rows from `end` on are the last row again, with the same results, but for 32 of
  // them, which have none (with one wave on a SIMD, they too).
  template <typename Out>
  static __device__ __forceinline__ void run(Shared& s, const Operand& a, const Operand& b, int32_t own, int32_t begin, int32_t end, Out& out) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int kTurn = CH < 16 ? CH - 1 : 15;
    if (begin >= end) return;
    chunk w[2][KS];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      int32_t row = own + (PAIR ? 0 : 32 * q) + in_order(lane & 31);
      row = row < a.rows ? row : a.rows - 1;
      const char* from = (PAIR && q ? a.second : a.first) + int64_t(row) * a.row_bytes;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const int c = 2 * kk + (lane >> 5);
        const chunk nothing = {};
        w[q][kk] = c < a.chunks ? *reinterpret_cast<const chunk*>(from + 16 * c) : nothing;
      }
    }
    const int32_t n = (end - begin + kRows - 1) / kRows;
    // Copy j of a thread: row tid / CH + j * kThreads / CH of the slot.  Where a copy's rows are a multiple of 16, which the turn repeats after, all of them have the same chunk.
    constexpr int kStep = kThreads / CH;
    auto chunk_of = [&](int j) __attribute__((always_inline)) { return ((tid + j * kThreads) % CH) ^ (turned((tid + (kStep % 16 ? j * kThreads : 0)) / CH) & kTurn); };
    auto list = [&](int32_t k) __attribute__((always_inline)) {
      if (b.order && wave == 0 && k < n)
        copy4(b.order + begin + k * kRows, min(lane, end - 1 - begin - k * kRows) * 4, __builtin_amdgcn_readfirstlane(lds_address(s.listed[k % (2 * SLOTS)])));
    };
    auto fetch = [&](int32_t k) __attribute__((always_inline)) {
      const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(s.rows[k % SLOTS]) + (tid & ~63) * 16);
      const int32_t row0 = begin + k * kRows;
      if (b.order) {
        list(k + SLOTS);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const int32_t row = s.listed[k % (2 * SLOTS)][min(tid / CH + j * kStep, end - 1 - row0)];
          const int c = chunk_of(j);
          copy16_from(c < b.chunks ? static_cast<const void*>(b.first + int64_t(row) * b.row_bytes + 16 * c) : kNothing, lds + j * kThreads * 16);
        }
      } else if (row0 + kRows <= end && b.chunks >= CH) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const char* from = b.first + int64_t(row0 + j * kStep) * b.row_bytes;
          copy16(in_all_lanes(from), uint32_t(tid / CH) * uint32_t(b.row_bytes) + 16 * chunk_of(j), lds + j * kThreads * 16);
        }
      } else {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          int32_t row = row0 + tid / CH + j * kStep;
          row = row < end ? row : end - 1;
          const int c = chunk_of(j);
          copy16_from(c < b.chunks ? static_cast<const void*>(b.first + int64_t(row) * b.row_bytes + 16 * c) : kNothing, lds + j * kThreads * 16);
        }
      }
    };
    if (b.order) {
#pragma unroll
      for (int k = 0; k < SLOTS; ++k) list(k);
      loads_done();
      together();
    }
#pragma unroll
    for (int k = 0; k < SLOTS - 1; ++k)
      if (k < n) fetch(k);
    const int at = (lane & 31) * CH + ((lane >> 5) ^ (turned(lane & 31) & kTurn));
    constexpr int kAhead = WAVES == 8 ? 2 : 3, kBlocks = kRows / 32;        // loads of operands ahead of their use; blocks in a slot
    const sums nothing = {};
    auto slot_ready = [&](int32_t k) __attribute__((always_inline)) {
      if (n - k >= SLOTS - 1) loads_left<(SLOTS - 2) * NC>();
      else loads_done();
      together();
    };
    chunk y[kAhead + 1];
    auto operand = [&](const char* tile, int i) __attribute__((always_inline)) { return *reinterpret_cast<const chunk*>(tile + ((at ^ (2 * (i % KS))) + i / KS * 32 * CH) * 16); };
    auto start = [&](auto of_ring, int32_t k) __attribute__((always_inline)) {
      constexpr int q = decltype(of_ring)::value, block = q % kBlocks;
      out.template start<q>(begin + k * kRows + 32 * block, s.listed[k % (2 * SLOTS)] + 32 * block);
    };
    out.template start<kRing - 1>(begin, s.listed[0]);
    out.next(begin, s.listed[0]);
    constexpr bool kTwo = WAVES == 8;
    const bool late = kTwo && wave >= WAVES / 2;
    sums acc[kTwo ? 1 : 2][2] = {};
    auto results = [&](auto of_ring, int32_t k) __attribute__((always_inline)) {       // of slot k
      constexpr int q = decltype(of_ring)::value, after = (q + 1) % kBlocks;
      if (begin + k * kRows + 32 * (q % kBlocks) >= end) return;
      each<16>([&](auto r) __attribute__((always_inline)) { out.template step<q, decltype(r)::value>(acc[kTwo ? 0 : q & 1]); });
      const int32_t then = after ? k : k + 1;
      out.next(begin + then * kRows + 32 * after, s.listed[then % (2 * SLOTS)] + 32 * after);
    };
    for (int32_t k0 = 0; k0 < n; k0 += kRing / kBlocks) {
      each<kRing>([&](auto of_ring) __attribute__((always_inline)) {
        constexpr int q = decltype(of_ring)::value, block = q % kBlocks, before = (q + kRing - 1) % kRing;
        const int32_t k = k0 + q / kBlocks;
        const char* tile = s.rows[k % SLOTS];
        if (block == 0) {
          if (k < n) slot_ready(k);
          if (kTwo ? late && k > 0 && k <= n : k == n) results(Int<before>(), k - 1);
        }
        if (k >= n) return;
        if (block == 0) each<kAhead>([&](auto i) __attribute__((always_inline)) { y[decltype(i)::value] = operand(tile, decltype(i)::value); });
        start(of_ring, k);
        each<KS>([&](auto step) __attribute__((always_inline)) {
          constexpr int kk = decltype(step)::value, here = block * KS + kk, ahead = here + kAhead, set = kTwo ? 0 : q & 1;
          if constexpr (ahead < kBlocks * KS) y[ahead % (kAhead + 1)] = operand(tile, ahead);
          acc[set][0] = Unit<T>::mfma(w[0][kk], y[here % (kAhead + 1)], kk ? acc[set][0] : nothing);
          // one wave: registers kk * 16 / KS ... of the results before
          if constexpr (!kTwo) each<(kk + 1) * 16 / KS - kk * 16 / KS>([&](auto r) __attribute__((always_inline)) {
            out.template step<before, kk * 16 / KS + decltype(r)::value>(acc[set ^ 1]);
          });
          if (!kTwo && kk + 1 == KS) out.next(begin + k * kRows + 32 * block, s.listed[k % (2 * SLOTS)] + 32 * block);
          acc[set][1] = Unit<T>::mfma(w[1][kk], y[here % (kAhead + 1)], kk ? acc[set][1] : nothing);
          __builtin_amdgcn_sched_barrier(0);
        });
        if (kTwo && (block + 1 < kBlocks || !late)) results(of_ring, k);
        __builtin_amdgcn_sched_barrier(0);
        if (block == kBlocks - 1 && k + SLOTS - 1 < n) fetch(k + SLOTS - 1);
      });
    }
    if ((!kTwo || late) && n % (kRing / kBlocks) == 0) results(Int<kRing - 1>(), n - 1);
  }
};

// Few rows of B: a workgroup has 16 rows of A (of each of a pair), which it reads once, and 16 of B.  Its eight waves take every eighth four chunks of the sum, straight
// to registers, many loads at a time, and are added in LDS in their order.  The result of A row r and B row c lies at sums[pair][c][r].
constexpr int kFewWaves = 8, kFewTokens = 32;
template <typename T, bool PAIR> struct Few {
  typedef typename Unit<T>::chunk chunk;
  typedef typename Unit<T>::sum sum;
  static constexpr int kPair = PAIR ? 2 : 1;
  struct Shared { sum sums[kFewWaves][kPair][16][17]; };
  static __device__ __forceinline__ void run(Shared& s, const Operand& a, const Operand& b, int32_t a_row, int32_t b_row) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const char* pa = a.first + int64_t(min(a_row + (lane & 15), a.rows - 1)) * a.row_bytes;
    const char* pa2 = PAIR ? a.second + int64_t(min(a_row + (lane & 15), a.rows - 1)) * a.row_bytes : nullptr;
    const char* pb = b.first + int64_t(min(b_row + (lane & 15), b.rows - 1)) * b.row_bytes;
    typename Unit<T>::few_sums acc[kPair] = {};
    const chunk nothing = {};
    constexpr int kAtOnce = PAIR ? 4 : 8;
    for (int32_t c0 = 4 * wave; c0 < a.chunks; c0 += 4 * kFewWaves * kAtOnce) {
      chunk x[kAtOnce], x2[kAtOnce], y[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int32_t c = c0 + 4 * kFewWaves * k + (lane >> 4);
        const bool in = c < a.chunks;
        x[k] = in ? *reinterpret_cast<const chunk*>(pa + 16 * int64_t(c)) : nothing;
        if (PAIR) x2[k] = in ? *reinterpret_cast<const chunk*>(pa2 + 16 * int64_t(c)) : nothing;
        y[k] = in ? *reinterpret_cast<const chunk*>(pb + 16 * int64_t(c)) : nothing;
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        acc[0] = Unit<T>::few(x[k], y[k], acc[0]);
        if (PAIR) acc[kPair - 1] = Unit<T>::few(x2[k], y[k], acc[kPair - 1]);
      }
    }
#pragma unroll
    for (int q = 0; q < kPair; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r) s.sums[wave][q][lane & 15][4 * (lane >> 4) + r] = acc[q][r];
    __syncthreads();
  }
  static __device__ __forceinline__ sum of(const Shared& s, int q, int c, int r) {
    sum x = s.sums[0][q][c][r];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) x += s.sums[w][q][c][r];
    return x;
  }
};

// Which tile a workgroup has: consecutive ones, which go to one XCD, are those of four tiles of B's rows with one of A's rows, then with the next: the 32 CUs of an XCD work on four by
// eight tiles at a time (65536 x 4096 with 4096 channels in 8 bits 1155 us; with two 1180, six 1160, eight by four 1222, sixteen 1300; 32768 rows of 2048 with 8192 hidden, a
// whole step: 8.60, 8.61, 8.67, 8.79 and 9.15 ms).
constexpr uint32_t kBeside = 4;
struct Tile { int32_t m, n, part; };
__device__ __forceinline__ Tile tile_of(uint32_t block, uint32_t blocks, int32_t tiles_m, int32_t tiles_n) {
  const uint32_t piece = piece_of(block, blocks), all = uint32_t(tiles_m) * uint32_t(tiles_n);
  Tile t;
  t.part = int32_t(piece / all);
  const uint32_t of = piece % all, group = of / (kBeside * uint32_t(tiles_m)), in = of % (kBeside * uint32_t(tiles_m));
  const uint32_t left = uint32_t(tiles_n) - group * kBeside, wide = left < kBeside ? left : kBeside;
  t.m = int32_t(in / wide);
  t.n = int32_t(group * kBeside + in % wide);
  return t;
}

}  // namespace
}  // namespace layer
}  // namespace lgp
