// What the operators of a model layer share: element types, the 32x32x16 matrix instruction and its operand order, documents and
// their tiles, host helpers of the entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "legion_prep.h"

namespace lgp {
namespace layer {

using f16 = _Float16;
using bf16 = __bf16;
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// The matrix instruction D[32, 32] += A[32, 16] B[16, 32].  Lane l holds of A row l % 32 and of B column l % 32, each at eight places of
// the sum; of D it holds column l % 32, register r being row 8 * (r / 4) + 4 * (l / 32) + r % 4.  Any order of the sum's places does as
// long as A and B agree, so registers 8 s .. 8 s + 7 of a D are, rounded, a B operand whose places are rows
// 16 s + 8 * (j / 4) + 4 * (l / 32) + j % 4: a product is handed to the next one without leaving the registers, and the other operand is
// read in that order (Places::across).
template <typename T> struct Elem;
template <> struct Elem<f16> {
  typedef f16 x8 __attribute__((ext_vector_type(8)));
  typedef f16 x4 __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ floatx16 mfma(x8 a, x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Elem<bf16> {
  typedef bf16 x8 __attribute__((ext_vector_type(8)));
  typedef bf16 x4 __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ floatx16 mfma(x8 a, x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <typename T> using vec8 = typename Elem<T>::x8;
template <typename T> using vec4 = typename Elem<T>::x4;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }     // one ulp, 0 and inf at the ends
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }

// Sum over groups of L lanes, the same in all of them.  Moves within rows of 16 lanes need no trip through LDS.
template <int CTRL> __device__ __forceinline__ float moved(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int L> __device__ __forceinline__ float sum_of_lanes(float x) {
  if constexpr (L >= 2) x += moved<0xb1>(x);        // quad_perm 1 0 3 2
  if constexpr (L >= 4) x += moved<0x4e>(x);        // quad_perm 2 3 0 1
  if constexpr (L >= 8) x += moved<0x141>(x);       // row_half_mirror: the other four of eight
  if constexpr (L >= 16) x += moved<0x140>(x);      // row_mirror: the other eight of sixteen
  if constexpr (L >= 32) x += __shfl_xor(x, 16, 64);
  return x;
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// A tile of rows x D elements of 16 bits in LDS, D 32 to 256: 16-byte chunk c of row r lies at place c ^ swizzle(r) of the row.  256 bytes lie in
// different banks, so 16 lanes that read the same chunk of 16 rows, and 32 lanes that read 64 bytes of four rows transposed, want different
// places there: the row's low bits, reversed, do both (for D of 128, chunks of 32 rows 3.6 -> 2.2 ns a wave and CU against the row's low bits
// as they are, transposed reads 3.5 -> 1.5).
template <int D> __device__ __forceinline__ int swizzle(int row) { return int(__brev(uint32_t(row)) >> 28) & (D / 8 >= 16 ? 15 : D / 8 - 1); }
template <int D> __device__ __forceinline__ int chunk_at(int row, int chunk) { return row * D + ((chunk ^ swizzle<D>(row)) << 3); }

// 16 bytes of each lane, `offset` bytes behind `from`, go to `lds` + 16 * lane, past the registers.  The compiler would wait for them before the
// next read of LDS, whichever tile that reads, so it is not told: what arrives may be read when the wave's loads are done (loads_done) and
// a barrier was passed.
__device__ __forceinline__ void copy16(const void* from, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(from) : "memory");       // m0 is never held across statements
}
template <typename T> __device__ __forceinline__ const T* in_all_lanes(const T* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const T*>(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x)))) | uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x >> 32)))) << 32);
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return uint32_t(uintptr_t((const __attribute__((address_space(3))) char*)p)); }

// Rows in memory, `row` elements apart; with fold = 2^log2_fold each is that many rows of a tile, `head` elements apart.  Strides are below
// 2^24, and those of up to 16 heads below 2^26, so that the 32 rows that a wave's lanes are in lie less than 2^32 bytes apart.
constexpr int64_t kMostStride = int64_t(1) << 24;
template <typename T> struct Rows {
  const T* from;
  int64_t row, head;
  int32_t log2_fold;
};

// ROWS rows of `dim` elements, from row `first` (a multiple of 16) on, into such a tile, by the THREADS threads of a workgroup.  A wave writes
// 64 consecutive chunks, and each lane reads the one that belongs there.  Rows from `there` on become zeros; what lies beyond dim is left as
// it is, which is zero (clear_tile).
template <typename T, int D, int ROWS, int THREADS>
__device__ __forceinline__ void copy_tile(T* tile, const Rows<T>& rows, int32_t first, int dim, int there, int tid) {
  constexpr int kStep = THREADS * 8 / D;         // rows that all threads write at once
  static_assert(ROWS % kStep == 0 || kStep % ROWS == 0, "whole waves");
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(tile) + (tid & ~63) * 16);
  const int r0 = tid / (D / 8), fold = 1 << rows.log2_fold;
  const T* from = rows.from + int64_t(first >> rows.log2_fold) * rows.row;
  if (kStep > ROWS && r0 >= ROWS) return;        // more threads than chunks
  constexpr int kSteps = kStep > ROWS ? 1 : ROWS / kStep;
#pragma unroll
  for (int c = 0; c < kSteps; ++c) {
    // with 16 rows and more at once the places in a row repeat, and so do the heads of a token
    const int r = kStep % 16 == 0 ? r0 : c * kStep + r0, d = ((tid % (D / 8)) ^ swizzle<D>(r)) * 8;
    const uint32_t offset = (uint32_t(r >> rows.log2_fold) * uint32_t(rows.row) + uint32_t(r & (fold - 1)) * uint32_t(rows.head) + d) * sizeof(T);
    const T* base = in_all_lanes(kStep % 16 == 0 ? from + int64_t(c * kStep >> rows.log2_fold) * rows.row : from);
    if (c * kStep + r0 < there && d < dim) copy16(base, offset, to + c * THREADS * 16);
  }
  if (there < ROWS) {
    const vec8<T> zero = {};
#pragma unroll
    for (int c = 0; c < kSteps; ++c)
      if (c * kStep + r0 >= there) reinterpret_cast<vec8<T>*>(tile)[c * THREADS + tid] = zero;
  }
}
template <typename T, int ELEMS, int THREADS> __device__ __forceinline__ void clear_tile(T* tile, int tid) {
  const vec8<T> zero = {};
  for (int i = tid; i < ELEMS / 8; i += THREADS) reinterpret_cast<vec8<T>*>(tile)[i] = zero;
}
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }       // vmcnt(0), the other counters as they are

// A tile may be read: the copies of all waves that share it are done, and so are everyone's reads of the tile that is overwritten next.
template <bool SHARED> __device__ __forceinline__ void tile_ready() {
  if constexpr (SHARED) {
    loads_done();
    __syncthreads();
  } else {
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
  }
}

// Division of numbers below 2^31 by a fixed one.
struct Divisor { uint32_t by, mul, shift; };
inline Divisor divisor(uint32_t by) {
  uint32_t l = 0;
  while ((1u << l) < by) ++l;
  return {by, by > 1 ? uint32_t(((uint64_t(1) << (31 + l)) + by - 1) / by) : 0, l ? l - 1 : 0};
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor& d) { return d.by == 1 ? n : __umulhi(n, d.mul) >> d.shift; }

// Where a lane finds its operands in such tiles.  Both places are those of the first of many, from which the others differ by a few bits or by
// whole rows: so two registers hold all addresses, if the compiler is kept from taking one for each (again(), once in a loop's body).
template <typename T, int D> struct Places {
  int row, col;
  __device__ __forceinline__ explicit Places(int lane) {
    const int r = lane & 31, i = lane & 15, r2 = 4 * (lane >> 5) + (i >> 2), c2 = 16 * ((lane >> 4) & 1) + 4 * (i & 3);
    row = chunk_at<D>(r, lane >> 5);
    col = chunk_at<D>(r2, c2 >> 3) + (c2 & 7);
  }
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(row), "+v"(col)); }
  // The operand whose rows are 32 rows of the tile and whose sum runs along them: elements 16 kk + 8 * (lane / 32) ... + 7 of row row0 + lane % 32.
  __device__ __forceinline__ vec8<T> along(const T* tile, int row0, int kk) const {
    return *reinterpret_cast<const vec8<T>*>(tile + row0 * D + (row ^ (kk << 4)));
  }
  // The operand whose rows are 32 columns of the tile and whose sum runs along its rows: column col0 + lane % 32 of rows row0 + 4 * (lane / 32) ... + 3
  // and of those eight further on (row0 a multiple of 16, col0 of 32).  Each 16 lanes read four rows of 16 columns, which the LDS hands out transposed.
  __device__ __forceinline__ vec8<T> across(const T* tile, int row0, int col0) const {
    typedef __attribute__((address_space(3))) shortx4* place;
    union { shortx4 s[2]; vec8<T> v; } u;
    const int at = col ^ col0;
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(tile + row0 * D + at));
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(tile + (row0 + 8) * D + (at ^ 8)));       // the swizzle of a row eight further on
    return u.v;
  }
};

// Documents: document d owns rows offsets[d] .. offsets[d + 1], the first lens[d] of which hold tokens.  The first begins at row 0 and the
// last ends at the last row, whatever the array says there; what else makes no sense is clamped, so no row outside is ever touched.
struct Side {
  const int32_t* offsets;
  const int32_t* lens;
  const int32_t* pos;
  int32_t rows;
};
struct Span { int32_t begin, tokens, owned; };       // first row, rows with a token, rows
__device__ __forceinline__ int32_t offset_of(const Side& s, int32_t d, int32_t n) {
  if (d <= 0) return 0;
  if (d >= n) return s.rows;
  const int32_t o = s.offsets[d];
  return o < 0 ? 0 : o > s.rows ? s.rows : o;
}
__device__ __forceinline__ Span span_between(const Side& s, int32_t d, int32_t begin, int32_t end) {       // d is the same in the whole wave
  Span x;
  x.begin = __builtin_amdgcn_readfirstlane(begin);
  end = __builtin_amdgcn_readfirstlane(end);
  x.owned = end > x.begin ? end - x.begin : 0;
  x.tokens = x.owned;
  if (s.lens) {
    const int32_t t = __builtin_amdgcn_readfirstlane(s.lens[d]);
    x.tokens = t < 0 ? 0 : t < x.owned ? t : x.owned;
  }
  return x;
}
__device__ __forceinline__ Span span_of(const Side& s, int32_t d, int32_t n) { return span_between(s, d, offset_of(s, d, n), offset_of(s, d + 1, n)); }

// Tiles of `size` rows, found without a list of them: with `fold` rows per token, document d has the tiles from
// floor(offset * fold / size) + d on, which leaves each at least as many as its rows take, and all of them rows * fold / size + n.  A wave
// looks at 64 documents around where the tile would be if all had as many rows, which also tells where the document begins and ends; if it
// is not among them, at 64 between the ends of what is left, until it is found.
__device__ __forceinline__ int32_t first_tile(int32_t offset, int32_t d, int32_t fold, int32_t size) { return int32_t(int64_t(offset) * fold / size) + d; }
struct Found { int32_t doc, first; Span span; };       // first: its first tile
__device__ __forceinline__ Found find_tile(const Side& s, int32_t n, float docs_per_tile, int32_t fold, int32_t size, int32_t tile, int lane) {
  Found f;
  int32_t lo = int32_t(float(tile) * docs_per_tile) - 31;
  lo = lo > n - 63 ? n - 63 : lo;
  lo = lo < 0 ? 0 : lo;
  int32_t at = lo + lane < n ? lo + lane : n, offset = offset_of(s, at, n);
  int known = __popcll(__ballot(lo + lane <= n && first_tile(offset, at, fold, size) <= tile));       // of them, begin no later than the tile
  if (known == 0 || known == 64) {
    int32_t hi = known ? n : lo;
    lo = known ? lo + 63 : 0;
    while (hi - lo > 1) {
      const int32_t step = (hi - lo + 63) / 64, d = lo + (lane + 1) * step;
      lo += step * __popcll(__ballot(d < hi && first_tile(offset_of(s, d, n), d, fold, size) <= tile));
      hi = hi < lo + step ? hi : lo + step;
    }
    at = lo + lane < n ? lo + lane : n;
    offset = offset_of(s, at, n);
    known = 1;
  }
  f.doc = __builtin_amdgcn_readfirstlane(lo + known - 1);
  const int32_t begin = __builtin_amdgcn_readlane(offset, __builtin_amdgcn_readfirstlane(known - 1));
  f.first = first_tile(begin, f.doc, fold, size);
  f.span = span_between(s, f.doc, begin, __builtin_amdgcn_readlane(offset, __builtin_amdgcn_readfirstlane(known & 63)));
  return f;
}
// The same document on the other side, which may be the same rows.
__device__ __forceinline__ Span other_side(const Side& other, const Side& s, const Found& f, int32_t n) {
  return other.offsets == s.offsets && other.lens == s.lens && other.rows == s.rows ? f.span : span_of(other, f.doc, n);
}
inline int64_t tiles_of(int64_t rows, int64_t fold, int64_t n, int64_t size) { return rows * fold / size + n; }

// Workgroups go to the eight XCDs in turn, and each XCD has an L2 of its own: consecutive pieces of work, which share rows, go to one XCD.
__device__ __forceinline__ uint32_t piece_of(uint32_t block, uint32_t blocks) {
  const uint32_t each = blocks / 8, more = blocks % 8, x = block % 8;
  return x * each + (x < more ? x : more) + block / 8;
}

inline int use_device(int device) {
  static const int devices = [] {
    int n = 0;
    return hipGetDeviceCount(&n) == hipSuccess ? n : 0;
  }();
  if (device < 0 || device >= devices || hipSetDevice(device) != hipSuccess) {
    (void)hipGetLastError();
    return LGP_EINVAL;
  }
  return LGP_OK;
}
// A launch has less than 2^32 threads, and what is beyond is dropped without an error: f(first workgroup, workgroups) for as many launches as it takes.
template <typename F> void in_launches(int64_t groups, int64_t threads, F f) {
  const int64_t most = (int64_t(1) << 31) / threads;
  for (int64_t g = 0; g < groups; g += most) f(uint32_t(g), uint32_t(groups - g < most ? groups - g : most));
}
inline int launched() { return hipGetLastError() == hipSuccess ? LGP_OK : LGP_EHIP; }
inline int compute_units(int device) {
  int n = 0;
  return hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) == hipSuccess && n > 0 ? n : 256;
}
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace layer
}  // namespace lgp
