// Attention inside documents: what the forward and the backward kernels share.
#pragma once

#include "layer_dev.hpp"

#include <type_traits>

namespace lgp {
namespace layer {

// Queries are handled as folded rows: the G query heads of a key head are G rows of each token, row t * G + g of key head hk being head
// hk * G + g of token t.  Keys and values are then read once for all of them, single tokens fill tiles, and the sum over the heads that
// share a key head is a sum over rows.
struct AttendParams {
  const void *q, *k, *v;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;
  Side qs, ks;
  int32_t n_docs, heads, kv_heads, group, dim;
  Divisor per_token;         // by group
  int32_t log2_fold;         // by keys: heads of a token that are folded, all of the group or one
  // Scores in powers of two: the product qk, capped, times z_mul = scale * log2(e), with the magnitude of the scale: where it is negative, q (by
  // keys: k) is negated as it is read.  z_mul is then positive (a scale of zero is taken as 1e-30), and the largest product is the largest score.
  float scale, z_mul;
  float t_mul, t_inv, tanh_c[4];         // scale / cap and its inverse, and kTanh with its powers: see capped_near
  float near;                // up to which product capped_near holds; negative where the powers leave the range of fp32
  bool negate;
  const float* slopes;
  float docs_per_tile;
  uint32_t first;            // workgroups of launches before this one
  int32_t tiles, splits;     // tiles of queries per key head (backward by keys: of keys); parts of the keys; attend_single.hip: workgroups with documents,
                             // and before them those that list the large ones
  // forward
  void *out, *rest;
  float* lse;
  float *part_o, *part_ml;   // [split][q_rows][heads][dim] and [split][q_rows][heads][2], if splits > 1
  // backward
  const void* d_out;
  const float* lse_in;
  void *dq, *dk, *dv;
  float* delta;              // [q_rows][heads]: d_out . out
  floatx4* sums;             // [split][q_rows][heads], if the gradient of the slopes is wanted: see dq_rows
  // documents of one query on average: those that are not left to single waves, see each_large
  bool any_large;            // there can be some
  int32_t* n_large;          // [survey], or NULL: documents are few
  uint16_t* large;           // [survey][kSurvey]: counted from the survey's first document
};

template <typename T> __device__ __forceinline__ vec8<T> load8(const T* p) { return *reinterpret_cast<const vec8<T>*>(p); }
template <typename T> __device__ __forceinline__ vec8<T> load8(const T* p, bool there, bool negate) {
  union { vec8<T> v; uint32_t w[4]; } u = {};
  if (there) u.v = load8(p);
  if (negate)
#pragma unroll
    for (int i = 0; i < 4; ++i) u.w[i] ^= 0x80008000u;
  return u.v;
}

// The cap: a product qk becomes tanh(x) / t_mul with x = qk * t_mul, which is qk where the cap is far.  Up to x = kNear that is
// qk (1 + c0 x^2 + c1 x^4 + c2 x^6 + c3 x^8), fitted by least squares of the relative error, reweighted until even: 1e-7 with its roundings, and it
// is where capped scores mostly are; the powers of t_mul are in the coefficients.  Beyond, tanh(x) = 1 - 2 / (e^2x + 1), which near zero would be 1e-7
// off in absolute terms, times the cap.  Scores of a tile go the short way together, if none is beyond.  Cap 30, scores of about 1, 4 and 16: 1024
// documents of 276, heads 8/8 of 32, 331, 342 and 437 us forward; 128 of 916, heads of 64, 428, 453 and 628.  Where the powers of t_mul leave the range of
// fp32 -- products of millions below a cap of a million, caps of millionths -- all go the other way, which takes x first.
constexpr float kNear = 0.55f;
constexpr float kTanh[4] = {-0.3333294689655304f, 0.13320724666118622f, -0.05267181620001793f, 0.016437582671642303f};
__device__ __forceinline__ float capped_near(const AttendParams& p, float s) {
  const float w = s * s;
  return s * fmaf(fmaf(fmaf(fmaf(p.tanh_c[3], w, p.tanh_c[2]), w, p.tanh_c[1]), w, p.tanh_c[0]), w, 1.f);
}
__device__ __forceinline__ float capped_any(const AttendParams& p, float s) {
  const float x = s * p.t_mul, w = x * x, far = (1.f - 2.f * rcp_fast(exp2_fast(x * (2.f * kLog2e)) + 1.f)) * p.t_inv;
  return fabsf(x) <= kNear ? s * fmaf(fmaf(fmaf(fmaf(kTanh[3], w, kTanh[2]), w, kTanh[1]), w, kTanh[0]), w, 1.f) : far;
}
template <bool CAP> __device__ __forceinline__ void cap(const AttendParams& p, floatx16& s) {
  if constexpr (CAP) {
    float most = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(s[r]));
    if (__any(most > p.near)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = capped_any(p, s[r]);
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = capped_near(p, s[r]);
    }
  }
}
template <bool CAP> __device__ __forceinline__ float capped(const AttendParams& p, float s) { return CAP ? capped_any(p, s) : s; }
// u times the cap's derivative, 1 - tanh^2, from the capped product.
template <bool CAP> __device__ __forceinline__ float through_cap(const AttendParams& p, float u, float s) {
  if constexpr (CAP) {
    const float t = s * p.t_mul;
    return fmaf(-u * t, t, u);
  }
  return u;
}

// The part of a document's keys that split s of `splits` takes: whole tiles of `size` keys, at most 256.  Counted in tiles: all parts together may be
// as many keys more than there are as to pass 2^31.
__host__ __device__ __forceinline__ void part_of(int32_t keys, int32_t size, int32_t s, int32_t splits, int32_t& begin, int32_t& end) {
  const int32_t tiles = (keys + size - 1) / size, each = (tiles + splits - 1) / splits, first = s * each, last = first + each;
  begin = first < tiles ? first * size : keys;
  end = last < tiles ? last * size : keys;
}

int check_attend(const lgp_documents* d, const lgp_attention* a);
AttendParams attend_params(const lgp_documents* d, const lgp_attention* a);

// Documents of one query and few keys on average (attend_single.hip).  The host knows no more of them; one that has many of both, or very many keys,
// would be one wave's work and take as long as its pairs one after the other.  So waves leave documents of more than kLargePairs pairs, if there can be
// any of more than kFewPairs, and a second launch of the tiled kernels goes through these: a workgroup counts all their tiles, 64 documents at a time,
// and takes every so many-th one.  Up to kOwnSurveys * kSurvey documents are looked through by every workgroup of it; of more, waves of the first
// launch list the large ones, kSurvey documents each (8192 documents, us a training step: looked through 61, listed 51 to 53).  Measured where none
// is large: a launch of 5 us, 3 for the host; 1024 documents of up to 10 keys, heads 8/8 of 32, forward 12.9 -> 16.3, trained 31 -> 37.5; 122 880 trained
// 582 -> 592.  2000 documents, bf16, heads 8/8 of 64: one of them 2000 rows and the others empty, forward 40 and backward 100; one of them a query over
// 60 000 keys, 390 and 1240, one workgroup for each head.
constexpr int kLargePairs = 512, kFewPairs = 2048, kSurvey = 512, kOwnSurveys = 8, kLargeGroups = 256;       // kLargeGroups: workgroups of the second launch
bool single_queries(const lgp_documents* d, const lgp_attention* a);
inline bool any_large(const lgp_documents* d) {
  const int64_t q = d->q_rows > 1 ? d->q_rows : 1, k = d->k_rows > 1 ? d->k_rows : 1;
  return q > kFewPairs || k > kFewPairs || q * k > kFewPairs;
}
inline int64_t surveys(const lgp_documents* d) { return any_large(d) && d->n_docs > kOwnSurveys * kSurvey ? (d->n_docs + kSurvey - 1) / kSurvey : 0; }
inline size_t survey_bytes(const lgp_documents* d) { return (size_t(surveys(d)) * (sizeof(int32_t) + kSurvey * sizeof(uint16_t)) + 15) / 16 * 16; }
inline void set_survey(AttendParams& p, const lgp_documents* d, void* at) {
  const int64_t n = surveys(d);
  p.any_large = any_large(d);
  p.n_large = n ? static_cast<int32_t*>(at) : nullptr;
  p.large = n ? reinterpret_cast<uint16_t*>(p.n_large + n) : nullptr;
}
void launch_single(const AttendParams& p, const lgp_attention* a, bool backward, hipStream_t s);
void launch_large(const AttendParams& p, const lgp_attention* a, hipStream_t s);       // of the forward pass
__device__ __forceinline__ bool is_large(int32_t q_owned, int32_t k_owned) {
  return int64_t(q_owned > 1 ? q_owned : 1) * (k_owned > 1 ? k_owned : 1) > kLargePairs;
}
// Rows of document d as span_of has them, none beyond the last one; without a branch, so that loads do not wait for each other.
__device__ __forceinline__ int32_t owned_of(const Side& s, int32_t d, int32_t n) {
  const int32_t a = d < n ? d : n, b = d < n ? d + 1 : n;
  int32_t begin = s.offsets[a], end = s.offsets[b];
  begin = a == 0 ? 0 : a == n ? s.rows : min(max(begin, 0), s.rows);
  end = b == n ? s.rows : min(max(end, 0), s.rows);
  return max(end - begin, 0);
}
// A wave lists the large ones of kSurvey documents, in their order, and counts them.
__device__ __forceinline__ void list_large(const AttendParams& p, int32_t survey, uint16_t* docs, int32_t* count) {
  constexpr int kAtOnce = kSurvey / 64;        // loads of a lane's documents are on their way together
  const int lane = threadIdx.x & 63;
  const int32_t d0 = survey * kSurvey + lane;
  bool large[kAtOnce];
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i)            // beyond the last one: no rows
    large[i] = is_large(owned_of(p.qs, d0 + 64 * i, p.n_docs), owned_of(p.ks, d0 + 64 * i, p.n_docs));
  int32_t n = 0;
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) {
    const uint64_t all = __ballot(large[i]);
    if (large[i]) docs[n + __popcll(all & ((uint64_t(1) << lane) - 1))] = uint16_t(64 * i + lane);
    n += __popcll(all);
  }
  if (lane == 0) *count = n;
}
// tiles(rows of queries, of keys) is what a document has of them; work(document, tile) is called by all waves of a workgroup of 256 alike.
template <typename Tiles, typename Work> __device__ __forceinline__ void each_large(const AttendParams& p, Tiles tiles, Work work) {
  __shared__ int32_t own_n[kOwnSurveys];
  __shared__ uint16_t own[kOwnSurveys * kSurvey];
  const int lane = threadIdx.x & 63;
  const int32_t n = (p.n_docs + kSurvey - 1) / kSurvey;
  const int32_t* counts = p.n_large;
  const uint16_t* docs = p.large;
  if (!counts) {
    for (int32_t at = threadIdx.x >> 6; at < n; at += 4) list_large(p, at, own + at * kSurvey, own_n + at);
    __syncthreads();
    counts = own_n;
    docs = own;
  }
  int64_t next = blockIdx.x;               // this workgroup's next tile, counted from the first of the documents that are looked at
  for (int32_t s0 = 0; s0 < n; s0 += 64) {
    const int32_t count = s0 + lane < n ? counts[s0 + lane] : 0;
    for (uint64_t some = __ballot(count > 0); some; some &= some - 1) {
      const int of = __builtin_ctzll(some);
      const int32_t listed = __builtin_amdgcn_readlane(count, of);
      for (int32_t i0 = 0; i0 < listed; i0 += 64) {
        const int32_t doc = i0 + lane < listed ? (s0 + of) * kSurvey + docs[int64_t(s0 + of) * kSurvey + i0 + lane] : -1;
        // in 64 bits: where offsets make no sense, every document may have all rows
        int64_t upto = doc >= 0 ? tiles(owned_of(p.qs, doc, p.n_docs), owned_of(p.ks, doc, p.n_docs)) : 0;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const int64_t before = __shfl_up(upto, d, 64);
          if (lane >= d) upto += before;
        }
        const int64_t all = __shfl(upto, 63, 64);
        for (; next < all; next += gridDim.x) {
          const int l = __popcll(__ballot(upto <= next));
          const int64_t first = l ? __shfl(upto, l - 1, 64) : 0;
          work(__builtin_amdgcn_readlane(doc, l), __builtin_amdgcn_readfirstlane(int32_t(next - first)));
          __syncthreads();                 // the next one has the same LDS
        }
        next -= all;
      }
    }
  }
}

// With fp16 a probability below 2^-14 would lose digits, and over 16 000 keys most are: where they are an operand of a product, the backward
// pass takes them times 2^12, which cannot overflow, and the result times 2^-12.
template <typename T> constexpr float kLift = 1.f;
template <> inline constexpr float kLift<f16> = 4096.f;
template <typename T> constexpr float kLiftLog2 = 0.f;
template <> inline constexpr float kLiftLog2<f16> = 12.f;

// dU has no such bound on either side: it is as small as the gradients of a mean over a batch and the probabilities together, or as large as those of
// a loss that was scaled up.  With fp16 it is taken times a power of two for each column of a product: 2^48 at first, and lowered, with what has been
// added up, when one comes out beyond kLiftedMost.  (Of numbers of fp16 the largest dU is 2^39, times a distance of 2^24 in the sums for the slopes.)
constexpr float kLiftFirstLog2 = 48.f, kLiftFirst = 0x1p48f, kLiftedMost = 32768.f;
// By what power of two: `most` then is 512 to 1024, which leaves room for larger ones.
__device__ __forceinline__ int lower_log2(float most) { return 10 - __builtin_amdgcn_frexp_expf(most); }

// Waves per SIMD that the kernels' registers are to leave room for: as many as their tiles in LDS do.
constexpr int waves_per_simd(int dim, int waves) { return dim == 32 ? 4 : dim == 64 ? (waves == 1 ? 2 : 3) : waves == 1 ? 1 : 2; }

// Launch shapes, chosen on the host by what it knows: rows and documents.
// Whether a workgroup is one wave of 32 rows, which waits for no other but has its tiles to itself: documents of up to 32 rows, and with heads of up
// to 32, whose tiles are small, of up to 320.  Four waves and one, us forward / backward, bf16, heads 8/8 of 32, half of the rows without a token: with cap
// and bias, 4000 documents of 100 rows 279 / 785 and 209 / 626, 1050 of 276 239 / 618 and 216 / 552, 781 of 320 188 / 546 and 188 / 506, 320 of 500
// 144 / 414 and 148 / 421; without, 245 / 617 and 199 / 551, 176 / 471 and 184 / 476, 153 / 408 and 167 / 432, 95 / 282 and 105 / 314.  With all rows full
// and neither cap nor bias four waves are ahead from 100 rows on (297 / 861 and 325 / 891; at 320 234 / 651 and 293 / 728), which the host cannot tell.
// 256 documents of 916 folded rows, heads of 64: forward 198 and 284.
inline bool one_wave(int64_t rows, int64_t docs, int32_t dim) { return rows <= (dim <= 32 ? 320 : 32) * docs; }
constexpr int kMostSplits = 256;        // a thread of join_kernel each
constexpr int kForwardRows = 32;        // folded rows of a wave
struct ForwardShape { int waves, key_waves; int64_t tiles; int splits; };      // waves of rows, and of parts of the keys, in a workgroup
ForwardShape forward_shape(int device, const lgp_documents* d, const lgp_attention* a);

}  // namespace layer
}  // namespace lgp
