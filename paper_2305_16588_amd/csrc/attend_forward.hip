// Attention inside documents, forward: out = softmax(scores) v in one pass over the keys with a running maximum and sum.
#include "attend.hpp"

#include <algorithm>
#include <cmath>

namespace lgp {
namespace layer {
namespace {

// A wave has 32 folded rows, as columns of the transposed scores S^T = K Q^T: every lane then holds scores of one row, so maximum and sum
// need one exchange between the halves of the wave, and the rounded probabilities are the operand of O^T = V^T P^T as they stand
// (layer_dev.hpp).  NW waves share the tiles of keys and values in LDS, where the next tile arrives while this one is worked on.  D is the
// head's dimension rounded up to 32, 64 or 128, with zeros.  Scores are taken against a base that is raised, and sums and results shrunk, only
// when a row's maximum has outgrown it by 2^kSlack: after the first tiles that is rare, and it would be a quarter of the arithmetic.  The base is
// settled before anything is taken off: a difference from a base that a tile leaves far behind would be rounded at the size of that distance.  The
// two places of a tile are two copies of the loop's body, so that no address is computed in it.
// Probabilities are rounded to the type of v for the second product, as the values themselves are: 32 bits there would want the fp32 matrix
// instructions, at a fraction of the rate.  Their sum is taken before, which lse wants; dividing by the sum of the rounded ones instead was level in error and 1 to 4 % dearer.  Error
// in the 2-norm of bf16 results 0.0024 where one rounding at the end has 0.0017, of fp16 2.9e-4 and 2.1e-4.
// Where a document has no more rows than a wave (NW 1), KW waves have the same rows and every KW-th tile of the keys each, in tiles of their own,
// and their results are joined in LDS.
// Measured: 4 documents of 8192 tokens, heads 8/4 of 128, bf16, bias: 1220 to 1250 us, 0.89 PFLOP/s, bound by matrix and vector instructions (41 and
// 60 % of the cycles); 1024 documents of 276 rows, heads 8/8 of 32, cap and bias: 260 us, bound by the vector instructions of cap, bias and exponent
// (70 %); 256 of 916, heads 4/2 of 64, cap: 158 us, likewise (88 %); 16 queries over 50 001 keys each, heads 16/2 of 128: 159 us, bound by bytes, 5.2 TB/s.
constexpr float kSlack = 8.f;
template <typename T, int D, bool CAP, bool BIAS, int NW, int KW, int BN>
__device__ __forceinline__ void attend_rows(const AttendParams& p, int32_t hk, int32_t split, int32_t row0, const Span qd, const Span kd) {
  constexpr int kThreads = 64 * NW;                           // that share tiles
  __shared__ __align__(16) T lds_tiles[KW][2][2][BN * D];     // of keys and values, two places each
  __shared__ __align__(16) float lds_at[KW][2][BIAS ? BN : 4];
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5, tid = threadIdx.x % kThreads, wave = NW > 1 ? threadIdx.x >> 6 : 0;
  const int part = KW > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  auto& lds_k = lds_tiles[part][0];
  auto& lds_v = lds_tiles[part][1];
  auto& lds_pos = lds_at[part];

  int32_t k_begin, k_end;
  part_of(row0 < qd.tokens * p.group ? kd.tokens : 0, BN, split * KW + part, p.splits * KW, k_begin, k_end);
  const Rows<T> k_rows = {static_cast<const T*>(p.k) + int64_t(kd.begin) * p.k_row + int64_t(hk) * p.k_head, p.k_row, 0, 0};
  const Rows<T> v_rows = {static_cast<const T*>(p.v) + int64_t(kd.begin) * p.v_row + int64_t(hk) * p.v_head, p.v_row, 0, 0};
  int32_t next_pos = 0;        // as it comes, so that nothing waits for it yet
  auto stage = [&](int32_t k0, int to) {
    if constexpr (BIAS) next_pos = tid < BN && k0 + tid < k_end ? p.ks.pos[kd.begin + k0 + tid] : 0;
    copy_tile<T, D, BN, kThreads>(lds_k[to], k_rows, k0, p.dim, k_end - k0, tid);
    copy_tile<T, D, BN, kThreads>(lds_v[to], v_rows, k0, p.dim, k_end - k0, tid);
  };
  if (p.dim < D) {
    clear_tile<T, 4 * BN * D, kThreads>(lds_k[0], tid);
    tile_ready<(NW > 1)>();
  }
  if (k_begin < k_end) stage(k_begin, 0);

  const int32_t row = row0 + 32 * wave + col;
  const bool live = row < qd.tokens * p.group;
  const int32_t of_doc = quotient(row, p.per_token), token = qd.begin + of_doc, head = hk * p.group + row - of_doc * p.group;
  vec8<T> qf[D / 16];
  {
    const T* q = static_cast<const T*>(p.q) + int64_t(token) * p.q_row + int64_t(head) * p.q_head;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = load8(q + 16 * kk + 8 * half, live && 16 * kk + 8 * half < p.dim, p.negate);
  }
  float slope = 0.f, at = 0.f;
  if constexpr (BIAS) {
    if (live) {
      slope = p.slopes[head] * kLog2e;
      at = float(p.qs.pos[token]);
    }
  }

  floatx16 o[D / 32] = {};
  // Scores are taken relative to `base`; a maximum beyond `limit` raises it: any, until the row has seen a score that is not infinite.
  float base = 0.f, limit = -3e38f, sum = 0.f;
  Places<T, D> at_tile(lane);
  const bool idle = row0 + 32 * wave >= qd.tokens * p.group;         // a wave of rows without tokens only copies
  // How far a score is above x, rounded once: without a bias from the product.  Only where a base passes 2^24, whose places are more than one, products
  // are made scores first: the largest is the base to the last digit then.
  float mul = p.z_mul;
  auto above = [&](float score, float x) { return BIAS ? score - x : fmaf(score, mul, -x); };
  auto step = [&](int32_t k0, auto stage_now) {
    constexpr int now = decltype(stage_now)::value;
    if constexpr (BIAS) {
      if (tid < BN) lds_pos[now][tid] = float(next_pos);
    }
    tile_ready<(NW > 1)>();
    if (k0 + BN < k_end) stage(k0 + BN, now ^ 1);
    if (idle) return;
    if constexpr (D == 128) at_tile.again();
    const T *tile_k = lds_k[now], *tile_v = lds_v[now];

    floatx16 s[BN / 32];
#pragma unroll
    for (int b = 0; b < BN / 32; ++b) {
      floatx16 acc = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) acc = Elem<T>::mfma(at_tile.along(tile_k, 32 * b, kk), qf[kk], acc);
      cap<CAP>(p, acc);
      s[b] = acc;
    }
    if constexpr (BIAS) {
#pragma unroll
      for (int b = 0; b < BN / 32; ++b)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const floatx4 kpos = *reinterpret_cast<const floatx4*>(&lds_pos[now][32 * b + 8 * r4 + 4 * half]);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[b][4 * r4 + i] = fmaf(s[b][4 * r4 + i], p.z_mul, -slope * fabsf(at - kpos[i]));
        }
    }
    auto make_scores = [&] {
#pragma unroll
      for (int b = 0; b < BN / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][r] *= p.z_mul;
    };
    if (!BIAS && mul != p.z_mul) make_scores();
    if (k0 + BN > k_end) {
#pragma unroll
      for (int b = 0; b < BN / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + 32 * b + 8 * (r / 4) + 4 * half + r % 4 >= k_end) s[b][r] = -INFINITY;
    }
    float most = s[0][0];
#pragma unroll
    for (int b = 0; b < BN / 32; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) most = fmaxf(most, s[b][r]);
    most = fmaxf(most, other_half(most));
    if (__any(above(most, base) > limit)) {
      // A row that has no base yet has nothing either, and 2^-by is inf where its first score is far below zero.  The row's state decides, not its sum:
      // a lane's sum is that of half of the keys so far, while its results are those of all.
      const bool raise = above(most, base) > limit;
      const float raised = BIAS ? most : most * mul, shrink = raise && limit == kSlack ? exp2_fast(base - raised) : 1.f;
      base = raise ? raised : base;
      limit = raise ? kSlack : limit;
      sum *= shrink;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= shrink;
      if (!BIAS && mul == p.z_mul && __any(fabsf(base) > 0x1p24f)) {
        make_scores();
        mul = 1.f;
      }
    }
#pragma unroll
    for (int b = 0; b < BN / 32; ++b) {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        vec8<T> pf;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float e = exp2_fast(above(s[b][8 * h2 + j], base));
          sum += e;
          pf[j] = T(e);
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db) o[db] = Elem<T>::mfma(at_tile.across(tile_v, 32 * b + 16 * h2, 32 * db), pf, o[db]);
      }
    }
  };
  for (int32_t k0 = k_begin; k0 < k_end; k0 += 2 * BN) {
    step(k0, std::integral_constant<int, 0>());
    if (k0 + BN < k_end) step(k0 + BN, std::integral_constant<int, 1>());
  }

  sum += other_half(sum);
  // Results of the waves that share the rows: of every four elements one wave adds up all.
  float* joined = reinterpret_cast<float*>(lds_tiles);        // [KW][D / 8][64][4]
  __shared__ float lds_stats[KW > 1 ? KW : 1][2][32];
  float weight[KW];
  if constexpr (KW > 1) {
    if (half == 0) {
      lds_stats[part][0][col] = sum == 0.f ? -INFINITY : base;
      lds_stats[part][1][col] = sum;
    }
    __syncthreads();                                          // and all are done with their tiles
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<floatx4*>(joined + ((part * (D / 8) + 4 * db + r4) * 64 + lane) * 4) = floatx4{o[db][4 * r4], o[db][4 * r4 + 1], o[db][4 * r4 + 2], o[db][4 * r4 + 3]};
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < KW; ++k) top = fmaxf(top, lds_stats[k][0][col]);
    base = top == -INFINITY ? 0.f : top;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      weight[k] = exp2_fast(lds_stats[k][0][col] - base);
      sum += weight[k] * lds_stats[k][1][col];
    }
    __syncthreads();
  }
  if (row >= qd.owned * p.group) return;
  const int64_t at_out = int64_t(token) * p.heads + head, at_part = int64_t(split) * p.qs.rows * p.heads + at_out;
  const float inv = sum > 0.f ? 1.f / sum : sum;        // zero keys: zeros; NaN stays
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int d = 32 * db + 8 * r4 + 4 * half;
      if ((KW > 1 && (4 * db + r4) % KW != part) || d >= p.dim) continue;
      floatx4 f = {o[db][4 * r4], o[db][4 * r4 + 1], o[db][4 * r4 + 2], o[db][4 * r4 + 3]};
      if constexpr (KW > 1) {
        f = floatx4{};
#pragma unroll
        for (int k = 0; k < KW; ++k) f += weight[k] * *reinterpret_cast<const floatx4*>(joined + ((k * (D / 8) + 4 * db + r4) * 64 + lane) * 4);
      }
      if (!live) f = floatx4{};
      if (p.splits > 1) {
        *reinterpret_cast<floatx4*>(p.part_o + at_part * p.dim + d) = f;
        continue;
      }
      vec4<T> x, y;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = T(live ? f[i] * inv : 0.f);
        y[i] = T(live ? f[i] * inv - float(x[i]) : 0.f);
      }
      *reinterpret_cast<vec4<T>*>(static_cast<T*>(p.out) + at_out * p.dim + d) = x;
      if (p.rest) *reinterpret_cast<vec4<T>*>(static_cast<T*>(p.rest) + at_out * p.dim + d) = y;
    }
  if (half || part) return;
  if (p.splits > 1) {
    p.part_ml[at_part * 2] = live && sum != 0.f ? base : -INFINITY;
    p.part_ml[at_part * 2 + 1] = live ? sum : 0.f;
  } else {
    p.lse[at_out] = live && sum != 0.f ? (base + log2_fast(sum)) * kLn2 : -INFINITY;
  }
}

template <typename T, int D, bool CAP, bool BIAS, int NW, int KW, int BN>
__global__ __launch_bounds__(64 * NW * KW, waves_per_simd(D, NW)) void attend_kernel(const AttendParams p) {
  constexpr int kRows = 32 * NW;
  uint32_t piece = p.first + piece_of(blockIdx.x, gridDim.x);
  int32_t split = 0, hk, tile;
  if constexpr (NW == 1) {          // short documents: the heads of a token lie side by side in memory
    hk = piece % p.kv_heads;
    piece /= p.kv_heads;
    split = piece % p.splits;
    tile = piece / p.splits;
  } else {                          // long ones: the tiles that share keys one after the other
    tile = piece % p.tiles;
    piece /= p.tiles;
    split = piece % p.splits;
    hk = piece / p.splits;
  }
  const Found doc = find_tile(p.qs, p.n_docs, p.docs_per_tile, p.group, kRows, tile, threadIdx.x & 63);
  const Span qd = doc.span, kd = other_side(p.ks, p.qs, doc, p.n_docs);
  const int32_t row0 = (tile - doc.first) * kRows;
  if (row0 < 0 || row0 >= qd.owned * p.group) return;
  attend_rows<T, D, CAP, BIAS, NW, KW, BN>(p, hk, split, row0, qd, kd);
}

// Large documents among those of one query on average, by four waves that share their keys.
template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, waves_per_simd(D < 64 ? 64 : D, 1)) void attend_large_kernel(const AttendParams p) {
  each_large(p, [&](int32_t q, int32_t) { return (q * p.group + 31) / 32 * p.kv_heads; },
             [&](int32_t doc, int32_t tile) {
               attend_rows<T, D, CAP, BIAS, 1, 4, 32>(p, tile % p.kv_heads, 0, tile / p.kv_heads * 32, span_of(p.qs, doc, p.n_docs), span_of(p.ks, doc, p.n_docs));
             });
}

// Joins the parts of a query: out = sum_s 2^(top_s - top) o_s / sum_s 2^(top_s - top) sum_s.  A workgroup has a row, eight groups of 32 lanes a
// part at a time, a lane four elements.  Measured: 256 rows of 128 in 30 parts: 5 us, of which a launch is most.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const AttendParams p) {
  __shared__ float weight[kMostSplits], high[4], added[4];
  __shared__ __align__(16) floatx4 sums[8][32];
  const int tid = threadIdx.x, lane = tid & 31, part = tid >> 5;
  const int64_t row = blockIdx.x, rows = int64_t(p.qs.rows) * p.heads;
  const bool in = tid < p.splits;
  const float top = in ? p.part_ml[(tid * rows + row) * 2] : -INFINITY, mine = in ? p.part_ml[(tid * rows + row) * 2 + 1] : 0.f;
  float most = top;
#pragma unroll
  for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
  if ((tid & 63) == 0) high[tid >> 6] = most;
  __syncthreads();
  most = fmaxf(fmaxf(high[0], high[1]), fmaxf(high[2], high[3]));
  const float w = exp2_fast(top - (most == -INFINITY ? 0.f : most));
  if (in) weight[tid] = w;
  float sum = in ? w * mine : 0.f;
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
  if ((tid & 63) == 0) added[tid >> 6] = sum;
  __syncthreads();
  sum = added[0] + added[1] + added[2] + added[3];
  floatx4 o = {};
  if (4 * lane < p.dim)
#pragma unroll 4
    for (int32_t s = part; s < p.splits; s += 8) o += weight[s] * *reinterpret_cast<const floatx4*>(p.part_o + (s * rows + row) * p.dim + 4 * lane);
  sums[part][lane] = o;
  __syncthreads();
  if (part || 4 * lane >= p.dim) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) o += sums[k][lane];
  const float inv = sum > 0.f ? 1.f / sum : sum;
  vec4<T> x, y;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = T(o[j] * inv);
    y[j] = T(o[j] * inv - float(x[j]));
  }
  *reinterpret_cast<vec4<T>*>(static_cast<T*>(p.out) + row * p.dim + 4 * lane) = x;
  if (p.rest) *reinterpret_cast<vec4<T>*>(static_cast<T*>(p.rest) + row * p.dim + 4 * lane) = y;
  if (lane == 0) p.lse[row] = sum != 0.f ? (most + log2_fast(sum)) * kLn2 : -INFINITY;
}

template <typename T, int D, bool CAP, bool BIAS> void launch(const AttendParams& p, const ForwardShape& f, hipStream_t s) {
  if (p.any_large) {
    attend_large_kernel<T, D, CAP, BIAS><<<uint32_t(f.tiles), 256, 0, s>>>(p);
    return;
  }
  in_launches(int64_t(p.tiles) * p.kv_heads * p.splits, 64 * f.waves * f.key_waves, [&](uint32_t first, uint32_t blocks) {
    AttendParams x = p;
    x.first = first;
    if (f.waves > 1) attend_kernel<T, D, CAP, BIAS, 4, 1, 64><<<blocks, 256, 0, s>>>(x);
    else if (f.key_waves > 1) attend_kernel<T, D, CAP, BIAS, 1, 4, 32><<<blocks, 256, 0, s>>>(x);
    else attend_kernel<T, D, CAP, BIAS, 1, 1, 32><<<blocks, 64, 0, s>>>(x);
  });
}
template <typename T, int D> void launch(const AttendParams& p, const ForwardShape& f, bool cap, hipStream_t s) {
  if (cap) p.slopes ? launch<T, D, true, true>(p, f, s) : launch<T, D, true, false>(p, f, s);
  else p.slopes ? launch<T, D, false, true>(p, f, s) : launch<T, D, false, false>(p, f, s);
}
template <typename T> void launch(const AttendParams& p, const ForwardShape& f, bool cap, hipStream_t s) {
  if (p.dim <= 32) launch<T, 32>(p, f, cap, s);
  else if (p.dim <= 64) launch<T, 64>(p, f, cap, s);
  else launch<T, 128>(p, f, cap, s);
  if (p.splits > 1) {
    join_kernel<T><<<uint32_t(p.qs.rows * p.heads), 256, 0, s>>>(p);
  }
}

}  // namespace

void launch_large(const AttendParams& p, const lgp_attention* a, hipStream_t s) {
  const ForwardShape f = {1, 4, kLargeGroups, 1};
  if (a->dtype == LGP_F16) launch<f16>(p, f, a->cap > 0.f, s);
  else launch<bf16>(p, f, a->cap > 0.f, s);
}

int check_attend(const lgp_documents* d, const lgp_attention* a) {
  if (!d || !a) return LGP_EINVAL;
  if (d->n_docs < 0 || d->q_rows < 0 || d->k_rows < 0 || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->dim < 1) return LGP_EINVAL;
  if (d->n_docs == 0 && (d->q_rows || d->k_rows)) return LGP_EINVAL;
  if (a->dtype != LGP_F16 && a->dtype != LGP_BF16) return LGP_EUNSUPPORTED;
  if (a->dim % 8 || a->dim > 128) return LGP_EUNSUPPORTED;
  if (!(a->cap >= 0.f) || !std::isfinite(a->cap) || !std::isfinite(a->scale)) return LGP_EINVAL;
  // folded rows and rows of tiles are counted in 32 bits
  const int64_t most = int64_t(1) << 31;
  if (a->heads > 65536 || d->n_docs >= most / 512 || d->q_rows >= most / a->heads || d->k_rows >= most) return LGP_EUNSUPPORTED;
  if (d->q_rows * a->heads + 256 * d->n_docs >= most || d->k_rows + 256 * d->n_docs >= most) return LGP_EUNSUPPORTED;
  if (d->n_docs && (!d->q_offsets || !d->k_offsets)) return LGP_EINVAL;
  if ((d->q_rows && !a->q) || (d->k_rows && (!a->k || !a->v))) return LGP_EINVAL;
  if (a->slopes && ((d->q_rows && !d->q_pos) || (d->k_rows && !d->k_pos))) return LGP_EINVAL;
  if (!aligned16(a->q) || !aligned16(a->k) || !aligned16(a->v)) return LGP_EINVAL;
  // rows of tiles lie less than 2^32 bytes apart (copy_tile), and so do the query heads that are folded into them; key heads are told apart in 64 bits
  for (int64_t stride : {a->q_row, a->k_row, a->v_row, int64_t(a->heads) * a->dim})
    if (stride < 0 || stride >= kMostStride) return LGP_EUNSUPPORTED;
  if (a->q_head < 0 || a->q_head >= 4 * kMostStride) return LGP_EUNSUPPORTED;
  for (int64_t stride : {a->k_head, a->v_head})
    if (stride < 0 || stride >= int64_t(1) << 40) return LGP_EUNSUPPORTED;
  if (a->q_row % 8 || a->q_head % 8 || a->k_row % 8 || a->k_head % 8 || a->v_row % 8 || a->v_head % 8) return LGP_EINVAL;
  return LGP_OK;
}

AttendParams attend_params(const lgp_documents* d, const lgp_attention* a) {
  AttendParams p = {};
  p.q = a->q; p.k = a->k; p.v = a->v;
  p.q_row = a->q_row; p.q_head = a->q_head; p.k_row = a->k_row; p.k_head = a->k_head; p.v_row = a->v_row; p.v_head = a->v_head;
  p.qs = {d->q_offsets, d->q_lens, d->q_pos, int32_t(d->q_rows)};
  p.ks = {d->k_offsets, d->k_lens, d->k_pos, int32_t(d->k_rows)};
  p.n_docs = int32_t(d->n_docs);
  p.heads = a->heads; p.kv_heads = a->kv_heads; p.group = a->heads / a->kv_heads; p.dim = a->dim;
  p.scale = a->scale;
  const float scale = std::fabs(a->scale);
  p.negate = a->scale < 0.f;
  p.z_mul = std::max(scale, 1e-30f) * kLog2e;
  p.t_mul = a->cap > 0.f ? std::min(scale / a->cap, 1e38f) : 0.f;
  p.t_inv = p.t_mul > 0.f ? 1.f / p.t_mul : 0.f;
  p.near = p.t_mul == 0.f || (p.t_mul >= 0x1p-12f && p.t_mul <= 0x1p12f) ? kNear / p.t_mul : -1.f;
  double power = 1.0;
  for (int i = 0; i < 4; ++i) p.tanh_c[i] = float(kTanh[i] * (power *= double(p.t_mul) * p.t_mul));
  p.per_token = divisor(uint32_t(p.group));
  while (16 % p.group == 0 && (1 << p.log2_fold) < p.group) ++p.log2_fold;
  p.slopes = a->slopes;
  p.splits = 1;
  return p;
}

// Where documents have up to 32 folded rows, a wave has them, or four share them where the keys are 64 and more; where they have more, four waves
// of 32 rows each share the keys, or are on their own where tiles are small and documents of a few waves leave others idle.  Few tiles over long
// documents are split over the keys until every CU has a few waves, at no less than 256 keys a part.
ForwardShape forward_shape(int device, const lgp_documents* d, const lgp_attention* a) {
  const int64_t group = a->heads / a->kv_heads, n = std::max<int64_t>(d->n_docs, 1), keys = d->k_rows / n;
  ForwardShape f;
  f.waves = one_wave(d->q_rows * group, n, a->dim) ? 1 : 4;
  f.key_waves = d->q_rows * group <= 32 * n && keys >= 64 ? 4 : 1;
  f.tiles = tiles_of(d->q_rows, group, d->n_docs, kForwardRows * f.waves);
  const int64_t waves = f.tiles * a->kv_heads * f.waves * f.key_waves, room = int64_t(compute_units(device)) * 8;
  f.splits = int(std::max<int64_t>(1, std::min({room / std::max<int64_t>(waves, 1), keys / 256 / f.key_waves, int64_t(kMostSplits)})));
  return f;
}

}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_attend(int device, const lgp_documents* docs, const lgp_attention* att, void* out, void* rest, float* lse, void* workspace,
               size_t workspace_bytes, void* stream) {
  if (int st = check_attend(docs, att)) return st;
  if (docs->q_rows && (!out || !lse || !aligned16(out) || !aligned16(rest))) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (docs->q_rows == 0) return LGP_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (single_queries(docs, att)) {
    AttendParams p = attend_params(docs, att);
    p.out = out;
    p.rest = rest;
    p.lse = lse;
    if (workspace_bytes < survey_bytes(docs)) return LGP_ECAPACITY;
    if (surveys(docs) && (!workspace || !aligned16(workspace))) return LGP_EINVAL;
    set_survey(p, docs, workspace);
    launch_single(p, att, false, s);
    if (p.any_large) launch_large(p, att, s);
    return launched();
  }
  const ForwardShape f = forward_shape(device, docs, att);
  if (f.tiles * att->kv_heads * f.splits >= int64_t(1) << 31) return LGP_EUNSUPPORTED;
  AttendParams p = attend_params(docs, att);
  p.tiles = int32_t(f.tiles);
  p.docs_per_tile = float(p.n_docs) / float(p.tiles);
  p.splits = f.splits;
  p.out = out;
  p.rest = rest;
  p.lse = lse;
  if (f.splits > 1) {
    const size_t rows = size_t(f.splits) * docs->q_rows * att->heads;
    if (workspace_bytes < rows * (att->dim + 2) * 4) return LGP_ECAPACITY;
    if (!workspace || !aligned16(workspace)) return LGP_EINVAL;
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o + rows * att->dim;
  }
  if (att->dtype == LGP_F16) launch<f16>(p, f, att->cap > 0.f, s);
  else launch<bf16>(p, f, att->cap > 0.f, s);
  return launched();
}

}  // extern "C"
