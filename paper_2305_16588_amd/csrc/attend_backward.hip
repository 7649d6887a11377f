// Attention inside documents, backward.  Scores are computed again, in two kernels: one has a wave per 32 queries and walks over the keys
// (gradients of q and of the slopes), the other a wave per 32 keys and walks over the queries (gradients of k and v).  Seven products
// instead of the five of a single kernel, and no sum in memory: nothing depends on the order in which workgroups finish.
#include "attend.hpp"

#include <algorithm>

namespace lgp {
namespace layer {
namespace {

// Gradient of q: with u = scale * q.k, z the score, P = exp(z - lse), dP = d_out . v and delta = d_out . out,
//     dS = P (dP - delta),  dU = dS (1 - tanh^2),  dq = scale * sum_j dU k_j.
// Everything is transposed, as in the forward kernel: columns are folded rows.  dU is rounded to the type of k for the last product, as k itself is; with
// fp16 it is lifted first (kLiftFirst).
// delta is taken from out and what its rounding took off, so it has the rounding of the probabilities that made out and not that of out.  The slope of a head has the gradient
//     - sum dS |distance| = - sum_rows (sum_j dS |distance| - (sum_j dS) (sum_j P |distance|) / sum_j P) / sum_j P,
// whose four sums per row go to `sums`: the second term is what the rounding of out and of lse left in dS, so the gradient depends on neither.
// Measured: 4 documents of 8192 tokens, heads 8/4 of 128, bf16, bias: 1595 to 1640 us, 1.02 PFLOP/s, matrix instructions 49 % and vector instructions
// 61 % of the cycles; 1024 documents of 276 rows, heads 8/8 of 32, cap and bias: 270 us, vector instructions 86 %.
template <typename T, int D, bool CAP, bool BIAS, int NW, int BN>
__device__ __forceinline__ void dq_rows(const AttendParams& p, int32_t hk, int32_t split, int32_t row0, const Span qd, const Span kd) {
  constexpr int kThreads = 64 * NW;
  __shared__ __align__(16) T lds_k[2][BN * D];
  __shared__ __align__(16) T lds_v[2][BN * D];
  __shared__ __align__(16) float lds_pos[2][BIAS ? BN : 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;

  int32_t k_begin, k_end;
  part_of(row0 < qd.tokens * p.group ? kd.tokens : 0, BN, split, p.splits, k_begin, k_end);
  const Rows<T> k_rows = {static_cast<const T*>(p.k) + int64_t(kd.begin) * p.k_row + int64_t(hk) * p.k_head, p.k_row, 0, 0};
  const Rows<T> v_rows = {static_cast<const T*>(p.v) + int64_t(kd.begin) * p.v_row + int64_t(hk) * p.v_head, p.v_row, 0, 0};
  int32_t next_pos = 0;        // as it comes, so that nothing waits for it yet
  auto stage = [&](int32_t k0, int to) {
    if constexpr (BIAS) next_pos = tid < BN && k0 + tid < k_end ? p.ks.pos[kd.begin + k0 + tid] : 0;
    copy_tile<T, D, BN, kThreads>(lds_k[to], k_rows, k0, p.dim, k_end - k0, tid);
    copy_tile<T, D, BN, kThreads>(lds_v[to], v_rows, k0, p.dim, k_end - k0, tid);
  };
  if (p.dim < D) {
    clear_tile<T, 2 * BN * D, kThreads>(lds_k[0], tid);
    clear_tile<T, 2 * BN * D, kThreads>(lds_v[0], tid);
    tile_ready<(NW > 1)>();
  }
  if (k_begin < k_end) stage(k_begin, 0);

  const int32_t row = row0 + 32 * wave + col;
  const bool live = row < qd.tokens * p.group;
  const int32_t of_doc = quotient(row, p.per_token), token = qd.begin + of_doc, head = hk * p.group + row - of_doc * p.group;
  const int64_t at_out = int64_t(token) * p.heads + head;
  vec8<T> qf[D / 16], df[D / 16];
  float delta = 0.f;
  {
    const T* q = static_cast<const T*>(p.q) + int64_t(token) * p.q_row + int64_t(head) * p.q_head;
    const T* g = static_cast<const T*>(p.d_out) + at_out * p.dim;
    const T* o = static_cast<const T*>(p.out) + at_out * p.dim;
    const T* o2 = static_cast<const T*>(p.rest) + at_out * p.dim;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const int d = 16 * kk + 8 * half;
      const bool there = live && d < p.dim;
      qf[kk] = load8(q + d, there, p.negate);
      df[kk] = load8(g + d, there, false);
      const vec8<T> of = load8(o + d, there, false), o2f = load8(o2 + d, there && p.rest, false);
#pragma unroll
      for (int i = 0; i < 8; ++i) delta += float(df[kk][i]) * (float(of[i]) + float(o2f[i]));
    }
  }
  delta += other_half(delta);
  float lse = INFINITY;           // no probability where there is no token or no key
  float slope = 0.f, at = 0.f;
  if (live) {
    lse = p.lse_in[at_out] * kLog2e;
    if (lse == -INFINITY) lse = INFINITY;
    if constexpr (BIAS) {
      slope = p.slopes[head] * kLog2e;
      at = float(p.qs.pos[token]);
    }
    if (split == 0 && half == 0) p.delta[at_out] = delta;
  }

  floatx16 dq[D / 32] = {};
  float sum_p = 0.f, sum_s = 0.f, sum_pf = 0.f, sum_sf = 0.f;
  constexpr bool kLifts = std::is_same<T, f16>::value;
  float lift = kLifts ? kLiftFirst : 1.f;        // of the probabilities, so of dU and of all four sums
  if constexpr (kLifts) lse -= kLiftFirstLog2;
  Places<T, D> at_tile(lane);
  const bool idle = row0 + 32 * wave >= qd.tokens * p.group;         // a wave of rows without tokens only copies
  auto step = [&](int32_t k0, int now, auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    if constexpr (BIAS) {
      if (tid < BN) lds_pos[now][tid] = float(next_pos);
    }
    tile_ready<(NW > 1)>();
    if (k0 + BN < k_end) stage(k0 + BN, now ^ 1);
    if (idle) return;
    at_tile.again();
    const T *tile_k = lds_k[now], *tile_v = lds_v[now];
#pragma unroll
    for (int b = 0; b < BN / 32; ++b) {
      floatx16 s = {}, g = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        s = Elem<T>::mfma(at_tile.along(tile_k, 32 * b, kk), qf[kk], s);
        g = Elem<T>::mfma(at_tile.along(tile_v, 32 * b, kk), df[kk], g);
      }
      const int32_t there = k0 + BN <= k_end ? BN : k_end - k0 - 32 * b - 4 * half;      // places of this block's half that are keys
      cap<CAP>(p, s);
      floatx4 of_tile = {};             // sums of sums: a lane's 16 scores first, for the digits of long ones
      vec8<T> uf[2];
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        floatx4 kpos = {};
        if constexpr (BIAS) kpos = *reinterpret_cast<const floatx4*>(&lds_pos[now][32 * b + 8 * r4 + 4 * half]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * r4 + i;
          float far = 0.f;
          if constexpr (BIAS) far = fabsf(at - kpos[i]);
          const float z = fmaf(s[r], p.z_mul, BIAS ? fmaf(-slope, far, -lse) : -lse);
          const float e = WHOLE || 8 * r4 + i < there ? exp2_fast(z) : 0.f, pd = e * g[r];
          float u = fmaf(-e, delta, pd);
          if constexpr (BIAS) {
            of_tile[0] += e;
            of_tile[1] += u;
            of_tile[2] = fmaf(e, far, of_tile[2]);
            of_tile[3] = fmaf(u, far, of_tile[3]);
          }
          u = through_cap<CAP>(p, u, s[r]);
          if constexpr (kLifts) s[r] = u;
          else uf[r / 8][r % 8] = T(u);
        }
      }
      if constexpr (BIAS) {
        sum_p += of_tile[0];
        sum_s += of_tile[1];
        sum_pf += of_tile[2];
        sum_sf += of_tile[3];
      }
      if constexpr (kLifts) {
        float most = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(s[r]));
        if (__any(most > kLiftedMost)) {
          most = fmaxf(most, other_half(most));
          const int by_log2 = most > kLiftedMost ? lower_log2(most) : 0;
          const float by = __builtin_amdgcn_ldexpf(1.f, by_log2);
          lift *= by;
          lse -= float(by_log2);
          sum_p *= by, sum_s *= by, sum_pf *= by, sum_sf *= by;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= by;
#pragma unroll
          for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) dq[db][r] *= by;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) uf[r / 8][r % 8] = T(s[r]);
      }
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) dq[db] = Elem<T>::mfma(at_tile.across(tile_k, 32 * b + 16 * h2, 32 * db), uf[h2], dq[db]);
    }
  };
  int32_t k0 = k_begin;
  for (; k0 + 2 * BN <= k_end; k0 += 2 * BN) {
    step(k0, 0, std::true_type());
    step(k0 + BN, 1, std::true_type());
  }
  for (int now = 0; k0 < k_end; k0 += BN, ++now) step(k0, now, std::false_type());

  if (row >= qd.owned * p.group) return;
  if constexpr (BIAS) {
    sum_p += other_half(sum_p);
    sum_s += other_half(sum_s);
    sum_pf += other_half(sum_pf);
    sum_sf += other_half(sum_sf);
    if (p.sums && half == 0) p.sums[int64_t(split) * p.qs.rows * p.heads + at_out] = live ? floatx4{sum_p, sum_s, sum_pf, sum_sf} * (1.f / lift) : floatx4{};
  }
  float* part = p.splits > 1 ? p.part_o + (int64_t(split) * p.qs.rows * p.heads + at_out) * p.dim : nullptr;
  T* out = static_cast<T*>(p.dq) + at_out * p.dim;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int d = 32 * db + 8 * r4 + 4 * half;
      if (d < p.dim) {
        floatx4 x = {};
        if (live) x = floatx4{dq[db][4 * r4], dq[db][4 * r4 + 1], dq[db][4 * r4 + 2], dq[db][4 * r4 + 3]} * (p.scale / lift);
        if (part) *reinterpret_cast<floatx4*>(part + d) = x;
        else *reinterpret_cast<vec4<T>*>(out + d) = vec4<T>{T(x[0]), T(x[1]), T(x[2]), T(x[3])};
      }
    }
}

template <typename T, int D, bool CAP, bool BIAS, int NW, int BN>
__global__ __launch_bounds__(64 * NW, waves_per_simd(D, NW)) void attend_dq_kernel(const AttendParams p) {
  constexpr int kRows = 32 * NW;
  uint32_t piece = p.first + piece_of(blockIdx.x, gridDim.x);
  int32_t split = 0, hk, tile;
  if constexpr (NW == 1) {
    hk = piece % p.kv_heads;
    piece /= p.kv_heads;
    split = piece % p.splits;
    tile = piece / p.splits;
  } else {
    tile = piece % p.tiles;
    piece /= p.tiles;
    split = piece % p.splits;
    hk = piece / p.splits;
  }
  const Found doc = find_tile(p.qs, p.n_docs, p.docs_per_tile, p.group, kRows, tile, threadIdx.x & 63);
  const Span qd = doc.span, kd = other_side(p.ks, p.qs, doc, p.n_docs);
  const int32_t row0 = (tile - doc.first) * kRows;
  if (row0 < 0 || row0 >= qd.owned * p.group) return;
  dq_rows<T, D, CAP, BIAS, NW, BN>(p, hk, split, row0, qd, kd);
}

// Adds the parts of dq, like join_kernel, and in its time.
template <typename T>
__global__ __launch_bounds__(256) void add_kernel(const AttendParams p) {
  __shared__ __align__(16) floatx4 sums[8][32];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int64_t row = blockIdx.x, rows = int64_t(p.qs.rows) * p.heads;
  floatx4 x = {};
  if (4 * lane < p.dim)
#pragma unroll 4
    for (int32_t s = part; s < p.splits; s += 8) x += *reinterpret_cast<const floatx4*>(p.part_o + (s * rows + row) * p.dim + 4 * lane);
  sums[part][lane] = x;
  __syncthreads();
  if (part || 4 * lane >= p.dim) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) x += sums[k][lane];
  *reinterpret_cast<vec4<T>*>(static_cast<T*>(p.dq) + row * p.dim + 4 * lane) = vec4<T>{T(x[0]), T(x[1]), T(x[2]), T(x[3])};
}

// Gradient of the slopes from the sums of all rows, in two steps of a fixed order: kSlopeThreads threads take rows a multiple of the number of
// heads apart, so that each adds up for one head, then a workgroup adds up what is there of a head.  Rows may cancel down to a small part of
// what one of them has, so they are added in 64 bits.  Measured: 282 624 rows of 8 heads, 9 and 5 us.
constexpr int64_t kSlopeThreads = 131072;
__global__ __launch_bounds__(256) void slopes_kernel(const AttendParams p, double* partial) {
  const int64_t rows = int64_t(p.qs.rows) * p.heads, each = kSlopeThreads / p.heads * p.heads, at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (at >= each) return;
  double x = 0.;
  for (int64_t r = at; r < rows; r += each) {
    floatx4 m = {};
    for (int32_t s = 0; s < p.splits; ++s) m += p.sums[s * rows + r];
    const float inv = m[0] != 0.f ? 1.f / m[0] : 0.f;
    x -= double((m[3] - m[1] * m[2] * inv) * inv);
  }
  partial[at % p.heads * (each / p.heads) + at / p.heads] = x;       // of a head side by side
}
constexpr int kEndThreads = 1024;
__global__ __launch_bounds__(kEndThreads) void slopes_end_kernel(const double* partial, int32_t heads, float* out) {
  __shared__ double lds[kEndThreads / 64];
  const int32_t each = int32_t(kSlopeThreads) / heads;
  double x = 0.;
#pragma unroll 8
  for (int32_t i = threadIdx.x; i < each; i += kEndThreads) x += partial[int64_t(blockIdx.x) * each + i];
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x) return;
#pragma unroll
  for (int k = 1; k < kEndThreads / 64; ++k) x += lds[k];
  out[blockIdx.x] = float(x);
}

// Gradients of k and v: a wave has 32 keys as columns and walks over the folded rows of their document, BQ at a time, in LDS.
//     dv_j = sum_i P_ij d_out_i,   dk_j = scale * sum_i dU_ij q_i.
// Measured, at the sizes of attend_dq_kernel: 2115 to 2180 us, 1.02 PFLOP/s, matrix instructions 45 % of the cycles of two waves per SIMD that wait for each
// other's tiles; 304 us, vector instructions 66 %.
// DELTA: delta is not there yet; eight threads take that of a row from d_out, out and rest.
template <typename T, int D, bool CAP, bool BIAS, int NW, int BQ, bool DELTA = false>
__device__ __forceinline__ void dkv_rows(const AttendParams& p, int32_t hk, int32_t key0, const Span kd, const Span qd) {
  constexpr int kThreads = 64 * NW, kKeys = 32 * NW;
  __shared__ __align__(16) T lds_q[2][BQ * D];
  __shared__ __align__(16) T lds_g[2][BQ * D];
  __shared__ __align__(16) float lds_row[2][4][BQ];       // lse, delta, slope, position
  // With heads of 128 the wave's keys, values and both results would be all registers there are: values are read from LDS.
  constexpr bool kHeld = D < 128 || NW == 1;
  __shared__ __align__(16) T lds_v[kHeld ? 8 : kKeys * D];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;

  // Up to 16 heads of a token, if they divide 16, are folded; otherwise the heads that share this one are gone through one after the other.
  const int32_t rows = key0 < kd.tokens ? qd.tokens << p.log2_fold : 0;
  static_assert(BQ <= kThreads && (!DELTA || 8 * BQ == kThreads), "a thread has a row, or eight");
  constexpr int kChunks = DELTA ? (D + 63) / 64 : 1;
  vec8<T> of_g[kChunks], of_o[kChunks], of_rest[kChunks];
  float next[3];               // as they come, so that nothing waits for them yet
  int32_t next_pos;
  auto stage = [&](int32_t h0, int32_t r0, int to) {
    next[0] = INFINITY, next[1] = next[2] = 0.f, next_pos = 0;
    if (tid < BQ && r0 + tid < rows) {
      const int32_t head = h0 + ((r0 + tid) & ((1 << p.log2_fold) - 1));
      const int64_t token = qd.begin + ((r0 + tid) >> p.log2_fold);
      next[0] = p.lse_in[token * p.heads + head];
      if constexpr (!DELTA) next[1] = p.delta[token * p.heads + head];
      if constexpr (BIAS) {
        next[2] = p.slopes[head];
        next_pos = p.qs.pos[token];
      }
    }
    if constexpr (DELTA) {
      const int32_t r = r0 + tid / 8;
      const int64_t d0 = ((qd.begin + int64_t(r >> p.log2_fold)) * p.heads + h0 + (r & ((1 << p.log2_fold) - 1))) * p.dim;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        const int d = 8 * (tid % 8 + 8 * j);
        const bool there = r < rows && d < p.dim;
        of_g[j] = load8(static_cast<const T*>(p.d_out) + d0 + d, there, false);
        of_o[j] = load8(static_cast<const T*>(p.out) + d0 + d, there, false);
        of_rest[j] = load8(static_cast<const T*>(p.rest) + d0 + d, there && p.rest, false);
      }
    }
    const Rows<T> q_rows = {static_cast<const T*>(p.q) + int64_t(qd.begin) * p.q_row + int64_t(h0) * p.q_head, p.q_row, p.q_head, p.log2_fold};
    const Rows<T> g_rows = {static_cast<const T*>(p.d_out) + (int64_t(qd.begin) * p.heads + h0) * p.dim, int64_t(p.heads) * p.dim, p.dim, p.log2_fold};
    copy_tile<T, D, BQ, kThreads>(lds_q[to], q_rows, r0, p.dim, rows - r0, tid);
    copy_tile<T, D, BQ, kThreads>(lds_g[to], g_rows, r0, p.dim, rows - r0, tid);
  };
  auto put_rows = [&](int to) {
    if (tid < BQ) {
      lds_row[to][0][tid] = (next[0] == -INFINITY ? INFINITY : next[0]) * kLog2e - kLiftLog2<T>;       // no probability where there is no key
      if constexpr (!DELTA) lds_row[to][1][tid] = next[1];
      lds_row[to][2][tid] = next[2] * kLog2e;
      lds_row[to][3][tid] = float(next_pos);
    }
    if constexpr (DELTA) {
      float delta = 0.f;
#pragma unroll
      for (int j = 0; j < kChunks; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) delta += float(of_g[j][i]) * (float(of_o[j][i]) + float(of_rest[j][i]));
      delta = sum_of_lanes<8>(delta);
      if (tid % 8 == 0) lds_row[to][1][tid / 8] = delta;
    }
  };
  if (p.dim < D) {
    clear_tile<T, 2 * BQ * D, kThreads>(lds_q[0], tid);
    clear_tile<T, 2 * BQ * D, kThreads>(lds_g[0], tid);
    tile_ready<(NW > 1)>();
  }
  if (rows > 0) stage(hk * p.group, 0, 0);

  const int32_t key = key0 + 32 * wave + col;
  const bool live = key < kd.tokens;
  const int64_t key_row = int64_t(kd.begin) + key;
  vec8<T> kf[D / 16], vf[kHeld ? D / 16 : 1];
  {
    const T* k = static_cast<const T*>(p.k) + key_row * p.k_row + int64_t(hk) * p.k_head;
    const T* v = static_cast<const T*>(p.v) + key_row * p.v_row + int64_t(hk) * p.v_head;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const int d = 16 * kk + 8 * half;
      kf[kk] = load8(k + d, live && d < p.dim, p.negate);
      const vec8<T> x = load8(v + d, live && d < p.dim, false);
      if constexpr (kHeld) vf[kk] = x;
      else *reinterpret_cast<vec8<T>*>(lds_v + chunk_at<D>(32 * wave + col, 2 * kk + half)) = x;
    }
  }
  float at = 0.f;
  if constexpr (BIAS) at = live ? float(p.ks.pos[key_row]) : 0.f;

  floatx16 dk[D / 32] = {}, dv[D / 32] = {};
  constexpr bool kLifts = std::is_same<T, f16>::value;
  float lift = (kLifts ? kLiftFirst : 1.f) / kLift<T>;        // of dU, less that of the probabilities
  Places<T, D> at_tile(lane);
  const bool idle = key0 + 32 * wave >= kd.tokens;                   // a wave of keys without tokens only copies
  int32_t h0 = hk * p.group, r0 = 0;
  auto step = [&](auto stage_now) {
    constexpr int now = decltype(stage_now)::value;
    put_rows(now);
    tile_ready<(NW > 1)>();
    r0 += BQ;
    if (r0 >= rows) r0 = 0, h0 += 1 << p.log2_fold;
    if (h0 < (hk + 1) * p.group) stage(h0, r0, now ^ 1);
    if (idle) return;
    at_tile.again();
    const T *tile_q = lds_q[now], *tile_g = lds_g[now];
#pragma unroll
    for (int b = 0; b < BQ / 32; ++b) {
      floatx16 s = {}, g = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        s = Elem<T>::mfma(at_tile.along(tile_q, 32 * b, kk), kf[kk], s);
        g = Elem<T>::mfma(at_tile.along(tile_g, 32 * b, kk),
                             kHeld ? vf[kHeld ? kk : 0] : at_tile.along(lds_v + 32 * wave * D, 0, kk), g);
      }
      cap<CAP>(p, s);
      vec8<T> pf[2], uf[2];
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int r_at = 32 * b + 8 * r4 + 4 * half;
        const floatx4 lse = *reinterpret_cast<const floatx4*>(&lds_row[now][0][r_at]), delta = *reinterpret_cast<const floatx4*>(&lds_row[now][1][r_at]);
        floatx4 slope = {}, pos = {};
        if constexpr (BIAS) {
          slope = *reinterpret_cast<const floatx4*>(&lds_row[now][2][r_at]);
          pos = *reinterpret_cast<const floatx4*>(&lds_row[now][3][r_at]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * r4 + i;
          const float e = exp2_fast(fmaf(s[r], p.z_mul, BIAS ? fmaf(-slope[i], fabsf(at - pos[i]), -lse[i]) : -lse[i]));             // times kLift
          float u = e * ((g[r] - delta[i]) * lift);
          u = through_cap<CAP>(p, u, s[r]);
          pf[r / 8][r % 8] = T(e);
          if constexpr (kLifts) s[r] = u;
          else uf[r / 8][r % 8] = T(u);
        }
      }
      if constexpr (kLifts) {
        float most = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(s[r]));
        if (__any(most > kLiftedMost)) {
          most = fmaxf(most, other_half(most));
          const float by = __builtin_amdgcn_ldexpf(1.f, most > kLiftedMost ? lower_log2(most) : 0);
          lift *= by;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= by;
#pragma unroll
          for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) dk[db][r] *= by;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) uf[r / 8][r % 8] = T(s[r]);
      }
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          dv[db] = Elem<T>::mfma(at_tile.across(tile_g, 32 * b + 16 * h2, 32 * db), pf[h2], dv[db]);
          dk[db] = Elem<T>::mfma(at_tile.across(tile_q, 32 * b + 16 * h2, 32 * db), uf[h2], dk[db]);
        }
    }
  };
  while (rows > 0 && h0 < (hk + 1) * p.group) {
    step(std::integral_constant<int, 0>());
    if (h0 < (hk + 1) * p.group) step(std::integral_constant<int, 1>());
  }

  if (key >= kd.owned) return;
  T* dk_out = static_cast<T*>(p.dk) + (key_row * p.kv_heads + hk) * p.dim;
  T* dv_out = static_cast<T*>(p.dv) + (key_row * p.kv_heads + hk) * p.dim;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int d = 32 * db + 8 * r4 + 4 * half;
      if (d < p.dim) {
        vec4<T> x, y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = T(live ? dk[db][4 * r4 + i] * (p.scale / (lift * kLift<T>)) : 0.f);
          y[i] = T(live ? dv[db][4 * r4 + i] * (1.f / kLift<T>) : 0.f);
        }
        *reinterpret_cast<vec4<T>*>(dk_out + d) = x;
        *reinterpret_cast<vec4<T>*>(dv_out + d) = y;
      }
    }
}

template <typename T, int D, bool CAP, bool BIAS, int NW, int BQ>
__global__ __launch_bounds__(64 * NW, waves_per_simd(D, NW)) void attend_dkv_kernel(const AttendParams p) {
  constexpr int kKeys = 32 * NW;
  uint32_t piece = p.first + piece_of(blockIdx.x, gridDim.x);
  int32_t hk, tile;
  if constexpr (NW == 1) {
    hk = piece % p.kv_heads;
    tile = piece / p.kv_heads;
  } else {
    tile = piece % p.tiles;
    hk = piece / p.tiles;
  }
  const Found doc = find_tile(p.ks, p.n_docs, p.docs_per_tile, 1, kKeys, tile, threadIdx.x & 63);
  const Span kd = doc.span, qd = other_side(p.qs, p.ks, doc, p.n_docs);
  const int32_t key0 = (tile - doc.first) * kKeys;
  if (key0 < 0 || key0 >= kd.owned) return;
  dkv_rows<T, D, CAP, BIAS, NW, BQ>(p, hk, key0, kd, qd);
}

// Large documents among those of one query on average.  Tiles of queries and of keys are taken side by side, so the latter take delta themselves.
template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void attend_backward_large_kernel(const AttendParams p) {
  each_large(p, [&](int32_t q, int32_t k) { return ((q * p.group + 127) / 128 + (k + 127) / 128) * p.kv_heads; },
             [&](int32_t doc, int32_t tile) {
               const Span qd = span_of(p.qs, doc, p.n_docs), kd = span_of(p.ks, doc, p.n_docs);
               const int32_t hk = tile % p.kv_heads, at = tile / p.kv_heads, of_q = (qd.owned * p.group + 127) / 128;
               if (at < of_q) dq_rows<T, D, CAP, BIAS, 4, 32>(p, hk, 0, at * 128, qd, kd);
               else dkv_rows<T, D, CAP, BIAS, 4, 32, true>(p, hk, (at - of_q) * 128, kd, qd);
             });
}

struct BackwardShape {
  ForwardShape q;             // of the kernel by queries
  int key_waves;              // of the kernel by keys
  int64_t key_tiles;
  size_t delta, sums, parts, partial, survey, bytes;      // offsets into the workspace, in floats; all of it, in bytes
};
BackwardShape backward_shape(int device, const lgp_documents* d, const lgp_attention* a) {
  BackwardShape b;
  b.q = forward_shape(device, d, a);
  b.q.splits = std::min(b.q.splits * b.q.key_waves, kMostSplits);        // this kernel's waves take parts of the keys as workgroups of their own
  if (b.q.key_waves > 1) b.q.splits = int(std::max<int64_t>(1, std::min<int64_t>(b.q.splits, d->k_rows / std::max<int64_t>(d->n_docs, 1) / 256)));
  if (single_queries(d, a)) b.q.splits = 1;
  b.key_waves = one_wave(d->k_rows, std::max<int64_t>(d->n_docs, 1), a->dim) ? 1 : 4;
  b.key_tiles = tiles_of(d->k_rows, 1, d->n_docs, 32 * b.key_waves);
  const size_t rows = size_t(d->q_rows) * a->heads;
  auto up = [](size_t x) { return (x + 3) / 4 * 4; };
  b.delta = 0;
  b.sums = up(rows);
  b.partial = b.sums + (a->slopes ? rows * 4 * b.q.splits : 0);
  b.parts = b.partial + (a->slopes ? 2 * size_t(kSlopeThreads) : 0);
  b.survey = b.parts + (b.q.splits > 1 ? rows * a->dim * b.q.splits : 0);
  b.bytes = b.survey * sizeof(float) + (single_queries(d, a) ? survey_bytes(d) : 0);
  return b;
}

template <typename T, int D, bool CAP, bool BIAS> void launch(const AttendParams& p, const BackwardShape& b, hipStream_t s) {
  if (p.any_large) {
    attend_backward_large_kernel<T, D, CAP, BIAS><<<kLargeGroups, 256, 0, s>>>(p);
    return;
  }
  AttendParams x = p;
  x.tiles = int32_t(b.q.tiles);
  x.docs_per_tile = float(p.n_docs) / float(std::max<int64_t>(b.q.tiles, 1));
  if (p.qs.rows) in_launches(b.q.tiles * p.kv_heads * p.splits, 64 * b.q.waves, [&](uint32_t first, uint32_t blocks) {
    x.first = first;
    if (b.q.waves == 1) attend_dq_kernel<T, D, CAP, BIAS, 1, 32><<<blocks, 64, 0, s>>>(x);
    else attend_dq_kernel<T, D, CAP, BIAS, 4, 32><<<blocks, 256, 0, s>>>(x);
  });
  x.tiles = int32_t(b.key_tiles);
  x.docs_per_tile = float(p.n_docs) / float(std::max<int64_t>(b.key_tiles, 1));
  if (p.ks.rows) in_launches(b.key_tiles * p.kv_heads, 64 * b.key_waves, [&](uint32_t first, uint32_t blocks) {
    x.first = first;
    if (b.key_waves == 1) attend_dkv_kernel<T, D, CAP, BIAS, 1, 32><<<blocks, 64, 0, s>>>(x);
    else attend_dkv_kernel<T, D, CAP, BIAS, 4, 32><<<blocks, 256, 0, s>>>(x);
  });
}
template <typename T, int D> void launch(const AttendParams& p, const BackwardShape& b, bool cap, hipStream_t s) {
  if (cap) p.slopes ? launch<T, D, true, true>(p, b, s) : launch<T, D, true, false>(p, b, s);
  else p.slopes ? launch<T, D, false, true>(p, b, s) : launch<T, D, false, false>(p, b, s);
}
template <typename T> void launch(const AttendParams& p, const BackwardShape& b, bool cap, hipStream_t s) {
  if (p.dim <= 32) launch<T, 32>(p, b, cap, s);
  else if (p.dim <= 64) launch<T, 64>(p, b, cap, s);
  else launch<T, 128>(p, b, cap, s);
  if (p.splits > 1 && p.qs.rows) {
    add_kernel<T><<<uint32_t(p.qs.rows * p.heads), 256, 0, s>>>(p);
  }
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_attend_workspace(int device, const lgp_documents* docs, const lgp_attention* att, int backward, size_t* bytes) {
  if (!bytes) return LGP_EINVAL;
  *bytes = 0;
  if (int st = check_attend(docs, att)) return st;
  if (backward) {
    *bytes = backward_shape(device, docs, att).bytes;
  } else {
    const ForwardShape f = forward_shape(device, docs, att);
    if (single_queries(docs, att)) *bytes = survey_bytes(docs);
    else if (f.splits > 1) *bytes = size_t(f.splits) * docs->q_rows * att->heads * (att->dim + 2) * sizeof(float);
  }
  return LGP_OK;
}

int lgp_attend_backward(int device, const lgp_documents* docs, const lgp_attention* att, const void* d_out, const void* out, const void* rest,
                        const float* lse, void* dq, void* dk, void* dv, float* d_slopes, void* workspace, size_t workspace_bytes, void* stream) {
  if (int st = check_attend(docs, att)) return st;
  if (docs->q_rows && (!d_out || !out || !lse || !dq)) return LGP_EINVAL;
  if (docs->k_rows && (!dk || !dv)) return LGP_EINVAL;
  if (d_slopes && !att->slopes) return LGP_EINVAL;
  if (!aligned16(d_out) || !aligned16(out) || !aligned16(rest) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv)) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  const BackwardShape b = backward_shape(device, docs, att);
  const int64_t most = int64_t(1) << 31;
  if (b.q.tiles * att->kv_heads * b.q.splits >= most || b.key_tiles * att->kv_heads >= most) return LGP_EUNSUPPORTED;
  if (workspace_bytes < b.bytes) return LGP_ECAPACITY;
  if (b.bytes && (!workspace || !aligned16(workspace))) return LGP_EINVAL;
  AttendParams p = attend_params(docs, att);
  float* w = static_cast<float*>(workspace);
  p.splits = b.q.splits;
  p.out = const_cast<void*>(out);
  p.rest = const_cast<void*>(rest);
  p.d_out = d_out;
  p.lse_in = lse;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  p.delta = w + b.delta;
  p.sums = d_slopes ? reinterpret_cast<floatx4*>(w + b.sums) : nullptr;
  p.part_o = w + b.parts;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool single = single_queries(docs, att);
  if (single) {
    set_survey(p, docs, w + b.survey);
    launch_single(p, att, true, s);
  }
  if (!single || p.any_large) att->dtype == LGP_F16 ? launch<f16>(p, b, att->cap > 0.f, s) : launch<bf16>(p, b, att->cap > 0.f, s);
  if (d_slopes) {
    double* partial = reinterpret_cast<double*>(w + b.partial);      // after the sums, so aligned to 16 bytes like them
    slopes_kernel<<<kSlopeThreads / 256, 256, 0, s>>>(p, partial);
    slopes_end_kernel<<<att->heads, kEndThreads, 0, s>>>(partial, att->heads, d_slopes);
  }
  return launched();
}

}  // extern "C"
