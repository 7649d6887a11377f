// Attention inside documents of one query and few keys each: a frontier vertex over its samples.  There the matrix instructions would have
// one row in 32 to work on and a wave per head little to read; here a wave takes all heads of a document, reads every key and value row once
// and end to end, and computes in fp32 lanes.  Both passes are bound by those bytes: the backward pass has one query per key, so the gradients of
// its row of k and v are ready as it is read and everything is read once and written once.  Measured: 122 880 documents of up to 10 keys, 8 heads
// of 32, fp16: 186 us forward, 399 backward, where the bytes take 577 together at the rate of a copy.
#include "attend.hpp"

#include <algorithm>

namespace lgp {
namespace layer {
namespace {

// L lanes have a head, eight elements each.  A wave has the heads of a chunk side by side, and as many keys at once as there are lanes left.
template <int L> struct Lanes {
  int c, head, key, keys_at_once;     // eight elements, head within the chunk, first key
  bool in;                            // a lane of a head there is
  int32_t doc, hk;
  __device__ __forceinline__ Lanes(const AttendParams& p, int32_t heads_at_once) {
    const int lane = threadIdx.x & 63, slot = lane / L;
    const int64_t unit = (int64_t(p.first) + piece_of(blockIdx.x - p.splits, p.tiles)) * 4 + (threadIdx.x >> 6);
    const int32_t chunks = (p.kv_heads + heads_at_once - 1) / heads_at_once;
    doc = __builtin_amdgcn_readfirstlane(int32_t(unit / chunks));
    c = lane % L;
    head = slot % heads_at_once;
    key = slot / heads_at_once;
    keys_at_once = (64 / L) / heads_at_once;
    hk = int32_t(unit - int64_t(doc) * chunks) * heads_at_once + head;
    in = key < keys_at_once && hk < p.kv_heads && 8 * c < p.dim;
  }
  // The lane with the same elements of the same head that has key k of those at once.
  __device__ __forceinline__ int twin(int k, int32_t heads_at_once) const { return (k * heads_at_once + head) * L + c; }
};

template <typename T> __device__ __forceinline__ float dot8(vec8<T> a, const float* b) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += float(a[i]) * b[i];
  return s;
}
template <typename T> __device__ __forceinline__ void widen(vec8<T> a, float* x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = float(a[i]);
}

constexpr int kSteps = 4;       // keys that a lane has in flight

// The first workgroups of a launch.
__device__ __forceinline__ void survey(const AttendParams& p) {
  const int32_t at = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at * kSurvey < p.n_docs) list_large(p, at, p.large + int64_t(at) * kSurvey, p.n_large + at);
}

template <typename T, int L, int G, bool CAP, bool BIAS>
__global__ __launch_bounds__(256) void single_kernel(const AttendParams p, int32_t heads_at_once) {
  if (blockIdx.x < uint32_t(p.splits)) return survey(p);
  const Lanes<L> a(p, heads_at_once);
  if (a.doc >= p.n_docs) return;
  const Span qd = span_of(p.qs, a.doc, p.n_docs), kd = span_of(p.ks, a.doc, p.n_docs);
  if (p.any_large && is_large(qd.owned, kd.owned)) return;
  const T* kp = static_cast<const T*>(p.k) + int64_t(a.hk) * p.k_head + 8 * a.c;
  const T* vp = static_cast<const T*>(p.v) + int64_t(a.hk) * p.v_head + 8 * a.c;
  for (int32_t row = 0; row < qd.owned; ++row) {
    const int64_t token = int64_t(qd.begin) + row;
    const bool live = row < qd.tokens;
    float q[G][8], acc[G][8] = {}, top[G], sum[G] = {}, slope[G] = {}, at = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      widen<T>(load8(static_cast<const T*>(p.q) + token * p.q_row + int64_t(a.hk * G + g) * p.q_head + 8 * a.c, a.in && live, p.negate), q[g]);
      top[g] = -INFINITY;
      if constexpr (BIAS) slope[g] = a.in ? p.slopes[a.hk * G + g] * kLog2e : 0.f;
    }
    if constexpr (BIAS) at = float(p.qs.pos[token]);
    const int32_t keys = live ? kd.tokens : 0;
    for (int32_t k0 = 0; k0 < keys; k0 += kSteps * a.keys_at_once) {
      vec8<T> kf[kSteps], vf[kSteps];
      float z[kSteps][G], far[kSteps] = {};
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int32_t key = k0 + i * a.keys_at_once + a.key;
        const bool there = a.in && key < keys;
        const int64_t key_row = int64_t(kd.begin) + key;
        kf[i] = load8(kp + key_row * p.k_row, there, false);
        vf[i] = load8(vp + key_row * p.v_row, there, false);
        if constexpr (BIAS) far[i] = there ? float(p.ks.pos[key_row]) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          z[i][g] = fmaf(capped<CAP>(p, sum_of_lanes<L>(dot8<T>(kf[i], q[g]))), p.z_mul, BIAS ? -slope[g] * fabsf(at - far[i]) : 0.f);
          if (k0 + i * a.keys_at_once + a.key >= keys) z[i][g] = -INFINITY;
        }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float most = top[g];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) most = fmaxf(most, z[i][g]);
        const float base = most == -INFINITY ? 0.f : most, shrink = exp2_fast(top[g] - base);
        top[g] = most;
        sum[g] *= shrink;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[g][j] *= shrink;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const float e = exp2_fast(z[i][g] - base);
          sum[g] += e;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[g][j] += e * float(vf[i][j]);
        }
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float most = top[g];
      for (int k = 0; k < a.keys_at_once; ++k) most = fmaxf(most, __shfl(top[g], a.twin(k, heads_at_once), 64));
      const float base = most == -INFINITY ? 0.f : most, shrink = exp2_fast(top[g] - base);
      sum[g] *= shrink;
      float total = 0.f, o[8] = {};
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[g][j] *= shrink;
      for (int k = 0; k < a.keys_at_once; ++k) {
        const int from = a.twin(k, heads_at_once);
        total += __shfl(sum[g], from, 64);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += __shfl(acc[g][j], from, 64);
      }
      if (!a.in || a.key != 0) continue;
      const float inv = total > 0.f ? 1.f / total : total;
      const int64_t at_out = token * p.heads + a.hk * G + g;
      vec8<T> x, y;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = T(o[j] * inv);
        y[j] = T(o[j] * inv - float(x[j]));
      }
      *reinterpret_cast<vec8<T>*>(static_cast<T*>(p.out) + at_out * p.dim + 8 * a.c) = x;
      if (p.rest) *reinterpret_cast<vec8<T>*>(static_cast<T*>(p.rest) + at_out * p.dim + 8 * a.c) = y;
      if (a.c == 0) p.lse[at_out] = total != 0.f ? (most + log2_fast(total)) * kLn2 : -INFINITY;
    }
  }
}

// One query row as the backward pass needs it.
template <typename T, int L, int G, bool BIAS> struct Query {
  float q[G][8], g[G][8], lse[G], delta[G], slope[G], at;
  __device__ __forceinline__ void load(const AttendParams& p, const Lanes<L>& a, int64_t token) {
    at = 0.f;
    if constexpr (BIAS) at = float(p.qs.pos[token]);
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const int64_t at_out = token * p.heads + a.hk * G + h;
      const int64_t d = at_out * p.dim + 8 * a.c;
      widen<T>(load8(static_cast<const T*>(p.q) + token * p.q_row + int64_t(a.hk * G + h) * p.q_head + 8 * a.c, a.in, p.negate), q[h]);
      widen<T>(load8(static_cast<const T*>(p.d_out) + d, a.in, false), g[h]);
      const vec8<T> o = load8(static_cast<const T*>(p.out) + d, a.in, false), o2 = load8(static_cast<const T*>(p.rest) + d, a.in && p.rest, false);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += g[h][i] * (float(o[i]) + float(o2[i]));
      delta[h] = sum_of_lanes<L>(s);
      lse[h] = a.in ? p.lse_in[at_out] * kLog2e : INFINITY;
      if (lse[h] == -INFINITY) lse[h] = INFINITY;
      slope[h] = 0.f;
      if constexpr (BIAS) slope[h] = a.in ? p.slopes[a.hk * G + h] * kLog2e : 0.f;
    }
  }
};

template <typename T, int L, int G, bool CAP, bool BIAS>
__global__ __launch_bounds__(256) void single_backward_kernel(const AttendParams p, int32_t heads_at_once) {
  if (blockIdx.x < uint32_t(p.splits)) return survey(p);
  const Lanes<L> a(p, heads_at_once);
  if (a.doc >= p.n_docs) return;
  const Span qd = span_of(p.qs, a.doc, p.n_docs), kd = span_of(p.ks, a.doc, p.n_docs);
  if (p.any_large && is_large(qd.owned, kd.owned)) return;
  const T* kp = static_cast<const T*>(p.k) + int64_t(a.hk) * p.k_head + 8 * a.c;
  const T* vp = static_cast<const T*>(p.v) + int64_t(a.hk) * p.v_head + 8 * a.c;
  const float back = fabsf(p.scale);        // q was negated as it was read where the scale is negative
  auto write_keys = [&](int32_t key, const float* dk, const float* dv) {
    vec8<T> x, y;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = T(dk[j]);
      y[j] = T(dv[j]);
    }
    const int64_t d = ((int64_t(kd.begin) + key) * p.kv_heads + a.hk) * p.dim + 8 * a.c;
    *reinterpret_cast<vec8<T>*>(static_cast<T*>(p.dk) + d) = x;
    *reinterpret_cast<vec8<T>*>(static_cast<T*>(p.dv) + d) = y;
  };
  const bool one = qd.tokens == 1;
  for (int32_t row = 0; row < qd.owned; ++row) {
    const int64_t token = int64_t(qd.begin) + row;
    const bool live = row < qd.tokens;
    float dq[G][8] = {};
    floatx4 sums[G] = {};
    if (live) {
      Query<T, L, G, BIAS> x;
      x.load(p, a, token);
      for (int32_t k0 = 0; k0 < kd.tokens; k0 += kSteps * a.keys_at_once) {
        vec8<T> kf[kSteps], vf[kSteps];
        float far[kSteps] = {};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const int32_t key = k0 + i * a.keys_at_once + a.key;
          const bool there = a.in && key < kd.tokens;
          const int64_t key_row = int64_t(kd.begin) + key;
          kf[i] = load8(kp + key_row * p.k_row, there, false);
          vf[i] = load8(vp + key_row * p.v_row, there, false);
          if constexpr (BIAS) far[i] = there ? fabsf(x.at - float(p.ks.pos[key_row])) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const int32_t key = k0 + i * a.keys_at_once + a.key;
          float dk[8] = {}, dv[8] = {};
#pragma unroll
          for (int h = 0; h < G; ++h) {
            const float t = capped<CAP>(p, sum_of_lanes<L>(dot8<T>(kf[i], x.q[h]))), z = fmaf(t, p.z_mul, BIAS ? fmaf(-x.slope[h], far[i], -x.lse[h]) : -x.lse[h]);
            const float e = key < kd.tokens ? exp2_fast(z) : 0.f, dp = sum_of_lanes<L>(dot8<T>(vf[i], x.g[h]));
            float u = e * (dp - x.delta[h]);
            if constexpr (BIAS) sums[h] += floatx4{e, u, e * far[i], u * far[i]};
            u = through_cap<CAP>(p, u, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              dq[h][j] += u * float(kf[i][j]);
              dk[j] += u * back * x.q[h][j];
              dv[j] += e * x.g[h][j];
            }
          }
          if (one && a.in && key < kd.tokens) write_keys(key, dk, dv);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < G; ++h) {
      float o[8] = {};
      floatx4 s = {};
      for (int k = 0; k < a.keys_at_once; ++k) {
        const int from = a.twin(k, heads_at_once);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += __shfl(dq[h][j], from, 64);
        if constexpr (BIAS) {
#pragma unroll
          for (int j = 0; j < 4; ++j) s[j] += __shfl(sums[h][j], from, 64);
        }
      }
      if (!a.in || a.key != 0) continue;
      const int64_t at_out = token * p.heads + a.hk * G + h;
      vec8<T> x;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = T(o[j] * p.scale);
      *reinterpret_cast<vec8<T>*>(static_cast<T*>(p.dq) + at_out * p.dim + 8 * a.c) = x;
      if constexpr (BIAS) {
        if (p.sums && a.c == 0) p.sums[at_out] = s;
      }
    }
  }
  // Keys whose document has not exactly one query: none, whose gradients are zero, or several, which are gone through for every key.
  for (int32_t key = a.key + (one ? kd.tokens : 0); key < kd.owned; key += a.keys_at_once) {
    float dk[8] = {}, dv[8] = {};
    if (key < kd.tokens && qd.tokens > 0) {
      const int64_t key_row = int64_t(kd.begin) + key;
      const vec8<T> kf = load8(kp + key_row * p.k_row, a.in, false), vf = load8(vp + key_row * p.v_row, a.in, false);
      float far = 0.f;
      if constexpr (BIAS) far = float(p.ks.pos[key_row]);
      for (int32_t row = 0; row < qd.tokens; ++row) {
        Query<T, L, G, BIAS> x;
        x.load(p, a, int64_t(qd.begin) + row);
#pragma unroll
        for (int h = 0; h < G; ++h) {
          const float t = capped<CAP>(p, sum_of_lanes<L>(dot8<T>(kf, x.q[h])));
          const float e = exp2_fast(fmaf(t, p.z_mul, BIAS ? fmaf(-x.slope[h], fabsf(x.at - far), -x.lse[h]) : -x.lse[h]));
          float u = e * (sum_of_lanes<L>(dot8<T>(vf, x.g[h])) - x.delta[h]);
          u = through_cap<CAP>(p, u, t);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            dk[j] += u * back * x.q[h][j];
            dv[j] += e * x.g[h][j];
          }
        }
      }
    }
    if (a.in) write_keys(key, dk, dv);
  }
}

template <typename T, int L, int G, bool CAP, bool BIAS> void launch(const AttendParams& p, bool backward, hipStream_t s) {
  const int32_t at_once = std::min(p.kv_heads, 64 / L), chunks = (p.kv_heads + at_once - 1) / at_once;
  in_launches((int64_t(p.n_docs) * chunks + 3) / 4, 256, [&](uint32_t first, uint32_t groups) {
    AttendParams x = p;
    x.first = first;
    x.tiles = int32_t(groups);
    x.splits = p.n_large && !first ? (p.n_docs + 4 * kSurvey - 1) / (4 * kSurvey) : 0;
    const uint32_t blocks = uint32_t(x.splits) + groups;
    if (backward) single_backward_kernel<T, L, G, CAP, BIAS><<<blocks, 256, 0, s>>>(x, at_once);
    else single_kernel<T, L, G, CAP, BIAS><<<blocks, 256, 0, s>>>(x, at_once);
  });
}
template <typename T, int L, int G> void launch(const AttendParams& p, bool cap, bool backward, hipStream_t s) {
  if (cap) p.slopes ? launch<T, L, G, true, true>(p, backward, s) : launch<T, L, G, true, false>(p, backward, s);
  else p.slopes ? launch<T, L, G, false, true>(p, backward, s) : launch<T, L, G, false, false>(p, backward, s);
}
template <typename T, int L> void launch(const AttendParams& p, bool cap, bool backward, hipStream_t s) {
  if (p.group == 1) launch<T, L, 1>(p, cap, backward, s);
  else launch<T, L, 2>(p, cap, backward, s);
}
template <typename T> void launch(const AttendParams& p, bool cap, bool backward, hipStream_t s) {
  if (p.dim <= 16) launch<T, 2>(p, cap, backward, s);
  else if (p.dim <= 32) launch<T, 4>(p, cap, backward, s);
  else if (p.dim <= 64) launch<T, 8>(p, cap, backward, s);
  else launch<T, 16>(p, cap, backward, s);
}

}  // namespace

// Up to two heads of a key head (a lane holds a query and a result for each of them) and 64 keys on average.  These kernels and the tiled ones, us
// forward / backward, fp16: heads 8/4 of 64, 78 125 documents of 10 keys 189 / 374 and 705 / 1769, 12 207 of 64 157 / 343 and 409 / 826; still ahead
// beyond, by less, 3051 of 256 144 / 334 and 168 / 690.  With four heads of a key head the tiled ones take 254 / 671 for 122 880 documents of 10 keys, heads
// 8/2 of 32, where these take 174 / 340 with heads 8/4.
bool single_queries(const lgp_documents* d, const lgp_attention* a) {
  return d->n_docs > 0 && a->heads <= 2 * a->kv_heads && d->q_rows <= d->n_docs && d->k_rows <= 64 * d->n_docs;
}
void launch_single(const AttendParams& p, const lgp_attention* a, bool backward, hipStream_t s) {
  if (a->dtype == LGP_F16) launch<f16>(p, a->cap > 0.f, backward, s);
  else launch<bf16>(p, a->cap > 0.f, backward, s);
}

}  // namespace layer
}  // namespace lgp
