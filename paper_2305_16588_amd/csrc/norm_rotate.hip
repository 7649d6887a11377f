// RMS norm of every query and key head with weights, and the rotation by the token's position, in one pass; and its backward pass.
#include "layer_dev.hpp"

#include <algorithm>
#include <cmath>

namespace lgp {
namespace layer {
namespace {

struct NormParams {
  const void *q, *k;
  int64_t q_row, q_head, k_row, k_head;
  int64_t tokens;
  int32_t heads, kv_heads, dim, rot, n_pos;
  const float *q_weight, *k_weight;
  const int32_t* pos;
  const float* table;        // [n_pos][rot]: cosines, then sines
  float eps;
  int32_t log2_side;         // 2^log2_side heads side by side
  bool apart;                // forward: queries and keys in workgroups of their own, where there are few
  void *q_out, *k_out;       // [tokens][heads][dim] and [tokens][kv_heads][dim]; backward: the gradients of q and k
  const void *dq, *dk;       // backward: like q_out and k_out
  float* partial;            // backward: [workgroup][2][dim]
};

template <typename T> __device__ __forceinline__ void read8(const T* p, float* x) {
  const vec8<T> v = *reinterpret_cast<const vec8<T>*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = float(v[i]);
}
template <> __device__ __forceinline__ void read8<float>(const float* p, float* x) {
  const floatx4 a = *reinterpret_cast<const floatx4*>(p), b = *reinterpret_cast<const floatx4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[i + 4] = b[i]; }
}
template <typename T> __device__ __forceinline__ void write8(T* p, const float* x) {
  vec8<T> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = T(x[i]);
  *reinterpret_cast<vec8<T>*>(p) = v;
}
template <> __device__ __forceinline__ void write8<float>(float* p, const float* x) {
  *reinterpret_cast<floatx4*>(p) = floatx4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<floatx4*>(p + 4) = floatx4{x[4], x[5], x[6], x[7]};
}

// Pair (i, i + rot / 2) turns by the angle of the position (back: the other way).  Lane c of a row has elements 8 c .. 8 c + 7, so the other
// half of its pairs are a lane's, rot / 16 lanes away.  A token's cosines and sines are read once for all its heads.  Every lane of the wave takes
// part in the exchange.
struct Turn {
  float co[8], si[8];         // sines with the sign of the lane's half
  int from;                   // the lane of the other half
  bool in;
  __device__ __forceinline__ Turn(const NormParams& p, int c, int lane, int32_t pos, bool known, bool back) {
    const int lanes = p.rot / 16;
    const bool low = c < lanes;
    in = c < 2 * lanes && known;
    from = c < 2 * lanes ? (low ? lane + lanes : lane - lanes) : lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) co[i] = 1.f, si[i] = 0.f;
    if (in) {
      const float* t = p.table + int64_t(pos) * p.rot + 8 * (low ? c : c - lanes);
      read8(t, co);
      read8(t + p.rot / 2, si);
      if (low != back)
#pragma unroll
        for (int i = 0; i < 8; ++i) si[i] = -si[i];
    }
  }
  __device__ __forceinline__ void operator()(float* y) const {
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = __shfl(y[i], from, 64);
    if (!in) return;          // not even times zero: what is not turned may be infinite
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] * co[i] + si[i] * z[i];
  }
};

// L lanes of a head, 2^log2_side heads of a token side by side (heads_side), so that a wave's loads are whole lines; a lane has eight
// elements of every so many heads, kAtOnce of them on their way at a time.  Bound by bytes.  Measured: 500 000 tokens, heads 8 and 2 of 128, fp16:
// 487 us, 5.2 TB/s; 282 624 tokens, heads 8 and 8 of 32, bf16, 30 % without a token: 119 us.
constexpr int kAtOnce = 4;
template <typename T, int L>
__global__ __launch_bounds__(256) void norm_rotate_kernel(const NormParams p) {
  const int lane = threadIdx.x & 63, c = lane % L, side = 1 << p.log2_side, first = lane / L & (side - 1);
  const int64_t at = (int64_t(blockIdx.x) * (256 / L) + threadIdx.x / L) >> p.log2_side, token = at < p.tokens ? at : p.tokens - 1;       // the last ones again
  const bool mine = 8 * c < p.dim;
  const int32_t pos = p.pos ? p.pos[token] : 0;
  const bool live = pos >= 0, known = p.rot == 0 || pos < p.n_pos;
  const Turn turn(p, c, lane, pos, live && known, false);
  auto rows = [&](const T* src, int64_t stride, int32_t heads, const float* weights, T* dst) {
    float w[8] = {};
    if (mine && heads) read8(weights + 8 * c, w);
    for (int32_t h0 = 0; h0 < heads; h0 += kAtOnce << p.log2_side) {
      float x[kAtOnce][8];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = 0.f;
        const int32_t h = h0 + j * side + first;
        if (live && mine && h < heads) read8(src + h * stride + 8 * c, x[j]);
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int32_t h = h0 + j * side + first;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[j][i] * x[j][i];
        const float r = known ? 1.f / sqrtf(sum_of_lanes<L>(sum) / float(p.dim) + p.eps) : NAN;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] *= r * w[i];
        if (p.rot) turn(x[j]);
        if (!mine || h >= heads || at >= p.tokens) continue;
        if (!live)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[j][i] = 0.f;
        write8(dst + int64_t(h) * p.dim + 8 * c, x[j]);
      }
    }
  };
  if (blockIdx.y == 0) rows(static_cast<const T*>(p.q) + token * p.q_row, p.q_head, p.heads, p.q_weight, static_cast<T*>(p.q_out) + token * p.heads * p.dim);
  if (blockIdx.y == gridDim.y - 1)
    rows(static_cast<const T*>(p.k) + token * p.k_row, p.k_head, p.kv_heads, p.k_weight, static_cast<T*>(p.k_out) + token * p.kv_heads * p.dim);
}

// Backward, with n = x r, r = 1 / sqrt(mean(x^2) + eps) and g = w * (dy turned back):  dx = r (g - n mean(g n)),  dw = sum over rows of n * (dy
// turned back).  Lanes as in the forward kernel, which go on to further tokens: a lane adds up the gradients of its own eight weights of queries
// and of keys in registers; the lanes of a workgroup are added in LDS and all workgroups in a second kernel, in a fixed order.  Bound by conversions
// and sums beside the bytes.  Measured: 282 624 tokens, heads 8 and 8 of 32, bf16, 30 % without a token: 175 us, and 5 for the second kernel.
template <typename T, int L>
__global__ __launch_bounds__(256) void norm_rotate_backward_kernel(const NormParams p) {
  constexpr int kGroups = 256 / L, kPairs = 2;           // heads of a lane on their way at a time
  __shared__ float lds[kGroups][8 * L + 1];
  const int lane = threadIdx.x & 63, c = lane % L, group = threadIdx.x / L, side = 1 << p.log2_side, first = group & (side - 1);
  const int tokens = kGroups >> p.log2_side;             // at a time
  const bool mine = 8 * c < p.dim;
  float dwq[8] = {}, dwk[8] = {};
  for (int64_t token0 = int64_t(blockIdx.x) * tokens; token0 < p.tokens; token0 += int64_t(gridDim.x) * tokens) {
    const int64_t at = token0 + (group >> p.log2_side), token = at < p.tokens ? at : p.tokens - 1;
    const bool in = at < p.tokens;
    const int32_t pos = p.pos ? p.pos[token] : 0;
    const bool live = in && pos >= 0, known = p.rot == 0 || pos < p.n_pos;
    const Turn turn(p, c, lane, pos, live && known, true);
    auto rows = [&](const T* src, int64_t stride, const T* grad, int32_t heads, const float* weights, T* dst, float* dw) {
      float w[8] = {};
      if (mine && heads) read8(weights + 8 * c, w);
      for (int32_t h0 = 0; h0 < heads; h0 += kPairs << p.log2_side) {
        float x[kPairs][8], g[kPairs][8];
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[j][i] = g[j][i] = 0.f;
          const int32_t h = h0 + j * side + first;
          if (live && mine && h < heads) {
            read8(src + h * stride + 8 * c, x[j]);
            read8(grad + int64_t(h) * p.dim + 8 * c, g[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          const int32_t h = h0 + j * side + first;
          float sum = 0.f, dot = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) sum += x[j][i] * x[j][i];
          // no norm where there is no head or no token: with an eps of zero it would be infinite, and its product with their zeros NaN
          sum = sum_of_lanes<L>(sum);
          const float r = live && h < heads ? 1.f / sqrtf(sum / float(p.dim) + p.eps) : 0.f;
          if (p.rot) turn(g[j]);
          if (live && !known && h < heads)
#pragma unroll
            for (int i = 0; i < 8; ++i) g[j][i] = NAN;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[j][i] *= r;
            dw[i] += g[j][i] * x[j][i];
            g[j][i] *= w[i];
            dot += g[j][i] * x[j][i];
          }
          dot = sum_of_lanes<L>(dot) / float(p.dim);
          if (!in || !mine || h >= heads) continue;
#pragma unroll
          for (int i = 0; i < 8; ++i) g[j][i] = live ? r * (g[j][i] - x[j][i] * dot) : 0.f;
          write8(dst + int64_t(h) * p.dim + 8 * c, g[j]);
        }
      }
    };
    rows(static_cast<const T*>(p.q) + token * p.q_row, p.q_head, static_cast<const T*>(p.dq) + token * p.heads * p.dim, p.heads, p.q_weight,
         static_cast<T*>(p.q_out) + token * p.heads * p.dim, dwq);
    rows(static_cast<const T*>(p.k) + token * p.k_row, p.k_head, static_cast<const T*>(p.dk) + token * p.kv_heads * p.dim, p.kv_heads, p.k_weight,
         static_cast<T*>(p.k_out) + token * p.kv_heads * p.dim, dwk);
  }
#pragma unroll
  for (int of_k = 0; of_k < 2; ++of_k) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) lds[group][8 * c + i] = of_k ? dwk[i] : dwq[i];
    __syncthreads();
    for (int d = threadIdx.x; d < p.dim; d += 256) {
      float s = 0.f;
      for (int g = 0; g < kGroups; ++g) s += lds[g][d];
      p.partial[(int64_t(blockIdx.x) * 2 + of_k) * p.dim + d] = s;
    }
  }
}

// Sum of the workgroups' weight gradients: a workgroup per weight of queries (y = 0) and keys.
__global__ __launch_bounds__(256) void weights_kernel(const float* partial, int32_t dim, int32_t groups, float* q, float* k) {
  __shared__ float lds[4];
  const int32_t d = blockIdx.x;
  float* out = blockIdx.y ? k : q;
  if (!out) return;
  float s = 0.f;
  for (int32_t g = threadIdx.x; g < groups; g += 256) s += partial[(int64_t(g) * 2 + blockIdx.y) * dim + d];
#pragma unroll
  for (int i = 32; i; i >>= 1) s += __shfl_xor(s, i, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) out[d] = lds[0] + lds[1] + lds[2] + lds[3];
}

int lanes_of(int32_t dim) {
  int l = 1;
  while (8 * l < dim) l *= 2;
  return l;
}
// Heads side by side.  Where there are too few tokens to fill the GPU, as many as a wave holds.  Else one in the forward pass, which then reads a
// token's angles least often, and in the backward pass, which reads and writes more, as many as make 16 lanes, 256 bytes of 16-bit elements (282624
// tokens, 8 + 8 heads of 32: forward 120 us, with four side by side 146; backward 193, with four 173).  Never more than there are heads.
bool few_tokens(int device, const lgp_heads* h) { return h->tokens * 16 < int64_t(compute_units(device)) * 512; }
int32_t heads_side(int device, const lgp_heads* h, bool backward) {
  const int l = lanes_of(h->dim), most = few_tokens(device, h) ? 64 : backward ? 16 : l;
  int side = 0;
  while ((l << side) < most && (1 << side) < std::max(h->heads, h->kv_heads)) ++side;
  return side;
}
template <typename T> void forward(const NormParams& whole, hipStream_t s) {
  const int l = lanes_of(whole.dim);
  const int64_t per_group = std::max(1, 256 / l >> whole.log2_side);        // tokens
  in_launches((whole.tokens + per_group - 1) / per_group, 256, [&](uint32_t first, uint32_t groups) {
    const int64_t t0 = first * per_group;
    NormParams p = whole;
    p.tokens = std::min(whole.tokens - t0, groups * per_group);
    p.q = static_cast<const T*>(whole.q) + t0 * whole.q_row;
    p.k = static_cast<const T*>(whole.k) + t0 * whole.k_row;
    p.q_out = static_cast<T*>(whole.q_out) + t0 * whole.heads * whole.dim;
    p.k_out = static_cast<T*>(whole.k_out) + t0 * whole.kv_heads * whole.dim;
    if (whole.pos) p.pos = whole.pos + t0;
    const dim3 blocks(groups, p.apart ? 2 : 1);
    switch (l) {
      case 1: norm_rotate_kernel<T, 1><<<blocks, 256, 0, s>>>(p); break;
      case 2: norm_rotate_kernel<T, 2><<<blocks, 256, 0, s>>>(p); break;
      case 4: norm_rotate_kernel<T, 4><<<blocks, 256, 0, s>>>(p); break;
      case 8: norm_rotate_kernel<T, 8><<<blocks, 256, 0, s>>>(p); break;
      case 16: norm_rotate_kernel<T, 16><<<blocks, 256, 0, s>>>(p); break;
      default: norm_rotate_kernel<T, 32><<<blocks, 256, 0, s>>>(p); break;
    }
  });
}
template <typename T> void backward(const NormParams& p, uint32_t blocks, hipStream_t s) {
  switch (lanes_of(p.dim)) {
    case 1: norm_rotate_backward_kernel<T, 1><<<blocks, 256, 0, s>>>(p); break;
    case 2: norm_rotate_backward_kernel<T, 2><<<blocks, 256, 0, s>>>(p); break;
    case 4: norm_rotate_backward_kernel<T, 4><<<blocks, 256, 0, s>>>(p); break;
    case 8: norm_rotate_backward_kernel<T, 8><<<blocks, 256, 0, s>>>(p); break;
    case 16: norm_rotate_backward_kernel<T, 16><<<blocks, 256, 0, s>>>(p); break;
    default: norm_rotate_backward_kernel<T, 32><<<blocks, 256, 0, s>>>(p); break;
  }
}

int check_norm(const lgp_heads* h) {
  if (!h) return LGP_EINVAL;
  if (h->tokens < 0 || h->heads < 0 || h->kv_heads < 0 || h->heads + h->kv_heads < 1 || h->dim < 1 || h->rot < 0 || h->rot > h->dim) return LGP_EINVAL;
  if (h->dtype != LGP_F32 && h->dtype != LGP_F16 && h->dtype != LGP_BF16) return LGP_EUNSUPPORTED;
  if (h->dim % 8 || h->dim > 256 || h->rot % 16) return LGP_EUNSUPPORTED;
  if (h->heads > 65536 || h->kv_heads > 65536 || h->tokens >= int64_t(1) << 33) return LGP_EUNSUPPORTED;
  if (h->tokens && ((h->heads && !h->q) || (h->kv_heads && !h->k))) return LGP_EINVAL;
  if ((h->heads && !h->q_weight) || (h->kv_heads && !h->k_weight)) return LGP_EINVAL;
  if (h->rot && (!h->table || h->n_pos < 1 || (h->tokens && !h->pos))) return LGP_EINVAL;
  if (!aligned16(h->q) || !aligned16(h->k) || !aligned16(h->q_weight) || !aligned16(h->k_weight) || !aligned16(h->table)) return LGP_EINVAL;
  if (h->q_row % 8 || h->q_head % 8 || h->k_row % 8 || h->k_head % 8) return LGP_EINVAL;
  return std::isfinite(h->eps) && h->eps >= 0.f ? LGP_OK : LGP_EINVAL;
}
NormParams norm_params(const lgp_heads* h) {
  NormParams p = {};
  p.q = h->q; p.k = h->k; p.q_row = h->q_row; p.q_head = h->q_head; p.k_row = h->k_row; p.k_head = h->k_head;
  p.tokens = h->tokens; p.heads = h->heads; p.kv_heads = h->kv_heads; p.dim = h->dim; p.rot = h->rot; p.n_pos = h->n_pos;
  p.q_weight = h->q_weight; p.k_weight = h->k_weight; p.pos = h->pos; p.table = h->table; p.eps = h->eps;
  return p;
}
// Workgroups of the backward kernel: at most four per CU.
int32_t backward_groups(int device, const lgp_heads* h) {
  const int64_t tokens = std::max(1, 256 / lanes_of(h->dim) >> heads_side(device, h, true));
  return int32_t(std::max<int64_t>(1, std::min((h->tokens + tokens - 1) / tokens, int64_t(compute_units(device)) * 4)));
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_norm_rotate(int device, const lgp_heads* in, void* q_out, void* k_out, void* stream) {
  if (int st = check_norm(in)) return st;
  if (in->tokens && ((in->heads && !q_out) || (in->kv_heads && !k_out))) return LGP_EINVAL;
  if (!aligned16(q_out) || !aligned16(k_out)) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (in->tokens == 0) return LGP_OK;
  NormParams p = norm_params(in);
  p.log2_side = heads_side(device, in, false);
  p.apart = few_tokens(device, in);
  p.q_out = q_out;
  p.k_out = k_out;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F32) forward<float>(p, s);
  else if (in->dtype == LGP_F16) forward<f16>(p, s);
  else forward<bf16>(p, s);
  return launched();
}

int lgp_norm_rotate_workspace(int device, const lgp_heads* in, size_t* bytes) {
  if (!bytes) return LGP_EINVAL;
  *bytes = 0;
  if (int st = check_norm(in)) return st;
  *bytes = size_t(backward_groups(device, in)) * 2 * in->dim * sizeof(float);
  return LGP_OK;
}

int lgp_norm_rotate_backward(int device, const lgp_heads* in, const void* dq_out, const void* dk_out, void* dq, void* dk, float* dq_weight,
                             float* dk_weight, void* workspace, size_t workspace_bytes, void* stream) {
  if (int st = check_norm(in)) return st;
  if (in->tokens && ((in->heads && (!dq_out || !dq)) || (in->kv_heads && (!dk_out || !dk)))) return LGP_EINVAL;
  if ((in->heads && !dq_weight) || (in->kv_heads && !dk_weight)) return LGP_EINVAL;
  if (!aligned16(dq_out) || !aligned16(dk_out) || !aligned16(dq) || !aligned16(dk)) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  NormParams p = norm_params(in);
  p.log2_side = heads_side(device, in, true);
  const int32_t groups = backward_groups(device, in);
  if (workspace_bytes < size_t(groups) * 2 * in->dim * sizeof(float)) return LGP_ECAPACITY;
  if (!workspace || !aligned16(workspace)) return LGP_EINVAL;
  p.dq = dq_out;
  p.dk = dk_out;
  p.q_out = dq;
  p.k_out = dk;
  p.partial = static_cast<float*>(workspace);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F32) backward<float>(p, groups, s);
  else if (in->dtype == LGP_F16) backward<f16>(p, groups, s);
  else backward<bf16>(p, groups, s);
  weights_kernel<<<dim3(in->dim, 2), 256, 0, s>>>(p.partial, in->dim, groups, in->heads ? dq_weight : nullptr, in->kv_heads ? dk_weight : nullptr);
  return launched();
}

}  // extern "C"
