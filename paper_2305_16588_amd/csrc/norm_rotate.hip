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
  void *q_out, *k_out;       // [tokens][heads][dim] and [tokens][kv_heads][dim]; backward: the gradients of q and k
  const void *dq, *dk;       // backward: like q_out and k_out
  float* partial;            // backward: [workgroup of q, then of k][dim]
  int32_t q_groups;          // backward: workgroups of q
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
// half of its pairs are a lane's, rot / 16 lanes away.  Every lane of the wave takes part in the exchange.
template <int L>
__device__ __forceinline__ void rotate(const NormParams& p, float* y, int c, int lane, int32_t pos, bool live, bool back) {
  if (p.rot == 0) return;
  const int lanes = p.rot / 16;
  const bool in = c < 2 * lanes, low = c < lanes;
  const int from = in ? (low ? lane + lanes : lane - lanes) : lane;
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = __shfl(y[i], from, 64);
  if (!in || !live) return;
  const float* t = p.table + int64_t(pos) * p.rot + 8 * (low ? c : c - lanes);
  float co[8], si[8];
  read8(t, co);
  read8(t + p.rot / 2, si);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = y[i] * co[i] + (low == back ? si[i] : -si[i]) * z[i];
}

// L lanes of a row of up to 8 L elements; 64 / L rows of a wave.
template <typename T, int L>
__global__ __launch_bounds__(256) void norm_rotate_kernel(const NormParams p) {
  const int lane = threadIdx.x & 63, c = lane % L;
  const uint32_t per_token = p.heads + p.kv_heads;
  const int64_t row = (int64_t(blockIdx.x) * 256 + threadIdx.x) / L, rows = p.tokens * per_token;
  const bool in = row < rows;
  const int64_t token = in ? row / per_token : 0;
  const int32_t h = in ? int32_t(row - token * per_token) : 0;
  const bool is_q = h < p.heads, mine = 8 * c < p.dim;
  const int32_t pos = p.pos ? p.pos[token] : 0;
  const bool live = in && pos >= 0, known = p.rot == 0 || pos < p.n_pos;
  float x[8] = {}, sum = 0.f;
  if (live && mine) {
    const T* src = is_q ? static_cast<const T*>(p.q) + token * p.q_row + h * p.q_head : static_cast<const T*>(p.k) + token * p.k_row + (h - p.heads) * p.k_head;
    read8(src + 8 * c, x);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
  sum = sum_of_lanes<L>(sum);
  const float r = 1.f / sqrtf(sum / float(p.dim) + p.eps);
  const float* w = is_q ? p.q_weight : p.k_weight;
  if (mine) {
    float wt[8];
    read8(w + 8 * c, wt);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= r * wt[i];
  }
  rotate<L>(p, x, c, lane, pos, live && known, false);
  if (!in || !mine) return;
  if (!live || !known) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = live ? NAN : 0.f;
  }
  T* dst = is_q ? static_cast<T*>(p.q_out) + (token * p.heads + h) * p.dim : static_cast<T*>(p.k_out) + (token * p.kv_heads + h - p.heads) * p.dim;
  write8(dst + 8 * c, x);
}

// Backward, with n = x r, r = 1 / sqrt(mean(x^2) + eps) and g = w * (dy turned back):  dx = r (g - n mean(g n)),  dw = sum over rows of n * (dy
// turned back).  A workgroup takes rows of queries or of keys, so that a lane adds up the gradient of its own eight weights in registers;
// its groups of lanes are added in LDS and all workgroups in a second kernel, in a fixed order.
template <typename T, int L>
__global__ __launch_bounds__(256) void norm_rotate_backward_kernel(const NormParams p) {
  constexpr int kRows = 256 / L;
  __shared__ float lds[kRows][8 * L + 1];
  const int lane = threadIdx.x & 63, c = lane % L, group = threadIdx.x / L;
  const bool is_q = int32_t(blockIdx.x) < p.q_groups, mine = 8 * c < p.dim;
  const int32_t heads = is_q ? p.heads : p.kv_heads, block = is_q ? blockIdx.x : blockIdx.x - p.q_groups;
  const int32_t blocks = is_q ? p.q_groups : gridDim.x - p.q_groups;
  const int64_t rows = p.tokens * heads, row_stride = is_q ? p.q_row : p.k_row, head_stride = is_q ? p.q_head : p.k_head;
  const T* src = static_cast<const T*>(is_q ? p.q : p.k);
  const T* grad = static_cast<const T*>(is_q ? p.dq : p.dk);
  T* dst = static_cast<T*>(is_q ? p.q_out : p.k_out);
  float w[8] = {}, dw[8] = {};
  if (mine) read8((is_q ? p.q_weight : p.k_weight) + 8 * c, w);
  for (int64_t row0 = int64_t(block) * kRows; row0 < rows; row0 += int64_t(blocks) * kRows) {
    const int64_t row = row0 + group;
    const bool in = row < rows;
    const int64_t token = in ? row / heads : 0;
    const int32_t h = in ? int32_t(row - token * heads) : 0;
    const int32_t pos = p.pos ? p.pos[token] : 0;
    const bool live = in && pos >= 0, known = p.rot == 0 || pos < p.n_pos;
    float x[8] = {}, g[8] = {}, sum = 0.f, dot = 0.f;
    if (live && mine) {
      read8(src + token * row_stride + h * head_stride + 8 * c, x);
      read8(grad + row * p.dim + 8 * c, g);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
    sum = sum_of_lanes<L>(sum);
    const float r = 1.f / sqrtf(sum / float(p.dim) + p.eps);
    rotate<L>(p, g, c, lane, pos, live && known, true);
    if (live && !known) {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = NAN;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] *= r;
      dw[i] += g[i] * x[i];
      g[i] *= w[i];
      dot += g[i] * x[i];
    }
    dot = sum_of_lanes<L>(dot) / float(p.dim);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = r * (g[i] - x[i] * dot);
    if (in && mine) {
      if (!live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 0.f;
      }
      write8(dst + row * p.dim + 8 * c, g);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) lds[group][8 * c + i] = dw[i];
  __syncthreads();
  for (int d = threadIdx.x; d < p.dim; d += 256) {
    float s = 0.f;
    for (int g = 0; g < kRows; ++g) s += lds[g][d];
    p.partial[int64_t(blockIdx.x) * p.dim + d] = s;
  }
}

// Sum of the workgroups' weight gradients: a workgroup per weight of queries (y = 0) and keys.
__global__ __launch_bounds__(256) void weights_kernel(const float* partial, int32_t dim, int32_t q_groups, int32_t k_groups, float* q, float* k) {
  __shared__ float lds[4];
  const int32_t d = blockIdx.x, groups = blockIdx.y ? k_groups : q_groups;
  const float* src = partial + (blockIdx.y ? int64_t(q_groups) * dim : 0);
  float s = 0.f;
  for (int32_t g = threadIdx.x; g < groups; g += 256) s += src[int64_t(g) * dim + d];
#pragma unroll
  for (int i = 32; i; i >>= 1) s += __shfl_xor(s, i, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) (blockIdx.y ? k : q)[d] = lds[0] + lds[1] + lds[2] + lds[3];
}

int lanes_of(int32_t dim) {
  int l = 1;
  while (8 * l < dim) l *= 2;
  return l;
}
template <typename T> void forward(const NormParams& p, hipStream_t s) {
  const int l = lanes_of(p.dim);
  const uint32_t blocks = uint32_t((p.tokens * (p.heads + p.kv_heads) * l + 255) / 256);
  switch (l) {
    case 1: norm_rotate_kernel<T, 1><<<blocks, 256, 0, s>>>(p); break;
    case 2: norm_rotate_kernel<T, 2><<<blocks, 256, 0, s>>>(p); break;
    case 4: norm_rotate_kernel<T, 4><<<blocks, 256, 0, s>>>(p); break;
    case 8: norm_rotate_kernel<T, 8><<<blocks, 256, 0, s>>>(p); break;
    case 16: norm_rotate_kernel<T, 16><<<blocks, 256, 0, s>>>(p); break;
    default: norm_rotate_kernel<T, 32><<<blocks, 256, 0, s>>>(p); break;
  }
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
  if (h->heads > 65536 || h->kv_heads > 65536 || h->tokens >= (int64_t(1) << 36) / (h->heads + h->kv_heads)) return LGP_EUNSUPPORTED;   // workgroups below 2^31
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
// Workgroups of the backward kernel that take queries and keys: at most four per CU, shared by the rows there are of each.
void backward_groups(int device, const lgp_heads* h, int32_t* q, int32_t* k) {
  const int64_t rows = 256 / lanes_of(h->dim), most = int64_t(compute_units(device)) * 4, all = std::max<int64_t>(1, h->heads + h->kv_heads);
  auto groups = [&](int64_t heads) {
    return heads == 0 ? 0 : int32_t(std::max<int64_t>(1, std::min((h->tokens * heads + rows - 1) / rows, most * heads / all)));
  };
  *q = groups(h->heads);
  *k = groups(h->kv_heads);
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
  int32_t q, k;
  backward_groups(device, in, &q, &k);
  *bytes = size_t(q + k) * in->dim * sizeof(float);
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
  int32_t q, k;
  backward_groups(device, in, &q, &k);
  if (workspace_bytes < size_t(q + k) * in->dim * sizeof(float)) return LGP_ECAPACITY;
  if (!workspace || !aligned16(workspace)) return LGP_EINVAL;
  p.dq = dq_out;
  p.dk = dk_out;
  p.q_out = dq;
  p.k_out = dk;
  p.partial = static_cast<float*>(workspace);
  p.q_groups = q;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F32) backward<float>(p, q + k, s);
  else if (in->dtype == LGP_F16) backward<f16>(p, q + k, s);
  else backward<bf16>(p, q + k, s);
  // without heads of one kind there are no workgroups of it, and nothing of it to write
  if (in->heads && in->kv_heads) weights_kernel<<<dim3(in->dim, 2), 256, 0, s>>>(p.partial, in->dim, q, k, dq_weight, dk_weight);
  else weights_kernel<<<dim3(in->dim, 1), 256, 0, s>>>(p.partial, in->dim, q + k, 0, in->heads ? dq_weight : dk_weight, nullptr);
  return launched();
}

}  // extern "C"
