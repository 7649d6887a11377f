// The residual's addition and the RMS norm of the sum in one pass, its result in 16, 32 or 8 bits, and the backward pass.
#include "rows_dev.hpp"

#include <algorithm>
#include <cmath>

namespace lgp {
namespace layer {
namespace {

struct AddParams {
  const void *x, *residual;
  int64_t x_row, residual_row, tokens;
  int32_t width;
  const float* weight;
  const int32_t* pos;
  float eps;
  void *y, *total;
  int8_t* values;
  float* scales;
  const void *dy, *d_total;        // backward
  void *dx, *d_residual;
  float* partial;                  // [workgroup][width]
};

// A row's sums over its L lanes: those of a wave, or a workgroup, which has a place for each of its waves in `lds`, used in turn so that one
// barrier is enough.
template <int L, int N> __device__ __forceinline__ void row_sums(float* x, float (*lds)[N][16], int turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = lanes_sum<(L > 64 ? 64 : L)>(x[i]);
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[turn][i][threadIdx.x >> 6] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = 0.f;
#pragma unroll
      for (int w = 0; w < L / 64; ++w) x[i] += lds[turn][i][w];
    }
  }
}

// Squares pass the range of 32 bits from 2^64 on and lose digits below 2^-63, where the norm does neither: a row whose mean square (with eps) says so is multiplied by a power of two
// in the registers, and its sums are taken again.  Infinities and NaN come here too, and stay.
__device__ __forceinline__ bool out_of_range(float mean) { return !(mean <= 3.402823466e+38f) || mean < 0x1p-100f; }
__device__ __forceinline__ float into_range(float mean) { return mean < 1.f ? 0x1p+100f : 0x1p-80f; }

// L lanes have a row, each of them every L-th eight elements, C of them: a row is read once and stays in registers, and a wave's loads are whole
// lines.  The sum of squares, the root and the products are in 32 bits; the total is rounded first, so that the backward pass, which reads it, has the
// gradients of what was computed.  Bound by bytes.  Measured: 400000 rows of 1024, fp16 with a residual in fp32: 855 us, 5.7 TB/s; 282624 rows of
// 256, bf16, 30 % without a token: 88 us, 5.6 TB/s, and 97 to 104 with the result in 8 bits (4.2 TB/s); rows packed alone: 282624 of 256, bf16, 38 us, 5.7 TB/s,
// 65536 of 4096 153 us, 5.3 TB/s.
enum { kNorm = 0, kNorm8 = 1, kPack8 = 2 };
template <typename T, typename S, int MODE, int L, int C>
__global__ __launch_bounds__(L > 256 ? L : 256) void add_norm_kernel(const AddParams p) {
  constexpr int kRows = (L > 256 ? L : 256) / L;
  __shared__ float lds[1][1][16];
  __shared__ uint32_t lds_top[16];
  const int c0 = threadIdx.x % L;
  const int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / L;
  const bool in = row < p.tokens, live = in && (!p.pos || p.pos[row] >= 0);
  float t[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = 8 * (c * L + c0), n = live ? p.width - at : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[c][i] = 0.f;
    if (n > 0) read_row(static_cast<const T*>(p.x) + row * p.x_row + at, n, t[c]);
  }
  if (MODE != kPack8 && p.residual) {
    float r[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = 8 * (c * L + c0), n = live ? p.width - at : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) r[c][i] = 0.f;
      if (n > 0) read_row(static_cast<const S*>(p.residual) + row * p.residual_row + at, n, r[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = 8 * (c * L + c0), n = in ? p.width - at : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) t[c][i] = float(S(t[c][i] + r[c][i]));
      if (n > 0) write_row(static_cast<S*>(p.total) + row * p.width + at, n, t[c]);
    }
  }
  if constexpr (MODE != kPack8) {
    float sum[1] = {};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[0] += t[c][i] * t[c][i];
    row_sums<L, 1>(sum, lds, 0);
    float mean = sum[0] / float(p.width) + p.eps;
    if (live && out_of_range(mean)) {          // in all lanes of a row
      const float by = into_range(mean);
      sum[0] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) t[c][i] *= by, sum[0] += t[c][i] * t[c][i];
      if constexpr (L > 64) __syncthreads();
      row_sums<L, 1>(sum, lds, 0);
      mean = sum[0] / float(p.width) + p.eps * by * by;
    }
    const float r = live ? 1.f / sqrtf(mean) : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = 8 * (c * L + c0), n = in ? p.width - at : 0;
      if (n <= 0) continue;
      float w[8];
      read_row(p.weight + at, n, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[c][i] = t[c][i] * r * w[i];
      if (MODE == kNorm) write_row(static_cast<T*>(p.y) + row * p.width + at, n, t[c]);
    }
  }
  if constexpr (MODE != kNorm) {
    uint32_t top = 0;              // as whole numbers infinities are larger than numbers, and NaN than they
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, t[c][i]) & 0x7fffffffu);
    top = lanes_max<(L > 64 ? 64 : L)>(top);
    if constexpr (L > 64) {
      if ((threadIdx.x & 63) == 0) lds_top[threadIdx.x >> 6] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < L / 64; ++w) top = max(top, lds_top[w]);
    }
    const bool finite = top < 0x7f800000u;
    const float scale = fmaxf(__builtin_bit_cast(float, top) / 127.f, 0x1p-126f), by = finite ? 1.f / scale : 0.f;
    const int pitch = (p.width + 15) / 16 * 16;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = 8 * (c * L + c0);
      if (!in || at >= pitch) continue;
      union { int8_t b[8]; uint64_t all; } v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.b[i] = finite ? int8_t(int(fminf(fmaxf(rintf(t[c][i] * by), -127.f), 127.f))) : int8_t(0);
      *reinterpret_cast<uint64_t*>(p.values + row * pitch + at) = v.all;
    }
    if (in && c0 == 0) p.scales[row] = !live ? 0.f : finite ? scale : NAN;
  }
}

// Backward: both sums of a row, of squares and of dy weight total, are taken together.  A workgroup goes on to further rows, whose weights' gradients
// a lane adds up for its own elements; the rows of a workgroup are added in LDS and all workgroups in a second kernel, in a fixed order.  Bound by bytes.  Measured: 400000 rows of
// 1024, fp16 with a residual in fp32: 1416 us, 4.6 TB/s; 282624 rows of 256, bf16, 30 % without a token: 121 to 125 us, 3.7 TB/s.
template <typename T, typename S, int L, int C>
__global__ __launch_bounds__(L > 256 ? L : 256) void add_norm_backward_kernel(const AddParams p) {
  constexpr int kThreads = L > 256 ? L : 256, kRows = kThreads / L;
  __shared__ float lds[2][2][16];
  __shared__ float lds_w[kRows > 1 ? kRows : 1][kRows > 1 ? 8 * L * C + 1 : 1];
  const int c0 = threadIdx.x % L, group = threadIdx.x / L;
  float w[C][8], dw[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = 8 * (c * L + c0);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[c][i] = dw[c][i] = 0.f;
    if (p.width > at) read_row(p.weight + at, p.width - at, w[c]);
  }
  int turn = 0;
  for (int64_t row0 = int64_t(blockIdx.x) * kRows; row0 < p.tokens; row0 += int64_t(gridDim.x) * kRows, turn ^= 1) {
    const int64_t row = row0 + group;
    const bool in = row < p.tokens, live = in && (!p.pos || p.pos[row] >= 0);
    float t[C][8], g[C][8], d[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = 8 * (c * L + c0), n = live ? p.width - at : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) t[c][i] = g[c][i] = d[c][i] = 0.f;
      if (n > 0) {
        read_row(static_cast<const S*>(p.residual) + row * p.residual_row + at, n, t[c]);
        read_row(static_cast<const T*>(p.dy) + row * p.width + at, n, g[c]);
        if (p.d_total) read_row(static_cast<const S*>(p.d_total) + row * p.width + at, n, d[c]);
      }
    }
    float sum[2] = {};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum[0] += t[c][i] * t[c][i];
        sum[1] += g[c][i] * w[c][i] * t[c][i];
      }
    row_sums<L, 2>(sum, lds, turn);
    float mean = sum[0] / float(p.width) + p.eps, by = 1.f;
    if (live && out_of_range(mean)) {
      by = into_range(mean);
      sum[0] = sum[1] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = t[c][i] * by;
          sum[0] += v * v;
          sum[1] += g[c][i] * w[c][i] * v;
        }
      if constexpr (L > 64) __syncthreads();
      row_sums<L, 2>(sum, lds, turn);
      mean = sum[0] / float(p.width) + p.eps * by * by;
    }
    const float r0 = live ? 1.f / sqrtf(mean) : 0.f;       // 0: with an eps of zero it would be infinite
    const float dot = sum[1] * r0 / float(p.width);
    const float r = r0 <= 3.402823466e+38f && r0 * by > 3.402823466e+38f ? 3.402823466e+38f : r0 * by;       // of rows without any normal number; NaN stays
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = 8 * (c * L + c0), n = in ? p.width - at : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float norm = t[c][i] * r;
        dw[c][i] += g[c][i] * norm;
        d[c][i] += r * (g[c][i] * w[c][i] - norm * dot);
      }
      if (n <= 0) continue;
      write_row(static_cast<S*>(p.d_residual) + row * p.width + at, n, d[c]);
      if (p.dx) write_row(static_cast<T*>(p.dx) + row * p.width + at, n, d[c]);
    }
  }
  float* out = p.partial + int64_t(blockIdx.x) * p.width;
  if constexpr (kRows > 1) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) lds_w[group][8 * (c * L + c0) + i] = dw[c][i];
    __syncthreads();
    for (int k = threadIdx.x; k < p.width; k += kThreads) {
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) s += lds_w[r][k];
      out[k] = s;
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (8 * (c * L + c0) + i < p.width) out[8 * (c * L + c0) + i] = dw[c][i];
  }
}

// Sum of the workgroups' weight gradients: a workgroup has 32 columns, each of them by 32 lanes.  Measured: 1024 workgroups' of 1024 columns, 6 us.
__global__ __launch_bounds__(1024) void add_groups_kernel(const float* partial, int32_t width, int32_t groups, float* out) {
  __shared__ float lds[32][33];
  const int at = threadIdx.x & 31, first = threadIdx.x >> 5;
  const int32_t k = blockIdx.x * 32 + at;
  float s = 0.f;
  if (k < width)
#pragma unroll 4
    for (int32_t g = first; g < groups; g += 32) s += partial[int64_t(g) * width + k];
  lds[first][at] = s;
  __syncthreads();
  s = sum_of_lanes<32>(lds[at][first]);
  if (at == 0 && blockIdx.x * 32 + first < width) out[blockIdx.x * 32 + first] = s;
}

// f(lanes of a row, groups of eight elements of each) for the least that hold `width`.
template <int N> using Int = std::integral_constant<int, N>;
template <typename F> void by_width(int32_t width, F f) {
  if (width <= 32) f(Int<4>(), Int<1>());
  else if (width <= 128) f(Int<16>(), Int<1>());
  else if (width <= 256) f(Int<32>(), Int<1>());
  else if (width <= 512) f(Int<64>(), Int<1>());
  else if (width <= 1024) f(Int<64>(), Int<2>());
  else if (width <= 2048) f(Int<64>(), Int<4>());
  else if (width <= 4096) f(Int<256>(), Int<2>());
  else if (width <= 8192) f(Int<256>(), Int<4>());
  else f(Int<512>(), Int<4>());
}
constexpr int32_t kMostWidth = 16384;
int32_t rows_at_once(int32_t width) {
  int32_t rows = 0;
  by_width(width, [&](auto l, auto) { rows = 256 / std::min(256, int(l)); });
  return rows;
}

template <typename T, typename S, int MODE> void forward(const AddParams& whole, hipStream_t s) {
  by_width(whole.width, [&](auto l, auto c) {
    constexpr int L = decltype(l)::value, C = decltype(c)::value, kThreads = L > 256 ? L : 256, kRows = kThreads / L;
    const int64_t pitch = (whole.width + 15) / 16 * 16;
    in_launches((whole.tokens + kRows - 1) / kRows, kThreads, [&](uint32_t first, uint32_t groups) {
      const int64_t t0 = int64_t(first) * kRows;
      AddParams p = whole;
      p.tokens = std::min(whole.tokens - t0, int64_t(groups) * kRows);
      p.x = static_cast<const T*>(whole.x) + t0 * whole.x_row;
      if (whole.residual) p.residual = static_cast<const S*>(whole.residual) + t0 * whole.residual_row;
      if (whole.total) p.total = static_cast<S*>(whole.total) + t0 * whole.width;
      if (whole.y) p.y = static_cast<T*>(whole.y) + t0 * whole.width;
      if (whole.values) p.values = whole.values + t0 * pitch;
      if (whole.scales) p.scales = whole.scales + t0;
      if (whole.pos) p.pos = whole.pos + t0;
      add_norm_kernel<T, S, MODE, L, C><<<groups, kThreads, 0, s>>>(p);
    });
  });
}
template <int MODE> void forward_by_type(int32_t dtype, int32_t stream_dtype, const AddParams& p, hipStream_t s) {
  if (dtype == LGP_F32) forward<float, float, MODE>(p, s);
  else if (dtype == LGP_F16) stream_dtype == LGP_F32 ? forward<f16, float, MODE>(p, s) : forward<f16, f16, MODE>(p, s);
  else stream_dtype == LGP_F32 ? forward<bf16, float, MODE>(p, s) : forward<bf16, bf16, MODE>(p, s);
}
template <typename T, typename S> void backward(const AddParams& p, uint32_t groups, hipStream_t s) {
  by_width(p.width, [&](auto l, auto c) {
    constexpr int L = decltype(l)::value, C = decltype(c)::value;
    add_norm_backward_kernel<T, S, L, C><<<groups, L > 256 ? L : 256, 0, s>>>(p);
  });
}

bool known(int32_t dtype) { return dtype == LGP_F32 || dtype == LGP_F16 || dtype == LGP_BF16; }
int check_residual(const lgp_residual* r) {
  if (!r || r->tokens < 0 || r->width < 1) return LGP_EINVAL;
  if (!known(r->dtype) || (r->stream_dtype != r->dtype && r->stream_dtype != LGP_F32)) return LGP_EUNSUPPORTED;
  if (r->width > kMostWidth || r->tokens >= int64_t(1) << 33) return LGP_EUNSUPPORTED;
  if (!r->weight || reinterpret_cast<uintptr_t>(r->weight) % 4) return LGP_EINVAL;
  return std::isfinite(r->eps) && r->eps >= 0.f ? LGP_OK : LGP_EINVAL;
}
int check_forward(const lgp_residual* r, const void* total) {
  if (int st = check_residual(r)) return st;
  if (r->tokens && (!r->x || (r->residual && !total))) return LGP_EINVAL;
  return !r->residual && r->stream_dtype != r->dtype ? LGP_EINVAL : LGP_OK;
}
int check_rows(const lgp_rows8* r) {
  if (!r || r->tokens < 0 || r->width < 1) return LGP_EINVAL;
  if (r->width > kMostWidth || r->tokens >= int64_t(1) << 33) return LGP_EUNSUPPORTED;
  if (r->tokens && (!r->values || !r->scales)) return LGP_EINVAL;
  return aligned16(r->values) ? LGP_OK : LGP_EINVAL;
}
AddParams add_params(const lgp_residual* r) {
  AddParams p = {};
  p.x = r->x; p.residual = r->residual; p.x_row = r->x_row; p.residual_row = r->residual_row; p.tokens = r->tokens; p.width = r->width;
  p.weight = r->weight; p.pos = r->pos; p.eps = r->eps;
  return p;
}
// Workgroups of the backward kernel: four per CU.
int32_t backward_groups(int device, const lgp_residual* r) {
  const int64_t rows = rows_at_once(r->width);
  return int32_t(std::max<int64_t>(1, std::min((r->tokens + rows - 1) / rows, int64_t(compute_units(device)) * 4)));
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_add_norm(int device, const lgp_residual* in, void* y, void* total, void* stream) {
  if (int st = check_forward(in, total)) return st;
  if (in->tokens && !y) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (in->tokens == 0) return LGP_OK;
  AddParams p = add_params(in);
  p.y = y;
  p.total = total;
  forward_by_type<kNorm>(in->dtype, in->stream_dtype, p, static_cast<hipStream_t>(stream));
  return launched();
}

int lgp_add_norm_rows8(int device, const lgp_residual* in, const lgp_rows8* out, void* total, void* stream) {
  if (int st = check_forward(in, total)) return st;
  if (int st = check_rows(out)) return st;
  if (out->tokens != in->tokens || out->width != in->width) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (in->tokens == 0) return LGP_OK;
  AddParams p = add_params(in);
  p.values = out->values;
  p.scales = out->scales;
  p.total = total;
  forward_by_type<kNorm8>(in->dtype, in->stream_dtype, p, static_cast<hipStream_t>(stream));
  return launched();
}

int lgp_add_norm_workspace(int device, const lgp_residual* in, size_t* bytes) {
  if (!bytes) return LGP_EINVAL;
  *bytes = 0;
  if (int st = check_residual(in)) return st;
  *bytes = size_t(backward_groups(device, in)) * in->width * sizeof(float);
  return LGP_OK;
}

int lgp_add_norm_backward(int device, const lgp_residual* in, const void* dy, const void* d_total, void* dx, void* d_residual, float* d_weight, void* workspace,
                          size_t workspace_bytes, void* stream) {
  if (int st = check_residual(in)) return st;
  if (in->tokens && (!in->residual || !dy || !d_residual)) return LGP_EINVAL;
  if (!d_weight || (in->dtype == in->stream_dtype ? dx != nullptr : in->tokens && !dx)) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  AddParams p = add_params(in);
  const int32_t groups = backward_groups(device, in);
  if (workspace_bytes < size_t(groups) * in->width * sizeof(float)) return LGP_ECAPACITY;
  if (!workspace || !aligned16(workspace)) return LGP_EINVAL;
  p.dy = dy;
  p.d_total = d_total;
  p.dx = dx;
  p.d_residual = d_residual;
  p.partial = static_cast<float*>(workspace);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F32) backward<float, float>(p, groups, s);
  else if (in->dtype == LGP_F16) in->stream_dtype == LGP_F32 ? backward<f16, float>(p, groups, s) : backward<f16, f16>(p, groups, s);
  else in->stream_dtype == LGP_F32 ? backward<bf16, float>(p, groups, s) : backward<bf16, bf16>(p, groups, s);
  add_groups_kernel<<<(in->width + 31) / 32, 1024, 0, s>>>(p.partial, in->width, groups, d_weight);
  return launched();
}

int lgp_pack_rows8(int device, const void* x, int64_t x_row, int32_t dtype, const lgp_rows8* out, void* stream) {
  if (int st = check_rows(out)) return st;
  if (!known(dtype)) return LGP_EUNSUPPORTED;
  if (out->tokens && !x) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (out->tokens == 0) return LGP_OK;
  AddParams p = {};
  p.x = x;
  p.x_row = x_row;
  p.tokens = out->tokens;
  p.width = out->width;
  p.pos = out->pos;
  p.values = out->values;
  p.scales = out->scales;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == LGP_F32) forward<float, float, kPack8>(p, s);
  else if (dtype == LGP_F16) forward<f16, f16, kPack8>(p, s);
  else forward<bf16, bf16, kPack8>(p, s);
  return launched();
}

}  // extern "C"
