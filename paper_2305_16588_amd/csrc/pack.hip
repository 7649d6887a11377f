// Activations held in 8 bits between the forward and the backward pass, and the gradients of a linear layer's weights and bias from them.
#include "layer_dev.hpp"

#include <algorithm>

namespace lgp {
namespace layer {
namespace {

constexpr int kGroup = 32;                    // values of a row that share a power of two
constexpr int kNotFinite = 255;               // its code where a value of the group is no finite number

// Rows need not be aligned to more than an element.
typedef f16 f16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef float floatx8_any __attribute__((ext_vector_type(8), aligned(4)));
template <typename T> struct Any;
template <> struct Any<f16> { typedef f16x8_any x8; };
template <> struct Any<bf16> { typedef bf16x8_any x8; };
template <> struct Any<float> { typedef floatx8_any x8; };
template <typename T> using any8 = typename Any<T>::x8;

template <typename T> __device__ __forceinline__ void read_any(const T* p, int n, float* x) {
  if (n >= 8) {
    const any8<T> v = *reinterpret_cast<const any8<T>*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? float(p[i]) : 0.f;
  }
}

struct PackParams {
  const void* x;
  int64_t tokens, x_row;
  int32_t width, pitch, groups, rows_each;     // rows_each: rows of a workgroup
  const int32_t* pos;
  int8_t* values;
  uint8_t* exps;
  void* out;
};

__device__ __forceinline__ float power_of(int code) { return __builtin_bit_cast(float, uint32_t(code) << 23); }   // 2^(code - 127); inf for 255

// A lane has eight values and four lanes a group.  The step is 2^(floor(log2(max |x|)) - 6), so that the largest value is 64 to 127 steps --
// what rounds to 128 is held as 127 -- and x / step, rounded to even, is exact up to that rounding.  The step is at least what the type's
// smallest numbers allow (2^-24 for fp16, 2^-126), so that a packed value is a number of the type x came in.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const PackParams p) {
  const uint32_t per_row = p.groups * 4;
  const int64_t row0 = int64_t(blockIdx.x) * p.rows_each;
  constexpr int kLeast = sizeof(T) == 2 && __is_same(T, f16) ? -24 : -126;
  for (uint32_t i = threadIdx.x; i < p.rows_each * per_row; i += 256) {
    const uint32_t r = i / per_row, c = i % per_row;
    const int64_t row = row0 + r;
    if (row >= p.tokens) break;                // whole groups of four lanes at once
    float x[8] = {};
    const int n = p.width - int(8 * c);
    if ((!p.pos || p.pos[row] >= 0) && n > 0) read_any(static_cast<const T*>(p.x) + row * p.x_row + 8 * c, n, x);
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __builtin_bit_cast(uint32_t, x[j]) & 0x7fffffffu);
    top = max(top, uint32_t(__shfl_xor(int(top), 1, 64)));
    top = max(top, uint32_t(__shfl_xor(int(top), 2, 64)));
    const int e = max(int(top >> 23) - 127 - 6, kLeast);
    const bool finite = top < 0x7f800000u;
    const float by = power_of(127 - e);
    union { int8_t b[8]; uint64_t all; } v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v.b[j] = finite ? int8_t(int(fminf(fmaxf(rintf(x[j] * by), -127.f), 127.f))) : int8_t(0);
    if (int(8 * c) < p.pitch) *reinterpret_cast<uint64_t*>(p.values + row * p.pitch + 8 * c) = v.all;
    if (c % 4 == 0) p.exps[row * p.groups + c / 4] = finite ? uint8_t(e + 127) : uint8_t(kNotFinite);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack_kernel(const PackParams p) {
  const uint32_t per_row = p.pitch / 8;
  const int64_t row0 = int64_t(blockIdx.x) * p.rows_each;
  for (uint32_t i = threadIdx.x; i < p.rows_each * per_row; i += 256) {
    const uint32_t r = i / per_row, c = i % per_row;
    const int64_t row = row0 + r;
    if (row >= p.tokens) break;
    const int n = p.width - int(8 * c);
    if (n <= 0) continue;
    union { int8_t b[8]; uint64_t all; } v;
    v.all = *reinterpret_cast<const uint64_t*>(p.values + row * p.pitch + 8 * c);
    const float step = power_of(p.exps[row * p.groups + c / 4]);      // 0 * inf: NaN
    any8<T> y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = T(float(v.b[j]) * step);
    T* out = static_cast<T*>(p.out) + row * p.width + 8 * c;
    if (n >= 8) {
      *reinterpret_cast<any8<T>*>(out) = y;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) out[j] = y[j];
    }
  }
}

struct GradParams {
  const int8_t* values;
  const uint8_t* exps;
  const void* dy;
  const int32_t* pos;
  int64_t tokens, dy_row, each;     // each: tokens of a part
  int32_t width, pitch, groups, out, tiles_w, tiles_n, parts;
  float *dw, *db;                   // [part][out][width] and [part][out]
};

// dw = dy^T x, a sum over tokens: a workgroup has 128 x 128 of dw and a part of the tokens, its four waves 64 x 64 each.  Both operands are
// read transposed from LDS.  value * 2^e has at most seven digits, so it is exact in the type of dy, and so are the products: the only
// rounding is that of the sums in 32 bits.  The workgroups of the first 128 columns add up the bias's gradient as they read dy.
template <typename T>
__global__ __launch_bounds__(256) void weight_grad_kernel(const GradParams p) {
  constexpr int BT = 64, D = 128;
  __shared__ __align__(16) T lds_y[BT * D];
  __shared__ __align__(16) T lds_x[BT * D];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t piece = piece_of(blockIdx.x, gridDim.x);
  const int32_t tw = piece % p.tiles_w, tn = piece / p.tiles_w % p.tiles_n, part = piece / p.tiles_w / p.tiles_n;
  const int32_t w0 = tw * D, n0 = tn * D;
  const int64_t t_begin = part * p.each, t_end = t_begin + p.each < p.tokens ? t_begin + p.each : p.tokens;
  floatx16 acc[2][2] = {};
  float bias[8] = {};
  const int c = tid % 16;           // a thread's eight columns
  for (int64_t t0 = t_begin; t0 < t_end; t0 += BT) {
#pragma unroll
    for (int j = 0; j < BT / 16; ++j) {
      const int r = tid / 16 + 16 * j;
      const int64_t t = t0 + r;
      float y[8] = {};
      vec8<T> xv = {}, yv;
      if (t < t_end && (!p.pos || p.pos[t] >= 0)) {
        const int n = p.out - n0 - 8 * c;
        if (n > 0) read_any(static_cast<const T*>(p.dy) + t * p.dy_row + n0 + 8 * c, n, y);
        if (w0 + 8 * c < p.pitch) {
          union { int8_t b[8]; uint64_t all; } v;
          v.all = *reinterpret_cast<const uint64_t*>(p.values + t * p.pitch + w0 + 8 * c);
          const float step = power_of(p.exps[t * p.groups + (w0 + 8 * c) / kGroup]);
#pragma unroll
          for (int i = 0; i < 8; ++i) xv[i] = T(float(v.b[i]) * step);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        yv[i] = T(y[i]);
        bias[i] += y[i];
      }
      *reinterpret_cast<vec8<T>*>(lds_y + chunk_at<D>(r, c)) = yv;
      *reinterpret_cast<vec8<T>*>(lds_x + chunk_at<D>(r, c)) = xv;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < BT / 16; ++s) {
      vec8<T> a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[i] = transposed8<T, D>(lds_y, 16 * s, 64 * (wave >> 1) + 32 * i, lane);
        b[i] = transposed8<T, D>(lds_x, 16 * s, 64 * (wave & 1) + 32 * i, lane);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = Elem<T>::mfma(a[i], b[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int n = n0 + 64 * (wave >> 1) + 32 * i + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, w = w0 + 64 * (wave & 1) + 32 * j + (lane & 31);
        if (n < p.out && w < p.width) p.dw[(int64_t(part) * p.out + n) * p.width + w] = acc[i][j][r];
      }
  if (tw == 0 && p.db) {
    float* sums = reinterpret_cast<float*>(lds_y);       // [16][128]
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[(tid / 16) * D + 8 * c + i] = bias[i];
    __syncthreads();
    if (tid < D && n0 + tid < p.out) {
      float s = 0.f;
      for (int r = 0; r < 16; ++r) s += sums[r * D + tid];
      p.db[int64_t(part) * p.out + n0 + tid] = s;
    }
  }
}

// Adds the parts, in their order.
__global__ __launch_bounds__(256) void add_parts_kernel(const float* dw_parts, const float* db_parts, int64_t n_dw, int64_t n_db, int32_t parts, float* dw, float* db) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const bool is_w = i < n_dw;
  if (i >= n_dw + n_db) return;
  const float* src = is_w ? dw_parts + i : db_parts + (i - n_dw);
  const int64_t step = is_w ? n_dw : n_db;
  float s = 0.f;
  for (int32_t k = 0; k < parts; ++k) s += src[k * step];
  (is_w ? dw[i] : db[i - n_dw]) = s;
}

int check_packed(const lgp_packed* a) {
  if (!a || a->tokens < 0 || a->width < 1) return LGP_EINVAL;
  if (a->dtype != LGP_F32 && a->dtype != LGP_F16 && a->dtype != LGP_BF16) return LGP_EUNSUPPORTED;
  if (a->width > (1 << 20) || a->tokens >= (int64_t(1) << 40)) return LGP_EUNSUPPORTED;
  if (a->tokens && (!a->values || !a->exps)) return LGP_EINVAL;
  return aligned16(a->values) ? LGP_OK : LGP_EINVAL;
}
int32_t pitch_of(int32_t width) { return (width + 15) / 16 * 16; }
PackParams pack_params(const lgp_packed* a, int32_t per_row) {
  PackParams p = {};
  p.tokens = a->tokens;
  p.width = a->width;
  p.pitch = pitch_of(a->width);
  p.groups = (a->width + kGroup - 1) / kGroup;
  p.pos = a->pos;
  p.values = a->values;
  p.exps = a->exps;
  p.rows_each = std::max<int32_t>(1, 1024 / per_row);      // about four rounds of 256 lanes
  return p;
}
// Parts of the tokens: two workgroups per CU, of at least 256 tokens each.
struct GradShape { int32_t tiles_w, tiles_n, parts; int64_t each; size_t bytes; };
GradShape grad_shape(int device, const lgp_packed* a, int32_t out) {
  GradShape g;
  g.tiles_w = (a->width + 127) / 128;
  g.tiles_n = (out + 127) / 128;
  const int64_t tiles = int64_t(g.tiles_w) * g.tiles_n, want = (int64_t(compute_units(device)) * 2 + tiles - 1) / tiles;
  const int64_t parts = std::max<int64_t>(1, std::min(want, a->tokens / 256));
  g.each = ((a->tokens + parts - 1) / parts + 63) / 64 * 64;
  g.parts = a->tokens ? int32_t((a->tokens + g.each - 1) / g.each) : 1;
  g.bytes = g.parts > 1 ? size_t(g.parts) * out * (size_t(a->width) + 1) * sizeof(float) : 0;
  return g;
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_pack_activations(int device, const void* x, int64_t x_row, const lgp_packed* out, void* stream) {
  if (int st = check_packed(out)) return st;
  if (out->tokens && !x) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (out->tokens == 0) return LGP_OK;
  PackParams p = pack_params(out, (out->width + kGroup - 1) / kGroup * 4);
  p.x = x;
  p.x_row = x_row;
  const int64_t blocks = (p.tokens + p.rows_each - 1) / p.rows_each;
  if (blocks >= int64_t(1) << 31) return LGP_EUNSUPPORTED;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (out->dtype == LGP_F32) pack_kernel<float><<<uint32_t(blocks), 256, 0, s>>>(p);
  else if (out->dtype == LGP_F16) pack_kernel<f16><<<uint32_t(blocks), 256, 0, s>>>(p);
  else pack_kernel<bf16><<<uint32_t(blocks), 256, 0, s>>>(p);
  return launched();
}

int lgp_unpack_activations(int device, const lgp_packed* in, void* x, void* stream) {
  if (int st = check_packed(in)) return st;
  if (in->tokens && !x) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (in->tokens == 0) return LGP_OK;
  PackParams p = pack_params(in, pitch_of(in->width) / 8);
  p.out = x;
  const int64_t blocks = (p.tokens + p.rows_each - 1) / p.rows_each;
  if (blocks >= int64_t(1) << 31) return LGP_EUNSUPPORTED;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F32) unpack_kernel<float><<<uint32_t(blocks), 256, 0, s>>>(p);
  else if (in->dtype == LGP_F16) unpack_kernel<f16><<<uint32_t(blocks), 256, 0, s>>>(p);
  else unpack_kernel<bf16><<<uint32_t(blocks), 256, 0, s>>>(p);
  return launched();
}

int lgp_packed_weight_grad_workspace(int device, const lgp_packed* x, int32_t out, size_t* bytes) {
  if (!bytes) return LGP_EINVAL;
  *bytes = 0;
  if (int st = check_packed(x)) return st;
  if (out < 1 || out > (1 << 20)) return LGP_EINVAL;
  *bytes = grad_shape(device, x, out).bytes;
  return LGP_OK;
}

int lgp_packed_weight_grad(int device, const lgp_packed* x, const void* dy, int64_t dy_row, int32_t dy_dtype, int32_t out, float* dw, float* db,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if (int st = check_packed(x)) return st;
  if (out < 1 || out > (1 << 20) || !dw || (x->tokens && !dy)) return LGP_EINVAL;
  if (dy_dtype != LGP_F16 && dy_dtype != LGP_BF16) return LGP_EUNSUPPORTED;
  if (dy_dtype == LGP_F16 && x->dtype != LGP_F16) return LGP_EUNSUPPORTED;      // fp16 cannot hold what was packed from a wider range
  if (int st = use_device(device)) return st;
  const GradShape g = grad_shape(device, x, out);
  if (workspace_bytes < g.bytes) return LGP_ECAPACITY;
  if (g.bytes && (!workspace || !aligned16(workspace))) return LGP_EINVAL;
  const int64_t blocks = int64_t(g.tiles_w) * g.tiles_n * g.parts;
  if (blocks >= int64_t(1) << 31) return LGP_EUNSUPPORTED;
  GradParams p = {};
  p.values = x->values;
  p.exps = x->exps;
  p.dy = dy;
  p.pos = x->pos;
  p.tokens = x->tokens;
  p.dy_row = dy_row;
  p.each = g.each;
  p.width = x->width;
  p.pitch = pitch_of(x->width);
  p.groups = (x->width + kGroup - 1) / kGroup;
  p.out = out;
  p.tiles_w = g.tiles_w;
  p.tiles_n = g.tiles_n;
  p.parts = g.parts;
  const int64_t n_dw = int64_t(out) * x->width;
  p.dw = g.parts > 1 ? static_cast<float*>(workspace) : dw;
  p.db = !db ? nullptr : g.parts > 1 ? static_cast<float*>(workspace) + n_dw * g.parts : db;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dy_dtype == LGP_F16) weight_grad_kernel<f16><<<uint32_t(blocks), 256, 0, s>>>(p);
  else weight_grad_kernel<bf16><<<uint32_t(blocks), 256, 0, s>>>(p);
  if (g.parts > 1) {
    const int64_t n_db = db ? out : 0;
    add_parts_kernel<<<uint32_t((n_dw + n_db + 255) / 256), 256, 0, s>>>(p.dw, p.db, n_dw, n_db, g.parts, dw, db);
  }
  return launched();
}

}  // extern "C"
