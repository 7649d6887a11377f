// Activations held in 8 bits between the forward and the backward pass, and the gradients of a linear layer's weights and bias from them.
#include "layer_dev.hpp"

#include <algorithm>
#include <type_traits>

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
// smallest numbers allow (2^-24 for fp16, 2^-126), so that a packed value is a number of the type x came in.  Bound by bytes.  Measured: 400 000 rows
// of 1024 values, fp16: 255 us, 4.9 TB/s.
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

// Values times their steps, exact; lanes as in pack_kernel.  Measured: 1024 rows of 100 values, fp32: 4.9 us, a launch.
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

// dw = dy^T x, a sum over tokens: a workgroup has NT x 128 of dw (NT 128 or 256) and a part of the tokens, its eight waves NT / 4 x 64 each.
// Both operands are read transposed from LDS.  While one tile of kTokens tokens is multiplied, the next is made ready -- its packed values
// are widened, rows without a token become zeros -- and the one after it is on its way to LDS (DMA: rows of dy are aligned to 16 bytes; else
// they go through registers).  value * 2^e has at most seven digits, so it is exact in the type of dy, and so are the products: the only
// rounding is that of the sums in 32 bits -- but for fp16 numbers below 2^-14, whose products lose what is below 2^-37 of the other
// factor (measured: activations of 1e-6 to 1e-5 with dy of 1 come out 1e-5 of the result off).  The workgroups of the first 128 columns add up the bias's gradient.  Columns beyond the
// operands' ends hold anything, and so do rows and columns of the result that are not written.  Measured, with 256 columns of dy: 400 000 rows of
// 1024 values, fp16: 373 to 386 us, 0.55 PFLOP/s; 1 000 003 of 256, bf16, 30 % without a token: 211 to 216 us.  No unit is full: matrix instructions have
// 34 and 30 % of the cycles, vector ones 40 and 41, LDS instructions are issued in 21 and 19; the rest are waits, for a tile at its barrier among them.
constexpr int kTokens = 32, kAhead = 256;        // of a tile; of which exponents and positions are held
template <typename T, int NT, bool DMA>
__global__ __launch_bounds__(512, 4) void weight_grad_kernel(const GradParams p) {
  constexpr int WT = 128, NB = NT / 128, NC = NT / 8, NJ = kTokens * NC / 512;       // NB: blocks of 32 rows of a wave; NC: chunks of eight in a row
  __shared__ __align__(16) T lds_y[3][kTokens * NT];
  __shared__ __align__(16) uint8_t lds_raw[3][kTokens * WT];
  __shared__ __align__(16) T lds_x[2][kTokens * WT];
  __shared__ uint32_t lds_exps[2][kAhead];
  __shared__ uint8_t lds_gone[2][kAhead];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t piece = piece_of(blockIdx.x, gridDim.x);
  const int32_t tw = piece % p.tiles_w, tn = piece / p.tiles_w % p.tiles_n, part = piece / p.tiles_w / p.tiles_n;
  const int32_t w0 = tw * WT, n0 = tn * NT;
  const int64_t t_begin = part * p.each, t_end = t_begin + p.each < p.tokens ? t_begin + p.each : p.tokens;
  const int32_t tokens = int32_t(t_end - t_begin), tiles = (tokens + kTokens - 1) / kTokens;
  const T* dy = static_cast<const T*>(p.dy) + t_begin * p.dy_row + n0;
  const int8_t* values = p.values + t_begin * p.pitch + w0;
  const bool sums = tw == 0 && p.db;
  const int yc = tid % NC, yr = tid / NC;        // a thread's chunk of dy, and its first row
  floatx16 acc[NB][2] = {};
  float bias[8] = {};
  const Places<T, NT> at_y(lane);
  const Places<T, WT> at_x(lane);

  vec8<T> held[DMA ? 1 : NJ];
  auto fetch = [&](int32_t i, int to) {
    if (i >= tiles) return;
    const int32_t t0 = i * kTokens;
    if constexpr (DMA) {
      copy_tile<T, NT, kTokens, 512>(lds_y[to], Rows<T>{dy, p.dy_row, 0, 0}, t0, p.out - n0, tokens - t0, tid);
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const T* src = dy + int64_t(min(t0 + yr + j * (512 / NC), tokens - 1)) * p.dy_row + 8 * yc;
        const int n = p.out - n0 - 8 * yc;
        vec8<T> v = {};
        if (n >= 8) v = *reinterpret_cast<const any8<T>*>(src);
        else
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (k < n) v[k] = src[k];
        held[j] = v;
      }
    }
    if (tid < kTokens * WT / 16) {
      const int r = tid / (WT / 16), c = tid % (WT / 16);
      if (w0 + 16 * c < p.pitch)
        copy16(values + int64_t(t0) * p.pitch, uint32_t(min(r, tokens - 1 - t0)) * p.pitch + 16 * c,
               __builtin_amdgcn_readfirstlane(lds_address(lds_raw[to]) + (tid & ~63) * 16));
    }
  };
  auto arrived = [&](int32_t i, int at) {        // in this wave: passed on by the next barrier
    loads_done();
    if constexpr (!DMA) {
      if (i < tiles)
#pragma unroll
        for (int j = 0; j < NJ; ++j) *reinterpret_cast<vec8<T>*>(lds_y[at] + chunk_at<NT>(yr + j * (512 / NC), yc)) = held[j];
    }
  };
  // Exponents of the four groups and the presence of each of the next kAhead tokens, a thread a token.
  uint32_t exps = 0;
  int32_t pos = 0;
  auto look = [&](int32_t block) {
    const int32_t t = block * kAhead + tid;
    exps = 0;
    pos = -1;
    if (tid < kAhead && t < tokens) {
      pos = p.pos ? p.pos[t_begin + t] : 0;
      const uint8_t* e = p.exps + (t_begin + t) * p.groups + w0 / kGroup;
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (w0 / kGroup + g < p.groups) exps |= uint32_t(e[g]) << (8 * g);
    }
  };
  auto note = [&](int32_t block) {
    if (tid < kAhead) {
      lds_exps[block & 1][tid] = exps;
      lds_gone[block & 1][tid] = pos < 0;
    }
  };
  auto ready = [&](int32_t i, int at, int to) {
    if (i >= tiles) return;
    const int block = i / (kAhead / kTokens) & 1, t0 = i % (kAhead / kTokens) * kTokens;
    {
      const int r = tid / (WT / 8), c = tid % (WT / 8);
      const uint64_t x = *reinterpret_cast<const uint64_t*>(lds_raw[at] + r * WT + 8 * c) ^ 0x8080808080808080ull;       // plus 128: bytes without a sign
      const float step = lds_gone[block][t0 + r] ? 0.f : power_of(lds_exps[block][t0 + r] >> (8 * (c / 4)) & 255);
      vec8<T> v;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = T((float(uint8_t(x >> (8 * k))) - 128.f) * step);        // not less 128 steps: those may be infinite
      *reinterpret_cast<vec8<T>*>(lds_x[to] + chunk_at<WT>(r, c)) = v;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int r = yr + j * (512 / NC);
      vec8<T>* y = reinterpret_cast<vec8<T>*>(lds_y[at] + chunk_at<NT>(r, yc));
      if (lds_gone[block][t0 + r]) {
        const vec8<T> zero = {};
        *y = zero;
      } else if (sums) {
        const vec8<T> v = *y;
#pragma unroll
        for (int k = 0; k < 8; ++k) bias[k] += float(v[k]);
      }
    }
  };
  if (tiles > 0) {
    look(0);
    fetch(0, 0);
    note(0);
    arrived(0, 0);
    __syncthreads();
    fetch(1, 1);
    ready(0, 0, 0);
  }
  auto step = [&](int32_t i, auto of_six) {
    constexpr int y_at = decltype(of_six)::value % 3, x_at = decltype(of_six)::value % 2, kEach = kAhead / kTokens;
    if (i % kEach == kEach / 2) note(i / kEach + 1);
    arrived(i + 1, (y_at + 1) % 3);
    __syncthreads();
    if (i % kEach == 0) look(i / kEach + 1);
    fetch(i + 2, (y_at + 2) % 3);
    ready(i + 1, (y_at + 1) % 3, x_at ^ 1);
#pragma unroll
    for (int s = 0; s < kTokens / 16; ++s) {
      vec8<T> a[NB], b[2];
#pragma unroll
      for (int k = 0; k < NB; ++k) a[k] = at_y.across(lds_y[y_at], 16 * s, NT / 4 * (wave >> 1) + 32 * k);
#pragma unroll
      for (int k = 0; k < 2; ++k) b[k] = at_x.across(lds_x[x_at], 16 * s, 64 * (wave & 1) + 32 * k);
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[k][j] = Elem<T>::mfma(a[k], b[j], acc[k][j]);
    }
  };
  for (int32_t i = 0; i < tiles; i += 6) {       // places of tiles are constants in each of six copies
    step(i, std::integral_constant<int, 0>());
    if (i + 1 < tiles) step(i + 1, std::integral_constant<int, 1>());
    if (i + 2 < tiles) step(i + 2, std::integral_constant<int, 2>());
    if (i + 3 < tiles) step(i + 3, std::integral_constant<int, 3>());
    if (i + 4 < tiles) step(i + 4, std::integral_constant<int, 4>());
    if (i + 5 < tiles) step(i + 5, std::integral_constant<int, 5>());
  }
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int n = n0 + NT / 4 * (wave >> 1) + 32 * i + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, w = w0 + 64 * (wave & 1) + 32 * j + (lane & 31);
        if (n < p.out && w < p.width) p.dw[(int64_t(part) * p.out + n) * p.width + w] = acc[i][j][r];
      }
  if (sums) {
    __syncthreads();
    float* rows = reinterpret_cast<float*>(lds_y);         // [512 / NC][NT]
#pragma unroll
    for (int i = 0; i < 8; ++i) rows[yr * NT + 8 * yc + i] = bias[i];
    __syncthreads();
    if (tid < NT && n0 + tid < p.out) {
      float s = 0.f;
      for (int r = 0; r < 512 / NC; ++r) s += rows[r * NT + tid];
      p.db[int64_t(part) * p.out + n0 + tid] = s;
    }
  }
}

// Adds the parts: eight lanes of a workgroup's 256 take every eighth part of a value each, and are added in their order.  Measured: 64 parts of
// 256 x 1024, 17 us; 253 of 256 x 256, 20 us.
__global__ __launch_bounds__(256) void add_parts_kernel(const float* dw_parts, const float* db_parts, int64_t n_dw, int64_t n_db, int32_t parts, float* dw, float* db) {
  __shared__ float lds[8][32];
  const int at = threadIdx.x & 31, first = threadIdx.x >> 5;
  const int64_t i = int64_t(blockIdx.x) * 32 + at;
  const bool is_w = i < n_dw, in = i < n_dw + n_db;
  const float* src = is_w ? dw_parts + i : db_parts + (i - n_dw);
  const int64_t step = is_w ? n_dw : n_db;
  float s = 0.f;
  if (in)
    for (int32_t k = first; k < parts; k += 8) s += src[k * step];
  lds[first][at] = s;
  __syncthreads();
  if (!in || first) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) s += lds[k][at];
  (is_w ? dw[i] : db[i - n_dw]) = s;
}

template <typename T> void launch_grad(const GradParams& p, int32_t rows, uint32_t blocks, hipStream_t s) {
  const bool dma = p.out % 8 == 0 && p.dy_row % 8 == 0 && p.dy_row >= 0 && p.dy_row < kMostStride && aligned16(p.dy);
  if (rows == 128) dma ? weight_grad_kernel<T, 128, true><<<blocks, 512, 0, s>>>(p) : weight_grad_kernel<T, 128, false><<<blocks, 512, 0, s>>>(p);
  else dma ? weight_grad_kernel<T, 256, true><<<blocks, 512, 0, s>>>(p) : weight_grad_kernel<T, 256, false><<<blocks, 512, 0, s>>>(p);
}

int check_packed(const lgp_packed* a) {
  if (!a || a->tokens < 0 || a->width < 1) return LGP_EINVAL;
  if (a->dtype != LGP_F32 && a->dtype != LGP_F16 && a->dtype != LGP_BF16) return LGP_EUNSUPPORTED;
  if (a->width > (1 << 20) || a->tokens >= int64_t(1) << 31) return LGP_EUNSUPPORTED;
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
  while (p.tokens / p.rows_each >= int64_t(1) << 23) p.rows_each *= 2;       // a launch has less than 2^32 threads
  return p;
}
// Parts of the tokens: two workgroups per CU, of at least 256 tokens each.
struct GradShape { int32_t rows, tiles_w, tiles_n, parts; int64_t each; size_t bytes; };
GradShape grad_shape(int device, const lgp_packed* a, int32_t out) {
  GradShape g;
  g.tiles_w = (a->width + 127) / 128;
  g.rows = out <= 128 ? 128 : 256;
  g.tiles_n = (out + g.rows - 1) / g.rows;
  const int64_t tiles = int64_t(g.tiles_w) * g.tiles_n, want = std::max<int64_t>(1, int64_t(compute_units(device)) * 2 / tiles);
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
  if (dy_dtype == LGP_F16) launch_grad<f16>(p, g.rows, uint32_t(blocks), s);
  else launch_grad<bf16>(p, g.rows, uint32_t(blocks), s);
  if (g.parts > 1) {
    const int64_t n_db = db ? out : 0;
    add_parts_kernel<<<uint32_t((n_dw + n_db + 31) / 32), 256, 0, s>>>(p.dw, p.db, n_dw, n_db, g.parts, dw, db);
  }
  return launched();
}

}  // extern "C"
