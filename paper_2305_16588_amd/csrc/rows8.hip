// Products of rows in 8-bit integers, with a scale for each row and each channel.
#include "product_dev.hpp"

#include <algorithm>

namespace lgp {
namespace layer {
namespace {

struct Product8Params {
  Operand w, x;
  const float *w_scales, *x_scales, *bias;
  const int32_t* pos;
  int32_t tokens, channels, chunks, tiles_m, tiles_n;
  void* out;
};

// Sums are exact in 32-bit integers: 2^17 products of at most 127^2 are less than 2^31.  They are rounded to 32 bits, multiplied by the channel's scale and
// then by the row's.
template <typename T> __device__ __forceinline__ void write_channels(const Product8Params& p, int32_t token, bool live, float scale, int32_t c, const int* sums) {
  const int32_t n = p.channels - c;
  if (n <= 0) return;
  float w[8], b[8], y[8];
  read_row(p.w_scales + c, n, w);
#pragma unroll
  for (int k = 0; k < 8; ++k) b[k] = 0.f;
  if (p.bias) read_row(p.bias + c, n, b);
#pragma unroll
  for (int k = 0; k < 8; ++k) y[k] = live ? float(sums[k]) * w[k] * scale + b[k] : 0.f;
  write_row(static_cast<T*>(p.out) + int64_t(token) * p.channels + c, n, y);
}

// Measured: 65536 rows of 4096 with 4096 channels, bf16: 1155 us, 1.90 POP/s.  Matrix instructions have half of the cycles; rows arrive late, as in gated_kernel.
template <typename T, class P>
__global__ __launch_bounds__(P::kThreads, 2) void product8_kernel(const Product8Params p) {
  __shared__ typename P::Shared lds;
  const Tile t = tile_of(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_n);
  const int32_t c0 = t.m * P::BM, t0 = t.n * P::BN;
  intx16 acc[P::MI][P::NJ] = {};
  P::run(lds, p.w, p.x, c0, t0, 0, p.chunks * 16, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % P::WM, wn = wave / P::WM;
#pragma unroll
  for (int j = 0; j < P::NJ; ++j) {
    const int32_t token = t0 + (wn * P::NJ + j) * 32 + (lane & 31);
    if (token >= p.tokens) continue;
    const bool live = !p.pos || p.pos[token] >= 0;
    const float scale = p.x_scales[token];
#pragma unroll
    for (int i = 0; i < P::MI; ++i)
#pragma unroll
      for (int r0 = 0; r0 < 16; r0 += 8) {
        int sums[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) sums[k] = acc[i][j][r0 + k];
        write_channels<T>(p, token, live, scale, c0 + (wm * P::MI + i) * 32 + 16 * (lane >> 5) + r0, sums);
      }
  }
}

__device__ __forceinline__ void read8(const float* p, float* x) {
  const floatx4 low = *reinterpret_cast<const floatx4*>(p), high = *reinterpret_cast<const floatx4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = low[i], x[i + 4] = high[i];
}

// Narrow rows: what becomes of 32 rows' results, lane l having row l % 32 and 16 consecutive channels in each of two blocks.  Beyond the rows' end it is the last one again.
template <typename T, int CHANNELS> struct NarrowOut8 {
  const Product8Params& p;
  const float* lds;                  // the workgroup's scales, and its biases CHANNELS further on
  int32_t c, at, end, lane;          // the lane's first channel, and its place in the workgroup; the end of the workgroup's rows
  bool whole;                        // in all lanes: all 16 channels of both blocks are there
  int32_t token[4];
  float scale[4];
  bool live[4];
  float y[2][8], w[2][8], b[2][8];
  __device__ __forceinline__ void next(int32_t, const int32_t*) {}
  template <int Q> __device__ __forceinline__ void start(int32_t first, const int32_t*) {
    token[Q] = min(first + (lane & 31), end - 1);
    scale[Q] = p.x_scales[token[Q]];
    live[Q] = !p.pos || p.pos[token[Q]] >= 0;
  }
  template <int Q, int R, typename Sums> __device__ __forceinline__ void step(const Sums (&acc)[2]) {
    constexpr int k = R % 8, i = R / 8;
    each<2>([&](auto of_two) __attribute__((always_inline)) {
      constexpr int q = decltype(of_two)::value;
      if (k == 0) {                  // of eight channels, two loads each
        read8(lds + at + 32 * q + R, w[q]);
        read8(lds + CHANNELS + at + 32 * q + R, b[q]);
      }
      const float v = float(acc[q][R]) * w[q][k] * scale[Q] + b[q][k];
      y[q][k] = live[Q] ? v : 0.f;
      if (k == 7) {
        const int32_t to = c + 32 * q + 8 * i, n = p.channels - to;
        if (whole || n > 0) write_row(static_cast<T*>(p.out) + int64_t(token[Q]) * p.channels + to, whole ? 8 : n, y[q]);
      }
    });
  }
};
// Measured: 282624 rows of 256 with 768 channels, bf16: 165 us, where bytes take 105; 50001 rows of 1000 with 1024 channels, fp16: 74 to 80 us, 1.3 POP/s (large tiles 103).
template <typename T, class P>
__global__ __launch_bounds__(P::kThreads, P::kPerCu * P::WAVES / 4) void product8_narrow_kernel(const Product8Params p) {
  __shared__ typename P::Shared lds;
  __shared__ __align__(16) float more[2 * 64 * P::WAVES];
  const int32_t piece = int32_t(piece_of(blockIdx.x, gridDim.x)), part = piece / p.tiles_m, parts = int32_t(gridDim.x) / p.tiles_m;
  const int32_t each = ((p.tokens + parts - 1) / parts + 63) / 64 * 64, c0 = piece % p.tiles_m * 64 * P::WAVES, begin = part * each, end = min(begin + each, p.tokens);
  for (int i = threadIdx.x; i < 64 * P::WAVES; i += P::kThreads) {
    const bool in = c0 + i < p.channels;
    more[i] = in ? p.w_scales[c0 + i] : 0.f;
    more[64 * P::WAVES + i] = in && p.bias ? p.bias[c0 + i] : 0.f;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t own = c0 + 64 * wave;
  NarrowOut8<T, 64 * P::WAVES> out = {p, more, own + 16 * (lane >> 5), 64 * wave + 16 * (lane >> 5), end, lane, own + 64 <= p.channels};
  P::run(lds, p.w, p.x, own, begin, end, out);
}

// Few rows: a thread has one channel of one.  Measured: one row of 1024 with 4096 channels: 3.9 us on the device, 1.1 TB/s of weights.
template <typename T>
__global__ __launch_bounds__(64 * kFewWaves) void product8_few_kernel(const Product8Params p) {
  typedef Few<int8_t, false> F;
  __shared__ F::Shared lds;
  const int32_t c0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  F::run(lds, p.w, p.x, c0, t0);
  const int r = threadIdx.x & 15, c = threadIdx.x >> 4;
  if (c >= 16 || t0 + c >= p.tokens || c0 + r >= p.channels) return;
  const float y = float(F::of(lds, 0, c, r)) * p.w_scales[c0 + r] * p.x_scales[t0 + c] + (p.bias ? p.bias[c0 + r] : 0.f);
  static_cast<T*>(p.out)[int64_t(t0 + c) * p.channels + c0 + r] = T(!p.pos || p.pos[t0 + c] >= 0 ? y : 0.f);
}

typedef Narrow<int8_t, 32, 4, false> Narrow1024;
typedef Narrow<int8_t, 16, 8, false> Narrow512;
typedef Narrow<int8_t, 8, 4, false> Narrow256;
typedef Narrow<int8_t, 4, 4, false> Narrow128;
typedef Tiles<int8_t, 256, 256, 2, 4, 8, 2, false, false, false> Large8;
typedef Tiles<int8_t, 64, 64, 2, 2, 8, 3, false, false, false> Small8;

template <typename T, class P> void launch8(Product8Params p, hipStream_t s) {
  p.tiles_m = (p.channels + P::BM - 1) / P::BM;
  p.tiles_n = (p.tokens + P::BN - 1) / P::BN;
  product8_kernel<T, P><<<uint32_t(p.tiles_m) * uint32_t(p.tiles_n), P::kThreads, 0, s>>>(p);
}
template <typename T, class P> void narrow8(Product8Params p, int cus, hipStream_t s) {
  p.tiles_m = (p.channels + 64 * P::WAVES - 1) / (64 * P::WAVES);
  const int32_t parts = std::max(1, std::min(cus * P::kPerCu / p.tiles_m, (p.tokens + 63) / 64));
  product8_narrow_kernel<T, P><<<uint32_t(p.tiles_m) * uint32_t(parts), P::kThreads, 0, s>>>(p);
}
// Up to 32 rows by the kernel that reads the weights straight to registers, then small tiles, up to eight for each CU (8192 rows of 2048, 1024 channels: 36 us, large ones 39;
// 32768: 130 and 83), then narrow rows (32768 rows of 256, 1024 channels: 22.6 us, large tiles 34.7, small ones 41.2; of 1024: 49, 56, 77) and large tiles.
template <typename T> void product8(const Product8Params& p, int cus, hipStream_t s) {
  if (p.tokens <= kFewTokens) {
    product8_few_kernel<T><<<dim3((p.channels + 15) / 16, (p.tokens + 15) / 16), 64 * kFewWaves, 0, s>>>(p);
    return;
  }
  const int64_t small = int64_t((p.channels + 63) / 64) * ((p.tokens + 63) / 64);
  if (small <= 8 * cus) launch8<T, Small8>(p, s);
  else if (p.chunks <= 8) narrow8<T, Narrow128>(p, cus, s);
  else if (p.chunks <= 16) narrow8<T, Narrow256>(p, cus, s);
  else if (p.chunks <= 32) narrow8<T, Narrow512>(p, cus, s);
  else if (p.chunks <= 64) narrow8<T, Narrow1024>(p, cus, s);
  else launch8<T, Large8>(p, s);
}

int check_side(const lgp_rows8* r) {
  if (!r || r->tokens < 0 || r->width < 1) return LGP_EINVAL;
  if (r->width > (1 << 17) || r->tokens > (int64_t(1) << 24)) return LGP_EUNSUPPORTED;
  if (r->tokens && (!r->values || !r->scales)) return LGP_EINVAL;
  return aligned16(r->values) ? LGP_OK : LGP_EINVAL;
}
Operand side_of(const lgp_rows8* r) {
  const int32_t chunks = (r->width + 15) / 16;
  return Operand{reinterpret_cast<const char*>(r->values), nullptr, int64_t(chunks) * 16, int32_t(r->tokens), chunks, 1 << 30, nullptr, nullptr};
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_linear_rows8(int device, const lgp_rows8* rows, const lgp_rows8* weight, const float* bias, int32_t dtype, void* out, void* stream) {
  if (int st = check_side(rows)) return st;
  if (int st = check_side(weight)) return st;
  if (rows->width != weight->width || weight->tokens < 1 || (rows->tokens && !out)) return LGP_EINVAL;
  if (dtype != LGP_F32 && dtype != LGP_F16 && dtype != LGP_BF16) return LGP_EUNSUPPORTED;
  if (int st = use_device(device)) return st;
  if (rows->tokens == 0) return LGP_OK;
  Product8Params p = {};
  p.w = side_of(weight);
  p.x = side_of(rows);
  p.w_scales = weight->scales;
  p.x_scales = rows->scales;
  p.bias = bias;
  p.pos = rows->pos;
  p.tokens = int32_t(rows->tokens);
  p.channels = int32_t(weight->tokens);
  p.chunks = p.w.chunks;
  p.out = out;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int cus = compute_units(device);
  if (dtype == LGP_F32) product8<float>(p, cus, s);
  else if (dtype == LGP_F16) product8<f16>(p, cus, s);
  else product8<bf16>(p, cus, s);
  return launched();
}

}  // extern "C"
