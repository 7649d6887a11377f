// The gated pair of projections, activation(x Wg^T) * (x Wu^T), and its gradients.
#include "product_dev.hpp"

#include <algorithm>

namespace lgp {
namespace layer {
namespace {

struct GatedParams {
  Operand w, x;                 // w: Wg and Wu
  const int32_t* pos;
  int32_t tokens, hidden, pitch;        // pitch: of half a row of `grads`
  int32_t width_chunks, tiles_m, tiles_n;
  void* h;
  const void* dh;
  void* grads;                  // [tokens][2][pitch]: the gradients of both projections' results, zeros behind hidden and where no token is
};

// a = act(g) and, for the backward pass, its slope.  silu: g s with s = 1 / (1 + exp(-g)), slope s + a (1 - s).  gelu: g P with P = erfc(-g / sqrt(2)) / 2, slope
// P + g exp(-g^2 / 2) / sqrt(2 pi).
template <int ACT, bool SLOPE> __device__ __forceinline__ float activated(float g, float& slope) {
  if constexpr (ACT == LGP_SILU) {
    const float s = rcp_fast(1.f + exp2_fast(-kLog2e * g)), a = g * s;
    if (SLOPE) slope = s + a * (1.f - s);
    return a;
  } else {
    const float p = 0.5f * erfcf(-0.70710678118654752440f * g);
    if (SLOPE) slope = p + g * (0.39894228040143267794f * exp2_fast(-0.5f * kLog2e * g * g));
    return g * p;
  }
}

template <typename T, int ACT, class P, bool BACK>
__global__ __launch_bounds__(P::kThreads, P::kThreads == 512 ? 2 : 2) void gated_kernel(const GatedParams p) {
  __shared__ typename P::Shared lds;
  const Tile t = tile_of(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_n);
  const int32_t f0 = t.m * (P::BM / 2), t0 = t.n * P::BN;
  floatx16 acc[P::MI][P::NJ] = {};
  P::run(lds, p.w, p.x, f0, t0, 0, p.width_chunks * 8, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % P::WM, wn = wave / P::WM;
#pragma unroll
  for (int j = 0; j < P::NJ; ++j) {
    const int32_t token = t0 + (wn * P::NJ + j) * 32 + (lane & 31);
    if (token >= p.tokens) continue;
    const bool live = !p.pos || p.pos[token] >= 0;
#pragma unroll
    for (int i = 0; i < P::MI / 2; ++i)
#pragma unroll
      for (int r0 = 0; r0 < 16; r0 += 8) {
        const int32_t f = f0 + (wm * (P::MI / 2) + i) * 32 + 16 * (lane >> 5) + r0, n = p.hidden - f;
        float y[8], z[8];
        if constexpr (BACK) {
          if (f >= p.pitch) continue;
          float dh[8] = {};
          if (live && n > 0) read_row(static_cast<const T*>(p.dh) + int64_t(token) * p.hidden + f, n, dh);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float slope;
            const float a = activated<ACT, true>(acc[i][j][r0 + k], slope);
            y[k] = live && k < n ? dh[k] * acc[i + P::MI / 2][j][r0 + k] * slope : 0.f;
            z[k] = live && k < n ? dh[k] * a : 0.f;
          }
          T* out = static_cast<T*>(p.grads) + int64_t(token) * 2 * p.pitch + f;
          write_row(out, 8, y);
          write_row(out + p.pitch, 8, z);
        } else {
          if (n <= 0) continue;
          float none;
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = live ? activated<ACT, false>(acc[i][j][r0 + k], none) * acc[i + P::MI / 2][j][r0 + k] : 0.f;
          write_row(static_cast<T*>(p.h) + int64_t(token) * p.hidden + f, n, y);
        }
      }
  }
}

// Few tokens: a thread has one element of h.
template <typename T, int ACT>
__global__ __launch_bounds__(64 * kFewWaves) void gated_few_kernel(const GatedParams p) {
  typedef Few<T, true> F;
  __shared__ typename F::Shared lds;
  const int32_t f0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  F::run(lds, p.w, p.x, f0, t0);
  const int r = threadIdx.x & 15, c = threadIdx.x >> 4;
  if (c >= 16 || t0 + c >= p.tokens || f0 + r >= p.hidden) return;
  float none;
  const float y = activated<ACT, false>(F::of(lds, 0, c, r), none) * F::of(lds, 1, c, r);
  static_cast<T*>(p.h)[int64_t(t0 + c) * p.hidden + f0 + r] = T(!p.pos || p.pos[t0 + c] >= 0 ? y : 0.f);
}

struct GradParams {
  Operand a, b;
  const int32_t* pos;           // of the rows of x's gradient
  int32_t rows, cols;           // of the result: tokens x width, or 2 x pitch rows of the weights' gradients x width
  int32_t hidden, pitch;        // weights: rows of each, and of each half of `rows`; x: hidden = 0
  int32_t each, sum;            // places of the sum of a part, and all of them
  int32_t tiles_m, tiles_n, parts;
  void *out, *second;
  float* partial;               // [part][rows][cols], of rows that there are
};

// dx = dg Wg + du Wu: A is the weights, across, B the gradients of the projections' results, along.  dWg = dg^T x and dWu = du^T x: A is x, across, and B those
// gradients, across.
template <typename T, class P>
__global__ __launch_bounds__(P::kThreads, 2) void grad_kernel(const GradParams p) {
  __shared__ typename P::Shared lds;
  const Tile t = tile_of(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_n);
  const int32_t c0 = t.m * P::BM, row0 = t.n * P::BN;
  floatx16 acc[P::MI][P::NJ] = {};
  const int32_t begin = t.part * p.each, end = min(begin + p.each, p.sum);
  P::run(lds, p.a, p.b, c0, row0, begin, end, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % P::WM, wn = wave / P::WM;
#pragma unroll
  for (int j = 0; j < P::NJ; ++j) {
    int32_t row = row0 + (wn * P::NJ + j) * 32 + (lane & 31);
    if (row >= p.rows) continue;
    T* out = static_cast<T*>(p.out);
    int64_t there = row;
    bool live = true;
    if (p.hidden) {
      if (row >= p.pitch) {
        row -= p.pitch;
        out = static_cast<T*>(p.second);
        there = p.hidden + row;
      }
      if (row >= p.hidden) continue;
    } else {
      live = !p.pos || p.pos[row] >= 0;
    }
#pragma unroll
    for (int i = 0; i < P::MI; ++i)
#pragma unroll
      for (int r0 = 0; r0 < 16; r0 += 8) {
        const int32_t c = c0 + (wm * P::MI + i) * 32 + 16 * (lane >> 5) + r0;
        if (c >= p.cols) continue;
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = live ? acc[i][j][r0 + k] : 0.f;
        if (p.parts > 1) write_row(p.partial + (int64_t(t.part) * (p.hidden ? 2 * int64_t(p.hidden) : p.rows) + there) * p.cols + c, 8, y);
        else write_row(out + int64_t(row) * p.cols + c, 8, y);
      }
  }
}

// Adds the parts of `n` elements each, eight a thread; those from `first` on go to `second`.
template <typename T> __global__ __launch_bounds__(256) void join_kernel(const float* partial, int64_t n, int32_t parts, T* out, int64_t first, T* second) {
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  float s[8] = {};
#pragma unroll 4
  for (int32_t k = 0; k < parts; ++k) {
    float x[8];
    read_row(partial + k * n + i, 8, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += x[e];
  }
  write_row(i < first ? out + i : second + (i - first), 8, s);
}

template <typename T> struct Forms {
  typedef Tiles<T, 256, 256, 2, 4, 4, 4, true, false, false> LargePair;
  typedef Tiles<T, 128, 256, 2, 2, 4, 3, true, false, false> MiddlePair;
  typedef Tiles<T, 128, 64, 2, 2, 8, 3, true, false, false> SmallPair;
  typedef Tiles<T, 256, 256, 2, 4, 4, 4, false, true, false> LargeX;
  typedef Tiles<T, 128, 256, 2, 2, 4, 3, false, true, false> MiddleX;
  typedef Tiles<T, 64, 64, 2, 2, 8, 3, false, true, false> SmallX;
  typedef Tiles<T, 256, 256, 2, 4, 4, 4, false, true, true> LargeW;
  typedef Tiles<T, 128, 256, 2, 2, 4, 3, false, true, true> MiddleW;
  typedef Tiles<T, 64, 64, 2, 2, 8, 3, false, true, true> SmallW;
};
enum { kLarge = 0, kMiddle = 1, kSmall = 2 };       // forms of a tile

template <typename T, int ACT, class P, bool BACK> void launch_gated(GatedParams p, hipStream_t s) {
  p.tiles_m = ((BACK ? p.pitch : p.hidden) + P::BM / 2 - 1) / (P::BM / 2);
  p.tiles_n = (p.tokens + P::BN - 1) / P::BN;
  gated_kernel<T, ACT, P, BACK><<<uint32_t(p.tiles_m) * uint32_t(p.tiles_n), P::kThreads, 0, s>>>(p);
}
template <typename T, int ACT, bool BACK> void gated_by_size(const GatedParams& p, hipStream_t s) {
  typedef Forms<T> F;
  const int f = p.tokens <= 1024 ? kSmall : kLarge;
  if (!BACK && p.tokens <= kFewTokens) {
    gated_few_kernel<T, ACT><<<dim3((p.hidden + 15) / 16, (p.tokens + 15) / 16), 64 * kFewWaves, 0, s>>>(p);
    return;
  }
  if (f == kLarge) launch_gated<T, ACT, typename F::LargePair, BACK>(p, s);
  else if (f == kMiddle) launch_gated<T, ACT, typename F::MiddlePair, BACK>(p, s);
  else launch_gated<T, ACT, typename F::SmallPair, BACK>(p, s);
}
template <typename T, bool BACK> void gated_by_act(int32_t act, const GatedParams& p, hipStream_t s) {
  if (act == LGP_SILU) gated_by_size<T, LGP_SILU, BACK>(p, s);
  else gated_by_size<T, LGP_GELU, BACK>(p, s);
}
struct GradShape { int32_t parts, each; int form; };
// Parts of the sum: as many as make 512 workgroups, of at least 512 places each.
GradShape grad_shape(int32_t rows, int32_t cols, int32_t sum, int f) {
  GradShape g;
  g.form = f;
  const int32_t bm = f == kLarge ? 256 : f == kMiddle ? 128 : 64, bn = f == kSmall ? 64 : 256;
  const int64_t tiles = std::max<int64_t>(1, int64_t((cols + bm - 1) / bm) * ((rows + bn - 1) / bn));
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(512 / tiles, sum / 512));
  g.each = std::max(64, int32_t(((sum + parts - 1) / parts + 63) / 64 * 64));
  g.parts = std::max(1, (sum + g.each - 1) / g.each);
  return g;
}
GradShape shape_x(const lgp_gated* g, int32_t pitch) { return grad_shape(int32_t(g->tokens), g->width, 2 * pitch, g->tokens <= 1024 ? kSmall : kLarge); }
GradShape shape_w(const lgp_gated* g, int32_t pitch) { return grad_shape(2 * pitch, g->width, int32_t(g->tokens), kLarge); }

template <typename T, class P> void launch_grad(GradParams p, const GradShape& g, hipStream_t s) {
  p.tiles_m = (p.cols + P::BM - 1) / P::BM;
  p.tiles_n = (p.rows + P::BN - 1) / P::BN;
  p.parts = g.parts;
  p.each = g.each;
  grad_kernel<T, P><<<uint32_t(p.tiles_m) * uint32_t(p.tiles_n) * uint32_t(g.parts), P::kThreads, 0, s>>>(p);
  if (g.parts > 1) {
    const int64_t first = p.hidden ? int64_t(p.hidden) * p.cols : int64_t(p.rows) * p.cols, n = p.hidden ? 2 * first : first;
    join_kernel<T><<<uint32_t((n / 8 + 255) / 256), 256, 0, s>>>(p.partial, n, g.parts, static_cast<T*>(p.out), first, static_cast<T*>(p.second));
  }
}

int32_t pitch_of(int32_t hidden) { return (hidden + 63) / 64 * 64; }
int check_gated(const lgp_gated* g) {
  if (!g || g->tokens < 0 || g->width < 1 || g->hidden < 1) return LGP_EINVAL;
  if (g->dtype != LGP_F16 && g->dtype != LGP_BF16) return LGP_EUNSUPPORTED;
  if (g->act != LGP_SILU && g->act != LGP_GELU) return LGP_EUNSUPPORTED;
  if (g->width % 8 || g->width > 65536 || g->hidden > 65536 || g->tokens > (int64_t(1) << 24)) return LGP_EUNSUPPORTED;
  if (!g->w_gate || !g->w_up || (g->tokens && !g->x)) return LGP_EINVAL;
  if (!aligned16(g->x) || !aligned16(g->w_gate) || !aligned16(g->w_up) || g->x_row % 8 || g->x_row < 0 || g->x_row >= (1 << 22)) return LGP_EINVAL;
  return LGP_OK;
}
GatedParams gated_params(const lgp_gated* g) {
  GatedParams p = {};
  p.w = Operand{static_cast<const char*>(g->w_gate), static_cast<const char*>(g->w_up), int64_t(g->width) * 2, g->hidden, g->width / 8, 1 << 30, nullptr};
  p.x = Operand{static_cast<const char*>(g->x), nullptr, g->x_row * 2, int32_t(g->tokens), g->width / 8, 1 << 30, nullptr};
  p.pos = g->pos;
  p.tokens = int32_t(g->tokens);
  p.hidden = g->hidden;
  p.pitch = pitch_of(g->hidden);
  p.width_chunks = g->width / 8;
  return p;
}
struct Space { size_t grads, x, w; };          // bytes of the projections' gradients, and of the parts of x's and the weights', which are not there at once
Space space_of(const lgp_gated* g) {
  const int32_t pitch = pitch_of(g->hidden);
  const GradShape x = shape_x(g, pitch), w = shape_w(g, pitch);
  return {size_t(g->tokens) * 2 * pitch * 2, x.parts > 1 ? size_t(x.parts) * g->tokens * g->width * 4 : 0, w.parts > 1 ? size_t(w.parts) * 2 * g->hidden * g->width * 4 : 0};
}

template <typename T> void backward(const lgp_gated* g, const void* dh, void* dx, void* dw_gate, void* dw_up, void* workspace, hipStream_t s) {
  typedef Forms<T> F;
  GatedParams p = gated_params(g);
  p.dh = dh;
  p.grads = workspace;
  const Space space = space_of(g);
  float* partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + space.grads);
  if (p.tokens) gated_by_act<T, true>(g->act, p, s);
  const char* grads = static_cast<const char*>(workspace);
  if (p.tokens) {
    GradParams d = {};
    d.a = Operand{p.w.first, p.w.second, p.w.row_bytes, g->hidden, g->width / 8, p.pitch, nullptr};
    d.b = Operand{grads, nullptr, int64_t(p.pitch) * 4, p.tokens, p.pitch / 4, 1 << 30, nullptr};
    d.pos = g->pos;
    d.rows = p.tokens;
    d.cols = g->width;
    d.sum = 2 * p.pitch;
    d.out = dx;
    d.partial = partial;
    const GradShape shape = shape_x(g, p.pitch);
    if (shape.form == kLarge) launch_grad<T, typename F::LargeX>(d, shape, s);
    else if (shape.form == kMiddle) launch_grad<T, typename F::MiddleX>(d, shape, s);
    else launch_grad<T, typename F::SmallX>(d, shape, s);
  }
  GradParams d = {};
  d.a = Operand{p.x.first, nullptr, p.x.row_bytes, p.tokens, g->width / 8, 1 << 30, g->pos};
  d.b = Operand{grads, nullptr, int64_t(p.pitch) * 4, p.tokens, p.pitch / 4, 1 << 30, nullptr};
  d.rows = 2 * p.pitch;
  d.cols = g->width;
  d.hidden = g->hidden;
  d.pitch = p.pitch;
  d.sum = p.tokens;
  d.out = dw_gate;
  d.second = dw_up;
  d.partial = partial;
  const GradShape shape = shape_w(g, p.pitch);
  if (shape.form == kLarge) launch_grad<T, typename F::LargeW>(d, shape, s);
  else if (shape.form == kMiddle) launch_grad<T, typename F::MiddleW>(d, shape, s);
  else launch_grad<T, typename F::SmallW>(d, shape, s);
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_gated_linear(int device, const lgp_gated* in, void* h, void* stream) {
  if (int st = check_gated(in)) return st;
  if (in->tokens && !h) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (in->tokens == 0) return LGP_OK;
  GatedParams p = gated_params(in);
  p.h = h;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F16) gated_by_act<f16, false>(in->act, p, s);
  else gated_by_act<bf16, false>(in->act, p, s);
  return launched();
}

int lgp_gated_linear_workspace(int device, const lgp_gated* in, size_t* bytes) {
  if (!bytes) return LGP_EINVAL;
  *bytes = 0;
  if (int st = check_gated(in)) return st;
  const Space s = space_of(in);
  *bytes = std::max<size_t>(16, s.grads + std::max(s.x, s.w));
  return device < 0 ? LGP_EINVAL : LGP_OK;
}

int lgp_gated_linear_backward(int device, const lgp_gated* in, const void* dh, void* dx, void* dw_gate, void* dw_up, void* workspace, size_t workspace_bytes, void* stream) {
  if (int st = check_gated(in)) return st;
  if ((in->tokens && (!dh || !dx)) || !dw_gate || !dw_up) return LGP_EINVAL;
  if (!aligned16(dx) || !aligned16(dw_gate) || !aligned16(dw_up)) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  const Space space = space_of(in);
  if (workspace_bytes < space.grads + std::max(space.x, space.w)) return LGP_ECAPACITY;
  if (!workspace || !aligned16(workspace)) return LGP_EINVAL;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F16) backward<f16>(in, dh, dx, dw_gate, dw_up, workspace, s);
  else backward<bf16>(in, dh, dx, dw_gate, dw_up, workspace, s);
  return launched();
}

}  // extern "C"
