// The gated pair of projections, activation(x Wg^T) * (x Wu^T), and its gradients.
#include "product_dev.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace lgp {
namespace layer {
namespace {

struct GatedParams {
  Operand w, x;                 // w: Wg and Wu
  const int32_t *pos, *count;           // with x.order, count: how many tokens there are, and pos is NULL
  int32_t tokens, hidden, pitch;        // pitch: of half a row of `grads`
  int32_t width_chunks, tiles_m, tiles_n;
  void* h;
  const void* dh;
  // [tokens][2][pitch]: the gradients of both projections' results, zeros behind hidden and where no token is.  They are rounded to 16 bits, as the matrix instructions want
  // them: gradients are off by 2.3e-3 (bf16) and 2.9e-4 (fp16) where a result that is rounded once is by 1.7e-3 and 2.1e-4; a second part of 16 bits for what the
  // rounding takes off would double the operations of both gradients' products, 3.9 of 8.8 ms for 32768 rows of 2048 with 8192 hidden.
  void* grads;
  const float* lift;            // fp16: what those are multiplied by, and its reciprocal; see lift_kernel
};
template <typename T> constexpr bool kLifted = std::is_same_v<T, f16>;

// a = act(g) and, for the backward pass, its slope.  silu: g s with s = 1 / (1 + exp(-g)), slope s + a (1 - s), where s is 1 from g of 17 on: a - a s in
// place of a (1 - s) would lose it beside an a of 2^24 and more.  gelu: g P with P = erfc(-g / sqrt(2)) / 2, slope
// P + g exp(-g^2 / 2) / sqrt(2 pi).  With x = |g| / sqrt(2) the smaller of P and 1 - P is exp(-x^2) t q(t), t = 1 / (1 + 0.36 x): a polynomial through t q(t) = exp(x^2) erfc(x) / 2 at
// the ten Chebyshev nodes of (0, 1], which is off by at most 5e-8 of it, so that the tail keeps its digits (calling erfcf instead: 32768 rows of 2048 with 8192 hidden, fp16,
// forward 2588 us).
template <int ACT, bool SLOPE> __device__ __forceinline__ float activated(float g, float& slope) {
  if constexpr (ACT == LGP_SILU) {
    const float s = rcp_fast(1.f + exp2_fast(-kLog2e * g)), a = g * s;
    if (SLOPE) slope = fmaf(a, 1.f - s, s);
    return a;
  } else {
    const float t = rcp_fast(1.f + 2.545584413e-01f * fabsf(g)), e = exp2_fast(g * g * (-0.5f * kLog2e));
    float q = 1.914578963e-02f;
    q = q * t - 7.248302199e-02f;
    q = q * t + 7.469616717e-02f;
    q = q * t - 1.753483407e-02f;
    q = q * t + 5.528966375e-02f;
    q = q * t + 6.070376850e-02f;
    q = q * t + 8.211907949e-02f;
    q = q * t + 9.495467540e-02f;
    q = q * t + 1.015546063e-01f;
    q = q * t + 1.015541227e-01f;
    const float tail = q * t * e, p = g < 0.f ? tail : 1.f - tail;
    if (SLOPE) slope = p + g * (0.39894228040143267794f * e);
    return g * p;
  }
}

// A tile of both projections, and what becomes of them.  Measured: 32768 rows of 2048 with 8192 hidden, fp16, gelu: 2200 to 2300 us, 0.98 PFLOP/s of products; with the projections' gradients
// in place of h 2570 to 2620 us.  Matrix instructions have half of the cycles; the activation is worked on after the products, and the next stage's rows arrive late (the same
// with rows that are always cached: a tenth less; without any copies: a quarter).
template <typename T, int ACT, class P, bool BACK>
__global__ __launch_bounds__(P::kThreads, 2) void gated_kernel(const GatedParams p) {
  __shared__ typename P::Shared lds;
  const int32_t tokens = p.count ? *fixed(p.count) : p.tokens, tiles_n = (tokens + P::BN - 1) / P::BN;
  if (int32_t(blockIdx.x) >= p.tiles_m * tiles_n) return;
  const Tile t = tile_of(blockIdx.x, p.tiles_m * tiles_n, p.tiles_m, tiles_n);
  const int32_t f0 = t.m * (P::BM / 2), t0 = t.n * P::BN;
  floatx16 acc[P::MI][P::NJ] = {};
  Operand x = p.x;
  x.rows = tokens;
  P::run(lds, p.w, x, f0, t0, 0, p.width_chunks * 8, acc);
  float lift = 1.f;
  if constexpr (BACK && kLifted<T>) lift = p.lift[0];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % P::WM, wn = wave / P::WM;
#pragma unroll
  for (int j = 0; j < P::NJ; ++j) {
    const int32_t row = t0 + (wn * P::NJ + j) * 32 + (lane & 31);
    if (row >= tokens) continue;
    const int32_t token = x.order ? x.order[row] : row;
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
            if (kLifted<T>) dh[k] *= lift;
            y[k] = live && k < n ? dh[k] * acc[i + P::MI / 2][j][r0 + k] * slope : 0.f;
            z[k] = live && k < n ? dh[k] * a : 0.f;
          }
          T* out = static_cast<T*>(p.grads) + int64_t(row) * 2 * p.pitch + f;
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

// Narrow rows: what becomes of 32 tokens' results, lane l having token l % 32 and 16 consecutive hidden elements.  Loads and stores are made whatever there is to load and
// store -- beyond the rows' end the last one's again -- but for what is behind hidden: the compiler counts those that are under way, and takes the fewest.
template <typename T, int ACT, bool BACK> struct NarrowOut {
  const GatedParams& p;
  int32_t f, end, lane;              // the lane's first hidden element; the end of the workgroup's rows
  bool whole;                        // in all lanes: 16 hidden elements are there
  float lift;
  int32_t row[4], token[4];          // of the list, and of memory
  vec8<T> dh[2], y, z;               // the gradients of h are on their way as soon as those before them are used
  float held_y, held_z;
  __device__ __forceinline__ int32_t clamped(int32_t first) const { return min(first + (lane & 31), end - 1); }
  __device__ __forceinline__ int32_t token_of(int32_t first, const int32_t* listed) const {
    return p.x.order ? listed[max(0, min(lane & 31, end - 1 - first))] : clamped(first);
  }
  template <int Q> __device__ __forceinline__ void start(int32_t first, const int32_t* listed) {
    row[Q] = clamped(first);
    if constexpr (!BACK) token[Q] = token_of(first, listed);
  }
  __device__ __forceinline__ void next(int32_t first, const int32_t* listed) {
    if constexpr (BACK) {
      if (first >= end) return;
      const T* from = static_cast<const T*>(p.dh) + int64_t(token_of(first, listed)) * p.hidden;
#pragma unroll
      for (int i = 0; i < 2; ++i) dh[i] = *reinterpret_cast<const typename AnyEight<T>::x8*>(from + min(f + 8 * i, p.hidden - 8));
    }
  }
  // Behind hidden the last eight of the row were read: those that are before these are shifted out.
  __device__ __forceinline__ void shift() {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int by = 16 * min(8, f + 8 * i - min(f + 8 * i, p.hidden - 8));
      union { vec8<T> v; uint64_t half[2]; } u;
      u.v = dh[i];
      if (by >= 64) u.half[0] = u.half[1], u.half[1] = 0;
      if (by >= 128) u.half[0] = 0;
      if (by & 63) u.half[0] = u.half[0] >> (by & 63) | u.half[1] << (64 - (by & 63)), u.half[1] >>= by & 63;
      dh[i] = u.v;
    }
  }
  template <int Q, int R, typename Sums> __device__ __forceinline__ void step(const Sums (&acc)[2]) {
    constexpr int k = R % 8, i = R / 8;
    float slope = 0.f;
    const float a = activated<ACT, BACK>(acc[0][R], slope);
    if constexpr (BACK) {
      if (R == 0 && !whole) shift();
      const float d = kLifted<T> ? float(dh[i][k]) * lift : float(dh[i][k]);           // zero behind hidden, and so are the results
      add<k>(y, held_y, d * acc[1][R] * slope);
      add<k>(z, held_z, d * a);
      if (k == 7) {
        T* out = static_cast<T*>(p.grads) + int64_t(row[Q]) * 2 * p.pitch + f + 8 * i;
        *reinterpret_cast<vec8<T>*>(out) = y;
        *reinterpret_cast<vec8<T>*>(out + p.pitch) = z;
      }
    } else {
      add<k>(y, held_y, a * acc[1][R]);
      if (k == 7) {
        T* out = static_cast<T*>(p.h) + int64_t(token[Q]) * p.hidden + f + 8 * i;
        const int n = p.hidden - f - 8 * i;
        if (whole || n >= 8) *reinterpret_cast<typename AnyEight<T>::x8*>(out) = y;
        else
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < n) out[e] = y[e];
      }
    }
  }
  // Two at a time are rounded, so that they take one register.
  template <int K> static __device__ __forceinline__ void add(vec8<T>& v, float& held, float x) {
    if constexpr (K % 2 == 0) held = x;
    else v[K - 1] = T(held), v[K] = T(x);
  }
};
// Measured: 282624 rows of 256, 30 % of them left out, 683 hidden, bf16, silu: h 187 us (tiles, of all rows: 335), the projections' gradients 345 us, where their bytes take 77 and 195.
template <typename T, int ACT, class P, bool BACK>
__global__ __launch_bounds__(P::kThreads, P::kPerCu * P::WAVES / 4) void gated_narrow_kernel(const GatedParams p) {
  __shared__ typename P::Shared lds;
  // workgroups of one part of the tokens, which read the same rows, are on one XCD
  const int32_t piece = int32_t(piece_of(blockIdx.x, gridDim.x)), part = piece / p.tiles_m, parts = int32_t(gridDim.x) / p.tiles_m;
  const int32_t rows = p.count ? *fixed(p.count) : p.tokens, each = ((rows + parts - 1) / parts + 63) / 64 * 64;
  const int32_t f0 = piece % p.tiles_m * 32 * P::WAVES, begin = part * each, end = min(begin + each, rows);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // waves behind the last hidden element do what those before them do
  const int32_t own = min(f0 + 32 * __builtin_amdgcn_readfirstlane(wave), ((BACK ? p.pitch : p.hidden) - 1) / 32 * 32);
  NarrowOut<T, ACT, BACK> out = {p, own + 16 * (lane >> 5), end, lane, own + 32 <= p.hidden, BACK && kLifted<T> ? p.lift[0] : 1.f};
  P::run(lds, p.w, p.x, own, begin, end, out);
}

// Tokens that there are, in order: a workgroup has kListed of them.  First it counts them, then, knowing how many come before, it lists them and fills the rows of
// `zeros` (cols wide) that have none.
// Measured: 282624 rows: counted in 5 us; listed, with zeros in 30 % of them, in 44 (683 wide) and 23 us (256).
constexpr int32_t kListed = 1024;
__global__ __launch_bounds__(256) void count_kernel(const int32_t* pos, int32_t tokens, int32_t* counts) {
  int32_t n = 0;
  for (int i = threadIdx.x; i < kListed; i += 256) {
    const int32_t t = blockIdx.x * kListed + i;
    n += __popcll(__ballot(t < tokens && pos[t < tokens ? t : 0] >= 0));
  }
  __shared__ int32_t lds[4];
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) counts[blockIdx.x] = lds[0] + lds[1] + lds[2] + lds[3];
}
template <typename T>
__global__ __launch_bounds__(256) void list_kernel(const int32_t* pos, int32_t tokens, const int32_t* counts, int32_t* order, int32_t* count, T* zeros, int32_t cols) {
  __shared__ int32_t lds[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t before = 0;
  for (uint32_t i = threadIdx.x; i < blockIdx.x; i += 256) before += counts[i];
#pragma unroll
  for (int i = 32; i; i >>= 1) before += __shfl_xor(before, i, 64);
  if (lane == 0) lds[wave] = before;
  __syncthreads();
  before = lds[0] + lds[1] + lds[2] + lds[3];
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *count = before + counts[blockIdx.x];
  for (int i = 0; i < kListed; i += 64) {        // every wave looks at all of them, and each fills rows of its own
    const int32_t t = blockIdx.x * kListed + i + lane;
    const uint64_t there = __ballot(t < tokens && pos[t < tokens ? t : 0] >= 0), all = __ballot(t < tokens);
    if (wave == 0 && (there >> lane & 1)) order[before + __popcll(there & ((uint64_t(1) << lane) - 1))] = t;
    before += __popcll(there);
    uint64_t gone = all & ~there & (uint64_t(0xffff) << (16 * wave));
    while (gone) {
      const int64_t row = int64_t(blockIdx.x) * kListed + i + __ffsll((unsigned long long)gone) - 1;
      gone &= gone - 1;
      const float nothing[8] = {};
      for (int32_t c = 8 * lane; c < cols; c += 512) write_row(zeros + row * cols + c, cols - c, nothing);
    }
  }
}

// fp16, backward.  The gradients of the projections' results are kept in 16 bits between the products, whose range is that of their inputs and results but not theirs: dh u
// act'(g) may pass 65504 or vanish below 2^-25 where dx and dW do neither.  All of them are lifted by one power of two, which both products take back from their sums:
// |dg| <= 1.13 |dh| |x| |w_up| and |du| <= |dh| |x| |w_gate| (|x|, |w|: norms of rows), so with B the largest |dh| |x| of a token times the largest |w| they end below
// 2^15, whatever they are.  The bound is some 2^3 beyond the largest, of 2^30 that fp16 has; what is below B 2^-27 is off by up to B 2^-38.  bf16 has the range.  Numbers that are not finite
// spoil their own rows and are left out.  Sixteen lanes read a row; bound by bytes.  Measured: 32768 rows of 2048 with 8192 hidden
// 160 us, 4.6 TB/s; 282624 of 256 with 683 hidden, 30 % left out, 137 us, 2.7 TB/s (odd rows); 300 rows 4.7, and 1.6 to 4.8 us for the power of two.
constexpr uint32_t kBoundGroups = 2048;
struct BoundParams {
  const char *x, *w_gate, *w_up;
  int64_t x_bytes;               // of a row
  const f16* dh;
  const int32_t* pos;
  int32_t tokens, width, hidden;
  float* partial;                // [2][workgroup]: of tokens, and of the weights' squares
};
__device__ __forceinline__ void finite8(const f16* p, int n, float* x) {
  read_row(p, n, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fabsf(x[i]) < INFINITY ? fabsf(x[i]) : 0.f;
}
__device__ __forceinline__ float group_max(float x, float* lds) {        // over 16 lanes each of the workgroup's sixteen groups, in all threads; no number is negative
  if ((threadIdx.x & 15) == 0) lds[threadIdx.x >> 4] = x;
  __syncthreads();
  x = lds[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) x = fmaxf(x, lds[i]);
  return x;
}
__global__ __launch_bounds__(256) void bound_kernel(const BoundParams p) {
  __shared__ float lds[2][16];
  const int lane = threadIdx.x & 15;
  float of_tokens = 0.f, of_weights = 0.f;
  for (int32_t r = int32_t(blockIdx.x) * 16 + (threadIdx.x >> 4); r < p.tokens + 2 * p.hidden; r += int32_t(gridDim.x) * 16) {
    const bool token = r < p.tokens;
    if (token && p.pos && p.pos[r] < 0) continue;
    const int32_t f = r - p.tokens;
    const char* row = token ? p.x + r * p.x_bytes : f < p.hidden ? p.w_gate + int64_t(f) * p.width * 2 : p.w_up + int64_t(f - p.hidden) * p.width * 2;
    float squares = 0.f, most = 0.f;
#pragma unroll 4
    for (int32_t c = 8 * lane; c < p.width; c += 128) {
      float x[8];
      finite8(reinterpret_cast<const f16*>(row) + c, 8, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) squares += x[i] * x[i];
    }
    squares = lanes_sum<16>(squares);
    if (token) {
#pragma unroll 4
      for (int32_t c = 8 * lane; c < p.hidden; c += 128) {
        float x[8];
        finite8(p.dh + int64_t(r) * p.hidden + c, p.hidden - c, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, x[i]);
      }
      most = __builtin_bit_cast(float, lanes_max<16>(__builtin_bit_cast(uint32_t, most)));
      of_tokens = fmaxf(of_tokens, most * sqrtf(squares));
    } else {
      of_weights = fmaxf(of_weights, squares);
    }
  }
  of_tokens = group_max(of_tokens, lds[0]);
  of_weights = group_max(of_weights, lds[1]);
  if (threadIdx.x == 0) p.partial[blockIdx.x] = of_tokens, p.partial[gridDim.x + blockIdx.x] = of_weights;
}
// lift[0]: the power of two, lift[1]: its reciprocal.
__global__ __launch_bounds__(256) void lift_kernel(const float* partial, int32_t groups, float* lift) {
  __shared__ float lds[2][16];
  float x[2] = {};
#pragma unroll 8
  for (int32_t i = threadIdx.x; i < groups; i += 256)
#pragma unroll
    for (int q = 0; q < 2; ++q) x[q] = fmaxf(x[q], partial[q * groups + i]);
#pragma unroll
  for (int q = 0; q < 2; ++q) x[q] = group_max(__builtin_bit_cast(float, lanes_max<16>(__builtin_bit_cast(uint32_t, x[q]))), lds[q]);
  const float bound = 1.2f * x[0] * sqrtf(x[1]);               // 1.13, and the rounding of the sums
  const int up = bound > 0.f ? 14 - (int(__builtin_bit_cast(uint32_t, bound) >> 23) - 127) : 0;
  if (threadIdx.x == 0) lift[0] = ldexpf(1.f, up), lift[1] = ldexpf(1.f, -up);
}

// Few tokens: a thread has one element of h.  Measured: one token, 1024 to 4096, bf16: 4.8 us on the device, 3.5 TB/s of weights.
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

// Few tokens, backward: the projections' gradients are kept in 32 bits, since hardly any sum would average their rounding, and both products that follow are memory's work: each
// weight is read, and each of its gradients written, once for eight tokens or all of them.
struct FewParams {
  const char *w_gate, *w_up, *x;
  int64_t x_bytes;               // of a row
  const int32_t* pos;
  int32_t tokens, width, hidden, pitch;
  float* grads;                  // [tokens][2][pitch], zeros where no token is
  float* partial;                // [part][tokens][width]
  void *dw_gate, *dw_up;
};
template <typename T, int ACT>
__global__ __launch_bounds__(64 * kFewWaves) void few_grads_kernel(const GatedParams p) {
  typedef Few<T, true> F;
  __shared__ typename F::Shared lds;
  const int32_t f0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  F::run(lds, p.w, p.x, f0, t0);
  const int r = threadIdx.x & 15, c = threadIdx.x >> 4;
  const int32_t f = f0 + r, token = t0 + c;
  if (c >= 16 || token >= p.tokens || f >= p.hidden) return;
  float dg = 0.f, du = 0.f;
  if (!p.pos || p.pos[token] >= 0) {
    const float dh = float(static_cast<const T*>(p.dh)[int64_t(token) * p.hidden + f]);
    float slope;
    const float a = activated<ACT, true>(F::of(lds, 0, c, r), slope);
    dg = dh * F::of(lds, 1, c, r) * slope;
    du = dh * a;
  }
  float* out = static_cast<float*>(p.grads) + int64_t(token) * 2 * p.pitch + f;
  out[0] = dg;
  out[p.pitch] = du;
}
// 256 columns of dx for eight tokens, from kFewHidden rows of both weights: a thread has eight columns and every eighth row, whose sums are added in LDS.
constexpr int kFewHidden = 128, kFewBack = 8;
template <typename T>
__global__ __launch_bounds__(256) void few_x_kernel(const FewParams p) {
  __shared__ float d[2][kFewHidden][8];
  __shared__ __align__(16) float sums[8][256];
  const int32_t t0 = blockIdx.y * 8, f0 = blockIdx.z * kFewHidden, n = min(kFewHidden, p.hidden - f0);
  for (int i = threadIdx.x; i < 2 * kFewHidden * 8; i += 256) {
    const int q = i / (kFewHidden * 8), f = i / 8 % kFewHidden, t = i % 8;
    d[q][f][t] = f < n && t0 + t < p.tokens ? p.grads[int64_t(t0 + t) * 2 * p.pitch + q * p.pitch + f0 + f] : 0.f;
  }
  __syncthreads();
  const int lane = threadIdx.x >> 5, c = blockIdx.x * 256 + 8 * (threadIdx.x & 31);
  float acc[8][8] = {};
  if (c < p.width) {
#pragma unroll 4
    for (int f = lane; f < n; f += 8) {
      float g[8], u[8];
      read_row(reinterpret_cast<const T*>(p.w_gate) + int64_t(f0 + f) * p.width + c, 8, g);
      read_row(reinterpret_cast<const T*>(p.w_up) + int64_t(f0 + f) * p.width + c, 8, u);
#pragma unroll
      for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[t][k] += d[0][f][t] * g[k] + d[1][f][t] * u[k];
    }
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) sums[lane][8 * (threadIdx.x & 31) + k] = acc[t][k];
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int l = 0; l < 8; ++l) s += sums[l][threadIdx.x];
    const int32_t at = blockIdx.x * 256 + threadIdx.x;
    if (at < p.width && t0 + t < p.tokens) p.partial[(int64_t(blockIdx.z) * p.tokens + t0 + t) * p.width + at] = s;
  }
}
// Eight columns of a row of both weights' gradients by each thread.
template <typename T>
__global__ __launch_bounds__(256) void few_weights_kernel(const FewParams p) {
  const int32_t f = blockIdx.x * 8 + (threadIdx.x >> 5), c = blockIdx.y * 256 + 8 * (threadIdx.x & 31);
  if (f >= p.hidden || c >= p.width) return;
  float g[8] = {}, u[8] = {};
#pragma unroll 4
  for (int32_t t = 0; t < p.tokens; ++t) {
    float x[8] = {};
    if (!p.pos || p.pos[t] >= 0) read_row(reinterpret_cast<const T*>(p.x + t * p.x_bytes) + c, 8, x);
    const float dg = p.grads[int64_t(t) * 2 * p.pitch + f], du = p.grads[(int64_t(t) * 2 + 1) * p.pitch + f];
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] += dg * x[k], u[k] += du * x[k];
  }
  write_row(static_cast<T*>(p.dw_gate) + int64_t(f) * p.width + c, 8, g);
  write_row(static_cast<T*>(p.dw_up) + int64_t(f) * p.width + c, 8, u);
}

struct GradParams {
  Operand a, b;
  const int32_t *pos, *order, *count;        // of the rows of x's gradient; with a list, how many rows (x) or places of the sum (weights) there are
  int32_t rows, cols;           // of the result: tokens x width, or 2 x pitch rows of the weights' gradients x width
  int32_t hidden, pitch;        // weights: rows of each, and of each half of `rows`; x: hidden = 0
  int32_t sum;                  // places of the sum
  int32_t tiles_m, tiles_n, parts;
  void *out, *second;
  float* partial;               // [part][rows][cols], of rows that there are
  const float* lift;            // as in GatedParams; NULL: nothing was multiplied
};

__host__ __device__ __forceinline__ int32_t part_of_sum(int32_t sum, int32_t parts) {       // places of a part: whole stages
  const int32_t each = ((sum + parts - 1) / parts + 63) / 64 * 64;
  return each > 64 ? each : 64;
}

// dx = dg Wg + du Wu: A is the weights, across, B the gradients of the projections' results, along.  dWg = dg^T x and dWu = du^T x: A is x, across, and B those
// gradients, across.  Measured: 32768 rows of 2048 with 8192 hidden, fp16: 1980 to 2040 and 1910 to 1980 us, 1.1 PFLOP/s; 282624 rows of 256, 30 % left out, 683 hidden, bf16: 222 and
// 231 us, where bytes take 139 each.
template <typename T, class P>
__global__ __launch_bounds__(P::kThreads, 2) void grad_kernel(const GradParams p) {
  __shared__ typename P::Shared lds;
  Operand a = p.a, b = p.b;
  int32_t rows = p.rows, sum = p.sum;
  if (p.count) {
    const int32_t n = *fixed(p.count);
    b.rows = n;
    if (p.hidden) sum = a.rows = n;
    else rows = n;
  }
  const int32_t tiles_n = (rows + P::BN - 1) / P::BN;
  if (int32_t(blockIdx.x) >= p.tiles_m * tiles_n * p.parts) return;
  const Tile t = tile_of(blockIdx.x, p.tiles_m * tiles_n * p.parts, p.tiles_m, tiles_n);
  const int32_t c0 = t.m * P::BM, row0 = t.n * P::BN;
  floatx16 acc[P::MI][P::NJ] = {};
  const int32_t each = part_of_sum(sum, p.parts), begin = t.part * each, end = min(begin + each, sum);
  P::run(lds, a, b, c0, row0, begin, end, acc);
  float drop = 1.f;
  if (kLifted<T> && p.lift) drop = p.lift[1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % P::WM, wn = wave / P::WM;
#pragma unroll
  for (int j = 0; j < P::NJ; ++j) {
    int32_t row = row0 + (wn * P::NJ + j) * 32 + (lane & 31);
    if (row >= rows) continue;
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
      if (p.order) there = row = p.order[row];
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
        for (int k = 0; k < 8; ++k) y[k] = live ? (kLifted<T> ? acc[i][j][r0 + k] * drop : acc[i][j][r0 + k]) : 0.f;
        if (p.parts > 1) write_row(p.partial + (int64_t(t.part) * (p.hidden ? 2 * int64_t(p.hidden) : p.rows) + there) * p.cols + c, 8, y);
        else write_row(out + int64_t(row) * p.cols + c, 8, y);
      }
  }
}

// Adds the parts of `n` elements each, eight a thread; those from `first` on go to `second`.  Measured: 85 parts of 2 x 683 x 256: 20 us.
// Rows (of `cols`) whose pos is negative become zeros.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const float* partial, int64_t n, int32_t parts, T* out, int64_t first, T* second, const int32_t* pos, int32_t cols) {
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  float s[8] = {};
  if (pos && pos[i / cols] < 0) parts = 0;
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
  typedef Narrow<T, 32, 4, true> Narrow512;
  typedef Narrow<T, 16, 8, true> Narrow256;
  typedef Narrow<T, 8, 8, true> Narrow128;
  typedef Narrow<T, 4, 8, true> Narrow64;
  typedef Tiles<T, 256, 256, 2, 4, 8, 2, true, false, false> LargePair;
  typedef Tiles<T, 128, 64, 2, 2, 8, 3, true, false, false> SmallPair;
  typedef Tiles<T, 256, 256, 2, 4, 8, 2, false, true, false> LargeX;
  typedef Tiles<T, 128, 256, 2, 2, 4, 3, false, true, false> MiddleX;
  typedef Tiles<T, 64, 64, 2, 2, 8, 3, false, true, false> SmallX;
  typedef Tiles<T, 256, 256, 2, 4, 8, 2, false, true, true> LargeW;
  typedef Tiles<T, 128, 256, 2, 2, 4, 3, false, true, true> MiddleW;
  typedef Tiles<T, 64, 64, 2, 2, 8, 3, false, true, true> SmallW;
};
enum { kLarge, kMiddle, kSmall };       // forms of a tile
// Tokens from which those that are there are listed.  Measured for bf16 with 30 % of the rows left out, forward and backward, listed and not: 4096 tokens of 256 with 704 hidden 36 + 65 and
// 11 + 61 us, 16384 of them 56 + 115 and 25 + 164; with 4096 hidden 4096 tokens 92 + 142 and 28 + 154, 8192 107 + 205 and 63 + 268 (with 5 % left out 64 + 236 and 58 + 270).  A step gains from some
// 10000 tokens on, or fewer with many hidden elements; a forward pass alone later.
constexpr int64_t kListFrom = 4096;

template <typename T, int ACT, class P, bool BACK> void launch_gated(GatedParams p, hipStream_t s) {
  p.tiles_m = ((BACK ? p.pitch : p.hidden) + P::BM / 2 - 1) / (P::BM / 2);
  p.tiles_n = (p.tokens + P::BN - 1) / P::BN;
  gated_kernel<T, ACT, P, BACK><<<uint32_t(p.tiles_m) * uint32_t(p.tiles_n), P::kThreads, 0, s>>>(p);
}
template <typename T, int ACT, class P, bool BACK> void launch_narrow(GatedParams p, int cus, hipStream_t s) {
  p.tiles_m = ((BACK ? p.pitch : p.hidden) + 32 * P::WAVES - 1) / (32 * P::WAVES);
  const int32_t parts = std::max(1, std::min(cus * P::kPerCu / p.tiles_m, (p.tokens + 63) / 64));
  gated_narrow_kernel<T, ACT, P, BACK><<<uint32_t(p.tiles_m) * uint32_t(parts), P::kThreads, 0, s>>>(p);
}
// Up to 32 tokens by the kernel that reads the weights straight to registers (32 tokens, 1024 to 4096: 8.4 us, small tiles 12.0; 64 tokens: 13.1 and 12.0).  Then small tiles, up
// to four for each CU (2048 tokens, 1024 to 2048, 1024 of them: 30.5 us, large ones 30.4; half as many tokens: 17.1 and 29.4; twice: 57 and 35).  Beyond that narrow rows,
// where every workgroup has four slots of them at least (32768 tokens, 256 to 1024, eight slots: 40.7 us, large tiles 51.0; 8192, two slots: 18.9 and 15.6), and large tiles.
template <typename T, int ACT, bool BACK> void gated_by_size(const GatedParams& p, int cus, hipStream_t s) {
  typedef Forms<T> F;
  if (!BACK && p.tokens <= kFewTokens) {
    gated_few_kernel<T, ACT><<<dim3((p.hidden + 15) / 16, (p.tokens + 15) / 16), 64 * kFewWaves, 0, s>>>(p);
    return;
  }
  const int64_t small = int64_t((p.hidden + 63) / 64) * ((p.tokens + 63) / 64);
  if (small <= 4 * cus) return launch_gated<T, ACT, typename F::SmallPair, BACK>(p, s);
  if (p.width_chunks > 64 || p.pos || p.hidden < 8) return launch_gated<T, ACT, typename F::LargePair, BACK>(p, s);
  const int64_t slots = int64_t(p.tokens + 63) / 64, groups = (p.hidden + (p.width_chunks <= 32 ? 255 : 127)) / (p.width_chunks <= 32 ? 256 : 128);
  if (slots * groups < 4 * cus) return launch_gated<T, ACT, typename F::LargePair, BACK>(p, s);
  if (p.width_chunks <= 8) launch_narrow<T, ACT, typename F::Narrow64, BACK>(p, cus, s);
  else if (p.width_chunks <= 16) launch_narrow<T, ACT, typename F::Narrow128, BACK>(p, cus, s);
  else if (p.width_chunks <= 32) launch_narrow<T, ACT, typename F::Narrow256, BACK>(p, cus, s);
  else launch_narrow<T, ACT, typename F::Narrow512, BACK>(p, cus, s);
}
template <typename T, bool BACK> void gated_by_act(int32_t act, const GatedParams& p, int cus, hipStream_t s) {
  if (act == LGP_SILU) gated_by_size<T, LGP_SILU, BACK>(p, cus, s);
  else gated_by_size<T, LGP_GELU, BACK>(p, cus, s);
}
// Small tiles for products of few operations, which large ones would leave to few CUs, and those between for the next ones.  Measured, by tokens, width and hidden, for whole
// backward passes: of x, 16384, 256, 704 (6e9 products): small 99 us, large 110; 4096, 1024, 2048 (2e10): 225, 250; 65536, 256, 704 (2e10): middle 279, small 307, large 332;
// 65536, 512, 1024 (7e10): large 524, middle 542.  Of the weights, 16384, 256, 704: small 107, large 111; 65536, 256, 704: middle 307, large 329, small 351; 65536, 512, 1024:
// middle 514, large 521; 65536, 1024, 2048 (3e11): large 1805, middle 1884.
struct GradShape { int32_t parts; int form; };
GradShape grad_shape(int32_t rows, int32_t cols, int32_t sum, double most_small, double most_middle) {
  GradShape g;
  const double products = double(rows) * cols * sum;
  g.form = products <= most_small ? kSmall : products <= most_middle ? kMiddle : kLarge;
  const int32_t bm = g.form == kLarge ? 256 : g.form == kMiddle ? 128 : 64, bn = g.form == kSmall ? 64 : 256;
  // parts of the sum: as many as make 512 workgroups, of at least 512 places each
  const int64_t tiles = std::max<int64_t>(1, int64_t((cols + bm - 1) / bm) * ((rows + bn - 1) / bn));
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(512 / tiles, sum / 512));
  const int32_t each = part_of_sum(sum, int32_t(parts));
  g.parts = std::max(1, (sum + each - 1) / each);
  return g;
}
GradShape shape_x(const lgp_gated* g, int32_t pitch) { return grad_shape(int32_t(g->tokens), g->width, 2 * pitch, 1.9e10, 5e10); }
GradShape shape_w(const lgp_gated* g, int32_t pitch) { return grad_shape(2 * pitch, g->width, int32_t(g->tokens), 8e9, 5e10); }

template <typename T, class P> void launch_grad(GradParams p, const GradShape& g, const int32_t* pos, hipStream_t s) {
  p.tiles_m = (p.cols + P::BM - 1) / P::BM;
  p.tiles_n = (p.rows + P::BN - 1) / P::BN;
  p.parts = g.parts;
  grad_kernel<T, P><<<uint32_t(p.tiles_m) * uint32_t(p.tiles_n) * uint32_t(g.parts), P::kThreads, 0, s>>>(p);
  if (g.parts > 1) {
    const int64_t first = p.hidden ? int64_t(p.hidden) * p.cols : int64_t(p.rows) * p.cols, n = p.hidden ? 2 * first : first;
    join_kernel<T><<<uint32_t((n / 8 + 255) / 256), 256, 0, s>>>(p.partial, n, g.parts, static_cast<T*>(p.out), first, static_cast<T*>(p.second), pos, p.cols);
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
  p.w = Operand{static_cast<const char*>(g->w_gate), static_cast<const char*>(g->w_up), int64_t(g->width) * 2, g->hidden, g->width / 8, 1 << 30, nullptr, nullptr};
  p.x = Operand{static_cast<const char*>(g->x), nullptr, g->x_row * 2, int32_t(g->tokens), g->width / 8, 1 << 30, nullptr, nullptr};
  p.pos = g->pos;
  p.tokens = int32_t(g->tokens);
  p.hidden = g->hidden;
  p.pitch = pitch_of(g->hidden);
  p.width_chunks = g->width / 8;
  return p;
}
// Where many rows may have no token, those that have one are listed, and the others cost nothing but their zeros.
bool lists(const lgp_gated* g) { return g->pos && g->tokens > kListFrom && g->tokens * g->x_row < int64_t(1) << 35; }       // places of x are counted in 32 bits, by 16 bytes
bool few_tokens(const lgp_gated* g) {
  return g->tokens > 0 && (g->tokens <= kFewBack || (g->tokens <= 64 && g->tokens * g->hidden <= 16384));
}
// Bytes of the list, of the lift, of the projections' gradients, and of the parts of x's and the weights' gradients, which are not there at once.
struct Space { size_t list, lift, grads, parts; };
Space space_of(const lgp_gated* g, bool backward) {
  const int32_t pitch = pitch_of(g->hidden);
  Space s = {};
  if (lists(g)) s.list = (size_t(g->tokens) + size_t(g->tokens + kListed - 1) / kListed + 1 + 63) / 64 * 64 * 4;
  if (!backward) return s;
  if (few_tokens(g)) {
    s.grads = size_t(g->tokens) * 2 * pitch * 4;
    s.parts = size_t((g->hidden + kFewHidden - 1) / kFewHidden) * g->tokens * g->width * 4;
    return s;
  }
  const GradShape x = shape_x(g, pitch), w = shape_w(g, pitch);
  if (g->dtype == LGP_F16 && g->tokens) s.lift = (64 + 2 * kBoundGroups) * sizeof(float);
  s.grads = size_t(g->tokens) * 2 * pitch * 2;
  s.parts = std::max(x.parts > 1 ? size_t(x.parts) * g->tokens * g->width * 4 : 0, w.parts > 1 ? size_t(w.parts) * 2 * g->hidden * g->width * 4 : 0);
  return s;
}
size_t bytes_of(const Space& s) { return s.list + s.lift + s.grads + s.parts; }

// Lists tokens, for `p` too, and fills the other rows of `zeros`.
template <typename T> void list_tokens(const lgp_gated* g, GatedParams& p, void* workspace, void* zeros, int32_t cols, hipStream_t s) {
  int32_t *order = static_cast<int32_t*>(workspace), *counts = order + g->tokens;
  const uint32_t groups = uint32_t((g->tokens + kListed - 1) / kListed);
  count_kernel<<<groups, 256, 0, s>>>(g->pos, p.tokens, counts);
  list_kernel<T><<<groups, 256, 0, s>>>(g->pos, p.tokens, counts, order, counts + groups, static_cast<T*>(zeros), cols);
  p.x.order = order;
  p.count = counts + groups;
  p.pos = nullptr;
}
// Finds the lift of the projections' gradients.
const float* lift_of(const lgp_gated* g, const GatedParams& p, const void* dh, float* space, hipStream_t s) {
  const uint32_t groups = uint32_t(std::min<int64_t>((g->tokens + 2 * g->hidden + 15) / 16, kBoundGroups));
  bound_kernel<<<groups, 256, 0, s>>>(BoundParams{p.x.first, p.w.first, p.w.second, p.x.row_bytes, static_cast<const f16*>(dh), g->pos, p.tokens, g->width, g->hidden, space + 64});
  lift_kernel<<<1, 256, 0, s>>>(space + 64, int32_t(groups), space);
  return space;
}
template <typename T> void forward(int device, const lgp_gated* g, void* h, void* workspace, hipStream_t s) {
  GatedParams p = gated_params(g);
  p.h = h;
  if (lists(g)) list_tokens<T>(g, p, workspace, h, g->hidden, s);
  gated_by_act<T, false>(g->act, p, compute_units(device), s);
}
// Up to eight tokens, and 64 with few hidden elements, want no lift either: the rounding of the projections' gradients to 16 bits would come out whole in the weights' gradients, which are sums over
// tokens (one token, bf16: 2.7e-3 of dw_up off, where a result rounded once, as here, is 1.7e-3 off; from nine on 1.47 times that at most, in 20 draws).  1024 to 4096, bf16: one
// token 32 us as with tiles, eight tokens 42, nine with tiles 35.
template <typename T> void few_backward(const lgp_gated* g, const void* dh, void* dx, void* dw_gate, void* dw_up, void* workspace, hipStream_t s) {
  GatedParams p = gated_params(g);
  p.dh = dh;
  p.grads = workspace;
  const dim3 blocks((g->hidden + 15) / 16, (p.tokens + 15) / 16);
  if (g->act == LGP_SILU) few_grads_kernel<T, LGP_SILU><<<blocks, 64 * kFewWaves, 0, s>>>(p);
  else few_grads_kernel<T, LGP_GELU><<<blocks, 64 * kFewWaves, 0, s>>>(p);
  FewParams f = {p.w.first, p.w.second, p.x.first, p.x.row_bytes, g->pos, p.tokens, g->width, g->hidden, p.pitch, static_cast<float*>(workspace), nullptr, dw_gate, dw_up};
  f.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + space_of(g, true).grads);
  const int32_t parts = (g->hidden + kFewHidden - 1) / kFewHidden;
  few_x_kernel<T><<<dim3((g->width + 255) / 256, (p.tokens + 7) / 8, parts), 256, 0, s>>>(f);
  const int64_t n = int64_t(p.tokens) * g->width;
  join_kernel<T><<<uint32_t((n / 8 + 255) / 256), 256, 0, s>>>(f.partial, n, parts, static_cast<T*>(dx), n, nullptr, g->pos, g->width);
  few_weights_kernel<T><<<dim3((g->hidden + 7) / 8, (g->width + 255) / 256), 256, 0, s>>>(f);
}
template <typename T> void backward(int device, const lgp_gated* g, const void* dh, void* dx, void* dw_gate, void* dw_up, void* workspace, hipStream_t s) {
  typedef Forms<T> F;
  if (few_tokens(g)) return few_backward<T>(g, dh, dx, dw_gate, dw_up, workspace, s);
  GatedParams p = gated_params(g);
  const Space space = space_of(g, true);
  char* grads = static_cast<char*>(workspace) + space.list + space.lift;
  float* partial = reinterpret_cast<float*>(grads + space.grads);
  p.dh = dh;
  p.grads = grads;
  const Operand of_grads = {grads, nullptr, int64_t(p.pitch) * 4, p.tokens, p.pitch / 4, 1 << 30, nullptr, nullptr};
  if (p.tokens) {
    if (kLifted<T>) p.lift = lift_of(g, p, dh, reinterpret_cast<float*>(static_cast<char*>(workspace) + space.list), s);
    if (lists(g)) list_tokens<T>(g, p, workspace, dx, g->width, s);
    gated_by_act<T, true>(g->act, p, compute_units(device), s);
    GradParams d = {};
    d.a = p.w;
    d.a.half = p.pitch;
    d.b = of_grads;
    d.pos = p.pos;
    d.order = p.x.order;
    d.count = p.count;
    d.rows = p.tokens;
    d.cols = g->width;
    d.sum = 2 * p.pitch;
    d.out = dx;
    d.partial = partial;
    d.lift = p.lift;
    const GradShape shape = shape_x(g, p.pitch);
    if (shape.form == kLarge) launch_grad<T, typename F::LargeX>(d, shape, g->pos, s);
    else if (shape.form == kMiddle) launch_grad<T, typename F::MiddleX>(d, shape, g->pos, s);
    else launch_grad<T, typename F::SmallX>(d, shape, g->pos, s);
  }
  GradParams d = {};
  d.a = p.x;
  d.a.pos = p.pos;
  d.b = of_grads;
  d.count = p.count;
  d.rows = 2 * p.pitch;
  d.cols = g->width;
  d.hidden = g->hidden;
  d.pitch = p.pitch;
  d.sum = p.tokens;
  d.out = dw_gate;
  d.second = dw_up;
  d.partial = partial;
  d.lift = p.lift;
  const GradShape shape = shape_w(g, p.pitch);
  if (shape.form == kLarge) launch_grad<T, typename F::LargeW>(d, shape, nullptr, s);
  else if (shape.form == kMiddle) launch_grad<T, typename F::MiddleW>(d, shape, nullptr, s);
  else launch_grad<T, typename F::SmallW>(d, shape, nullptr, s);
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_gated_linear(int device, const lgp_gated* in, void* h, void* workspace, size_t workspace_bytes, void* stream) {
  if (int st = check_gated(in)) return st;
  if (in->tokens && !h) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (in->tokens == 0) return LGP_OK;
  const size_t bytes = bytes_of(space_of(in, false));
  if (workspace_bytes < bytes) return LGP_ECAPACITY;
  if (bytes && (!workspace || !aligned16(workspace))) return LGP_EINVAL;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F16) forward<f16>(device, in, h, workspace, s);
  else forward<bf16>(device, in, h, workspace, s);
  return launched();
}

int lgp_gated_linear_workspace(int device, const lgp_gated* in, int backward, size_t* bytes) {
  if (!bytes) return LGP_EINVAL;
  *bytes = 0;
  if (int st = check_gated(in)) return st;
  *bytes = bytes_of(space_of(in, backward != 0));
  return device < 0 ? LGP_EINVAL : LGP_OK;
}

int lgp_gated_linear_backward(int device, const lgp_gated* in, const void* dh, void* dx, void* dw_gate, void* dw_up, void* workspace, size_t workspace_bytes, void* stream) {
  if (int st = check_gated(in)) return st;
  if ((in->tokens && (!dh || !dx)) || !dw_gate || !dw_up) return LGP_EINVAL;
  if (!aligned16(dx) || !aligned16(dw_gate) || !aligned16(dw_up)) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  const size_t bytes = bytes_of(space_of(in, true));
  if (workspace_bytes < bytes) return LGP_ECAPACITY;
  if (bytes && (!workspace || !aligned16(workspace))) return LGP_EINVAL;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (in->dtype == LGP_F16) backward<f16>(device, in, dh, dx, dw_gate, dw_up, workspace, s);
  else backward<bf16>(device, in, dh, dx, dw_gate, dw_up, workspace, s);
  return launched();
}

}  // extern "C"
