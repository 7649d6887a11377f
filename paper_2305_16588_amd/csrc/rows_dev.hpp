// Rows of a matrix by groups of lanes: reads and writes of eight elements at any alignment, sums and largest values over a group.
#pragma once

#include "layer_dev.hpp"

namespace lgp {
namespace layer {
namespace {

template <typename T> struct AnyEight;
template <> struct AnyEight<f16> { typedef f16 x8 __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct AnyEight<bf16> { typedef bf16 x8 __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct AnyEight<float> { typedef float x8 __attribute__((ext_vector_type(8), aligned(4))); };

// Eight elements of a row that has n from here on, zeros behind them.
template <typename T> __device__ __forceinline__ void read_row(const T* p, int n, float* x) {
  if (n >= 8) {
    const typename AnyEight<T>::x8 v = *reinterpret_cast<const typename AnyEight<T>::x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? float(p[i]) : 0.f;
  }
}
template <typename T> __device__ __forceinline__ void write_row(T* p, int n, const float* x) {
  if (n >= 8) {
    typename AnyEight<T>::x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = T(x[i]);
    *reinterpret_cast<typename AnyEight<T>::x8*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = T(x[i]);
  }
}

// Over L lanes of a wave, the same in all of them.
template <int L> __device__ __forceinline__ float lanes_sum(float x) {
  x = sum_of_lanes<(L > 32 ? 32 : L)>(x);
  if constexpr (L >= 64) x += __shfl_xor(x, 32, 64);
  return x;
}
template <int CTRL> __device__ __forceinline__ uint32_t moved_bits(uint32_t x) { return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xf, 0xf, true)); }
template <int L> __device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  if constexpr (L >= 2) x = max(x, moved_bits<0xb1>(x));
  if constexpr (L >= 4) x = max(x, moved_bits<0x4e>(x));
  if constexpr (L >= 8) x = max(x, moved_bits<0x141>(x));
  if constexpr (L >= 16) x = max(x, moved_bits<0x140>(x));
  if constexpr (L >= 32) x = max(x, uint32_t(__shfl_xor(int(x), 16, 64)));
  if constexpr (L >= 64) x = max(x, uint32_t(__shfl_xor(int(x), 32, 64)));
  return x;
}

}  // namespace
}  // namespace layer
}  // namespace lgp
