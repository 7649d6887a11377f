// The norm over all gradients of a model, and the gradients scaled down to a largest norm.
#include "rows_dev.hpp"

#include <algorithm>
#include <cmath>
#include <vector>

namespace lgp {
namespace layer {
namespace {

// What a launch works on comes with its arguments, of which there are at most 4096 bytes: nothing is copied to the GPU beforehand, and a captured
// launch holds it.
constexpr int kTensors = 120;
struct Tensors {
  const void* grad[kTensors];
  void* out[kTensors];
  int64_t n_type[kTensors];              // elements * 4 + type
  uint32_t chunk[kTensors + 1];          // the first chunk of each, and all of them
  int32_t count;
  int32_t n_partial;                     // sums of squares: one of each workgroup of all launches
  double* partial;                       // norm: of this launch; scale: of all
  double most;
  float* norm;                           // scale: written by the first workgroup of the first launch, else NULL
};
static_assert(sizeof(Tensors) <= 4096, "arguments of a launch");

constexpr int kThreads = 256, kChunk = 16384, kPartials = 2048;      // elements of a chunk; workgroups of all launches of the first pass

// The sum of x over the workgroup, the same in all threads.
__device__ __forceinline__ double group_sum(double x, double* lds) {
#pragma unroll
  for (int i = 32; i; i >>= 1) x += __shfl_xor(x, i, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// f(elements, n) of this thread's share of a chunk: eight at a time.
template <typename F> __device__ __forceinline__ void eights(int64_t n, F f) {
#pragma unroll 4
  for (int64_t i = threadIdx.x * 8; i < n; i += kThreads * 8) f(i, n - i < 8 ? int(n - i) : 8);
}
struct Place { int tensor; int64_t begin, n; };
__device__ __forceinline__ Place place_of(const Tensors& t, uint32_t chunk) {
  int lo = 0, hi = t.count;              // the last tensor that begins at this chunk or before it, and has any
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.chunk[mid] <= chunk) lo = mid; else hi = mid;
  }
  const int64_t begin = int64_t(chunk - t.chunk[lo]) * kChunk, n = (t.n_type[lo] >> 2) - begin;
  return {lo, begin, n < kChunk ? n : kChunk};
}

// Squares of 32-bit numbers are exact in 64 bits, where no sum of them overflows or loses small ones.  Bound by bytes: 476 million bf16 gradients in 218 tensors, this pass and the
// next in 611 us, 4.7 TB/s of what is read twice and written once; 200000 fp32 ones in 11 tensors 4.8 and 7 us.
template <typename T> __device__ __forceinline__ double squares(const T* g, int64_t n) {
  double s = 0;
  eights(n, [&](int64_t i, int have) {
    float x[8];
    read_row(g + i, have, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) s += double(x[k]) * double(x[k]);
  });
  return s;
}
__global__ __launch_bounds__(kThreads) void squares_kernel(const Tensors t) {
  __shared__ double lds[4];
  double s = 0;
  for (uint32_t c = blockIdx.x; c < t.chunk[t.count]; c += gridDim.x) {
    const Place p = place_of(t, c);
    const void* g = t.grad[p.tensor];
    const int type = int(t.n_type[p.tensor] & 3);
    if (type == LGP_F32) s += squares(static_cast<const float*>(g) + p.begin, p.n);
    else if (type == LGP_F16) s += squares(static_cast<const f16*>(g) + p.begin, p.n);
    else s += squares(static_cast<const bf16*>(g) + p.begin, p.n);
  }
  s = group_sum(s, lds);
  if (threadIdx.x == 0) t.partial[blockIdx.x] = s;
}

// v cut to 14 places behind the first, the last of which is set where anything was cut off: that is a number of 32 bits (from 2^-135 on; what is less becomes zero), and as a number of 16 bits
// it is rounded as v would be, since those, and what lies half way between them, have at most 11 (v in 32 bits, rounded, may land half way: 717 of 12.7 million results were off).
__device__ __forceinline__ float cut(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t high = uint32_t(bits >> 32), rest = (high & 0x3fu) | uint32_t(bits);
  return float(__builtin_bit_cast(double, uint64_t((high & ~0x3fu) | (rest ? 0x40u : 0u)) << 32));
}

// Every workgroup adds the sums up again, in the same order, which is less than a launch for it, and scales its share, the chunks that were read last first: they
// are the likeliest to be cached.  The factor and the products are in 64 bits, so that a result is rounded once.
template <typename T> __device__ __forceinline__ void scale(const T* g, T* out, int64_t n, double by) {
  eights(n, [&](int64_t i, int have) {
    float x[8];
    read_row(g + i, have, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const double v = double(x[k]) * by;
      x[k] = sizeof(T) == 2 ? cut(v) : float(v);
    }
    write_row(out + i, have, x);
  });
}
__global__ __launch_bounds__(kThreads) void scale_kernel(const Tensors t) {
  __shared__ double lds[4];
  double s = 0;
  for (int i = threadIdx.x; i < t.n_partial; i += kThreads) s += t.partial[i];
  const double exact = sqrt(group_sum(s, lds));
  const float norm = float(exact);
  if (t.norm && blockIdx.x == 0 && threadIdx.x == 0) *t.norm = norm;
  const bool finite = norm < INFINITY;
  const double by = finite && exact > t.most ? t.most / exact : 1.0;
  const uint32_t chunks = t.chunk[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Place p = place_of(t, chunks - 1 - c);
    const void* g = t.grad[p.tensor];
    void* out = t.out[p.tensor];
    if (by == 1.0 && out == g) continue;
    const int type = int(t.n_type[p.tensor] & 3);
    if (type == LGP_F32) scale(static_cast<const float*>(g) + p.begin, static_cast<float*>(out) + p.begin, p.n, by);
    else if (type == LGP_F16) scale(static_cast<const f16*>(g) + p.begin, static_cast<f16*>(out) + p.begin, p.n, by);
    else scale(static_cast<const bf16*>(g) + p.begin, static_cast<bf16*>(out) + p.begin, p.n, by);
  }
}

int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }
int64_t size_of(int64_t dtype) { return dtype == LGP_F32 ? 4 : 2; }

// Whether a range that is written overlaps another, but for a gradient that stays where it is.
bool overlap(const lgp_gradient* list, int64_t n) {
  struct Range { uintptr_t begin, end; bool written; };
  std::vector<Range> ranges;
  ranges.reserve(size_t(2 * n));
  for (int64_t i = 0; i < n; ++i) {
    if (!list[i].n) continue;
    const uintptr_t g = reinterpret_cast<uintptr_t>(list[i].grad), o = reinterpret_cast<uintptr_t>(list[i].out);
    const uintptr_t bytes = uintptr_t(list[i].n * size_of(list[i].dtype));
    ranges.push_back({o, o + bytes, true});
    if (o != g) ranges.push_back({g, g + bytes, false});
  }
  std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t end = 0, written_end = 0;
  for (const Range& r : ranges) {
    if (r.begin < (r.written ? end : written_end)) return true;
    end = std::max(end, r.end);
    if (r.written) written_end = std::max(written_end, r.end);
  }
  return false;
}

int clip(int device, const lgp_gradient* list, int64_t n, double most, float* norm, void* workspace, size_t workspace_bytes, hipStream_t s) {
  if (n < 0 || (n && !list) || !norm || std::isnan(most) || most < 0) return LGP_EINVAL;
  if (n > 65536) return LGP_EUNSUPPORTED;
  const bool scales = !std::isinf(most);
  bool copies = false;
  for (int64_t i = 0; i < n; ++i) {
    const lgp_gradient& g = list[i];
    if (g.dtype != LGP_F32 && g.dtype != LGP_F16 && g.dtype != LGP_BF16) return LGP_EUNSUPPORTED;
    if (g.n < 0 || (g.n && (!g.grad || !g.out))) return LGP_EINVAL;
    if (g.n >= int64_t(1) << 38) return LGP_EUNSUPPORTED;          // chunks of a launch are counted in 32 bits
    if ((reinterpret_cast<uintptr_t>(g.grad) | reinterpret_cast<uintptr_t>(g.out)) % size_of(g.dtype)) return LGP_EINVAL;
    copies = copies || (g.n && g.out != g.grad);
  }
  if ((scales || copies) && overlap(list, n)) return LGP_EINVAL;
  if (int st = use_device(device)) return st;
  if (workspace_bytes < kPartials * sizeof(double)) return LGP_ECAPACITY;
  if (!workspace || !aligned16(workspace)) return LGP_EINVAL;
  const int32_t launches = int32_t(std::max<int64_t>(1, (n + kTensors - 1) / kTensors)), most_groups = kPartials / launches;       // two at least
  double* partial = static_cast<double*>(workspace);
  Tensors t;
  int32_t n_partial = 0;
  auto pass = [&](bool second) {
    for (int32_t l = 0; l < launches; ++l) {
      const int32_t which = second ? launches - 1 - l : l;
      const int64_t first = int64_t(which) * kTensors;
      t.count = int32_t(std::min<int64_t>(kTensors, n - first));
      int64_t chunks = 0;
      for (int32_t i = 0; i < t.count; ++i) {
        const lgp_gradient& g = list[first + i];
        t.grad[i] = g.grad;
        t.out[i] = g.out;
        t.n_type[i] = g.n * 4 + g.dtype;
        t.chunk[i] = uint32_t(chunks);
        chunks += chunks_of(g.n);
      }
      t.chunk[t.count] = uint32_t(chunks);
      const uint32_t groups = uint32_t(std::max<int64_t>(1, std::min<int64_t>(chunks, most_groups)));
      if (!second) {
        t.partial = partial + n_partial;
        n_partial += int32_t(groups);
        squares_kernel<<<groups, kThreads, 0, s>>>(t);
      } else {
        t.partial = partial;
        t.n_partial = n_partial;
        t.most = most;
        t.norm = l == 0 ? norm : nullptr;
        const bool idle = !scales && !copies;
        scale_kernel<<<idle ? 1 : uint32_t(std::max<int64_t>(1, std::min<int64_t>(chunks, kPartials))), kThreads, 0, s>>>(t);
        if (idle) break;
      }
    }
  };
  pass(false);
  pass(true);
  return launched();
}

}  // namespace
}  // namespace layer
}  // namespace lgp

using namespace lgp::layer;

extern "C" {

int lgp_clip_gradients_workspace(int device, size_t* bytes) {
  if (!bytes) return LGP_EINVAL;
  *bytes = kPartials * sizeof(double);
  return device < 0 ? LGP_EINVAL : LGP_OK;
}

int lgp_clip_gradients(int device, const lgp_gradient* list, int64_t n, double most, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    return clip(device, list, n, most, norm, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
  } catch (...) {          // the host's memory
    return LGP_ENOMEM;
  }
}

}  // extern "C"
