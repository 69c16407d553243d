// The global norm of many gradients, and clipping them by it: the C entry points
// tlf_grad_norm_ws_bytes, tlf_grad_norm and tlf_grad_clip and their kernels.
//
//   norm = sqrt(sum over all tensors of g^2),  scale = min(1, max_norm / norm)
//
// Squares are exact in float64 and are summed in it, so that no square leaves the
// range and the sum of 10^9 elements has float32's precision.  Each workgroup's sum
// goes to a place of its own and they are added in a fixed order: no atomics, and
// nothing has to be cleared.  The scale stays on the device.
//
// Bound by HBM: 176M bf16 elements 55 us (6.3 TB/s; what the memory-side cache still holds
// of them helps), 4.6 us for the sums; a pass that does not clip ends with a launch that
// reads one value (2.5-4.5 us), one that clips with one of 109 us (6.5 TB/s).  4096
// workgroups take the pieces of 8192 in turn: a workgroup for each took 69 us in all
// against 64, with sums for 21000 workgroups.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

#include "common.h"
#include "tlf.h"

namespace tlf {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8192;                     // elements of a workgroup
constexpr int kTensors = 160;                  // of a launch: its arguments stay below 4 KiB
constexpr int64_t kGroups = 4096;              // workgroups of a launch, which take its pieces in turn
constexpr int kTotalThreads = 1024;
constexpr int64_t kMost = (int64_t)1 << 35;    // elements of a tensor
static_assert(kTensors * (kMost / kPer) < INT32_MAX, "pieces of a launch");

struct GradArgs {
  void* g[kTensors];
  int64_t n[kTensors];              // times four, plus the flags below
  int32_t first[kTensors + 1];      // pieces before each tensor
  int32_t count;
  double* part;
  const float* scale;
};
enum { kBf16 = 1, kVector = 2 };
static_assert(sizeof(GradArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ int tensor_of(const GradArgs& a, int block) {
  int lo = 0, hi = a.count - 1;  // the last tensor whose pieces start at or before this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= block) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// 16 bytes as they lie, and as floats.
template <typename T> struct Chunk;
template <> struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(uint4 v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <> struct Chunk<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(uint4 v, float (&f)[8]) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[2 * k] = __uint_as_float(w[k] << 16);
      f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
};

template <typename T> __device__ __forceinline__ double squares(const T* g, int64_t n, int64_t base, bool vec) {
  using C = Chunk<T>;
  constexpr int U = kPer / (kThreads * C::N);
  double s[2] = {0.0, 0.0};
  if (vec && base + kPer <= n) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const uint4*>(g + base + (u * kThreads + threadIdx.x) * C::N);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[C::N];
      C::get(v[u], f);
#pragma unroll
      for (int e = 0; e < C::N; ++e) s[e & 1] = fma((double)f[e], (double)f[e], s[e & 1]);
    }
  } else {
    for (int64_t e = base + threadIdx.x; e < n && e < base + kPer; e += kThreads) {
      const double f = (double)to_f<T>(g[e]);
      s[0] = fma(f, f, s[0]);
    }
  }
  return s[0] + s[1];
}

__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

__global__ __launch_bounds__(kThreads) void k_grad_squares(GradArgs a) {
  __shared__ double sums[kThreads / kWave];
  double s = 0.0;
  for (int block = blockIdx.x; block < a.first[a.count]; block += gridDim.x) {
    const int k = tensor_of(a, block);
    const int64_t n = a.n[k] >> 2, base = (int64_t)(block - a.first[k]) * kPer;
    const bool vec = a.n[k] & kVector;
    s += a.n[k] & kBf16 ? squares(reinterpret_cast<const bf16*>(a.g[k]), n, base, vec)
                        : squares(reinterpret_cast<const float*>(a.g[k]), n, base, vec);
  }
  s = wave_total(s);
  if (lane_id() == 0) sums[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.part[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// All workgroups' sums, the norm and the scale.
__global__ __launch_bounds__(kTotalThreads) void k_grad_total(const double* part, int64_t n, double max_norm, float* norm, float* scale) {
  __shared__ double sums[kTotalThreads / kWave];
  double s = 0.0;
#pragma unroll 8
  for (int64_t k = threadIdx.x; k < n; k += kTotalThreads) s += part[k];
  s = wave_total(s);
  if (lane_id() == 0) sums[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x > 0) return;
  s = sums[0];
  for (int w = 1; w < kTotalThreads / kWave; ++w) s += sums[w];
  s = sqrt(s);
  *norm = (float)s;
  // 0 or NaN of a sum that is not finite; NaN where the limit is infinite too
  if (scale) *scale = s <= max_norm && s < INFINITY ? 1.f : (float)(max_norm / s);
}

template <typename T> __device__ __forceinline__ void scale_all(T* g, int64_t n, int64_t base, bool vec, float f) {
  using C = Chunk<T>;
  constexpr int U = kPer / (kThreads * C::N);
  if (vec && base + kPer <= n) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const uint4*>(g + base + (u * kThreads + threadIdx.x) * C::N);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[C::N];
      C::get(v[u], x);
#pragma unroll
      for (int e = 0; e < C::N; ++e) x[e] *= f;
      *reinterpret_cast<uint4*>(g + base + (u * kThreads + threadIdx.x) * C::N) = C::put(x);
    }
  } else {
    for (int64_t e = base + threadIdx.x; e < n && e < base + kPer; e += kThreads) g[e] = from_f<T>(to_f<T>(g[e]) * f);
  }
}

// Gradients within the limit are neither read nor written.
__global__ __launch_bounds__(kThreads) void k_grad_scale(GradArgs a) {
  const float f = *a.scale;
  if (f == 1.f) return;
  for (int block = blockIdx.x; block < a.first[a.count]; block += gridDim.x) {
    const int k = tensor_of(a, block);
    const int64_t n = a.n[k] >> 2, base = (int64_t)(block - a.first[k]) * kPer;
    const bool vec = a.n[k] & kVector;
    if (a.n[k] & kBf16) scale_all(reinterpret_cast<bf16*>(a.g[k]), n, base, vec, f);
    else scale_all(reinterpret_cast<float*>(a.g[k]), n, base, vec, f);
  }
}

int64_t blocks_of(int64_t n) { return (n + kPer - 1) / kPer; }

int check(const tlf_grad* grads, int32_t count) {
  if (count < 0 || (count > 0 && !grads)) return TLF_E_INVALID_ARG;
  int st = TLF_OK;
  for (int i = 0; i < count; ++i) {
    const tlf_grad& t = grads[i];
    if (t.n < 0 || (t.dtype != TLF_DTYPE_F32 && t.dtype != TLF_DTYPE_BF16)) return TLF_E_INVALID_ARG;
    if (t.n > 0 && (!t.d_grad || ((uintptr_t)t.d_grad & (t.dtype == TLF_DTYPE_BF16 ? 1u : 3u)) != 0)) return TLF_E_INVALID_ARG;
    if (t.n > kMost) st = TLF_E_UNSUPPORTED;
  }
  return st;
}

// The launches over all tensors, as many of them at a time as the arguments hold:
// go(arguments, workgroups) for each.
template <typename F> int launches(const tlf_grad* grads, int32_t count, F go) {
  GradArgs a{};
  for (int i = 0; i <= count; ++i) {
    const tlf_grad* t = i < count ? &grads[i] : nullptr;
    const int64_t blocks = t ? blocks_of(t->n) : 0;
    if (a.count > 0 && (!t || a.count == kTensors)) {  // full, or done; its pieces are less than 2^31
      const int st = go(a, (int)std::min<int64_t>(a.first[a.count], kGroups));
      if (st != TLF_OK) return st;
      a.count = 0;
    }
    if (blocks == 0) continue;
    const bool vec = ((uintptr_t)t->d_grad & 15u) == 0;
    a.g[a.count] = t->d_grad;
    a.n[a.count] = t->n << 2 | (t->dtype == TLF_DTYPE_BF16 ? kBf16 : 0) | (vec ? kVector : 0);
    a.first[a.count + 1] = a.first[a.count] + (int32_t)blocks;
    ++a.count;
  }
  return TLF_OK;
}

// Workgroups of all launches, each of which has a sum.
int64_t sums_of(const tlf_grad* grads, int32_t count) {
  int64_t n = 0;
  launches(grads, count, [&](GradArgs&, int groups) {
    n += groups;
    return TLF_OK;
  });
  return n;
}

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_grad_norm_ws_bytes(const tlf_grad* h_grads, int32_t count, size_t* ws_bytes) {
  const int st = tlf::check(h_grads, count);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  *ws_bytes = (size_t)tlf::sums_of(h_grads, count) * sizeof(double);
  return TLF_OK;
}

int tlf_grad_norm(const tlf_grad* h_grads, int32_t count, double max_norm, float* d_norm, float* d_scale, void* d_workspace,
                  size_t ws_bytes, void* stream) {
  int st = tlf::check(h_grads, count);
  if (st != TLF_OK) return st;
  if (!(max_norm > 0.0) || !d_norm || ((uintptr_t)d_norm & 3u) != 0 || ((uintptr_t)d_scale & 3u) != 0) return TLF_E_INVALID_ARG;
  const int64_t sums = tlf::sums_of(h_grads, count);
  if (sums > 0 && (!d_workspace || ((uintptr_t)d_workspace & 7u) != 0 || ws_bytes < (size_t)sums * sizeof(double)))
    return TLF_E_INVALID_ARG;
  const hipStream_t s = (hipStream_t)stream;
  double* part = (double*)d_workspace;
  st = tlf::launches(h_grads, count, [&](tlf::GradArgs& a, int groups) {
    a.part = part;
    part += groups;
    hipLaunchKernelGGL(tlf::k_grad_squares, dim3(groups), dim3(tlf::kThreads), 0, s, a);
    return hipGetLastError() == hipSuccess ? TLF_OK : TLF_E_HIP;
  });
  if (st != TLF_OK) return st;
  hipLaunchKernelGGL(tlf::k_grad_total, dim3(1), dim3(tlf::kTotalThreads), 0, s, (const double*)d_workspace, sums, max_norm,
                     d_norm, d_scale);
  return hipGetLastError() == hipSuccess ? TLF_OK : TLF_E_HIP;
}

int tlf_grad_clip(const tlf_grad* h_grads, int32_t count, const float* d_scale, void* stream) {
  const int st = tlf::check(h_grads, count);
  if (st != TLF_OK) return st;
  if (!d_scale || ((uintptr_t)d_scale & 3u) != 0) return TLF_E_INVALID_ARG;
  // workgroups run in no order: what they write overlaps nothing else of the call
  struct Range {
    uintptr_t begin, end;
  };
  const std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[(size_t)count + 1]);
  if (!ranges) return TLF_E_HIP;
  size_t n = 0;
  ranges[n++] = Range{(uintptr_t)d_scale, (uintptr_t)d_scale + sizeof(float)};
  for (int i = 0; i < count; ++i)
    if (h_grads[i].n > 0) {
      const uintptr_t p = (uintptr_t)h_grads[i].d_grad;
      ranges[n++] = Range{p, p + (uintptr_t)h_grads[i].n * (h_grads[i].dtype == TLF_DTYPE_BF16 ? 2 : 4)};
    }
  std::sort(ranges.get(), ranges.get() + n, [](const Range& a, const Range& b) { return a.begin < b.begin; });
  for (size_t k = 1; k < n; ++k)
    if (ranges[k].begin < ranges[k - 1].end) return TLF_E_INVALID_ARG;
  return tlf::launches(h_grads, count, [&](tlf::GradArgs& a, int groups) {
    a.scale = d_scale;
    hipLaunchKernelGGL(tlf::k_grad_scale, dim3(groups), dim3(tlf::kThreads), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TLF_OK : TLF_E_HIP;
  });
}

}  // extern "C"
