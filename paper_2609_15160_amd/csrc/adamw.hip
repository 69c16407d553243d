// One AdamW step over many tensors (Appendix A's training recipe): the C entry
// point tlf_adamw and its kernels.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Every element is read and written once.  The tensors of a launch are
// described in its arguments (nothing is copied to the device beforehand), a
// workgroup finds its tensor from the workgroup counts before it.
//
// Moments in 8 bits share one float32 scale per 256 elements: m is e4m3 of
// m / s with s = max|m| / 448, v is e5m2 of v / s with s = max v / 57344, so
// that each block's largest value is the format's largest; a v that is not
// zero does not become zero (its m / sqrt(v) would grow without bound).  They
// are computed in float64 up to that rounding, each product and sum rounded by
// itself: in float32 a value next to a border between two codes would fall to
// either side, and a fused product and sum fall to another side of a tie.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

#include "common.h"
#include "tlf.h"

namespace tlf {

namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamUnroll = 4;
constexpr int kAdamPer = kAdamThreads * 4 * kAdamUnroll;  // elements of a workgroup
constexpr int kAdamTensors = 40;                          // tensors of a launch: its arguments stay below 4 KiB
constexpr int kAdamBlocks = (1 << 24) - 1;                // of a launch, which has fewer than 2^32 threads
constexpr int kBlock = TLF_ADAMW_BLOCK;
static_assert(kBlock == 4 * kWave, "one wave per block of 8-bit moments");

// Nothing is read twice, so loads and stores pass the caches by (10^8 elements
// with float32 moments: 510 us through them, 463 past them, 6.0 TB/s; with 8 bits
// 349 and 340, and 314, 5.1 TB/s, with reciprocals for divisions).
struct AdamTensor {
  float* p;
  bf16* copy;
  const void* g;
  void* m;
  void* v;
  float* ms;
  float* vs;
  int64_t n;
  float decay, rate, root;  // 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  int32_t flags;
};
enum { kGradBf16 = 1, kVector = 2 };

struct AdamArgs {
  AdamTensor t[kAdamTensors];
  int32_t first[kAdamTensors + 1];  // workgroups before each tensor
  int32_t count;
  double b1, b2;
  const float* scale;  // of the gradients, or NULL
  float eps;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ int tensor_of(const AdamArgs& a, int block) {
  int lo = 0, hi = a.count - 1;  // the last tensor whose workgroups start at or before this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= block) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The hardware's reciprocal is off by one of the float32 roundings that the step's
// other operations make too.
__device__ __forceinline__ float update(float p, float m, float v, const AdamTensor& t, float eps) {
  return p * t.decay - t.rate * m * __builtin_amdgcn_rcpf(sqrtf(v) * t.root + eps);  // eps is normal
}

// SCALED: gradients count times *a.scale (clipping), which costs no pass of their own
// (40M float32 elements: 163 us, 7.0 TB/s; with the norm before it 200).
template <bool SCALED> __global__ __launch_bounds__(kAdamThreads) void k_adamw(AdamArgs a) {
  const int k = tensor_of(a, blockIdx.x);
  const AdamTensor& t = a.t[k];
  const float b1 = (float)a.b1, b2 = (float)a.b2, c1 = (float)(1.0 - a.b1), c2 = (float)(1.0 - a.b2);
  float* m = reinterpret_cast<float*>(t.m);
  float* v = reinterpret_cast<float*>(t.v);
  const int64_t base = (int64_t)(blockIdx.x - a.first[k]) * kAdamPer;
  const float scale = SCALED ? *a.scale : 1.f;
  if ((t.flags & kVector) && base + kAdamPer <= t.n) {
    f32x4 p4[kAdamUnroll], g4[kAdamUnroll], m4[kAdamUnroll], v4[kAdamUnroll];
#pragma unroll
    for (int u = 0; u < kAdamUnroll; ++u) {
      const int64_t e = base + (u * kAdamThreads + threadIdx.x) * 4;
      p4[u] = Stream4<float>::load(t.p + e);
      m4[u] = Stream4<float>::load(m + e);
      v4[u] = Stream4<float>::load(v + e);
      g4[u] = t.flags & kGradBf16 ? Stream4<bf16>::load(reinterpret_cast<const bf16*>(t.g) + e)
                                  : Stream4<float>::load(reinterpret_cast<const float*>(t.g) + e);
    }
#pragma unroll
    for (int u = 0; u < kAdamUnroll; ++u) {
      const int64_t e = base + (u * kAdamThreads + threadIdx.x) * 4;
      if (SCALED) g4[u] *= scale;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        m4[u][r] = b1 * m4[u][r] + c1 * g4[u][r];
        v4[u][r] = b2 * v4[u][r] + c2 * (g4[u][r] * g4[u][r]);
        p4[u][r] = update(p4[u][r], m4[u][r], v4[u][r], t, a.eps);
      }
      Stream4<float>::store(t.p + e, p4[u]);
      Stream4<float>::store(m + e, m4[u]);
      Stream4<float>::store(v + e, v4[u]);
      if (t.copy) Stream4<bf16>::store(t.copy + e, p4[u]);
    }
    return;
  }
  for (int64_t e = base + threadIdx.x; e < t.n && e < base + kAdamPer; e += kAdamThreads) {
    float g = t.flags & kGradBf16 ? (float)reinterpret_cast<const bf16*>(t.g)[e] : reinterpret_cast<const float*>(t.g)[e];
    if (SCALED) g *= scale;
    const float m1 = b1 * m[e] + c1 * g, v1 = b2 * v[e] + c2 * (g * g);
    const float p = update(t.p[e], m1, v1, t, a.eps);
    t.p[e] = p;
    m[e] = m1;
    v[e] = v1;
    if (t.copy) t.copy[e] = (bf16)p;
  }
}

// Magnitudes are compared as their bits: NaN is above infinity and is not lost.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ float wave_max(unsigned v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, shfl_xor(v, o));
  return __uint_as_float(v);
}

// v / s, at most `most` in magnitude (s may have lost bits where it is subnormal)
__device__ __forceinline__ float scaled(double v, double inv, float most) {
  const float t = (float)(v * inv);
  return t > most ? most : t < -most ? -most : t;
}

// 1 / s to the last bit or so: two steps x <- x + x (1 - s x).  v / s is
// rounded to float32 next, which an error of 2^-51 does not reach.
__device__ __forceinline__ double inverse(double s) {
  double x = __builtin_amdgcn_rcp(s);
  x = fma(x, fma(-s, x, 1.0), x);
  return fma(x, fma(-s, x, 1.0), x);
}

__device__ __forceinline__ double moment(double b, double old, double c, double x) {
#pragma clang fp contract(off)
  return b * old + c * x;
}

// One wave per block of 256 elements, four per lane.
template <bool SCALED> __global__ __launch_bounds__(kAdamThreads) void k_adamw8(AdamArgs a) {
  const int k = tensor_of(a, blockIdx.x);
  const AdamTensor& t = a.t[k];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  uint8_t* m = reinterpret_cast<uint8_t*>(t.m);
  uint8_t* v = reinterpret_cast<uint8_t*>(t.v);
  const double c1 = 1.0 - a.b1, c2 = 1.0 - a.b2;
  const double scale = SCALED ? (double)*a.scale : 1.0;
#pragma unroll 1
  for (int u = 0; u < kAdamUnroll; ++u) {
    const int64_t blk = (int64_t)(blockIdx.x - a.first[k]) * (kAdamPer / kBlock) + u * (kAdamThreads / kWave) + wave;
    const int64_t base = blk * kBlock;
    if (base >= t.n) return;
    // whole blocks: four consecutive elements per lane; else every 64th element
    const bool vec = (t.flags & kVector) && base + kBlock <= t.n;
    f32x4 p4, g4;
    unsigned mc = 0, vc = 0;
    if (vec) {
      const int64_t e = base + lane * 4;
      p4 = Stream4<float>::load(t.p + e);
      g4 = t.flags & kGradBf16 ? Stream4<bf16>::load(reinterpret_cast<const bf16*>(t.g) + e)
                               : Stream4<float>::load(reinterpret_cast<const float*>(t.g) + e);
      mc = __builtin_nontemporal_load(reinterpret_cast<const unsigned*>(m + e));
      vc = __builtin_nontemporal_load(reinterpret_cast<const unsigned*>(v + e));
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t e = base + r * kWave + lane;
        const bool in = e < t.n;
        p4[r] = in ? t.p[e] : 0.f;
        g4[r] = !in ? 0.f : t.flags & kGradBf16 ? (float)reinterpret_cast<const bf16*>(t.g)[e] : reinterpret_cast<const float*>(t.g)[e];
        mc |= in ? (unsigned)m[e] << (8 * r) : 0u;
        vc |= in ? (unsigned)v[e] << (8 * r) : 0u;
      }
    }
    const float ms = t.ms[blk], vs = t.vs[blk];
    const f32x2 m01 = __builtin_amdgcn_cvt_pk_f32_fp8(mc, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(mc, true);
    const f32x2 v01 = __builtin_amdgcn_cvt_pk_f32_bf8(vc, false), v23 = __builtin_amdgcn_cvt_pk_f32_bf8(vc, true);
    const float mo[4] = {m01[0], m01[1], m23[0], m23[1]}, vo[4] = {v01[0], v01[1], v23[0], v23[1]};
    double m1[4], v1[4];
    unsigned mtop = 0, vtop = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const double g = SCALED ? g4[r] * scale : (double)g4[r];
      m1[r] = moment(a.b1, (double)mo[r] * ms, c1, g);
      v1[r] = moment(a.b2, (double)vo[r] * vs, c2, g * g);
      mtop = max(mtop, magnitude((float)m1[r]));
      vtop = max(vtop, magnitude((float)v1[r]));
      p4[r] = update(p4[r], (float)m1[r], (float)v1[r], t, a.eps);
    }
    // an infinite or NaN scale spoils its block: every code times it is infinite or NaN
    const float mm = (float)((double)wave_max(mtop) / 448.0), vm = (float)((double)wave_max(vtop) / 57344.0);
    const double mi = mm > 0.f && mm < INFINITY ? inverse(mm) : 0.0, vi = vm > 0.f && vm < INFINITY ? inverse(vm) : 0.0;
    float mt[4], vt[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      mt[r] = scaled(m1[r], mi, 448.f);
      vt[r] = scaled(v1[r], vi, 57344.f);
      if (v1[r] > 0.0 && vi > 0.0 && vt[r] < 0x1p-16f) vt[r] = 0x1p-16f;  // by v1: vt may have become zero in float32
    }
    mc = __builtin_amdgcn_cvt_pk_fp8_f32(mt[0], mt[1], 0, false);
    mc = __builtin_amdgcn_cvt_pk_fp8_f32(mt[2], mt[3], mc, true);
    vc = __builtin_amdgcn_cvt_pk_bf8_f32(vt[0], vt[1], 0, false);
    vc = __builtin_amdgcn_cvt_pk_bf8_f32(vt[2], vt[3], vc, true);
    if (lane == 0) {
      t.ms[blk] = mm;
      t.vs[blk] = vm;
    }
    if (vec) {
      const int64_t e = base + lane * 4;
      Stream4<float>::store(t.p + e, p4);
      if (t.copy) Stream4<bf16>::store(t.copy + e, p4);
      __builtin_nontemporal_store(mc, reinterpret_cast<unsigned*>(m + e));
      __builtin_nontemporal_store(vc, reinterpret_cast<unsigned*>(v + e));
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t e = base + r * kWave + lane;
        if (e >= t.n) break;
        t.p[e] = p4[r];
        if (t.copy) t.copy[e] = (bf16)p4[r];
        m[e] = (uint8_t)(mc >> (8 * r));
        v[e] = (uint8_t)(vc >> (8 * r));
      }
    }
  }
}

bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

int check(const tlf_adamw_tensor& t) {
  if (t.n < 0 || t.step < 1 || !(t.weight_decay >= 0.f) || !(t.weight_decay < INFINITY)) return TLF_E_INVALID_ARG;
  if ((t.grad_dtype != TLF_DTYPE_F32 && t.grad_dtype != TLF_DTYPE_BF16) || (t.state_bits != 32 && t.state_bits != 8))
    return TLF_E_INVALID_ARG;
  if (t.n == 0) return TLF_OK;
  if (!t.d_param || !t.d_grad || !t.d_m || !t.d_v || (t.state_bits == 8 && (!t.d_m_scale || !t.d_v_scale)))
    return TLF_E_INVALID_ARG;
  const bool g16 = t.grad_dtype == TLF_DTYPE_BF16;
  if (!aligned(t.d_param, 4) || !aligned(t.d_copy, 2) || !aligned(t.d_grad, g16 ? 2 : 4) || !aligned(t.d_m_scale, 4) ||
      !aligned(t.d_v_scale, 4) || (t.state_bits == 32 && (!aligned(t.d_m, 4) || !aligned(t.d_v, 4))))
    return TLF_E_INVALID_ARG;
  return t.n > ((int64_t)1 << 35) ? TLF_E_UNSUPPORTED : TLF_OK;
}

// What the step updates must overlap nothing else of the call, since the
// workgroups run in no order; gradients may overlap each other.
int check_overlap(const tlf_adamw_tensor* tensors, int32_t count, const float* scale) {
  struct Range {
    uintptr_t begin, end;
    bool updated;
  };
  const std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[7 * (size_t)count + 2]);
  if (!ranges) return TLF_E_HIP;
  size_t n = 0;
  if (scale) ranges[n++] = Range{(uintptr_t)scale, (uintptr_t)scale + sizeof(float), false};
  for (int i = 0; i < count; ++i) {
    const tlf_adamw_tensor& t = tensors[i];
    auto add = [&](const void* p, int64_t bytes, bool updated) {
      if (p && bytes > 0) ranges[n++] = Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, updated};
    };
    const int64_t moment = t.state_bits / 8, scales = t.state_bits == 8 ? (t.n + kBlock - 1) / kBlock : 0;
    add(t.d_param, t.n * 4, true);
    add(t.d_copy, t.n * 2, true);
    add(t.d_grad, t.n * (t.grad_dtype == TLF_DTYPE_BF16 ? 2 : 4), false);
    add(t.d_m, t.n * moment, true);
    add(t.d_v, t.n * moment, true);
    add(t.d_m_scale, scales * 4, true);
    add(t.d_v_scale, scales * 4, true);
  }
  std::sort(ranges.get(), ranges.get() + n, [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t any = 0, updated = 0;  // where the ranges so far end, and those that are updated
  for (size_t k = 0; k < n; ++k) {
    const Range& r = ranges[k];
    if (r.begin < (r.updated ? any : updated)) return TLF_E_INVALID_ARG;
    any = std::max(any, r.end);
    if (r.updated) updated = std::max(updated, r.end);
  }
  return TLF_OK;
}

int step(const tlf_adamw_tensor* h_tensors, int32_t count, double lr, double beta1, double beta2, double eps,
         const float* d_grad_scale, void* stream) {
  if (count < 0 || (count > 0 && !h_tensors) || !(lr >= 0.0) || !(lr < INFINITY) || !(beta1 >= 0.0) || !(beta1 < 1.0) ||
      !(beta2 >= 0.0) || !(beta2 < 1.0) || !((float)eps >= FLT_MIN) || !((float)eps < INFINITY) || !aligned(d_grad_scale, 4))
    return TLF_E_INVALID_ARG;
  for (int i = 0; i < count; ++i) {
    const int st = check(h_tensors[i]);
    if (st != TLF_OK) return st;
  }
  const int st = check_overlap(h_tensors, count, d_grad_scale);
  if (st != TLF_OK) return st;
  for (int bits : {32, 8}) {
    AdamArgs a{};
    a.b1 = beta1;
    a.b2 = beta2;
    a.eps = (float)eps;
    a.scale = d_grad_scale;
    for (int i = 0; i <= count; ++i) {
      const tlf_adamw_tensor* t = i < count ? &h_tensors[i] : nullptr;
      const bool take = t && t->state_bits == bits && t->n > 0;
      const int64_t blocks = take ? (t->n + kAdamPer - 1) / kAdamPer : 0;
      // full, or done
      if (a.count > 0 && (!t || (take && (a.count == kAdamTensors || a.first[a.count] + blocks > kAdamBlocks)))) {
        auto* kernel = bits == 32 ? (d_grad_scale ? k_adamw<true> : k_adamw<false>) : (d_grad_scale ? k_adamw8<true> : k_adamw8<false>);
        hipLaunchKernelGGL(kernel, dim3(a.first[a.count]), dim3(kAdamThreads), 0, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return TLF_E_HIP;
        a.count = 0;
      }
      if (!take) continue;
      const bool g16 = t->grad_dtype == TLF_DTYPE_BF16;
      const bool vec = aligned(t->d_param, 16) && aligned(t->d_copy, 8) && aligned(t->d_grad, g16 ? 8 : 16) &&
                       aligned(t->d_m, bits == 32 ? 16 : 4) && aligned(t->d_v, bits == 32 ? 16 : 4);
      AdamTensor& o = a.t[a.count];
      o.p = t->d_param;
      o.copy = (bf16*)t->d_copy;
      o.g = t->d_grad;
      o.m = t->d_m;
      o.v = t->d_v;
      o.ms = t->d_m_scale;
      o.vs = t->d_v_scale;
      o.n = t->n;
      o.decay = (float)(1.0 - lr * t->weight_decay);
      o.rate = (float)(lr / (1.0 - pow(beta1, (double)t->step)));
      o.root = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)t->step)));
      o.flags = (g16 ? kGradBf16 : 0) | (vec ? kVector : 0);
      a.first[a.count + 1] = a.first[a.count] + (int32_t)blocks;
      ++a.count;
    }
  }
  return TLF_OK;
}

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_adamw(const tlf_adamw_tensor* h_tensors, int32_t count, double lr, double beta1, double beta2, double eps,
              void* stream) {
  return tlf::step(h_tensors, count, lr, beta1, beta2, eps, nullptr, stream);
}

int tlf_adamw_scaled(const tlf_adamw_tensor* h_tensors, int32_t count, double lr, double beta1, double beta2, double eps,
                     const float* d_grad_scale, void* stream) {
  return d_grad_scale ? tlf::step(h_tensors, count, lr, beta1, beta2, eps, d_grad_scale, stream) : TLF_E_INVALID_ARG;
}

}  // extern "C"
