// RMSNorm of the training rows (Appendix A) with the AdaLN scale of a row's
// group (Section 3.1), forward and backward: the C entry points tlf_rms_norm
// and tlf_rms_norm_grad and their kernels.
//
//   r = 1 / sqrt(mean x^2 + eps),  y = x r (1 + gamma[group])
//   h = dy (1 + gamma[group]),  dx = r (h - x r^2 mean(h x)),
//   dgamma[k] = sum over the rows of group k of dy x r
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "tlf.h"

namespace tlf {

namespace {

constexpr int kNormWaves = 4;      // rows of a workgroup
constexpr int kGammaCols = 256;    // columns of a gamma-gradient workgroup
constexpr int kGammaChunks = 128;  // at most so many row chunks of partial sums

struct NormArgs {
  const void* x;
  const void* dy;
  const float* gamma;
  const int32_t* group;
  float* rstd;
  void* out;  // y or dx
  int rows, d, groups;
  float eps;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += shfl_xor(v, o);
  return v;
}

// The row's gamma, or NULL where its group lies outside [0, groups).
__device__ __forceinline__ const float* gamma_of(const float* gamma, const int32_t* group, int groups, int row, int d) {
  const int k = group ? group[row] : 0;
  return gamma && k >= 0 && k < groups ? gamma + (int64_t)k * d : nullptr;
}

// One wave per row, the row in registers: 4 NV elements per lane.
template <typename TX, typename TY, int NV> __global__ __launch_bounds__(kNormWaves* kWave) void k_norm(NormArgs a) {
  const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * kNormWaves + threadIdx.x / kWave), lane = lane_id();
  if (row >= a.rows) return;
  const TX* x = reinterpret_cast<const TX*>(a.x) + (int64_t)row * a.d;
  const float* gm = gamma_of(a.gamma, a.group, a.groups, row, a.d);
  f32x4 v[NV];
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    v[k] = c < a.d ? Vec4<TX>::load(x + c) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) ss += (v[k][0] * v[k][0] + v[k][1] * v[k][1]) + (v[k][2] * v[k][2] + v[k][3] * v[k][3]);
  const float r = 1.f / sqrtf(wave_sum(ss) / (float)a.d + a.eps);
  if (a.rstd && lane == 0) a.rstd[row] = r;
  TY* y = reinterpret_cast<TY*>(a.out) + (int64_t)row * a.d;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    if (c >= a.d) continue;
    f32x4 o = v[k] * r;
    if (gm) o *= 1.f + Vec4<float>::load(gm + c);
    Vec4<TY>::store(y + c, o);
  }
}

template <typename TX, typename TY, int NV> __global__ __launch_bounds__(kNormWaves* kWave) void k_norm_dx(NormArgs a) {
  const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * kNormWaves + threadIdx.x / kWave), lane = lane_id();
  if (row >= a.rows) return;
  const TX* x = reinterpret_cast<const TX*>(a.x) + (int64_t)row * a.d;
  const TY* dy = reinterpret_cast<const TY*>(a.dy) + (int64_t)row * a.d;
  const float* gm = gamma_of(a.gamma, a.group, a.groups, row, a.d);
  const float r = a.rstd[row];
  f32x4 v[NV], h[NV];
  float hx = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    v[k] = h[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (c < a.d) {
      v[k] = Vec4<TX>::load(x + c);
      h[k] = Vec4<TY>::load(dy + c);
      if (gm) h[k] *= 1.f + Vec4<float>::load(gm + c);
    }
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
    hx += (v[k][0] * h[k][0] + v[k][1] * h[k][1]) + (v[k][2] * h[k][2] + v[k][3] * h[k][3]);
  const float s = r * r * (wave_sum(hx) / (float)a.d);
  TX* dx = reinterpret_cast<TX*>(a.out) + (int64_t)row * a.d;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    if (c < a.d) Vec4<TX>::store(dx + c, r * (h[k] - v[k] * s));
  }
}

// gamma's gradient of one row chunk and 256 columns: each wave adds its rows
// into its own LDS sums (one lane owns a column, so the order is fixed), the
// waves' sums are added in order.
template <typename TX, typename TY>
__global__ __launch_bounds__(kNormWaves* kWave) void k_norm_dgamma(NormArgs a, int chunk, float* part) {
  __shared__ __align__(16) float sum[kNormWaves][TLF_NORM_MAX_GROUPS][kGammaCols];
  const int lane = lane_id(), wave = threadIdx.x / kWave, c = blockIdx.y * kGammaCols + lane * 4;
  for (int k = 0; k < a.groups; ++k) Vec4<float>::store(&sum[wave][k][lane * 4], f32x4{0.f, 0.f, 0.f, 0.f});
  const int r0 = blockIdx.x * chunk, r1 = min(a.rows, r0 + chunk);
  if (c < a.d) {
    for (int row = r0 + wave; row < r1; row += kNormWaves) {
      const int k = a.group ? a.group[row] : 0;
      if (k < 0 || k >= a.groups) continue;
      const int64_t o = (int64_t)row * a.d + c;
      const f32x4 t = Vec4<TY>::load(reinterpret_cast<const TY*>(a.dy) + o) *
                      (Vec4<TX>::load(reinterpret_cast<const TX*>(a.x) + o) * a.rstd[row]);
      float* s = &sum[wave][k][lane * 4];
      Vec4<float>::store(s, Vec4<float>::load(s) + t);
    }
  }
  __syncthreads();
  for (int k = wave; k < a.groups; k += kNormWaves) {
    if (c >= a.d) break;
    f32x4 t = Vec4<float>::load(&sum[0][k][lane * 4]);
#pragma unroll
    for (int w = 1; w < kNormWaves; ++w) t += Vec4<float>::load(&sum[w][k][lane * 4]);
    Vec4<float>::store(part + ((int64_t)blockIdx.x * a.groups + k) * a.d + c, t);
  }
}

// The chunks' sums, added in order.
__global__ __launch_bounds__(256) void k_norm_join(const float* part, int chunks, int n, float* out) {
  const int e = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= n) return;
  f32x4 t = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < chunks; ++k) t += Vec4<float>::load(part + (int64_t)k * n + e);
  Vec4<float>::store(out + e, t);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

int gamma_chunk(int rows) {
  int c = (rows + kGammaChunks - 1) / kGammaChunks;
  return c < 16 ? 16 : c;
}
int gamma_chunks(int rows) { return (rows + gamma_chunk(rows) - 1) / gamma_chunk(rows); }

bool is_dtype(int32_t t) { return t == TLF_DTYPE_F32 || t == TLF_DTYPE_BF16; }

int check(int32_t x_dtype, int32_t y_dtype, int32_t groups, int32_t rows, int32_t d) {
  if (!is_dtype(x_dtype) || !is_dtype(y_dtype) || groups < 0 || rows < 0 || d <= 0 || d % 4 != 0) return TLF_E_INVALID_ARG;
  return d > TLF_NORM_MAX_D || groups > TLF_NORM_MAX_GROUPS ? TLF_E_UNSUPPORTED : TLF_OK;
}

template <typename TX, typename TY, bool GRAD> hipError_t launch_rows(const NormArgs& a, hipStream_t s) {
  const dim3 grid((a.rows + kNormWaves - 1) / kNormWaves), block(kNormWaves * kWave);
#define TLF_NORM(NV)                                                                   \
  if (GRAD) hipLaunchKernelGGL((k_norm_dx<TX, TY, NV>), grid, block, 0, s, a);         \
  else hipLaunchKernelGGL((k_norm<TX, TY, NV>), grid, block, 0, s, a)
  if (a.d <= 256) { TLF_NORM(1); }
  else if (a.d <= 512) { TLF_NORM(2); }
  else if (a.d <= 1024) { TLF_NORM(4); }
  else if (a.d <= 2048) { TLF_NORM(8); }
  else { TLF_NORM(16); }
#undef TLF_NORM
  return hipGetLastError();
}

template <typename TX, typename TY> hipError_t launch_grad(const NormArgs& a, void* dx, float* dgamma, float* part, hipStream_t s) {
  if (dx && a.rows > 0) {
    NormArgs b = a;
    b.out = dx;
    const hipError_t e = launch_rows<TX, TY, true>(b, s);
    if (e != hipSuccess) return e;
  }
  if (dgamma) {
    const int chunks = gamma_chunks(a.rows), n = a.groups * a.d;
    if (chunks > 0)
      hipLaunchKernelGGL((k_norm_dgamma<TX, TY>), dim3(chunks, (a.d + kGammaCols - 1) / kGammaCols),
                         dim3(kNormWaves * kWave), 0, s, a, gamma_chunk(a.rows), part);
    hipLaunchKernelGGL(k_norm_join, dim3((n / 4 + 255) / 256), dim3(256), 0, s, part, chunks, n, dgamma);
  }
  return hipGetLastError();
}

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_rms_norm(const void* d_x, int32_t x_dtype, const float* d_gamma, const int32_t* d_group, int32_t groups,
                 int32_t rows, int32_t d, float eps, void* d_y, int32_t y_dtype, float* d_rstd, void* stream) {
  const int st = tlf::check(x_dtype, y_dtype, groups, rows, d);
  if (st != TLF_OK) return st;
  if (!(eps > 0.f) || (groups > 0) != (d_gamma != nullptr)) return TLF_E_INVALID_ARG;
  if (rows == 0) return TLF_OK;
  if (!d_x || !d_y || (groups > 1 && !d_group)) return TLF_E_INVALID_ARG;
  if (!tlf::aligned16(d_x) || !tlf::aligned16(d_y) || !tlf::aligned16(d_gamma)) return TLF_E_INVALID_ARG;
  tlf::NormArgs a{d_x, nullptr, d_gamma, d_group, d_rstd, d_y, rows, d, groups, eps};
  const hipStream_t s = (hipStream_t)stream;
  const bool xb = x_dtype == TLF_DTYPE_BF16, yb = y_dtype == TLF_DTYPE_BF16;
  const hipError_t e = xb ? (yb ? tlf::launch_rows<bf16, bf16, false>(a, s) : tlf::launch_rows<bf16, float, false>(a, s))
                          : (yb ? tlf::launch_rows<float, bf16, false>(a, s) : tlf::launch_rows<float, float, false>(a, s));
  return e == hipSuccess ? TLF_OK : TLF_E_HIP;
}

int tlf_rms_norm_grad_ws_bytes(int32_t groups, int32_t rows, int32_t d, size_t* ws_bytes) {
  const int st = tlf::check(TLF_DTYPE_F32, TLF_DTYPE_F32, groups, rows, d);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  *ws_bytes = (size_t)tlf::gamma_chunks(rows) * groups * d * sizeof(float);
  return TLF_OK;
}

int tlf_rms_norm_grad(const void* d_dy, int32_t y_dtype, const void* d_x, int32_t x_dtype, const float* d_gamma,
                      const int32_t* d_group, int32_t groups, const float* d_rstd, int32_t rows, int32_t d, void* d_dx,
                      float* d_dgamma, void* d_workspace, size_t ws_bytes, void* stream) {
  const int st = tlf::check(x_dtype, y_dtype, groups, rows, d);
  if (st != TLF_OK) return st;
  if ((groups > 0) != (d_gamma != nullptr) || (d_dgamma && groups == 0)) return TLF_E_INVALID_ARG;
  if (!d_dx && !d_dgamma) return TLF_OK;
  if (rows > 0 && (!d_dy || !d_x || !d_rstd || (groups > 1 && !d_group))) return TLF_E_INVALID_ARG;
  for (const void* p : {d_dy, d_x, (const void*)d_gamma, (const void*)d_dx, (const void*)d_dgamma, (const void*)d_workspace})
    if (!tlf::aligned16(p)) return TLF_E_INVALID_ARG;
  size_t need = 0;
  tlf_rms_norm_grad_ws_bytes(groups, rows, d, &need);
  if (d_dgamma && need > 0 && (!d_workspace || ws_bytes < need)) return TLF_E_INVALID_ARG;
  tlf::NormArgs a{d_x, d_dy, d_gamma, d_group, const_cast<float*>(d_rstd), nullptr, rows, d, groups, 0.f};
  const hipStream_t s = (hipStream_t)stream;
  float* part = (float*)d_workspace;
  const bool xb = x_dtype == TLF_DTYPE_BF16, yb = y_dtype == TLF_DTYPE_BF16;
  const hipError_t e = xb ? (yb ? tlf::launch_grad<bf16, bf16>(a, d_dx, d_dgamma, part, s)
                                : tlf::launch_grad<bf16, float>(a, d_dx, d_dgamma, part, s))
                          : (yb ? tlf::launch_grad<float, bf16>(a, d_dx, d_dgamma, part, s)
                                : tlf::launch_grad<float, float>(a, d_dx, d_dgamma, part, s));
  return e == hipSuccess ? TLF_OK : TLF_E_HIP;
}

}  // extern "C"
