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

constexpr int kNormWaves = 4;    // rows of a workgroup, a wave each
constexpr int kGradRows = 2;     // rows that a gradient workgroup has in flight
constexpr int kGammaCols = 256;  // columns of a wave
constexpr int kJoinCols = 64;    // columns of a joining workgroup

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

template <int CTRL> __device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, false));
}

// Sum over the 64 lanes of a wave, in the VALU; every lane gets the total.
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp<0xB1>(v);   // lane ^ 1
  v += dpp<0x4E>(v);   // lane ^ 2
  v += dpp<0x141>(v);  // other quad of the 8
  v += dpp<0x140>(v);  // other half of the 16
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Where the call's tensors are more than the memory-side cache holds, the rows are
// loaded past the caches, which else give up what they could serve (us through and
// past them, both gradients, 8 groups: 20000 x 1024 42, 50; 24576 63, 57; 32768 84,
// 71; 65536 154, 140; dx alone 24576 37, 42; 40000 77, 64; forward 40000 38, 45; 65536
// 73, 68; 131072 139, 118).  What is written is read next and stays in them.
constexpr int64_t kCacheBytes = 256ll << 20;
template <bool PAST, typename T> __device__ __forceinline__ f32x4 load4(const T* p) {
  if constexpr (PAST) return Stream4<T>::load(p);
  else return Vec4<T>::load(p);
}

// Four elements as they lie in memory, converted where they are used: a
// conversion next to the load would wait for it there.
template <typename T> struct Raw4;
template <> struct Raw4<float> {
  f32x4 v;
  template <bool PAST> __device__ __forceinline__ void load(const void* p, int64_t at) {
    v = load4<PAST>(reinterpret_cast<const float*>(p) + at);
  }
  __device__ __forceinline__ void zero() { v = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ f32x4 get() const { return v; }
};
template <> struct Raw4<bf16> {
  uint2 v;
  template <bool PAST> __device__ __forceinline__ void load(const void* p, int64_t at) {
    const bf16* s = reinterpret_cast<const bf16*>(p) + at;
    if constexpr (PAST) {
      const auto r = Stream4<bf16>::raw(s);
      v = make_uint2(r[0], r[1]);
    } else {
      v = *reinterpret_cast<const uint2*>(s);
    }
  }
  __device__ __forceinline__ void zero() { v = make_uint2(0, 0); }
  __device__ __forceinline__ f32x4 get() const {
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                 __uint_as_float(v.y & 0xFFFF0000u)};
  }
};

// The row's gamma, or NULL where its group lies outside [0, groups).
__device__ __forceinline__ const float* gamma_of(const float* gamma, const int32_t* group, int groups, int row, int d) {
  const int k = group ? group[row] : 0;
  return gamma && k >= 0 && k < groups ? gamma + (int64_t)k * d : nullptr;
}

// One wave per row, the row in registers: 4 NV elements per lane.  Bound by HBM:
// 32768 x 1024 from float32 to bf16, 8 groups, 41 us behind the gradient's pass
// (4.9 TB/s), 33 again and again on the same rows, of which the memory-side cache
// then holds a part; bf16 rows 28, without gamma 21 (6.3 TB/s).
template <typename TX, typename TY, int NV, bool PAST>
__global__ __launch_bounds__(kNormWaves* kWave) void k_norm(NormArgs a) {
  const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * kNormWaves + threadIdx.x / kWave), lane = lane_id();
  if (row >= a.rows) return;
  const TX* x = reinterpret_cast<const TX*>(a.x) + (int64_t)row * a.d;
  const float* gm = gamma_of(a.gamma, a.group, a.groups, row, a.d);
  f32x4 v[NV];
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    v[k] = c < a.d ? load4<PAST>(x + c) : f32x4{0.f, 0.f, 0.f, 0.f};
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

template <typename TX, typename TY, int NV, bool PAST>
__global__ __launch_bounds__(kNormWaves* kWave) void k_norm_dx(NormArgs a) {
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
      v[k] = load4<PAST>(x + c);
      h[k] = load4<PAST>(dy + c);
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

// Both gradients in one pass: a workgroup takes a run of rows, RU at a time, a
// thread four columns of each (a wave per 256 columns), so that a column of
// gamma's gradient has one owner, which adds its rows in order, each group's in
// registers of its own (the row's group is uniform, a scalar branch picks them;
// with the sums in LDS 108 us where these took 90).  The row's mean goes over the
// waves through LDS, one barrier for RU rows; the next RU rows are on their way
// meanwhile, and the groups of those after them.  x and dy are read once, dx is
// written; the workgroups' sums add 4 groups d bytes each.  32768 x 1024, float32
// x, bf16 dy, both gradients with their sums joined: 71 us for 8 groups (5.2 TB/s
// with the sums), dx alone 54 (6.2 TB/s); bf16 rows the same 71 us for 201 MB, dx
// alone 32 (6.2 TB/s): what is left is the loads' latency between two barriers.
template <typename TX, typename TY, int GMAX, int MAXT, int RU, bool PAST>
__global__ __launch_bounds__(MAXT) void k_norm_grad(NormArgs a, int chunk, float* part) {
  __shared__ __align__(16) float red[2][MAXT / kWave][RU];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave, nw = blockDim.x / kWave, c = tid * 4;
  const bool own = c < a.d;
  const int r0 = blockIdx.x * chunk, r1 = min(a.rows, r0 + chunk);
  const f32x4 zero = f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 sum[GMAX], gain = zero;
#pragma unroll
  for (int k = 0; k < GMAX; ++k) sum[k] = zero;
  if (GMAX == 1 && own) gain = 1.f + Vec4<float>::load(a.gamma + c);
  struct Row {
    Raw4<TX> x;
    Raw4<TY> dy;
    f32x4 gamma;
    float r;
    int k;
  };
  auto group_of = [&](int row) __attribute__((always_inline)) { return a.group ? a.group[min(row, r1 - 1)] : 0; };
  // `group` is made uniform here, a step after its load: at the load it would wait for every load before it
  auto fetch = [&](int row, int group, Row& o) __attribute__((always_inline)) {
    const int g = __builtin_amdgcn_readfirstlane(group), k = g >= 0 && g < a.groups ? g : -1;
    o.k = k;
    o.r = a.rstd[min(row, r1 - 1)];
    o.x.zero();
    o.dy.zero();
    o.gamma = zero;
    if (own && row < r1) {
      o.x.template load<PAST>(a.x, (int64_t)row * a.d + c);
      o.dy.template load<PAST>(a.dy, (int64_t)row * a.d + c);
      if (GMAX > 1 && k >= 0) o.gamma = Vec4<float>::load(a.gamma + (int64_t)k * a.d + c);
    }
  };
  Row cur[RU], next[RU];
  int kn[RU];
#pragma unroll
  for (int u = 0; u < RU; ++u) {
    fetch(r0 + u, group_of(r0 + u), cur[u]);
    kn[u] = group_of(r0 + RU + u);
  }
  for (int row = r0, it = 0; row < r1; row += RU, it ^= 1) {
    f32x4 h[RU];
    float m[RU];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      fetch(row + RU + u, kn[u], next[u]);
      kn[u] = group_of(row + 2 * RU + u);
    }
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      const f32x4 x = cur[u].x.get();
      h[u] = cur[u].dy.get();
      if (GMAX > 1) h[u] *= 1.f + cur[u].gamma;
      else if (cur[u].k >= 0) h[u] *= gain;
      m[u] = wave_sum((x[0] * h[u][0] + x[1] * h[u][1]) + (x[2] * h[u][2] + x[3] * h[u][3]));
    }
    if (lane == 0) {
#pragma unroll
      for (int u = 0; u < RU; ++u) red[it][wave][u] = m[u];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int u = 0; u < RU; ++u) m[u] = red[it][0][u];
    for (int w = 1; w < nw; ++w)
#pragma unroll
      for (int u = 0; u < RU; ++u) m[u] += red[it][w][u];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      if (row + u >= r1) break;
      const float r = cur[u].r, s = r * r * (m[u] / (float)a.d);
      const f32x4 x = cur[u].x.get(), t = cur[u].dy.get() * (x * r);
      if (own && a.out) Vec4<TX>::store(reinterpret_cast<TX*>(a.out) + (int64_t)(row + u) * a.d + c, r * (h[u] - x * s));
#pragma unroll
      for (int k = 0; k < GMAX; ++k)
        if (cur[u].k == k) sum[k] += t;
    }
#pragma unroll
    for (int u = 0; u < RU; ++u) cur[u] = next[u];
  }
  if (!own) return;
  float* o = part + (int64_t)blockIdx.x * a.groups * a.d + c;
#pragma unroll
  for (int k = 0; k < GMAX; ++k)
    if (k < a.groups) Vec4<float>::store(o + k * a.d, sum[k]);
}

// The workgroups' sums, kJoinCols columns of them: each of 16 waves' four 16 lanes
// add every 64th one, those 64 sums are added in a fixed order (32768 x 1024, 8
// groups, 1024 workgroups' sums of 32 KB: 6.9 us, with 256 columns and 16 sums 12).
__global__ __launch_bounds__(1024) void k_norm_join(const float* part, int chunks, int n, float* out) {
  __shared__ __align__(16) float sum[64][kJoinCols];
  const int lane = lane_id(), wave = threadIdx.x / kWave, own = wave * 4 + (lane >> 4), c = (lane & 15) * 4;
  const int e = blockIdx.x * kJoinCols + c;
  f32x4 t = f32x4{0.f, 0.f, 0.f, 0.f};
  if (e < n) {
#pragma unroll 4
    for (int k = own; k < chunks; k += 64) t += Vec4<float>::load(part + (int64_t)k * n + e);
  }
  Vec4<float>::store(&sum[own][c], t);
  __syncthreads();
  if (wave > 0) return;
  t = Vec4<float>::load(&sum[lane >> 4][c]);
#pragma unroll
  for (int k = 4; k < 64; k += 4) t += Vec4<float>::load(&sum[k + (lane >> 4)][c]);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    t[r] += shfl_xor(t[r], 16);
    t[r] += shfl_xor(t[r], 32);
  }
  if (lane < 16 && e < n) Vec4<float>::store(out + e, t);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Rows of a workgroup: 16 waves per compute unit where the rows allow it (8 with
// twice the rows in flight were slower: 32768 x 1024, 8 groups, 107 against 90
// us), and 8 rows at least, so that the sums stay a small part of the traffic
// and few rows still spread (300 x 1024: 16 rows 16 us, 8 rows 12).
int grad_chunk(int rows, int d) {
  const int waves = (d + kGammaCols - 1) / kGammaCols, most = 4096 / waves;
  const int c = (rows + most - 1) / most;
  return c < 8 ? 8 : c;
}
int grad_chunks(int rows, int d) { return (rows + grad_chunk(rows, d) - 1) / grad_chunk(rows, d); }

bool is_dtype(int32_t t) { return t == TLF_DTYPE_F32 || t == TLF_DTYPE_BF16; }

int check(int32_t x_dtype, int32_t y_dtype, int32_t groups, int32_t rows, int32_t d) {
  if (!is_dtype(x_dtype) || !is_dtype(y_dtype) || groups < 0 || rows < 0 || d <= 0 || d % 4 != 0) return TLF_E_INVALID_ARG;
  return d > TLF_NORM_MAX_D || groups > TLF_NORM_MAX_GROUPS || rows > TLF_NORM_MAX_ROWS ? TLF_E_UNSUPPORTED : TLF_OK;
}

constexpr int kLaunchRows = 1 << 24;  // a launch has fewer than 2^32 threads

template <typename TX, typename TY, bool GRAD, bool PAST> hipError_t launch_rows(NormArgs a, hipStream_t s) {
  if (a.rows > kLaunchRows) {
    NormArgs head = a;
    head.rows = kLaunchRows;
    const hipError_t e = launch_rows<TX, TY, GRAD, PAST>(head, s);
    if (e != hipSuccess) return e;
    const int64_t n = (int64_t)kLaunchRows * a.d;
    a.x = reinterpret_cast<const TX*>(a.x) + n;
    if (GRAD) a.dy = reinterpret_cast<const TY*>(a.dy) + n;
    a.out = reinterpret_cast<char*>(a.out) + n * (GRAD ? sizeof(TX) : sizeof(TY));
    if (a.group) a.group += kLaunchRows;
    if (a.rstd) a.rstd += kLaunchRows;
    a.rows -= kLaunchRows;
    return launch_rows<TX, TY, GRAD, PAST>(a, s);
  }
  const dim3 grid((a.rows + kNormWaves - 1) / kNormWaves), block(kNormWaves * kWave);
#define TLF_NORM(NV)                                                                   \
  if (GRAD) hipLaunchKernelGGL((k_norm_dx<TX, TY, NV, PAST>), grid, block, 0, s, a);   \
  else hipLaunchKernelGGL((k_norm<TX, TY, NV, PAST>), grid, block, 0, s, a)
  if (a.d <= 256) { TLF_NORM(1); }
  else if (a.d <= 512) { TLF_NORM(2); }
  else if (a.d <= 1024) { TLF_NORM(4); }
  else if (a.d <= 2048) { TLF_NORM(8); }
  else { TLF_NORM(16); }
#undef TLF_NORM
  return hipGetLastError();
}

template <typename TX, typename TY, bool GRAD> hipError_t launch_rows(const NormArgs& a, hipStream_t s) {
  const int64_t bytes = (int64_t)a.rows * a.d * (int64_t)(GRAD ? 2 * sizeof(TX) + sizeof(TY) : sizeof(TX) + sizeof(TY));
  return bytes > kCacheBytes ? launch_rows<TX, TY, GRAD, true>(a, s) : launch_rows<TX, TY, GRAD, false>(a, s);
}

template <typename TX, typename TY, int MAXT, int RU, bool PAST>
void launch_sums(const NormArgs& a, int chunk, int chunks, float* part, hipStream_t s) {
  const dim3 grid(chunks), block((a.d + kGammaCols - 1) / kGammaCols * kWave);
  if (a.groups == 1) hipLaunchKernelGGL((k_norm_grad<TX, TY, 1, MAXT, RU, PAST>), grid, block, 0, s, a, chunk, part);
  else if (a.groups <= 8) hipLaunchKernelGGL((k_norm_grad<TX, TY, 8, MAXT, RU, PAST>), grid, block, 0, s, a, chunk, part);
  else hipLaunchKernelGGL((k_norm_grad<TX, TY, TLF_NORM_MAX_GROUPS, MAXT, RU, PAST>), grid, block, 0, s, a, chunk, part);
}

template <typename TX, typename TY, bool PAST>
void launch_width(const NormArgs& a, int chunk, int chunks, float* part, hipStream_t s) {
  if (a.d <= 1024) launch_sums<TX, TY, 256, kGradRows, PAST>(a, chunk, chunks, part, s);
  else if (a.d <= 2048) launch_sums<TX, TY, 512, kGradRows, PAST>(a, chunk, chunks, part, s);
  else launch_sums<TX, TY, 1024, kGradRows, PAST>(a, chunk, chunks, part, s);
}

template <typename TX, typename TY> hipError_t launch_grad(const NormArgs& a, void* dx, float* dgamma, float* part, hipStream_t s) {
  NormArgs b = a;
  b.out = dx;
  if (!dgamma) return a.rows > 0 ? launch_rows<TX, TY, true>(b, s) : hipSuccess;
  const int chunk = grad_chunk(a.rows, a.d), chunks = grad_chunks(a.rows, a.d), n = a.groups * a.d;
  if (chunks > 0) {
    const int64_t row = (int64_t)a.d * (int64_t)(2 * sizeof(TX) + sizeof(TY)), sums = (int64_t)chunks * n * 4;
    if (a.rows * row + sums > kCacheBytes) launch_width<TX, TY, true>(b, chunk, chunks, part, s);
    else launch_width<TX, TY, false>(b, chunk, chunks, part, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_norm_join, dim3((n + kJoinCols - 1) / kJoinCols), dim3(1024), 0, s, part, chunks, n, dgamma);
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
  *ws_bytes = (size_t)tlf::grad_chunks(rows, d) * groups * d * sizeof(float);
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
