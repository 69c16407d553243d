// The gated residual of the training rows with the norm that follows it (Section
// 3.1, Appendix A), forward and backward: the C entry points tlf_residual_norm and
// tlf_residual_norm_grad and their kernels.
//
//   t = y, or y ry with ry = 1 / sqrt(mean y^2 + eps)  (post_norm)
//   h = x + (1 + alpha[group]) t,  r = 1 / sqrt(mean h^2 + eps),  z = h r (1 + gamma[group])
//
// With u = dz (1 + gamma[group]), and e = dh + r (u - h r^2 mean(u h)), h's whole gradient:
//   dx = e,  dt = e (1 + alpha[group]),  dy = dt, or ry (dt - y ry^2 mean(dt y))
//   dalpha[k] = sum over the rows of group k of e t,  dgamma[k] = of dz h r
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "rownorm.h"
#include "tlf.h"

namespace tlf {

namespace {

constexpr int kRowWaves = 4;  // rows of a workgroup, a wave each
constexpr int kMaxSums = 8;   // groups whose sums a thread holds

struct ResidArgs {
  const float* x;  // h in the backward pass
  const void* y;
  const float *alpha, *gamma;
  const int32_t* group;
  const float* dh;
  const void* dz;
  float *h, *rstd, *ystd;  // h: dx in the backward pass
  void* z;                 // dy in the backward pass
  int rows, d, groups;
  float eps;
};

__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return (a[0] * b[0] + a[1] * b[1]) + (a[2] * b[2] + a[3] * b[3]); }

// One wave per row, the row in registers: 4 NV elements of x and of y per lane, so that
// nothing is read twice and no row waits for another.  Bound by HBM: 32768 x 1024 bf16 y,
// 8 groups 76 us, 5.3 TB/s (a copy of 1 GiB: 5.1); 9999 x 2048 float32, post_norm 69 us, 4.7.
template <typename T, int NV, bool POST, bool PAST>
__global__ __launch_bounds__(kRowWaves* kWave) void k_resid(ResidArgs a) {
  const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * kRowWaves + threadIdx.x / kWave), lane = lane_id();
  if (row >= a.rows) return;
  const int64_t at = (int64_t)row * a.d;
  const float* al = gamma_of(a.alpha, a.group, a.groups, row, a.d);
  const float* gm = gamma_of(a.gamma, a.group, a.groups, row, a.d);
  f32x4 h[NV];
  Raw4<T> y[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    h[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    y[k].zero();
    if (c < a.d) {
      y[k].template load<PAST>(a.y, at + c);
      h[k] = load4<PAST>(a.x + at + c);
    }
  }
  float ry = 1.f;
  if (POST) {
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) ss += dot4(y[k].get(), y[k].get());
    ry = 1.f / sqrtf(wave_sum(ss) / (float)a.d + a.eps);
    if (a.ystd && lane == 0) a.ystd[row] = ry;
  }
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    f32x4 t = y[k].get();
    if (POST) t *= ry;
    if (al && c < a.d) t *= 1.f + Vec4<float>::load(al + c);
    h[k] += t;
    ss += dot4(h[k], h[k]);
  }
  const float r = 1.f / sqrtf(wave_sum(ss) / (float)a.d + a.eps);
  if (a.rstd && lane == 0) a.rstd[row] = r;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    if (c >= a.d) continue;
    Vec4<float>::store(a.h + at + c, h[k]);
    f32x4 o = h[k] * r;
    if (gm) o *= 1.f + Vec4<float>::load(gm + c);
    Vec4<T>::store(reinterpret_cast<T*>(a.z) + at + c, o);
  }
}

// The rows' gradients alone, a wave per row.  The second mean, of dt y, is linear in
// the first: all sums of a row are taken at once.
template <typename T, int NV, bool POST, bool PAST>
__global__ __launch_bounds__(kRowWaves* kWave) void k_resid_dx(ResidArgs a) {
  const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * kRowWaves + threadIdx.x / kWave), lane = lane_id();
  if (row >= a.rows) return;
  const int64_t at = (int64_t)row * a.d;
  const float* al = gamma_of(a.alpha, a.group, a.groups, row, a.d);
  const float* gm = gamma_of(a.gamma, a.group, a.groups, row, a.d);
  const float r = a.rstd[row], ry = POST ? a.ystd[row] : 1.f;
  f32x4 h[NV], e[NV];  // e: dh + r u, then dx
  Raw4<T> y[NV];
  float uh = 0.f, ey = 0.f, hy = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    h[k] = e[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    y[k].zero();
    if (c >= a.d) continue;
    if (POST) y[k].template load<PAST>(a.y, at + c);
    h[k] = load4<PAST>(a.x + at + c);
    f32x4 u = f32x4{0.f, 0.f, 0.f, 0.f};
    if (a.dz) u = load4<PAST>(reinterpret_cast<const T*>(a.dz) + at + c);
    if (a.dh) e[k] = load4<PAST>(a.dh + at + c);
    if (gm) u *= 1.f + Vec4<float>::load(gm + c);
    uh += dot4(u, h[k]);
    e[k] += r * u;
    if (POST) {
      f32x4 ya = y[k].get();
      if (al) ya *= 1.f + Vec4<float>::load(al + c);
      ey += dot4(e[k], ya);
      hy += dot4(h[k], ya);
    }
  }
  const float s = r * (r * r * (wave_sum(uh) / (float)a.d));  // r's cube alone may leave float32's range
  float q = 0.f;
  if (POST) q = ry * ry * ((wave_sum(ey) - s * wave_sum(hy)) / (float)a.d);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * kWave + lane) * 4;
    if (c >= a.d) continue;
    e[k] -= h[k] * s;
    Vec4<float>::store(a.h + at + c, e[k]);
    f32x4 o = e[k];
    if (al) o *= 1.f + Vec4<float>::load(al + c);
    if (POST) o = ry * (o - y[k].get() * q);
    Vec4<T>::store(reinterpret_cast<T*>(a.z) + at + c, o);
  }
}

// The rows' gradients and the sums of alpha's and gamma's in one pass: a workgroup
// takes a run of rows, RU at a time, a thread four columns of each, so that a column
// of the sums has one owner that adds its rows in order, the groups from `first` on in
// registers of their own.  The rows' sums go over the waves through LDS, one barrier
// for RU rows; the next RU rows are on their way meanwhile.  With more groups than
// kMaxSums the pass is made again for those behind them, without the rows' gradients.
// Bound by HBM, and by the loads' latency between two barriers: 32768 x 1024 bf16 y, 8
// groups 122-125 us, 4.9 TB/s; 9999 x 2048 float32, post_norm, 3 groups 100 us, 4.9.
template <typename T, int GMAX, int MAXT, int RU, bool POST, bool PAST>
__global__ __launch_bounds__(MAXT) void k_resid_grad(ResidArgs a, int chunk, int first, float* part) {
  constexpr int SUMS = POST ? 3 : 1;
  __shared__ __align__(16) float red[2][MAXT / kWave][RU][SUMS];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave, nw = blockDim.x / kWave, c = tid * 4;
  const bool own = c < a.d;
  const int r0 = blockIdx.x * chunk, r1 = min(a.rows, r0 + chunk);
  const f32x4 zero = f32x4{0.f, 0.f, 0.f, 0.f}, one = f32x4{1.f, 1.f, 1.f, 1.f};
  f32x4 sa[GMAX], sg[GMAX], gain_a = one, gain_g = one;
#pragma unroll
  for (int k = 0; k < GMAX; ++k) sa[k] = sg[k] = zero;
  if (GMAX == 1 && own) {
    if (a.alpha) gain_a = 1.f + Vec4<float>::load(a.alpha + c);
    if (a.gamma) gain_g = 1.f + Vec4<float>::load(a.gamma + c);
  }
  struct Row {
    f32x4 h, dh, alpha, gamma;
    Raw4<T> y, dz;
    float r, ry;
    int k;
  };
  auto group_of = [&](int row) __attribute__((always_inline)) { return a.group ? a.group[min(row, r1 - 1)] : 0; };
  // `group` is made uniform here, a step after its load: at the load it would wait for every load before it
  auto fetch = [&](int row, int group, Row& o) __attribute__((always_inline)) {
    const int g = __builtin_amdgcn_readfirstlane(group), k = g >= 0 && g < a.groups ? g : -1;
    o.k = k;
    o.r = a.rstd[min(row, r1 - 1)];
    o.ry = POST ? a.ystd[min(row, r1 - 1)] : 1.f;
    o.h = o.dh = o.alpha = o.gamma = zero;
    o.y.zero();
    o.dz.zero();
    if (own && row < r1) {
      const int64_t at = (int64_t)row * a.d + c;
      o.h = load4<PAST>(a.x + at);
      o.y.template load<PAST>(a.y, at);
      if (a.dz) o.dz.template load<PAST>(a.dz, at);
      if (a.dh) o.dh = load4<PAST>(a.dh + at);
      if (GMAX > 1 && k >= 0) {
        if (a.alpha) o.alpha = Vec4<float>::load(a.alpha + (int64_t)k * a.d + c);
        if (a.gamma) o.gamma = Vec4<float>::load(a.gamma + (int64_t)k * a.d + c);
      }
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
    f32x4 e[RU], al[RU];
    float m[RU][SUMS];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      fetch(row + RU + u, kn[u], next[u]);
      kn[u] = group_of(row + 2 * RU + u);
    }
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      f32x4 w = cur[u].dz.get();
      if (GMAX > 1) w *= 1.f + cur[u].gamma;
      else if (cur[u].k >= 0) w *= gain_g;
      al[u] = GMAX > 1 ? 1.f + cur[u].alpha : cur[u].k >= 0 ? gain_a : one;
      m[u][0] = wave_sum(dot4(w, cur[u].h));
      e[u] = cur[u].dh + cur[u].r * w;
      if constexpr (POST) {
        const f32x4 ya = cur[u].y.get() * al[u];
        m[u][1] = wave_sum(dot4(e[u], ya));
        m[u][2] = wave_sum(dot4(cur[u].h, ya));
      }
    }
    if (lane == 0) {
#pragma unroll
      for (int u = 0; u < RU; ++u)
#pragma unroll
        for (int x = 0; x < SUMS; ++x) red[it][wave][u][x] = m[u][x];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int u = 0; u < RU; ++u)
#pragma unroll
      for (int x = 0; x < SUMS; ++x) m[u][x] = red[it][0][u][x];
    for (int w = 1; w < nw; ++w)
#pragma unroll
      for (int u = 0; u < RU; ++u)
#pragma unroll
        for (int x = 0; x < SUMS; ++x) m[u][x] += red[it][w][u][x];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      if (row + u >= r1) break;
      const float r = cur[u].r, ry = cur[u].ry, s = r * (r * r * (m[u][0] / (float)a.d));
      const f32x4 y = cur[u].y.get();
      e[u] -= cur[u].h * s;
      if (own && first == 0) {
        const int64_t at = (int64_t)(row + u) * a.d + c;
        f32x4 o = e[u] * al[u];
        if constexpr (POST) o = ry * (o - y * (ry * ry * ((m[u][1] - s * m[u][2]) / (float)a.d)));
        Vec4<float>::store(a.h + at, e[u]);
        Vec4<T>::store(reinterpret_cast<T*>(a.z) + at, o);
      }
      const f32x4 ta = POST ? e[u] * (y * ry) : e[u] * y, tg = cur[u].dz.get() * (cur[u].h * r);
#pragma unroll
      for (int k = 0; k < GMAX; ++k)
        if (cur[u].k == first + k) {
          sa[k] += ta;
          sg[k] += tg;
        }
    }
#pragma unroll
    for (int u = 0; u < RU; ++u) cur[u] = next[u];
  }
  if (!own) return;
  // [workgroup][alpha's, then gamma's groups][d], of those that there are
  const int sets = (a.alpha != nullptr) + (a.gamma != nullptr);
  float* o = part + (int64_t)blockIdx.x * sets * a.groups * a.d + c;
  if (a.alpha) {
#pragma unroll
    for (int k = 0; k < GMAX; ++k)
      if (first + k < a.groups) Vec4<float>::store(o + (int64_t)(first + k) * a.d, sa[k]);
    o += (int64_t)a.groups * a.d;
  }
  if (a.gamma) {
#pragma unroll
    for (int k = 0; k < GMAX; ++k)
      if (first + k < a.groups) Vec4<float>::store(o + (int64_t)(first + k) * a.d, sg[k]);
  }
}

// Rows of a workgroup: 8 waves per compute unit where the rows allow it, all that the
// registers let run at a time, and 8 rows at least, so that the sums stay a small part
// of the traffic and few rows still spread.  Twice as many workgroups write twice the
// sums (32768 x 1024, 8 groups: the join 11.8 us, so 6.8; the rows' pass the same).
int resid_chunk(int rows, int d) {
  const int waves = (d + kGammaCols - 1) / kGammaCols, most = 2048 / waves;
  const int c = (rows + most - 1) / most;
  return c < 8 ? 8 : c;
}

constexpr int kLaunchRows = 1 << 24;  // a launch has fewer than 2^32 threads

template <typename T, bool GRAD, bool POST, bool PAST> hipError_t launch_rows(ResidArgs a, hipStream_t s) {
  for (;;) {
    ResidArgs b = a;
    b.rows = a.rows < kLaunchRows ? a.rows : kLaunchRows;
    const dim3 grid((b.rows + kRowWaves - 1) / kRowWaves), block(kRowWaves * kWave);
#define TLF_RESID(NV)                                                                        \
  if (GRAD) hipLaunchKernelGGL((k_resid_dx<T, NV, POST, PAST>), grid, block, 0, s, b);       \
  else hipLaunchKernelGGL((k_resid<T, NV, POST, PAST>), grid, block, 0, s, b)
    if (a.d <= 256) { TLF_RESID(1); }
    else if (a.d <= 512) { TLF_RESID(2); }
    else if (a.d <= 1024) { TLF_RESID(4); }
    else if (a.d <= 2048) { TLF_RESID(8); }
    else { TLF_RESID(16); }
#undef TLF_RESID
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.rows <= kLaunchRows) return e;
    const int64_t n = (int64_t)kLaunchRows * a.d;
    auto on = [n](const void* p, size_t each) { return p ? (const char*)p + n * (int64_t)each : nullptr; };
    a.x = (const float*)on(a.x, 4);
    a.y = on(a.y, sizeof(T));
    a.dh = (const float*)on(a.dh, 4);
    a.dz = on(a.dz, sizeof(T));
    a.h = (float*)on(a.h, 4);
    a.z = (void*)on(a.z, sizeof(T));
    if (a.group) a.group += kLaunchRows;
    if (a.rstd) a.rstd += kLaunchRows;
    if (a.ystd) a.ystd += kLaunchRows;
    a.rows -= kLaunchRows;
  }
}

template <typename T, int MAXT, int RU, bool POST, bool PAST>
void launch_sums(const ResidArgs& a, int chunk, int chunks, float* part, hipStream_t s) {
  const dim3 grid(chunks), block((a.d + kGammaCols - 1) / kGammaCols * kWave);
  if (a.groups == 1) hipLaunchKernelGGL((k_resid_grad<T, 1, MAXT, RU, POST, PAST>), grid, block, 0, s, a, chunk, 0, part);
  else
    for (int first = 0; first < a.groups; first += kMaxSums)
      hipLaunchKernelGGL((k_resid_grad<T, kMaxSums, MAXT, RU, POST, PAST>), grid, block, 0, s, a, chunk, first, part);
}

template <typename T, bool POST, bool PAST>
hipError_t launch_grad(const ResidArgs& a, float* dalpha, float* dgamma, float* part, hipStream_t s) {
  if (!dalpha && !dgamma) return a.rows > 0 ? launch_rows<T, true, POST, PAST>(a, s) : hipSuccess;
  const int chunk = resid_chunk(a.rows, a.d), chunks = (a.rows + chunk - 1) / chunk, n = a.groups * a.d;
  if (chunks > 0) {
    if (a.d <= 1024) launch_sums<T, 256, 2, POST, PAST>(a, chunk, chunks, part, s);
    else if (a.d <= 2048) launch_sums<T, 512, 2, POST, PAST>(a, chunk, chunks, part, s);
    else launch_sums<T, 1024, 1, POST, PAST>(a, chunk, chunks, part, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int all = n * ((a.alpha != nullptr) + (a.gamma != nullptr));
  float* out = a.alpha ? dalpha : dgamma;
  hipLaunchKernelGGL(k_norm_join, dim3((all + kJoinCols - 1) / kJoinCols), dim3(1024), 0, s, part, chunks, all, out, n, dgamma);
  return hipGetLastError();
}

template <typename T, bool GRAD>
hipError_t launch(const ResidArgs& a, bool post, float* dalpha, float* dgamma, float* part, hipStream_t s) {
  // past the caches where the call's tensors exceed them, as the norm's
  const bool past = (int64_t)a.rows * a.d * (int64_t)((GRAD ? 3 : 2) * 4 + (GRAD ? 3 : 2) * sizeof(T)) > kCacheBytes;
  if constexpr (GRAD) {
    if (post) return past ? launch_grad<T, true, true>(a, dalpha, dgamma, part, s) : launch_grad<T, true, false>(a, dalpha, dgamma, part, s);
    return past ? launch_grad<T, false, true>(a, dalpha, dgamma, part, s) : launch_grad<T, false, false>(a, dalpha, dgamma, part, s);
  } else {
    if (post) return past ? launch_rows<T, false, true, true>(a, s) : launch_rows<T, false, true, false>(a, s);
    return past ? launch_rows<T, false, false, true>(a, s) : launch_rows<T, false, false, false>(a, s);
  }
}

int check(int32_t y_dtype, int32_t groups, int32_t rows, int32_t d) {
  if ((y_dtype != TLF_DTYPE_F32 && y_dtype != TLF_DTYPE_BF16) || groups < 0 || rows < 0 || d <= 0 || d % 4 != 0)
    return TLF_E_INVALID_ARG;
  return d > TLF_NORM_MAX_D || groups > TLF_NORM_MAX_GROUPS || rows > TLF_NORM_MAX_ROWS ? TLF_E_UNSUPPORTED : TLF_OK;
}

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_residual_norm(const float* d_x, const void* d_y, int32_t y_dtype, const float* d_alpha, const float* d_gamma,
                      const int32_t* d_group, int32_t groups, int32_t rows, int32_t d, int32_t post_norm, float eps,
                      float* d_h, void* d_z, float* d_rstd, float* d_ystd, void* stream) {
  const int st = tlf::check(y_dtype, groups, rows, d);
  if (st != TLF_OK) return st;
  if (!(eps > 0.f) || (groups > 0) != (d_alpha || d_gamma)) return TLF_E_INVALID_ARG;
  if (rows == 0) return TLF_OK;
  if (!d_x || !d_y || !d_h || !d_z || (groups > 1 && !d_group)) return TLF_E_INVALID_ARG;
  for (const void* p : {(const void*)d_x, d_y, (const void*)d_alpha, (const void*)d_gamma, (const void*)d_h, (const void*)d_z})
    if (!tlf::aligned16(p)) return TLF_E_INVALID_ARG;
  if (!tlf::aligned4(d_group) || !tlf::aligned4(d_rstd) || !tlf::aligned4(d_ystd)) return TLF_E_INVALID_ARG;
  const tlf::ResidArgs a{d_x, d_y, d_alpha, d_gamma, d_group, nullptr, nullptr, d_h, d_rstd, d_ystd, d_z, rows, d, groups, eps};
  const hipStream_t s = (hipStream_t)stream;
  const hipError_t e = y_dtype == TLF_DTYPE_BF16 ? tlf::launch<bf16, false>(a, post_norm != 0, nullptr, nullptr, nullptr, s)
                                                 : tlf::launch<float, false>(a, post_norm != 0, nullptr, nullptr, nullptr, s);
  return e == hipSuccess ? TLF_OK : TLF_E_HIP;
}

int tlf_residual_norm_grad_ws_bytes(int32_t groups, int32_t rows, int32_t d, size_t* ws_bytes) {
  const int st = tlf::check(TLF_DTYPE_F32, groups, rows, d);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  const int chunk = tlf::resid_chunk(rows, d);
  *ws_bytes = (size_t)((rows + chunk - 1) / chunk) * 2 * groups * d * sizeof(float);
  return TLF_OK;
}

int tlf_residual_norm_grad(const float* d_dh, const void* d_dz, const float* d_h, const void* d_y, int32_t y_dtype,
                           const float* d_alpha, const float* d_gamma, const int32_t* d_group, int32_t groups,
                           const float* d_rstd, const float* d_ystd, int32_t rows, int32_t d, int32_t post_norm, float* d_dx,
                           void* d_dy, float* d_dalpha, float* d_dgamma, void* d_workspace, size_t ws_bytes, void* stream) {
  const int st = tlf::check(y_dtype, groups, rows, d);
  if (st != TLF_OK) return st;
  if ((groups > 0) != (d_alpha || d_gamma)) return TLF_E_INVALID_ARG;
  const bool sums = d_dalpha || d_dgamma;  // all scales' gradients or none
  if (sums && ((d_dalpha != nullptr) != (d_alpha != nullptr) || (d_dgamma != nullptr) != (d_gamma != nullptr)))
    return TLF_E_INVALID_ARG;
  if (rows > 0 && (!d_h || !d_y || !d_rstd || (post_norm && !d_ystd) || !d_dx || !d_dy || (groups > 1 && !d_group)))
    return TLF_E_INVALID_ARG;
  for (const void* p : {(const void*)d_dh, d_dz, (const void*)d_h, d_y, (const void*)d_alpha, (const void*)d_gamma,
                        (const void*)d_dx, (const void*)d_dy, (const void*)d_dalpha, (const void*)d_dgamma, (const void*)d_workspace})
    if (!tlf::aligned16(p)) return TLF_E_INVALID_ARG;
  if (!tlf::aligned4(d_group) || !tlf::aligned4(d_rstd) || !tlf::aligned4(d_ystd)) return TLF_E_INVALID_ARG;
  size_t need = 0;
  tlf_residual_norm_grad_ws_bytes(groups, rows, d, &need);
  if (sums && need > 0 && (!d_workspace || ws_bytes < need)) return TLF_E_INVALID_ARG;
  const tlf::ResidArgs a{d_h, d_y, d_alpha, d_gamma, d_group, d_dh, d_dz, d_dx, const_cast<float*>(d_rstd),
                         const_cast<float*>(d_ystd), d_dy, rows, d, groups, 0.f};
  const hipStream_t s = (hipStream_t)stream;
  float* part = (float*)d_workspace;
  const hipError_t e = y_dtype == TLF_DTYPE_BF16 ? tlf::launch<bf16, true>(a, post_norm != 0, d_dalpha, d_dgamma, part, s)
                                                 : tlf::launch<float, true>(a, post_norm != 0, d_dalpha, d_dgamma, part, s);
  return e == hipSuccess ? TLF_OK : TLF_E_HIP;
}

}  // extern "C"
