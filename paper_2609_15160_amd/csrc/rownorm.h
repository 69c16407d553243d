// Row reductions and the sums of rows by group, shared by the norm kernels of the
// training operators (gfx950 only).
#pragma once

#include "common.h"

namespace tlf {

namespace {

constexpr int kGammaCols = 256;  // columns of a wave
constexpr int kJoinCols = 64;    // columns of a joining workgroup

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

// The workgroups' sums, kJoinCols columns of them: each of 16 waves' four 16 lanes
// add every 64th one, those 64 sums are added in a fixed order (32768 x 1024, 8
// groups, 1024 workgroups' sums of 32 KB: 6.9 us, with 256 columns and 16 sums 12).
// The first n0 sums go to out, the others to out1.
__global__ __launch_bounds__(1024) void k_norm_join(const float* part, int chunks, int n, float* out, int n0, float* out1) {
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
  if (lane < 16 && e < n) Vec4<float>::store(e < n0 ? out + e : out1 + (e - n0), t);
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Rows of a workgroup: 16 waves per compute unit where the rows allow it (8 with
// twice the rows in flight were slower: 32768 x 1024, 8 groups, 107 against 90
// us), and 8 rows at least, so that the sums stay a small part of the traffic
// and few rows still spread (300 x 1024: 16 rows 16 us, 8 rows 12).
inline int grad_chunk(int rows, int d) {
  const int waves = (d + kGammaCols - 1) / kGammaCols, most = 4096 / waves;
  const int c = (rows + most - 1) / most;
  return c < 8 ? 8 : c;
}
inline int grad_chunks(int rows, int d) { return (rows + grad_chunk(rows, d) - 1) / grad_chunk(rows, d); }

}  // namespace

}  // namespace tlf
