// Staging through LDS, accumulators to memory and the order of workgroups, shared
// by the tile kernels of the training operators (gfx950 only).
#pragma once

#include "common.h"

namespace tlf {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ unsigned lds_offset(const void* p) {
  return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// 16 bytes per lane from base + off into 64 consecutive 16-byte places from LDS
// byte `lds` (wave-uniform, in M0).  Counts toward vmcnt; the compiler does not
// wait for it.  It does not look into the text for hazards either: a scalar
// write of M0 must be one wait state ahead of the load, and a vector write of
// the scalar base (a spilled one comes back by v_readlane) five.
__device__ __forceinline__ void stage16(const void* base, unsigned off, unsigned lds) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}

// 4 bytes per lane, likewise.
__device__ __forceinline__ void stage4(const void* base, unsigned off, unsigned lds) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}

// At most N of this wave's vector-memory operations outstanding and its LDS
// operations done, then the barrier.
template <int N> __device__ __forceinline__ void wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// This wave's LDS operations done, then the barrier.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Two neighbouring accumulators (columns 0..15 and 16..31 of 16 rows, four
// columns of a row per lane) to row-major memory; `row` is the address of the
// lane's row at column 0.  bf16: lane rows 0 and 1, 2 and 3 exchange halves, so
// that a lane has eight columns, 16 bytes, and four lanes 64.
template <typename T> __device__ __forceinline__ void store_pair(T* row, f32x4 u, f32x4 v, int lane);
template <> __device__ __forceinline__ void store_pair<float>(float* row, f32x4 u, f32x4 v, int lane) {
  Vec4<float>::store(row + (lane >> 4) * 4, u);
  Vec4<float>::store(row + 16 + (lane >> 4) * 4, v);
}
template <> __device__ __forceinline__ void store_pair<bf16>(bf16* row, f32x4 u, f32x4 v, int lane) {
  const auto a = __builtin_amdgcn_permlane16_swap(pack_bf16x2(u[0], u[1]), pack_bf16x2(v[0], v[1]), false, false);
  const auto b = __builtin_amdgcn_permlane16_swap(pack_bf16x2(u[2], u[3]), pack_bf16x2(v[2], v[3]), false, false);
  const int g = lane >> 4;
  *reinterpret_cast<uint4*>(row + (g & 1) * 16 + (g >> 1) * 8) = make_uint4(a[0], b[0], a[1], b[1]);
}

// Workgroup L runs on XCD L % 8, and each XCD has its own L2: every XCD gets
// a run of consecutive tiles.
__device__ __forceinline__ int xcd_run(int L, int n) {
  const int x = L & 7, i = L >> 3, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + i;
}

}  // namespace tlf
