// Training of the gated FFN (Appendix A with SwiGLU), the C entry points
// tlf_ffn and tlf_ffn_grad and their kernels:
//
//   g | u = x [W_gate | W_up]^T,  a = silu(g) u,  y = a W_down^T
//   da = dy W_down,  dg = da u s (1 + g (1 - s)),  du = da g s,  s = 1 / (1 + exp(-g))
//   dx = [dg | du] [W_gate ; W_up],  d[W_gate ; W_up] = [dg | du]^T x,  dW_down = dy^T a
//
// Both projections, the activation and the product are one kernel (a tile
// holds the same columns of gate and up), the activation's derivative is the
// epilogue of the product with W_down.  Everything is one tile kernel on the
// matrix cores over C[m][n] = sum_k A(m, k) B(n, k) whose operands lie either
// with k or with m (n) contiguous, so no operand is transposed in memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "tlf.h"

namespace tlf {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ unsigned lds_offset(const void* p) {
  return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// 16 bytes per lane from base + off into 64 consecutive 16-byte places from LDS
// byte `lds` (wave-uniform, in M0; a write of M0 needs one wait state before
// the load).  Counts toward vmcnt; the compiler does not wait for it.
__device__ __forceinline__ void stage16(const void* base, unsigned off, unsigned lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}

// At most N of this wave's vector-memory operations outstanding and its LDS
// operations done, then the barrier.
template <int N> __device__ __forceinline__ void wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

enum Epi {
  E_STORE = 0,   // out[m][n] = C
  E_SWIGLU = 1,  // columns are gate and up: out[m][f] = silu(g) u, gu[m][f], gu[m][F + f] = g, u
  E_DSWIGLU = 2, // C = da: dgu[m][f], dgu[m][F + f] from it and the stored g, u
  E_PART = 3     // float32 partial sums of one K range: part[range][m][n]
};

struct FArgs {
  const void* A;  // k contiguous: [M][lda]; m contiguous: [K][lda]
  const void* B;  // k contiguous: [N][ldb]; n contiguous: [K][ldb]
  int64_t lda, ldb, ldo;
  int M, N, K;        // E_SWIGLU: N = F
  void* out;          // E_STORE, E_SWIGLU
  void* gu;           // E_SWIGLU: written unless NULL; E_DSWIGLU: dgu, written
  const void* gu_in;  // E_DSWIGLU
  float* part;        // E_PART
  int splits;         // K ranges (E_PART)
};

// 1 / (1 + exp(-g)); the float32 operators take the correctly rounded division
template <typename T> __device__ __forceinline__ float sigmoid(float g);
template <> __device__ __forceinline__ float sigmoid<bf16>(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }
template <> __device__ __forceinline__ float sigmoid<float>(float g) { return 1.f / (1.f + expf(-g)); }

// One operand of a stage: ROWS rows of m (or n) times 128 bytes of k, in
// 16-byte chunks that the 64 lanes of a load put into consecutive places.
//
// k contiguous: LDS row = one row's 8 chunks, chunk c at place c ^ (row & 7),
// so the rows of a fragment's 16-byte reads lie in distinct banks.
// m contiguous: LDS row = one k with ROWS elements; pieces of 16 elements lie
// at place c ^ key(k), so that the k of a transposed read do.
template <typename T, bool TR, int ROWS> struct Operand {
  static constexpr int EPC = 16 / (int)sizeof(T);  // elements of a chunk
  static constexpr int BK = 8 * EPC;               // k of a stage
  static constexpr int BYTES = ROWS * 128;
  static constexpr int CPP = 16 / EPC;             // chunks of a 16-element piece
  static constexpr int CPR = ROWS / EPC;           // TR: chunks of an LDS row
  static __device__ __forceinline__ int key(int k) {
    const int x = sizeof(T) == 2 ? (k & 3) | ((k >> 3) & 3) << 2 : (k >> 2) & 3;
    return x & (ROWS / 16 - 1);
  }
  // source of chunk q: row (m relative to the tile) or k of the stage, and the element of it
  static __device__ __forceinline__ void place(int q, int& line, int& elem) {
    if constexpr (TR) {
      line = q / CPR;
      const int p = q % CPR;
      elem = ((((p / CPP) ^ key(line)) * CPP) + p % CPP) * EPC;
    } else {
      line = q >> 3;
      elem = ((q & 7) ^ (line & 7)) * EPC;
    }
  }
};

// Fragment of 16 rows (m) from row r0 and one half of the stage's k.
template <typename T, bool TR, int ROWS> struct Frag;
template <bool TR, int ROWS> struct Frag<bf16, TR, ROWS> {
  bf16x8 v;
  static __device__ __forceinline__ Frag load(const char* s, int r0, int half, int lane) {
    Frag f;
    const int g = lane >> 4, i = lane & 15;
    if constexpr (!TR) {
      f.v = *reinterpret_cast<const bf16x8*>(s + (r0 + i) * 128 + (((half * 4 + g) ^ (i & 7)) << 4));
    } else {
      // a group of 16 lanes reads 4 k x 16 m, lane i receives the 4 k of m = i
      const int k = half * 32 + g * 8 + (i >> 2);
      const char* p = s + k * (ROWS * 2) + (((r0 >> 4) ^ Operand<bf16, TR, ROWS>::key(k)) << 5) + (i & 3) * 8;
      union { s16x4 h[2]; bf16x8 v; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * ROWS * 2));
      f.v = u.v;
    }
    return f;
  }
};
template <bool TR, int ROWS> struct Frag<float, TR, ROWS> {
  float v[4];  // k = 4 (lane / 16) + j of the half for the j-th instruction
  static __device__ __forceinline__ Frag load(const char* s, int r0, int half, int lane) {
    Frag f;
    const int g = lane >> 4, i = lane & 15;
    if constexpr (!TR) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(s + (r0 + i) * 128 + (((half * 4 + g) ^ (i & 7)) << 4));
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = x[j];
    } else {
      const int k = half * 16 + g * 4;
      const char* p = s + k * (ROWS * 4) + (((r0 >> 4) ^ Operand<float, TR, ROWS>::key(k)) << 6) + i * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = *reinterpret_cast<const float*>(p + j * ROWS * 4);
    }
    return f;
  }
};
template <typename T, bool TA, int RA, bool TB, int RB>
__device__ __forceinline__ f32x4 mma(const Frag<T, TA, RA>& a, const Frag<T, TB, RB>& b, f32x4 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
  }
}

template <int BM_, int BN_, int WM_, int WN_> struct FShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NTH = WM_ * WN_ * kWave;
};

// Workgroup L runs on XCD L % 8, and each XCD has its own L2: every XCD gets
// a run of consecutive tiles.
__device__ __forceinline__ int xcd_run(int L, int n) {
  const int x = L & 7, i = L >> 3, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + i;
}

template <typename T, bool TA, bool TB, int EK, typename SH>
__global__ __launch_bounds__(SH::NTH) void k_ffn(FArgs g) {
  constexpr int BM = SH::BM, BN = SH::BN, NTH = SH::NTH;
  constexpr int MT = BM / SH::WM / 16, NT = BN / SH::WN / 16;
  using OA = Operand<T, TA, BM>;
  using OB = Operand<T, TB, BN>;
  using FA = Frag<T, TA, BM>;
  using FB = Frag<T, TB, BN>;
  constexpr int BK = OA::BK, STAGE = OA::BYTES + OB::BYTES;
  constexpr int ACH = BM * 8 / NTH, BCH = BN * 8 / NTH;
  static_assert(BM * 8 % NTH == 0 && BN * 8 % NTH == 0 && 2 * STAGE <= 160 * 1024, "chunks");
  static_assert(EK != E_SWIGLU || (NT % 2 == 0 && !TB), "gate and up");
  __shared__ __align__(16) char lds[2 * STAGE];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / SH::WN, wn = wave % SH::WN;
  const int wbase = __builtin_amdgcn_readfirstlane(tid & ~(kWave - 1));
  constexpr int TN = EK == E_SWIGLU ? BN / 2 : BN;  // columns of N that a tile covers
  const int tm = (g.M + BM - 1) / BM, tn = (g.N + TN - 1) / TN;
  int t = xcd_run(blockIdx.x, gridDim.x), split = 0;
  if constexpr (EK == E_PART) {
    split = t / (tm * tn);
    t %= tm * tn;
  }
  // eight row tiles at a time, so that the tiles of a run share columns and rows
  const int band = t / (8 * tn), bh = min(8, tm - band * 8), in = t - band * 8 * tn;
  const int m0 = (band * 8 + in % bh) * BM, n0 = (in / bh) * TN;
  const int KT = (g.K + BK - 1) / BK;  // stages; the last one of an m-contiguous operand may be short
  int k0 = 0, k1 = KT;
  if constexpr (EK == E_PART) {
    k0 = (int)((int64_t)KT * split / g.splits);
    k1 = (int)((int64_t)KT * (split + 1) / g.splits);
  }

  // byte offsets of this thread's chunks from the stage's first element; rows
  // and columns past the matrix read the last one (their results are not stored)
  unsigned ao[ACH], bo[BCH];
#pragma unroll
  for (int c = 0; c < ACH; ++c) {
    int line, e;
    OA::place(tid + c * NTH, line, e);
    if constexpr (TA) ao[c] = (unsigned)((line * g.lda + min(m0 + e, g.M - OA::EPC)) * sizeof(T));
    else ao[c] = (unsigned)(((min(m0 + line, g.M - 1) - m0) * g.lda + e) * sizeof(T));
  }
#pragma unroll
  for (int c = 0; c < BCH; ++c) {
    int line, e;
    OB::place(tid + c * NTH, line, e);
    if constexpr (TB) {
      bo[c] = (unsigned)((line * g.ldb + min(n0 + e, g.N - OB::EPC)) * sizeof(T));
    } else {
      int row = line;
      if constexpr (EK == E_SWIGLU) row = line < TN ? min(n0 + line, g.N - 1) - n0 : g.N + min(n0 + line - TN, g.N - 1) - n0;
      else row = min(n0 + line, g.N - 1) - n0;
      bo[c] = (unsigned)((row * g.ldb + e) * sizeof(T));
    }
  }
  const char* ab = reinterpret_cast<const char*>(g.A) + (TA ? 0 : m0 * g.lda * (int64_t)sizeof(T));
  const char* bb = reinterpret_cast<const char*>(g.B) + (TB ? 0 : n0 * g.ldb * (int64_t)sizeof(T));
  const int64_t astep = TA ? BK * g.lda * (int64_t)sizeof(T) : 128, bstep = TB ? BK * g.ldb * (int64_t)sizeof(T) : 128;
  const unsigned lbase = lds_offset(lds);

  auto issue = [&](int kt) __attribute__((always_inline)) {
    const unsigned s = lbase + ((kt - k0) & 1) * STAGE;
    if ((TA || TB) && kt == KT - 1 && g.K % BK != 0) {
      // short stage: k past the end are zeros
#pragma unroll
      for (int c = 0; c < ACH; ++c) {
        int line, e;
        OA::place(tid + c * NTH, line, e);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (kt * BK + (TA ? line : e) < g.K) v = *reinterpret_cast<const uint4*>(ab + kt * astep + ao[c]);
        *reinterpret_cast<uint4*>(lds + ((kt - k0) & 1) * STAGE + (tid + c * NTH) * 16) = v;
      }
#pragma unroll
      for (int c = 0; c < BCH; ++c) {
        int line, e;
        OB::place(tid + c * NTH, line, e);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (kt * BK + (TB ? line : e) < g.K) v = *reinterpret_cast<const uint4*>(bb + kt * bstep + bo[c]);
        *reinterpret_cast<uint4*>(lds + ((kt - k0) & 1) * STAGE + OA::BYTES + (tid + c * NTH) * 16) = v;
      }
      return;
    }
    const char* as = ab + kt * astep;
    const char* bs = bb + kt * bstep;
#pragma unroll
    for (int c = 0; c < ACH; ++c) stage16(as, ao[c], s + (c * NTH + wbase) * 16);
#pragma unroll
    for (int c = 0; c < BCH; ++c) stage16(bs, bo[c], s + OA::BYTES + (c * NTH + wbase) * 16);
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto bcol = [&](int j) __attribute__((always_inline)) {  // LDS row of B's fragment j
    if constexpr (EK == E_SWIGLU)
      return (j < NT / 2 ? 0 : TN) + wn * (TN / SH::WN) + (j % (NT / 2)) * 16;
    else
      return wn * (BN / SH::WN) + j * 16;
  };
  auto fetch = [&](FA (&a)[MT], FB (&b)[NT], int st, int half) __attribute__((always_inline)) {
    const char* s = lds + st * STAGE;
#pragma unroll
    for (int j = 0; j < NT; ++j) b[j] = FB::load(s + OA::BYTES, bcol(j), half, lane);
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = FA::load(s, wm * (BM / SH::WM) + i * 16, half, lane);
  };
  // B is the instruction's first operand, so that a lane holds four consecutive columns of one row
  auto multiply = [&](FA (&a)[MT], FB (&b)[NT]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = mma(b[j], a[i], acc[i][j]);
  };

  // Two stages and two sets of fragments: while a half stage is multiplied, the
  // next half's fragments are read.  The barrier in the middle ends every
  // wave's reads of stage kt and every wave's loads of stage kt + 1; stage kt + 2
  // then goes where kt was.
  FA a0[MT], a1[MT];
  FB b0[NT], b1[NT];
  if (k0 < k1) {
    issue(k0);
    wait_barrier<0>();
    if (k0 + 1 < k1) issue(k0 + 1);
    fetch(a0, b0, 0, 0);
    for (int kt = k0; kt < k1; ++kt) {
      const int st = (kt - k0) & 1;
      fetch(a1, b1, st, 1);
      multiply(a0, b0);
      wait_barrier<0>();
      if (kt + 2 < k1) issue(kt + 2);
      if (kt + 1 < k1) fetch(a0, b0, st ^ 1, 0);
      multiply(a1, b1);
    }
  }

  // lane: row m0 + .. + lane % 16, columns .. + 4 (lane / 16) + 0..3
  const int rq = lane & 15, cq = (lane >> 4) * 4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = m0 + wm * (BM / SH::WM) + i * 16 + rq;
    if (m >= g.M) continue;
    if constexpr (EK == E_SWIGLU) {
#pragma unroll
      for (int j = 0; j < NT / 2; ++j) {
        const int f = n0 + wn * (TN / SH::WN) + j * 16 + cq;
        if (f >= g.N) continue;
        const f32x4 gt = acc[i][j], up = acc[i][j + NT / 2];
        f32x4 h;
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = gt[r] * sigmoid<T>(gt[r]) * up[r];
        Vec4<T>::store(reinterpret_cast<T*>(g.out) + m * g.ldo + f, h);
        if (g.gu) {
          T* o = reinterpret_cast<T*>(g.gu) + (int64_t)m * 2 * g.N + f;
          Vec4<T>::store(o, gt);
          Vec4<T>::store(o + g.N, up);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int n = n0 + wn * (BN / SH::WN) + j * 16 + cq;
        if (n >= g.N) continue;
        if constexpr (EK == E_STORE) {
          Vec4<T>::store(reinterpret_cast<T*>(g.out) + m * g.ldo + n, acc[i][j]);
        } else if constexpr (EK == E_PART) {
          Vec4<float>::store(g.part + ((int64_t)split * g.M + m) * g.N + n, acc[i][j]);
        } else {
          const int64_t o = (int64_t)m * 2 * g.N + n;
          const f32x4 gt = Vec4<T>::load(reinterpret_cast<const T*>(g.gu_in) + o);
          const f32x4 up = Vec4<T>::load(reinterpret_cast<const T*>(g.gu_in) + o + g.N);
          f32x4 dg, du;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float s = sigmoid<T>(gt[r]), da = acc[i][j][r];
            dg[r] = da * up[r] * s * (1.f + gt[r] * (1.f - s));
            du[r] = da * gt[r] * s;
          }
          Vec4<T>::store(reinterpret_cast<T*>(g.gu) + o, dg);
          Vec4<T>::store(reinterpret_cast<T*>(g.gu) + o + g.N, du);
        }
      }
    }
  }
}

// The K ranges' partial sums added in order, rounded once.
template <typename T> __global__ __launch_bounds__(256) void k_ffn_join(const float* part, int splits, int64_t n, T* out) {
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= n) return;
  f32x4 v = Vec4<float>::load(part + e);
  for (int s = 1; s < splits; ++s) v += Vec4<float>::load(part + s * n + e);
  Vec4<T>::store(out + e, v);
}

template <typename T, bool TA, bool TB, int EK, typename SH> hipError_t launch_shape(const FArgs& g, hipStream_t s) {
  constexpr int TN = EK == E_SWIGLU ? SH::BN / 2 : SH::BN;
  const int64_t tiles = (int64_t)((g.M + SH::BM - 1) / SH::BM) * ((g.N + TN - 1) / TN) * (EK == E_PART ? g.splits : 1);
  if (tiles <= 0 || tiles > INT32_MAX) return tiles == 0 ? hipSuccess : hipErrorInvalidValue;
  hipLaunchKernelGGL((k_ffn<T, TA, TB, EK, SH>), dim3((unsigned)tiles), dim3(SH::NTH), 0, s, g);
  return hipGetLastError();
}

using Big = FShape<256, 256, 2, 4>;
using Mid = FShape<128, 128, 2, 2>;
using Small = FShape<64, 64, 2, 2>;

template <typename T, bool TA, bool TB, int EK> hipError_t launch_ffn(const FArgs& g, hipStream_t s) {
  const int64_t mid = (int64_t)((g.M + 127) / 128) * ((g.N + 127) / 128) * (EK == E_SWIGLU ? 2 : 1);
  if constexpr (sizeof(T) == 2) {
    if (mid * (EK == E_PART ? g.splits : 1) >= 768) return launch_shape<T, TA, TB, EK, Big>(g, s);
  }
  if (mid * (EK == E_PART ? g.splits : 1) >= 200) return launch_shape<T, TA, TB, EK, Mid>(g, s);
  return launch_shape<T, TA, TB, EK, Small>(g, s);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

int check(int32_t dtype, int32_t rows, int32_t d, int32_t f) {
  if (dtype != TLF_DTYPE_F32 && dtype != TLF_DTYPE_BF16) return TLF_E_INVALID_ARG;
  if (rows < 0 || d <= 0 || f <= 0) return TLF_E_INVALID_ARG;
  // up to this width the byte offsets inside a tile and from gate to up stay below 2^32
  if (d % 64 != 0 || f % 64 != 0 || d > TLF_FFN_MAX_WIDTH || f > TLF_FFN_MAX_WIDTH) return TLF_E_UNSUPPORTED;
  return TLF_OK;
}

// K ranges of a weight gradient: enough workgroups for every compute unit
// while a range still has work for its start and its partial sums.
int grad_splits(int64_t m, int64_t n, int64_t rows) {
  const int64_t tiles = ((m + 127) / 128) * ((n + 127) / 128);
  const int64_t steps = rows / 512;
  int64_t s = 512 / tiles;
  if (s > steps) s = steps;
  return (int)(s < 1 ? 1 : s > 32 ? 32 : s);
}

template <typename T>
int ffn_forward(const void* x, const void* wgu, const void* wd, int rows, int d, int f, void* gu, void* a, void* y,
                hipStream_t s) {
  FArgs p{};
  p.A = x; p.B = wgu; p.lda = d; p.ldb = d; p.ldo = f;
  p.M = rows; p.N = f; p.K = d; p.out = a; p.gu = gu;
  if (launch_ffn<T, false, false, E_SWIGLU>(p, s) != hipSuccess) return TLF_E_HIP;
  FArgs q{};
  q.A = a; q.B = wd; q.lda = f; q.ldb = f; q.ldo = d;
  q.M = rows; q.N = d; q.K = f; q.out = y;
  return launch_ffn<T, false, false, E_STORE>(q, s) == hipSuccess ? TLF_OK : TLF_E_HIP;
}

template <typename T>
hipError_t weight_grad(const void* a, int m, const void* b, int n, int rows, void* out, float* part, hipStream_t s) {
  FArgs p{};
  p.A = a; p.B = b; p.lda = m; p.ldb = n; p.ldo = n;
  p.M = m; p.N = n; p.K = rows; p.out = out; p.part = part; p.splits = grad_splits(m, n, rows);
  if (p.splits == 1) return launch_ffn<T, true, true, E_STORE>(p, s);
  hipError_t e = launch_ffn<T, true, true, E_PART>(p, s);
  if (e != hipSuccess) return e;
  const int64_t all = (int64_t)m * n;
  hipLaunchKernelGGL(k_ffn_join<T>, dim3((unsigned)((all + 1023) / 1024)), dim3(256), 0, s, part, p.splits, all,
                     reinterpret_cast<T*>(out));
  return hipGetLastError();
}

size_t part_bytes(int64_t m, int64_t n, int64_t rows) {
  const int s = grad_splits(m, n, rows);
  return s > 1 ? (size_t)(m * n * s) * sizeof(float) : 0;
}

size_t dgu_bytes(int32_t dtype, int64_t rows, int64_t f) {
  return (size_t)(rows * 2 * f) * (dtype == TLF_DTYPE_BF16 ? 2 : 4);
}

template <typename T>
int ffn_backward(const void* dy, const void* x, const void* wgu, const void* wd, const void* gu, const void* a, int rows,
                 int d, int f, void* dx, void* dwgu, void* dwd, char* ws, hipStream_t s) {
  void* dgu = ws;
  float* part = reinterpret_cast<float*>(ws + dgu_bytes(sizeof(T) == 2 ? TLF_DTYPE_BF16 : TLF_DTYPE_F32, rows, f));
  if (rows > 0 && (dx || dwgu)) {
    FArgs p{};
    p.A = dy; p.B = wd; p.lda = d; p.ldb = f;
    p.M = rows; p.N = f; p.K = d; p.gu = dgu; p.gu_in = gu;
    if (launch_ffn<T, false, true, E_DSWIGLU>(p, s) != hipSuccess) return TLF_E_HIP;
  }
  if (dx) {
    FArgs p{};
    p.A = dgu; p.B = wgu; p.lda = 2 * f; p.ldb = d; p.ldo = d;
    p.M = rows; p.N = d; p.K = 2 * f; p.out = dx;
    if (launch_ffn<T, false, true, E_STORE>(p, s) != hipSuccess) return TLF_E_HIP;
  }
  if (dwgu && weight_grad<T>(dgu, 2 * f, x, d, rows, dwgu, part, s) != hipSuccess) return TLF_E_HIP;
  if (dwd && weight_grad<T>(dy, d, a, f, rows, dwd, part, s) != hipSuccess) return TLF_E_HIP;
  return TLF_OK;
}

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_ffn(const void* d_x, const void* d_w_gate_up, const void* d_w_down, int32_t dtype, int32_t rows, int32_t d,
            int32_t f, void* d_gu, void* d_a, void* d_y, void* stream) {
  const int st = tlf::check(dtype, rows, d, f);
  if (st != TLF_OK) return st;
  if (rows == 0) return TLF_OK;
  if (!d_x || !d_w_gate_up || !d_w_down || !d_a || !d_y) return TLF_E_INVALID_ARG;
  for (const void* p : {d_x, d_w_gate_up, d_w_down, (const void*)d_gu, (const void*)d_a, (const void*)d_y})
    if (!tlf::aligned16(p)) return TLF_E_INVALID_ARG;
  return dtype == TLF_DTYPE_BF16
             ? tlf::ffn_forward<bf16>(d_x, d_w_gate_up, d_w_down, rows, d, f, d_gu, d_a, d_y, (hipStream_t)stream)
             : tlf::ffn_forward<float>(d_x, d_w_gate_up, d_w_down, rows, d, f, d_gu, d_a, d_y, (hipStream_t)stream);
}

int tlf_ffn_grad_ws_bytes(int32_t dtype, int32_t rows, int32_t d, int32_t f, size_t* ws_bytes) {
  const int st = tlf::check(dtype, rows, d, f);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  const size_t gu = tlf::part_bytes(2 * (int64_t)f, d, rows), dn = tlf::part_bytes(d, f, rows);
  *ws_bytes = tlf::dgu_bytes(dtype, rows, f) + (gu > dn ? gu : dn);
  return TLF_OK;
}

int tlf_ffn_grad(const void* d_dy, const void* d_x, const void* d_w_gate_up, const void* d_w_down, const void* d_gu,
                 const void* d_a, int32_t dtype, int32_t rows, int32_t d, int32_t f, void* d_dx, void* d_dw_gate_up,
                 void* d_dw_down, void* d_workspace, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int st = tlf_ffn_grad_ws_bytes(dtype, rows, d, f, &need);
  if (st != TLF_OK) return st;
  if (!d_dx && !d_dw_gate_up && !d_dw_down) return TLF_OK;
  if (rows > 0) {
    if (!d_dy || !d_x || !d_w_gate_up || !d_w_down || !d_gu || !d_a) return TLF_E_INVALID_ARG;
    if (need > 0 && (!d_workspace || ws_bytes < need)) return TLF_E_INVALID_ARG;
  }
  for (const void* p : {d_dy, d_x, d_w_gate_up, d_w_down, d_gu, d_a, (const void*)d_dx, (const void*)d_dw_gate_up,
                        (const void*)d_dw_down, (const void*)d_workspace})
    if (!tlf::aligned16(p)) return TLF_E_INVALID_ARG;
  if (rows == 0) d_dx = nullptr;  // no rows; the weights' gradients are zeros
  return dtype == TLF_DTYPE_BF16
             ? tlf::ffn_backward<bf16>(d_dy, d_x, d_w_gate_up, d_w_down, d_gu, d_a, rows, d, f, d_dx, d_dw_gate_up,
                                       d_dw_down, (char*)d_workspace, (hipStream_t)stream)
             : tlf::ffn_backward<float>(d_dy, d_x, d_w_gate_up, d_w_down, d_gu, d_a, rows, d, f, d_dx, d_dw_gate_up,
                                        d_dw_down, (char*)d_workspace, (hipStream_t)stream);
}

}  // extern "C"
