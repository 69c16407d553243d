// Training of the gated FFN (Appendix A with SwiGLU), the C entry points
// tlf_ffn and tlf_ffn_grad and their kernels:
//
//   g | u = x [W_gate | W_up]^T,  a = silu(g) u,  y = a W_down^T
//   dg = da q, du = da p with da = dy W_down, p = silu(g), q = u silu'(g) = u s (1 + g (1 - s)),
//   s = 1 / (1 + exp(-g));
//   dx = [dg | du] [W_gate ; W_up],  d[W_gate ; W_up] = [dg | du]^T x,  dW_down = dy^T a
//
// The forward pass keeps q and p instead of g and u: the gradient then takes
// two products per element and no exponential, and one rounding each.
//
// Both projections, the activation and the product are one kernel (a tile
// holds the same columns of gate and up), the activation's derivative is the
// epilogue of the product with W_down.  Everything is one tile kernel on the
// matrix cores over C[m][n] = sum_k A(m, k) B(n, k) whose operands lie either
// with k or with m (n) contiguous, so no operand is transposed in memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "common.h"
#include "tlf.h"

namespace tlf {

namespace {

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

// At most N of this wave's vector-memory operations outstanding and its LDS
// operations done, then the barrier.
template <int N> __device__ __forceinline__ void wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// This wave's LDS operations done, then the barrier.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

enum Epi {
  E_STORE = 0,   // out[m][n] = C
  E_SWIGLU = 1,  // columns are gate and up: out[m][f] = silu(g) u; kept: q, p
  E_DSWIGLU = 2  // C = da: out[m][f], out[m][F + f] = da q, da p
};

struct FArgs {
  const void* A;  // k contiguous: [M][lda]; m contiguous: [K][lda]
  const void* B;  // k contiguous: [N][ldb]; n contiguous: [K][ldb]
  int64_t lda, ldb, ldo;
  int M, N, K;    // E_SWIGLU: N = F
  void* out;
  void* kept;     // E_SWIGLU: written unless NULL; E_DSWIGLU: read
  float* part;    // sums over `splits` ranges of k, [range][tile], each as its accumulators lie
  int splits;
};

// q and p between the passes.  float32: as they are.  bf16: float32's sign, exponent
// and 9 bits of mantissa, 18 bits, so that what operands of bf16 give between the
// ends of their range (infinity and NaN too) comes back as it was up to 2^-10 of
// it.  Rounded to bf16 their 2^-8 would be the larger part of the gradients' error
// (dx and dW_gate_up 0.0030 from 64 bits relative to their norm, 0.0024 with 2^-10);
// 9 bits of mantissa within 16 would leave 6 for the exponent, which loses gates
// and products past 2^32 and below 2^-30.
__device__ __forceinline__ unsigned kept18(float v) {  // in the upper 18 bits, the others are not zeros
  const unsigned b = v == v ? __float_as_uint(v) : 0x7FC00000u;
  return b + 0x1FFFu + ((b >> 14) & 1u);  // nearest, ties to even
}
// They lie as the lanes of two neighbouring 16 x 16 accumulators hold them: first
// the upper 16 bits, [row / 16][f / 16][lane][4 q, 4 p], behind those of all rows the
// other two, [row / 16][f / 32][lane][16 of them], so that a wave reads and writes
// whole lines (row by row it moved 8 bytes per lane in 32-byte pieces), past the
// caches, which keep a and the weights instead (16384 x 1024 x 2816, measured when
// q and p were 16 bits: gate/up 224 -> 217 us, down 88 -> 83).  `pair` counts the
// pairs of accumulators, row bands of 16 first, of which there are `pairs`.
template <typename T> struct Kept;
template <> struct Kept<float> {
  struct Raw { f32x4 q[2], p[2]; };
  static __device__ __forceinline__ void load(const void* base, int64_t, int64_t pair, int lane, Raw& o) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float* s = reinterpret_cast<const float*>(base) + ((2 * pair + x) * kWave + lane) * 8;
      o.q[x] = Vec4<float>::load(s);
      o.p[x] = Vec4<float>::load(s + 4);
    }
  }
  static __device__ __forceinline__ void get(const Raw& o, int x, f32x4& q, f32x4& p) { q = o.q[x], p = o.p[x]; }
  static __device__ __forceinline__ void store(void* base, int64_t, int64_t pair, int lane, const f32x4 (&q)[2],
                                               const f32x4 (&p)[2]) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float* s = reinterpret_cast<float*>(base) + ((2 * pair + x) * kWave + lane) * 8;
      Vec4<float>::store(s, q[x]);
      Vec4<float>::store(s + 4, p[x]);
    }
  }
};
template <> struct Kept<bf16> {
  struct Raw {
    u32x4 high[2];
    unsigned low;  // element r of q and of p of accumulator x: bits 8 x + 2 r and 16 + 8 x + 2 r
  };
  static __device__ __forceinline__ void load(const void* base, int64_t pairs, int64_t pair, int lane, Raw& o) {
    const u32x4* high = reinterpret_cast<const u32x4*>(base);
#pragma unroll
    for (int x = 0; x < 2; ++x) o.high[x] = __builtin_nontemporal_load(high + (2 * pair + x) * kWave + lane);
    o.low = __builtin_nontemporal_load(reinterpret_cast<const unsigned*>(high + 2 * pairs * kWave) + pair * kWave + lane);
  }
  static __device__ __forceinline__ float value(unsigned two, int r, unsigned low, int at) {
    const unsigned l = at < 14 ? low << (14 - at) : low >> (at - 14);
    return __uint_as_float((r & 1 ? two & 0xFFFF0000u : two << 16) | (l & 0xC000u));
  }
  static __device__ __forceinline__ void get(const Raw& c, int x, f32x4& q, f32x4& p) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      q[r] = value(c.high[x][r >> 1], r, c.low, 8 * x + 2 * r);
      p[r] = value(c.high[x][2 + (r >> 1)], r, c.low, 16 + 8 * x + 2 * r);
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t pairs, int64_t pair, int lane, const f32x4 (&q)[2],
                                               const f32x4 (&p)[2]) {
    u32x4* high = reinterpret_cast<u32x4*>(base);
    unsigned low = 0;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      unsigned b[8];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        b[r] = kept18(q[x][r]);
        b[4 + r] = kept18(p[x][r]);
        low |= (b[r] >> 14 & 3u) << (8 * x + 2 * r) | (b[4 + r] >> 14 & 3u) << (16 + 8 * x + 2 * r);
      }
      u32x4 h;
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = b[2 * k] >> 16 | (b[2 * k + 1] & 0xFFFF0000u);
      __builtin_nontemporal_store(h, high + (2 * pair + x) * kWave + lane);
    }
    __builtin_nontemporal_store(low, reinterpret_cast<unsigned*>(high + 2 * pairs * kWave) + pair * kWave + lane);
  }
};

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

// 1 / (1 + exp(-g)); the float32 operators take the correctly rounded division.
// bf16: the exponential and reciprocal of the hardware are off by some 2^-22 and
// |g| 2^-24 of the value, far below the 2^-8 and 2^-10 that its uses are rounded to.
template <typename T> __device__ __forceinline__ float sigmoid(float g);
template <> __device__ __forceinline__ float sigmoid<bf16>(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }
template <> __device__ __forceinline__ float sigmoid<float>(float g) { return 1.f / (1.f + expf(-g)); }

// One operand of a stage: ROWS rows of m (or n) times 128 bytes of k, a whole line,
// in 16-byte chunks that the 64 lanes of a load put into consecutive places.
//
// k contiguous: LDS row = one row's chunks, chunk c at place c ^ key(row), so
// that the 8 rows which a fragment's 16-byte reads take at a time lie in
// distinct banks.
// m contiguous: LDS row = one k with ROWS elements; the piece c of 16 elements
// lies at place c ^ key(k), so that the k of a transposed read do.
// (No bank conflicts counted for either.)
template <typename T, bool TR, int ROWS> struct Operand {
  static constexpr int KB = 128;
  static constexpr int EPC = 16 / (int)sizeof(T);        // elements of a chunk
  static constexpr int BK = KB / (int)sizeof(T);         // k of a stage
  static constexpr int BYTES = ROWS * KB;
  static constexpr int CPP = 16 / EPC;                   // chunks of a 16-element piece
  static constexpr int CPR = TR ? ROWS / EPC : KB / 16;  // chunks of an LDS row
  static __device__ __forceinline__ int key(int line) {
    if constexpr (!TR) return line & 7;
    const int x = sizeof(T) == 2 ? (line & 3) | ((line >> 3) & 3) << 2 : (line >> 2) & 3;
    return x & (ROWS / 16 - 1);
  }
  // source of chunk q: row (relative to the tile) or k of the stage, and the element of it
  static __device__ __forceinline__ void place(int q, int& line, int& elem) {
    line = q / CPR;
    const int c = q % CPR;
    if constexpr (TR) elem = ((((c / CPP) ^ key(line)) * CPP) + c % CPP) * EPC;
    else elem = (c ^ key(line)) * EPC;
  }
};

// Fragment of 16 rows (m) from row r0 and 64 bytes of k, the h-th half of the stage.
template <typename T, bool TR, int ROWS> struct Frag;
template <bool TR, int ROWS> struct Frag<bf16, TR, ROWS> {
  bf16x8 v;  // k = 32 h + 8 (lane / 16) + 0..7
  static __device__ __forceinline__ Frag load(const char* s, int r0, int h, int lane) {
    using O = Operand<bf16, TR, ROWS>;
    Frag f;
    const int g = lane >> 4, i = lane & 15;
    if constexpr (!TR) {
      f.v = *reinterpret_cast<const bf16x8*>(s + (r0 + i) * O::KB + (((h * 4 + g) ^ O::key(i)) << 4));
    } else {
      // a group of 16 lanes reads 4 k x 16 m, lane i receives the 4 k of m = i
      const int k = g * 8 + (i >> 2);
      const char* p = s + (h * 32 + k) * (ROWS * 2) + (((r0 >> 4) ^ O::key(k)) << 5) + (i & 3) * 8;
      union { s16x4 h[2]; bf16x8 v; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * ROWS * 2));
      f.v = u.v;
    }
    return f;
  }
};
template <bool TR, int ROWS> struct Frag<float, TR, ROWS> {
  float v[4];  // k = 16 h + 4 (lane / 16) + j for the j-th instruction
  static __device__ __forceinline__ Frag load(const char* s, int r0, int h, int lane) {
    using O = Operand<float, TR, ROWS>;
    Frag f;
    const int g = lane >> 4, i = lane & 15;
    if constexpr (!TR) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(s + (r0 + i) * O::KB + (((h * 4 + g) ^ O::key(i)) << 4));
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = x[j];
    } else {
      const char* p = s + (h * 16 + g * 4) * (ROWS * 4) + (((r0 >> 4) ^ O::key(g * 4)) << 6) + i * 4;
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

// Tile of BM x BN by WM x WN waves, RA stages of A and RB of B in LDS; WK groups
// of such waves share the tile's stages (their sums are added in LDS afterwards,
// in a fixed order).
template <int BM_, int BN_, int WM_, int WN_, int RA_, int RB_, int WK_> struct FShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, RA = RA_, RB = RB_, WK = WK_;
  static constexpr int GTH = WM * WN * kWave, NTH = GTH * WK;
};

// Workgroup L runs on XCD L % 8, and each XCD has its own L2: every XCD gets
// a run of consecutive tiles.
__device__ __forceinline__ int xcd_run(int L, int n) {
  const int x = L & 7, i = L >> 3, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + i;
}

// Tiles of a product, eight row tiles at a time, so that the tiles of a run share columns and rows.
struct Tiles {
  int tm, tn;
  __device__ __forceinline__ void at(int t, int& row, int& col) const {
    const int band = t / (8 * tn), bh = min(8, tm - band * 8), in = t - band * 8 * tn;
    row = band * 8 + in % bh;
    col = in / bh;
  }
};

template <typename T, bool TA, bool TB, int EK, typename SH, bool SPLIT> struct Tile {
  static constexpr int BM = SH::BM, BN = SH::BN, NTH = SH::GTH, RA = SH::RA, RB = SH::RB, WK = SH::WK;
  static constexpr int MT = BM / SH::WM / 16, NT = BN / SH::WN / 16;
  using OA = Operand<T, TA, BM>;
  using OB = Operand<T, TB, BN>;
  using FA = Frag<T, TA, BM>;
  using FB = Frag<T, TB, BN>;
  static constexpr int BK = OA::BK, ALL = RA * OA::BYTES + RB * OB::BYTES;
  static constexpr int ACH = OA::BYTES / 16 / NTH, BCH = OB::BYTES / 16 / NTH;
  static constexpr int TN = EK == E_SWIGLU ? BN / 2 : BN;  // columns of N that a tile covers
  static_assert(OA::BYTES % (16 * NTH) == 0 && OB::BYTES % (16 * NTH) == 0, "chunks");
  static_assert(NT % 2 == 0 && (EK != E_SWIGLU || (NT % 4 == 0 && !TB)), "pairs of columns, of gate and of up");
  static constexpr int LDS = WK * ALL;
  static_assert((WK - 1) * BM * BN * 4 <= LDS && LDS <= 160 * 1024, "LDS");

  // Stages [first, last) of the tile at (m0, n0); the sums go to the epilogue, or
  // (SPLIT) to `part` as they are.
  static __device__ __forceinline__ void run(const FArgs& g, int m0, int n0, int first, int last, float* part, char* lds0) {
    const int grp = WK == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NTH);
    const int tid = threadIdx.x - grp * NTH, lane = tid & 63, wave = tid >> 6, wm = wave / SH::WN, wn = wave % SH::WN;
    const int wbase = __builtin_amdgcn_readfirstlane(tid & ~(kWave - 1));
    char* lds = lds0 + grp * ALL;  // RA places of A, then RB of B
    // this group's stages [k0, k1); all groups go through `turns` of them
    const int turns_n = (last - first + WK - 1) / WK, k0 = min(first + grp * turns_n, last), k1 = min(k0 + turns_n, last);

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
    const int64_t astep = TA ? BK * g.lda * (int64_t)sizeof(T) : OA::KB, bstep = TB ? BK * g.ldb * (int64_t)sizeof(T) : OB::KB;
    const unsigned lbase = lds_offset(lds);

    // chunk c of A's of stage kt into place `slot`, and of B's
    auto load_a = [&](int kt, int slot, int c) __attribute__((always_inline)) {
      stage16(ab + kt * astep, ao[c], lbase + slot * OA::BYTES + (c * NTH + wbase) * 16);
    };
    auto load_b = [&](int kt, int slot, int c) __attribute__((always_inline)) {
      stage16(bb + kt * bstep, bo[c], lbase + RA * OA::BYTES + slot * OB::BYTES + (c * NTH + wbase) * 16);
    };
    // any stage, the short last one of a sum over rows too: k past the end are
    // zeros, and none of its loads is left (the waits below count loads)
    const int kfull = TA && TB ? min(k1, g.K / BK) : k1;
    auto any_a = [&](int kt, int slot) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < ACH; ++c) {
        if ((TA && TB) && kt >= kfull) {
          const int q = tid + c * NTH;
          int line, e;
          OA::place(q, line, e);
          uint4 v = make_uint4(0, 0, 0, 0);
          if (kt * BK + line < g.K) v = *reinterpret_cast<const uint4*>(ab + kt * astep + ao[c]);
          *reinterpret_cast<uint4*>(lds + slot * OA::BYTES + q * 16) = v;
        } else {
          load_a(kt, slot, c);
        }
      }
      if ((TA && TB) && kt >= kfull) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    auto any_b = [&](int kt, int slot) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < BCH; ++c) {
        if ((TA && TB) && kt >= kfull) {
          const int q = tid + c * NTH;
          int line, e;
          OB::place(q, line, e);
          uint4 v = make_uint4(0, 0, 0, 0);
          if (kt * BK + line < g.K) v = *reinterpret_cast<const uint4*>(bb + kt * bstep + bo[c]);
          *reinterpret_cast<uint4*>(lds + RA * OA::BYTES + slot * OB::BYTES + q * 16) = v;
        } else {
          load_b(kt, slot, c);
        }
      }
      if ((TA && TB) && kt >= kfull) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto bcol = [&](int j) __attribute__((always_inline)) {  // LDS row of B's fragment j
      if constexpr (EK == E_SWIGLU) return (j < NT / 2 ? 0 : TN) + wn * (TN / SH::WN) + (j % (NT / 2)) * 16;
      else return wn * (BN / SH::WN) + j * 16;
    };
    auto fetch = [&](FA (&a)[MT], FB (&b)[NT], int sa, int sb, int h) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NT; ++j) b[j] = FB::load(lds + RA * OA::BYTES + sb * OB::BYTES, bcol(j), h, lane);
#pragma unroll
      for (int i = 0; i < MT; ++i) a[i] = FA::load(lds + sa * OA::BYTES, wm * (BM / SH::WM) + i * 16, h, lane);
    };
    // B is the instruction's first operand, so that a lane holds four consecutive columns of one row
    auto multiply = [&](FA (&a)[MT], FB (&b)[NT], int i) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = mma(b[j], a[i], acc[i][j]);
    };

    if (first < last) {
      if constexpr (NTH == 512) {
        // Three stages of A in LDS and two of B.  Two waves on each SIMD take turns:
        // while one multiplies half a stage, the other reads the fragments of its
        // next half, then they change places at a barrier (waves 4 to 7 start one
        // barrier later).  When the late waves have read the last half of stage k,
        // its places are free for B of k + 2 and A of k + 3: the late waves load them
        // between the products of that half, the early ones, whose turn it is to
        // read, between those of their next.  A stage's loads of B have three to four
        // turns to arrive, those of A seven to eight: the weights are in L2, the rows
        // come from memory.  At the last turn before stage k + 1 everyone waits for
        // its own loads of it, which leaves those of A of k + 2.
        static_assert(WK == 1 && RA == 3 && RB == 2 && MT == ACH + BCH, "loads between the products");
        const bool is_late = wbase >= 256;
        any_a(k0, 0);
        any_b(k0, 0);
        if (k0 + 1 < k1) any_a(k0 + 1, 1);
        if (is_late && k0 + 1 < k1) any_b(k0 + 1, 1);
        if (is_late && k0 + 2 < k1) any_a(k0 + 2, 2);
        if (k0 + 2 >= kfull) wait_barrier<0>();
        else if (is_late) wait_barrier<2 * ACH + BCH>();
        else wait_barrier<ACH>();
        auto turns = [&](auto late_) __attribute__((always_inline)) {
          constexpr bool late = decltype(late_)::value;
          FA a[MT];
          FB b[NT];
          if (late) wait_reads();
          int kt = k0, sa = 0, sb = 0;
          auto next3 = [](int s) __attribute__((always_inline)) { return s == 2 ? 0 : s + 1; };
          // one stage; its loads are of B of kb and A of kb + 1, both whole
          for (; kt + (late ? 3 : 2) < kfull; ++kt) {
            const int sp = sa == 0 ? 2 : sa - 1;  // A of kt - 1, and of kt + 2
            fetch(a, b, sa, sb, 0);
            wait_reads();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              multiply(a, b, i);
              if (!late && i < BCH) load_b(kt + 1, sb ^ 1, i);
              else if (!late) load_a(kt + 2, sp, i - BCH);
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            wait_reads();
            __builtin_amdgcn_sched_barrier(0);
            fetch(a, b, sa, sb, 1);
            if (late) wait_barrier<ACH>();
            else wait_reads();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              multiply(a, b, i);
              if (late && i < BCH) load_b(kt + 2, sb, i);
              else if (late) load_a(kt + 3, sa, i - BCH);
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            if (late) wait_reads();
            else wait_barrier<ACH>();
            __builtin_amdgcn_sched_barrier(0);
            sa = next3(sa);
            sb ^= 1;
          }
          for (; kt < k1; ++kt) {
            const int sp = sa == 0 ? 2 : sa - 1;
            fetch(a, b, sa, sb, 0);
            wait_reads();
            __builtin_amdgcn_sched_barrier(0);
            if (!late && kt + 1 < k1) any_b(kt + 1, sb ^ 1);
            if (!late && kt + 2 < k1) any_a(kt + 2, sp);
#pragma unroll
            for (int i = 0; i < MT; ++i) multiply(a, b, i);
            __builtin_amdgcn_sched_barrier(0);
            wait_reads();
            __builtin_amdgcn_sched_barrier(0);
            fetch(a, b, sa, sb, 1);
            if (late) wait_barrier<0>();
            else wait_reads();
            __builtin_amdgcn_sched_barrier(0);
            if (late && kt + 2 < k1) any_b(kt + 2, sb);
            if (late && kt + 3 < k1) any_a(kt + 3, sa);
#pragma unroll
            for (int i = 0; i < MT; ++i) multiply(a, b, i);
            __builtin_amdgcn_sched_barrier(0);
            if (late) wait_reads();
            else wait_barrier<0>();
            __builtin_amdgcn_sched_barrier(0);
            sa = next3(sa);
            sb ^= 1;
          }
          if (!late) wait_reads();
        };
        if (is_late) turns(std::true_type{});
        else turns(std::false_type{});
      } else {
        // Two sets of fragments: while half a stage is multiplied, the next half's
        // fragments are read.  The barrier in the middle ends every wave's reads of
        // stage kt and every wave's loads of kt + 1; kt + RA then goes where kt was.
        static_assert(RA == RB, "one ring");
        constexpr int LPT = ACH + BCH;
        FA a0[MT], a1[MT];
        FB b0[NT], b1[NT];
#pragma unroll
        for (int k = 0; k < RA; ++k)
          if (k0 + k < k1) {
            any_a(k0 + k, k);
            any_b(k0 + k, k);
          }
        if (k0 + RA - 1 < kfull) wait_barrier<(RA - 1) * LPT>();
        else wait_barrier<0>();
        if (WK == 1 || k0 < k1) fetch(a0, b0, 0, 0, 0);
        int st = 0;
        for (int it = 0; it < turns_n; ++it) {
          const int kt = k0 + it, sn = st + 1 == RA ? 0 : st + 1;
          const bool on = WK == 1 || kt < k1;
          if (on) {
            fetch(a1, b1, st, st, 1);
#pragma unroll
            for (int i = 0; i < MT; ++i) multiply(a0, b0, i);
          }
          if (RA > 2 && kt + RA - 1 < kfull) wait_barrier<(RA - 2) * LPT>();
          else wait_barrier<0>();
          if (kt + RA < k1) {
            any_a(kt + RA, st);
            any_b(kt + RA, st);
          }
          if (kt + 1 < k1) fetch(a0, b0, sn, sn, 0);
          if (on) {
#pragma unroll
            for (int i = 0; i < MT; ++i) multiply(a1, b1, i);
          }
          st = sn;
        }
      }
    }
    if constexpr (WK > 1) {
      // groups 1 .. WK - 1 hand their sums to group 0
      float* sums = reinterpret_cast<float*>(lds0);
      __syncthreads();
      if (grp > 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
            Vec4<float>::store(sums + (grp - 1) * (BM * BN) + (((wave * MT + i) * NT + j) * kWave + lane) * 4, acc[i][j]);
      }
      __syncthreads();
      if (grp > 0) return;
#pragma unroll
      for (int k = 1; k < WK; ++k)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
            acc[i][j] += Vec4<float>::load(sums + (k - 1) * (BM * BN) + (((wave * MT + i) * NT + j) * kWave + lane) * 4);
    }

    // lane: row m0 + .. + lane % 16, columns .. + 4 (lane / 16) + 0..3
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) Vec4<float>::store(part + (((wave * MT + i) * NT + j) * kWave + lane) * 4, acc[i][j]);
      return;
    }
    // q and p are on their way kAhead rows of accumulators early, since the compiler
    // moves no load past a store (da of 16384 x 1024 x 2816 148 -> 146 us, of 2000 x
    // 1024 x 2816 30 -> 28; all 8 rows early spill: 173)
    constexpr int kAhead = MT < 4 ? MT : 4;
    const int64_t pairs = (int64_t)((g.M + 15) >> 4) * (g.N >> 5);
    typename Kept<T>::Raw raw[MT][NT / 2];
    auto early = [&](int i) __attribute__((always_inline)) {
      const int mb = m0 + wm * (BM / SH::WM) + i * 16, n = n0 + wn * (BN / SH::WN);
      if (mb >= g.M) return;
#pragma unroll
      for (int j = 0; j < NT / 2; ++j)
        if (n + j * 32 < g.N)
          Kept<T>::load(g.kept, pairs, (int64_t)(mb >> 4) * (g.N >> 5) + (n >> 5) + j, lane, raw[i][j]);
    };
    if constexpr (EK == E_DSWIGLU) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) early(i);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int mb = m0 + wm * (BM / SH::WM) + i * 16, m = mb + (lane & 15);
      if (mb >= g.M) break;
      if constexpr (EK == E_DSWIGLU) {
        if (i + kAhead < MT) early(i + kAhead);
      }
      const bool in = m < g.M;
      if constexpr (EK == E_SWIGLU) {
#pragma unroll
        for (int j = 0; j < NT / 2; j += 2) {
          const int f = n0 + wn * (TN / SH::WN) + j * 16;
          if (f >= g.N) break;
          f32x4 h[2], q[2], p[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const f32x4 gt = acc[i][j + x], up = acc[i][j + x + NT / 2];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float s = sigmoid<T>(gt[r]);
              p[x][r] = gt[r] * s;
              q[x][r] = up[r] * (s * (1.f + gt[r] * (1.f - s)));
              h[x][r] = p[x][r] * up[r];
            }
          }
          if (g.kept) Kept<T>::store(g.kept, pairs, (int64_t)(mb >> 4) * (g.N >> 5) + (f >> 5), lane, q, p);
          if (in) store_pair<T>(reinterpret_cast<T*>(g.out) + m * g.ldo + f, h[0], h[1], lane);
        }
      } else {
#pragma unroll
        for (int j = 0; j < NT; j += 2) {
          const int n = n0 + wn * (BN / SH::WN) + j * 16;
          if (n >= g.N) break;
          if constexpr (EK == E_STORE) {
            if (in) store_pair<T>(reinterpret_cast<T*>(g.out) + m * g.ldo + n, acc[i][j], acc[i][j + 1], lane);
          } else {
            f32x4 q[2], p[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) Kept<T>::get(raw[i][j / 2], x, q[x], p[x]);
            T* o = reinterpret_cast<T*>(g.out) + m * g.ldo + n;
            if (in) {
              store_pair<T>(o, acc[i][j] * q[0], acc[i][j + 1] * q[1], lane);
              store_pair<T>(o + g.N, acc[i][j] * p[0], acc[i][j + 1] * p[1], lane);
            }
          }
        }
      }
    }
  }
};

// bf16 on 256 x 256 tiles, us and TFLOP/s of kernels that run one at a time: 16384 x
// 1024 x 2816 gate/up 216 (875), down 78 (1215), da 151 (625), dx 145 (1300); 8191 x
// 2048 x 5504 356 (1040), 142 (1300), 222 (830), 280 (1320); traced right behind each
// other they take up to a tenth more.  The matrix cores are busy 36, 49, 25 and 56%
// of the first four, no LDS read meets a bank conflict.  The loads into LDS bound the
// products: without them 135, 50, 139 and 91 us of the first four (then 231, 91, 153,
// 155), alone 131 of gate/up, 73 of down, 126 of dx, of which 37 of down's where all
// of it is in L2.  Gate/up writes 300 MB in its epilogue and da reads and writes 392:
// one workgroup fills a compute unit, so nothing else runs on it meanwhile, and it
// does not load its next tile then, though the epilogue needs none of the LDS.
template <typename T, bool TA, bool TB, int EK, typename SH> __global__ __launch_bounds__(SH::NTH) void k_ffn(FArgs g) {
  using TL = Tile<T, TA, TB, EK, SH, false>;
  __shared__ __align__(16) char lds[TL::LDS];
  const Tiles ts{(g.M + SH::BM - 1) / SH::BM, (g.N + TL::TN - 1) / TL::TN};
  int row, col;
  ts.at(xcd_run(blockIdx.x, gridDim.x), row, col);
  TL::run(g, row * SH::BM, col * TL::TN, 0, (g.K + TL::BK - 1) / TL::BK, nullptr, lds);
}

// Products with few tiles and a long sum, in `splits` ranges of k.  The tiles of
// one range follow each other, so that an XCD's workgroups read the same k at a
// time (with ranges that begin at any k, every tile's share of the same length,
// dW_gate_up of 16384 x 1024 x 2816 took 243 us where these took 205, and take 191
// with stages of whole lines: without reuse in L2).
template <typename T, bool TA, bool TB, typename SH> __global__ __launch_bounds__(SH::NTH) void k_ffn_split(FArgs g) {
  using TL = Tile<T, TA, TB, E_STORE, SH, true>;
  __shared__ __align__(16) char lds[TL::LDS];
  const Tiles ts{(g.M + SH::BM - 1) / SH::BM, (g.N + SH::BN - 1) / SH::BN};
  const int u = xcd_run(blockIdx.x, gridDim.x), n = ts.tm * ts.tn, s = u / n, KT = (g.K + TL::BK - 1) / TL::BK;
  int row, col;
  ts.at(u - s * n, row, col);
  TL::run(g, row * SH::BM, col * SH::BN, (int)((int64_t)KT * s / g.splits), (int)((int64_t)KT * (s + 1) / g.splits),
          g.part + (int64_t)u * (SH::BM * SH::BN), lds);
}

// The ranges' sums added in order and rounded once; a workgroup per 1024
// elements of a tile, in the accumulators' order.
template <typename T, typename SH> __global__ __launch_bounds__(256) void k_ffn_join(FArgs g) {
  constexpr int MT = SH::BM / SH::WM / 16, NT = SH::BN / SH::WN / 16;
  const Tiles ts{(g.M + SH::BM - 1) / SH::BM, (g.N + SH::BN - 1) / SH::BN};
  int row, col;
  ts.at(blockIdx.y, row, col);
  const int v = blockIdx.x * 256 + threadIdx.x, lane = v & 63, f = v >> 6;  // fragment of the tile
  const int j = f % NT, i = f / NT % MT, wave = f / (NT * MT);
  const int m = row * SH::BM + wave / SH::WN * (SH::BM / SH::WM) + i * 16 + (lane & 15);
  const int n = col * SH::BN + wave % SH::WN * (SH::BN / SH::WN) + j * 16 + (lane >> 4) * 4;
  const float* p = g.part + (int64_t)blockIdx.y * (SH::BM * SH::BN) + (int64_t)v * 4;
  const int64_t step = (int64_t)gridDim.y * (SH::BM * SH::BN);
  f32x4 c = Vec4<float>::load(p);
#pragma unroll 4
  for (int s = 1; s < g.splits; ++s) c += Vec4<float>::load(p + s * step);
  if (m < g.M && n < g.N) Vec4<T>::store(reinterpret_cast<T*>(g.out) + m * g.ldo + n, c);
}

using Big = FShape<256, 256, 2, 4, 3, 2, 1>;
using Mid = FShape<128, 128, 2, 2, 2, 2, 1>;
using Small = FShape<64, 64, 4, 1, 3, 3, 1>;
using Deep = FShape<64, 64, 4, 1, 2, 2, 4>;

template <typename T, bool TA, bool TB, int EK, typename SH> hipError_t launch_shape(const FArgs& g, hipStream_t s) {
  constexpr int TN = EK == E_SWIGLU ? SH::BN / 2 : SH::BN;
  const int64_t tiles = (int64_t)((g.M + SH::BM - 1) / SH::BM) * ((g.N + TN - 1) / TN);
  if (tiles <= 0 || tiles > INT32_MAX) return tiles == 0 ? hipSuccess : hipErrorInvalidValue;
  hipLaunchKernelGGL((k_ffn<T, TA, TB, EK, SH>), dim3((unsigned)tiles), dim3(SH::NTH), 0, s, g);
  return hipGetLastError();
}

constexpr int64_t kCus = 256;  // compute units

int64_t tiles_of(int64_t m, int64_t n, int64_t b) { return ((m + b - 1) / b) * ((n + b - 1) / b); }

// Whether tiles of 256 x 256, one per compute unit at a time, leave less than a
// third of the compute units' time unused.
bool big_fits(int64_t tiles) {
  const int64_t rounds = (tiles + kCus - 1) / kCus;
  return 3 * tiles >= 2 * kCus * rounds;
}

// The fused products: Big where it fits, Mid from 300 tiles of its size, else
// Small.  bf16, us with Small, Mid and Big, gate/up with the product down
// behind it and da with dx: 333 x 768 x 2048 19, 25, 37 and 29, 38, 53; 1000 x
// 768 x 2048 27, 27, 38 and 31, 39, 54; 4096 x 1024 x 2816 109, 101, 102 and 131,
// 131, 125; 8191 x 2048 x 5504 624, 555, 468 and 606, 539, 490.  float32 is bound
// by its matrix instructions and takes Small (1000 x 256 x 512: 24 and 36, Mid 36
// and 51).
template <typename T, bool TA, bool TB, int EK> hipError_t launch_fused(const FArgs& g, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    const int64_t n = EK == E_SWIGLU ? 2 * (int64_t)g.N : g.N;
    if (big_fits(tiles_of(g.M, n, 256))) return launch_shape<T, TA, TB, EK, Big>(g, s);
    if (tiles_of(g.M, n, 128) >= 300) return launch_shape<T, TA, TB, EK, Mid>(g, s);
  }
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

// Up to this many elements every launch has fewer than 2^32 threads.
bool launchable(int32_t rows, int32_t d, int32_t f) { return rows * (int64_t)(d > f ? d : f) < (int64_t)1 << 35; }

// How a product that is only stored is computed.
enum { P_SMALL = 0, P_MID = 1, P_BIG = 2, P_DEEP = 3 };
struct Plan {
  int shape;
  int splits;      // ranges of k that are summed apart, 1: none
  size_t part;     // bytes of their sums
};

int tile_of(int shape) { return shape == P_BIG ? 256 : shape == P_MID ? 128 : 64; }

Plan plan_of(int shape, int64_t m, int64_t n, int64_t splits) {
  const int64_t b = tile_of(shape);
  return {shape, (int)splits, splits > 1 ? (size_t)(splits * tiles_of(m, n, b) * b * b) * sizeof(float) : 0};
}

// y and dx, m rows, n columns, `stages` of 128 bytes of k.
//
// bf16, large tiles where they fill the device, those of 128 x 128 with one on
// most compute units or with so many that few of them having two does not matter:
// us of the forward pass and of da with dx with Small, Mid and Big 3001 x 1024 x
// 2816 (192 tiles of 128 x 128) 82, 88, 112 and 106, 111, 160; 3580 x 1024 x 2816
// (224) 92, 88, 113 and 128, 112, 160; 2000 x 2048 x 5504 (256) 180, 171, 214 and 225,
// 191, 278; 4400 x 1024 x 2816 (280) 106, 109, 123 and 135, 133, 158; 8191 x 2048 x
// 5504 (1024) 589, 515, 456 and 890, 597, 486.  From 257 to 299 tiles of 128 x 128 the
// sides are level: 280 above, and the y of 6000 x 768 x 2048 (282) 76-78 with Small in
// the whole pass, 79 with Mid.
//
// Else tiles of 64 x 64, by four waves where there are more than compute units,
// by 16, which share the sum, below (1300 x 768 x 2048, 252 tiles, 33 and 31, 37 and
// 35; 1500 x 768 x 2048, 288 tiles, 35 and 41, 44 and 51), and by four with the sum in
// ranges where few tiles have a long one (16 waves and ranges: 1 x 2048 x 5504 32, 22
// and 57, 28; 10 x 768 x 2048 16, 14 and 23, 16; 333 x 768 x 2048 19, 19 and 29, 23; 256
// x 2048 x 5504 45, 38 and 67, 47; not 1000 x 768 x 2048 26, 27 and 31, 33).  float32,
// whose products take more of the time, the same with other limits (300 x 256 x
// 512 21, 17 and 31, 20; 1000 x 256 x 512 23, 19 and 33, 23; 3001 x 256 x 512 32, 36 and
// 36, 39).
Plan store_plan(bool half, int64_t m, int64_t n, int64_t stages) {
  if (half && big_fits(tiles_of(m, n, 256))) return plan_of(P_BIG, m, n, 1);
  const int64_t mid = tiles_of(m, n, 128), tiles = tiles_of(m, n, 64);
  if (half && ((mid >= 208 && mid <= kCus) || mid >= 300)) return plan_of(P_MID, m, n, 1);
  if (tiles == 0 || tiles > kCus) return plan_of(P_SMALL, m, n, 1);
  const int64_t wide = (half ? 2 : 1) * kCus / tiles, deep = stages / (half ? 6 : 3), s = wide < deep ? wide : deep;
  if (s >= 2 && (!half || tiles <= 64 || (tiles <= 176 && stages >= 40))) return plan_of(P_SMALL, m, n, s < 16 ? s : 16);
  return plan_of(P_DEEP, m, n, 1);
}

// Estimated ns of a weight gradient with tiles of b x b, `slots` of which the
// device holds: per round, the stages (64 rows) and a start and an end.
int64_t rounds_time(int64_t tiles, int64_t slots, int64_t stages, int64_t stage_ns, int64_t base_ns) {
  return (tiles + slots - 1) / slots * (stages * stage_ns + base_ns);
}

// A weight gradient [m][n], a sum over `rows` rows.  bf16: the shape of the least
// estimated time, tiles of 256 x 256 also in ranges of rows, whose sums are
// written and read again at 4.5 TB/s.  The times per stage are fitted to
// dW_down, measured us with Small, Mid, Big whole and Big in ranges: 1000 x 768 x
// 2048 13, 20, 30, 25 (2); 3001 x 1024 x 2816 36, 51, 69, 40 (5); 6000 x 768 x 2048
// 57, 92, 123, 40 (8); 1000 x 2048 x 5504 50, 42, 33, 66 (2); 8191 x 2048 x 5504
// 331, 268, 171, 214 (2); 16384 x 1024 x 2816 176, 242, 310, 91 (5).  float32: 64 x 64,
// the rows in ranges for a workgroup on each compute unit, or two with 375 rows or
// more (3001 x 256 x 512, ranges for one and for two: dW_down 17, 19, dW_gate_up 42
// with da, 39; 8000 rows 34, 30 and 89, 76; 1000 rows 11, 13 and 24, 26; whole 3001
// rows take 80 and 96; ranges of 375 rows were faster and of 125 slower, those in
// between are not measured).
Plan grad_plan(bool half, int64_t m, int64_t n, int64_t rows) {
  const int64_t stages = (rows + 63) / 64, small = tiles_of(m, n, 64), mid = tiles_of(m, n, 128), big = tiles_of(m, n, 256);
  if (!half) {
    const int64_t one = (kCus + small - 1) / small, few = rows / 64, two = 2 * kCus / small, long_ = rows / 375;
    const int64_t a = one < few ? one : few, b = two < long_ ? two : long_, s = a > b ? a : b;
    return plan_of(P_SMALL, m, n, rows < 256 || s < 1 ? 1 : s < 64 ? s : 64);
  }
  Plan best = plan_of(P_SMALL, m, n, 1);
  int64_t t = rounds_time(small, 3 * kCus, stages, small <= kCus ? 400 : small <= 2 * kCus ? 500 : 680, 3500);
  const int64_t tm = rounds_time(mid, 2 * kCus, stages, mid <= kCus ? 850 : 930, 5000);
  if (tm < t) {
    t = tm;
    best = plan_of(P_MID, m, n, 1);
  }
  for (int64_t s = 1; s <= 12 && (s == 1 || stages >= 4 * s); ++s) {
    const int64_t parts = s > 1 ? s * big * 117 + 5000 : 0;  // 2 x 256 KB each
    const int64_t tb = rounds_time(big * s, kCus, (stages + s - 1) / s, 1400, 6000) + parts;
    if (tb < t) {
      t = tb;
      best = plan_of(P_BIG, m, n, s);
    }
  }
  return best;
}

size_t dgu_bytes(int32_t dtype, int64_t rows, int64_t f) {
  return (size_t)(rows * 2 * f) * (dtype == TLF_DTYPE_BF16 ? 2 : 4);
}

template <typename T, bool TA, bool TB, typename SH> hipError_t launch_split(const FArgs& p, hipStream_t s) {
  if (p.splits == 1) return launch_shape<T, TA, TB, E_STORE, SH>(p, s);
  const int64_t tiles = tiles_of(p.M, p.N, SH::BM);
  hipLaunchKernelGGL((k_ffn_split<T, TA, TB, SH>), dim3((unsigned)(tiles * p.splits)), dim3(SH::NTH), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_ffn_join<T, SH>), dim3(SH::BM * SH::BN / 1024, (unsigned)tiles), dim3(256), 0, s, p);
  return hipGetLastError();
}

template <typename T, bool TA, bool TB> hipError_t launch_store(FArgs p, const Plan& plan, hipStream_t s) {
  p.splits = plan.splits;
  if constexpr (sizeof(T) == 2) {
    if (plan.shape == P_BIG) {
      if constexpr (TA) return launch_split<T, TA, TB, Big>(p, s);
      else return launch_shape<T, TA, TB, E_STORE, Big>(p, s);
    }
    if (plan.shape == P_MID) return launch_shape<T, TA, TB, E_STORE, Mid>(p, s);
  }
  if constexpr (!TA) {
    if (plan.shape == P_DEEP) return launch_shape<T, TA, TB, E_STORE, Deep>(p, s);
  }
  if constexpr (TA && sizeof(T) == 2) return launch_shape<T, TA, TB, E_STORE, Small>(p, s);
  else return launch_split<T, TA, TB, Small>(p, s);
}

template <typename T>
int ffn_forward(const void* x, const void* wgu, const void* wd, int rows, int d, int f, void* kept, void* a, void* y,
                float* part, hipStream_t s) {
  FArgs p{};
  p.A = x; p.B = wgu; p.lda = d; p.ldb = d; p.ldo = f;
  p.M = rows; p.N = f; p.K = d; p.out = a; p.kept = kept;
  if (launch_fused<T, false, false, E_SWIGLU>(p, s) != hipSuccess) return TLF_E_HIP;
  FArgs q{};
  q.A = a; q.B = wd; q.lda = f; q.ldb = f; q.ldo = d;
  q.M = rows; q.N = d; q.K = f; q.out = y; q.part = part;
  const Plan plan = store_plan(sizeof(T) == 2, rows, d, (int64_t)f * (int64_t)sizeof(T) / 128);
  return launch_store<T, false, false>(q, plan, s) == hipSuccess ? TLF_OK : TLF_E_HIP;
}

template <typename T>
hipError_t weight_grad(const void* a, int m, const void* b, int n, int rows, void* out, float* part, hipStream_t s) {
  FArgs p{};
  p.A = a; p.B = b; p.lda = m; p.ldb = n; p.ldo = n;
  p.M = m; p.N = n; p.K = rows; p.out = out; p.part = part;
  return launch_store<T, true, true>(p, grad_plan(sizeof(T) == 2, m, n, rows), s);
}

template <typename T>
int ffn_backward(const void* dy, const void* x, const void* wgu, const void* wd, const void* kept, const void* a, int rows,
                 int d, int f, void* dx, void* dwgu, void* dwd, char* ws, hipStream_t s) {
  void* dgu = ws;
  float* part = reinterpret_cast<float*>(ws + dgu_bytes(sizeof(T) == 2 ? TLF_DTYPE_BF16 : TLF_DTYPE_F32, rows, f));
  if (rows > 0 && (dx || dwgu)) {
    FArgs p{};
    p.A = dy; p.B = wd; p.lda = d; p.ldb = f; p.ldo = 2 * f;
    p.M = rows; p.N = f; p.K = d; p.out = dgu; p.kept = const_cast<void*>(kept);
    if (launch_fused<T, false, true, E_DSWIGLU>(p, s) != hipSuccess) return TLF_E_HIP;
  }
  if (dx) {
    FArgs p{};
    p.A = dgu; p.B = wgu; p.lda = 2 * f; p.ldb = d; p.ldo = d;
    p.M = rows; p.N = d; p.K = 2 * f; p.out = dx; p.part = part;
    const Plan plan = store_plan(sizeof(T) == 2, rows, d, 2 * (int64_t)f * (int64_t)sizeof(T) / 128);
    if (launch_store<T, false, true>(p, plan, s) != hipSuccess) return TLF_E_HIP;
  }
  if (dwgu && weight_grad<T>(dgu, 2 * f, x, d, rows, dwgu, part, s) != hipSuccess) return TLF_E_HIP;
  if (dwd && weight_grad<T>(dy, d, a, f, rows, dwd, part, s) != hipSuccess) return TLF_E_HIP;
  return TLF_OK;
}

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_ffn_ws_bytes(int32_t dtype, int32_t rows, int32_t d, int32_t f, size_t* ws_bytes) {
  const int st = tlf::check(dtype, rows, d, f);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  const bool half = dtype == TLF_DTYPE_BF16;
  *ws_bytes = tlf::store_plan(half, rows, d, (int64_t)f * (half ? 2 : 4) / 128).part;
  return TLF_OK;
}

int tlf_ffn(const void* d_x, const void* d_w_gate_up, const void* d_w_down, int32_t dtype, int32_t rows, int32_t d,
            int32_t f, void* d_kept, void* d_a, void* d_y, void* d_workspace, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int st = tlf_ffn_ws_bytes(dtype, rows, d, f, &need);
  if (st != TLF_OK) return st;
  if (rows == 0) return TLF_OK;
  if (!tlf::launchable(rows, d, f)) return TLF_E_UNSUPPORTED;
  if (!d_x || !d_w_gate_up || !d_w_down || !d_a || !d_y) return TLF_E_INVALID_ARG;
  if (need > 0 && (!d_workspace || ws_bytes < need)) return TLF_E_INVALID_ARG;
  for (const void* p : {d_x, d_w_gate_up, d_w_down, (const void*)d_kept, (const void*)d_a, (const void*)d_y,
                        (const void*)d_workspace})
    if (!tlf::aligned16(p)) return TLF_E_INVALID_ARG;
  return dtype == TLF_DTYPE_BF16
             ? tlf::ffn_forward<bf16>(d_x, d_w_gate_up, d_w_down, rows, d, f, d_kept, d_a, d_y, (float*)d_workspace,
                                      (hipStream_t)stream)
             : tlf::ffn_forward<float>(d_x, d_w_gate_up, d_w_down, rows, d, f, d_kept, d_a, d_y, (float*)d_workspace,
                                       (hipStream_t)stream);
}

int tlf_ffn_grad_ws_bytes(int32_t dtype, int32_t rows, int32_t d, int32_t f, size_t* ws_bytes) {
  const int st = tlf::check(dtype, rows, d, f);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  const bool half = dtype == TLF_DTYPE_BF16;
  size_t part = 0;  // of the three products that may be split, one after the other
  for (const tlf::Plan& p : {tlf::store_plan(half, rows, d, 2 * (int64_t)f * (half ? 2 : 4) / 128),
                             tlf::grad_plan(half, 2 * (int64_t)f, d, rows), tlf::grad_plan(half, d, f, rows)})
    part = p.part > part ? p.part : part;
  *ws_bytes = tlf::dgu_bytes(dtype, rows, f) + part;
  return TLF_OK;
}

int tlf_ffn_grad(const void* d_dy, const void* d_x, const void* d_w_gate_up, const void* d_w_down, const void* d_kept,
                 const void* d_a, int32_t dtype, int32_t rows, int32_t d, int32_t f, void* d_dx, void* d_dw_gate_up,
                 void* d_dw_down, void* d_workspace, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int st = tlf_ffn_grad_ws_bytes(dtype, rows, d, f, &need);
  if (st != TLF_OK) return st;
  if (!d_dx && !d_dw_gate_up && !d_dw_down) return TLF_OK;
  if (rows > 0) {
    if (!tlf::launchable(rows, d, f)) return TLF_E_UNSUPPORTED;
    if (!d_dy || !d_x || !d_w_gate_up || !d_w_down || !d_kept || !d_a) return TLF_E_INVALID_ARG;
    if (need > 0 && (!d_workspace || ws_bytes < need)) return TLF_E_INVALID_ARG;
  }
  for (const void* p : {d_dy, d_x, d_w_gate_up, d_w_down, d_kept, d_a, (const void*)d_dx, (const void*)d_dw_gate_up,
                        (const void*)d_dw_down, (const void*)d_workspace})
    if (!tlf::aligned16(p)) return TLF_E_INVALID_ARG;
  if (rows == 0) d_dx = nullptr;  // no rows; the weights' gradients are zeros
  return dtype == TLF_DTYPE_BF16
             ? tlf::ffn_backward<bf16>(d_dy, d_x, d_w_gate_up, d_w_down, d_kept, d_a, rows, d, f, d_dx, d_dw_gate_up,
                                       d_dw_down, (char*)d_workspace, (hipStream_t)stream)
             : tlf::ffn_backward<float>(d_dy, d_x, d_w_gate_up, d_w_down, d_kept, d_a, rows, d, f, d_dx, d_dw_gate_up,
                                        d_dw_down, (char*)d_workspace, (hipStream_t)stream);
}

}  // extern "C"
