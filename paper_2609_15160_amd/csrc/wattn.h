// Causal attention of ragged rows with a sliding window and sinks: what its
// forward and backward kernels share (gfx950 only).
//
// Sequence b has query rows [q_off[b], q_off[b + 1]) and n keys from row k_off[b];
// its last query stands at its last key, query j at position p = n - nq + j.  The
// key at position x is visible to the query at p when
//   x <= p and (p - x < window or x < sinks).
//
// All products are MFMA of 16 x 16 tiles.  A row-major LDS tile (rows of keys or of
// queries) gives both operands: rows as they lie (contraction over the head's
// dimensions), and transposed (contraction over rows).  Scores are computed so that
// a lane's accumulators are four rows of one column; as operand of the next product
// they are the rows 4 g .. 4 g + 3 (g = lane / 16) of one or two tiles, and the
// other operand is read in the same order of rows, so scores never leave registers.
#pragma once

#include "common.h"
#include "stage.h"
#include "visible.h"

namespace tlf {

struct WAttnArgs {
  const void *q, *k, *v, *o, *dout;
  void *out, *dq, *dk, *dv;
  void* low;                        // [rows_q] as o: what its rounding took, or NULL
  float* lse;                       // [heads][rows_q]: log2 of the softmax sums
  float *nlse, *ndelta;             // [heads][rows_q]: -lse in units of q . k, -o . do
  float* part;
  const int32_t *q_off, *k_off, *k_len;
  int64_t qs, ks, vs, os;           // elements between rows; gradients lie as what they belong to
  int batch, heads, kv_heads, rows_q, rows_k, window, sinks;
  int slots;                        // tiles of rows, an upper bound
  int splits;
  float scale, scale_log2;
};

struct WSeq {
  int q0, nq, k0, n, cap;  // first rows, queries, keys, rows that the keys have room in
};

// Waves per SIMD that the registers of the kernels leave room for.  Up to 256
// registers a wave's products take their accumulators as they take other values;
// with more, scores are copied from and to registers that only products reach.
template <typename T, int D> constexpr int kRoom = sizeof(T) == 4 && D == 128 ? 1 : 2;

// Waves of a workgroup of the tile kernels.  One wave each, which would spread few rows
// over more compute units, was slower at every size (12 x 64 heads, bf16, forward, dq and
// dkv, us with four and with one: 4 x 200 rows 9, 10, 11 and 10, 10, 12; 8 x 800 26, 30,
// 36 and 48, 46, 59; float32 4 x 200 21, 28, 36 and 21, 28, 35).
constexpr int kTileWaves = 4;

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Tiles of STEP rows: sequence b's begin at slot off[b] / STEP + b + 1, which leaves
// each at least as many slots as it has tiles and needs no plan on the device.  The rows
// ahead of the first sequence are one more, number -1, and those behind the last are
// number `batch`: sequences without keys.
template <int STEP> __device__ __forceinline__ int slot_of(const int32_t* off, int rows, int b) {
  return b < 0 ? 0 : clampi(off[b], 0, rows) / STEP + b + 1;
}
template <int STEP> inline int64_t slots_of(int64_t rows, int64_t batch) { return rows / STEP + batch + 2; }

// The last b in [-1, batch] whose slots begin at or before `slot`, 64 at a time.
template <int STEP> __device__ __forceinline__ int seq_of(const int32_t* off, int rows, int batch, int slot) {
  int lo = -1, hi = batch;
  while (hi > lo) {
    const int step = (hi - lo + kWave - 1) / kWave, b = lo + (lane_id() + 1) * step;
    const bool before = b <= hi && slot_of<STEP>(off, rows, min(b, hi)) <= slot;
    lo += __builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) * step;
    hi = min(hi, lo + step - 1);
  }
  return lo;
}

__device__ __forceinline__ WSeq load_seq(const WAttnArgs& a, int b) {
  WSeq s;
  s.q0 = b < 0 ? 0 : clampi(a.q_off[b], 0, a.rows_q);
  s.k0 = b < 0 ? 0 : clampi(a.k_off[b], 0, a.rows_k);
  if (b < a.batch) {
    s.nq = clampi(a.q_off[b + 1], s.q0, a.rows_q) - s.q0;
    s.cap = clampi(a.k_off[b + 1], s.k0, a.rows_k) - s.k0;
    s.n = b < 0 ? 0 : a.k_len ? clampi(a.k_len[b], 0, s.cap) : s.cap;
  } else {
    s.nq = a.rows_q - s.q0;
    s.cap = a.rows_k - s.k0;
    s.n = 0;
  }
  return s;
}

// What a tile's scores are masked by.  Each comparison is with a constant of the
// unrolled code and is used up by one select: differences and combined masks would
// take more instructions than the products, and more scalar registers than there are.
enum Mask {
  M_NONE = 0,   // every pair is visible
  M_UPPER = 1,  // keys behind the query are not
  M_LOWER = 2,  // keys before the window are not
  M_ALL = 3     // both (M_UPPER | M_LOWER), and sinks
};
__device__ __forceinline__ int reach(int x, int window, int sinks) { return x < sinks ? INT32_MAX : window; }
__device__ __forceinline__ bool sees(int p, int x, int far) { return (unsigned)(p - x) < (unsigned)far; }

// The mask of queries at positions [p0, p1] and keys [k0, k1], or -1: nothing is visible.
__device__ __forceinline__ int mask_of(int p0, int p1, int k0, int k1, int window, int sinks) {
  if (k0 > p1 || (p0 - k1 >= window && k0 >= sinks)) return -1;
  const bool low = p1 - k0 >= window && k1 >= sinks, up = k1 > p0;
  return !low ? (up ? M_UPPER : M_NONE) : up || k0 < sinks ? M_ALL : M_LOWER;
}

// Operands of 16 bytes per lane: bf16, eight values of one MFMA over 32; float32,
// four values of one MFMA over 4 each.
template <typename T> struct Opnd;
template <> struct Opnd<bf16> {
  typedef bf16x8 frag;
  static constexpr int TILES = 2;  // score tiles of one operand
  static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ frag ones() { return __builtin_bit_cast(frag, make_uint4(kOnes, kOnes, kOnes, kOnes)); }
  static constexpr unsigned kOnes = 0x3F803F80u;
  static __device__ __forceinline__ frag pack(const f32x4* s) {  // the rows of two score tiles
    return __builtin_bit_cast(frag, make_uint4(pack_bf16x2(s[0][0], s[0][1]), pack_bf16x2(s[0][2], s[0][3]),
                                               pack_bf16x2(s[1][0], s[1][1]), pack_bf16x2(s[1][2], s[1][3])));
  }
};
template <> struct Opnd<float> {
  typedef f32x4 frag;
  static constexpr int TILES = 1;
  static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ frag pack(const f32x4* s) { return s[0]; }
};

// LDS rows of one head: D elements in 16-byte chunks, chunk c of row r at place
// c ^ key(r).  The keys of 16 rows are distinct where 16 rows span the banks
// twice, those of rows 0..7 differ by pairs of chunks: reads of 16 rows' chunks and
// transposed reads of 8 rows' chunk pairs both fall into distinct banks.
template <typename T, int D> struct HeadRows {
  using O = Opnd<T>;
  typedef typename O::frag frag;
  static constexpr int EPC = 16 / (int)sizeof(T);
  static constexpr int RB = D * (int)sizeof(T);      // bytes of a row
  static constexpr int CPR = RB / 16;                // its chunks
  static constexpr int KSTEPS = CPR / 4;             // contraction steps over D
  static constexpr int DT = D / 16;
  static constexpr int ROWS = 16 * O::TILES;         // rows of one transposed operand
  static constexpr int PER = RB >= 256 ? 1 : 256 / RB, KEYS = CPR < 16 ? CPR : 16;
  static_assert(CPR % 4 == 0 && D % 16 == 0, "head width");
  static __device__ __forceinline__ int key(int r) {
    const int x = (r / PER) & (KEYS - 1);
    return (x & (KEYS / 2 - 1)) << 1 | x / (KEYS / 2);
  }
  // This lane's byte offsets in a tile at a multiple of RB * 16: of row i's chunk of step
  // 0, and of the transposed reads of dimension tile 0.  The others differ by the bits
  // that the key is added to, so they need no register.
  static __device__ __forceinline__ unsigned direct(int lane) {
    const int i = lane & 15, g = lane >> 4;
    return i * RB + ((g ^ key(i)) << 4);
  }
  static __device__ __forceinline__ unsigned transposed(int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (sizeof(T) == 2) {
      const int r = 4 * g + (i >> 2);  // a group of 16 lanes reads 4 rows x 16 dimensions, lane i gets dimension i
      return r * RB + ((((i >> 1) & 1) ^ key(r)) << 4) + (i & 1) * 8;
    } else {
      return 4 * g * RB + (((i >> 2) ^ key(4 * g)) << 4) + (i & 3) * 4;
    }
  }
  // A tile's read addresses: its LDS address plus direct() or transposed() for step ks or
  // dimension tile dt; rows that are multiples of 16 further on are an offset to it.
  static __device__ __forceinline__ unsigned step(unsigned at, int ks) { return at ^ (ks << 6); }
  static __device__ __forceinline__ unsigned tile(unsigned at, int dt) { return at ^ (dt << (sizeof(T) == 2 ? 5 : 6)); }
  static __device__ __forceinline__ frag load(unsigned at, int row) {
    return *(const __attribute__((address_space(3))) frag*)(at + row * RB);
  }
  // the ROWS rows from `row` on
  static __device__ __forceinline__ frag load_t(unsigned at, int row) {
    if constexpr (sizeof(T) == 2) {
      union { s16x4 h[2]; frag v; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + row * RB));
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + (row + 16) * RB));
      return u.v;
    } else {
      frag v;  // rows 4 g + j: their keys differ from that of 4 g
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *(const __attribute__((address_space(3))) float*)((at ^ (key_step(j) << 4)) + (row + j) * RB);
      return v;
    }
  }
  // key(4 g + j) ^ key(4 g), which is the same for every g
  static constexpr int key_step(int j) {
    const int x = (j / PER) & (KEYS - 1);
    return (x & (KEYS / 2 - 1)) << 1 | x / (KEYS / 2);
  }
};

// Transposed operands on their way: the first kAhead dimension tiles are read before
// the softmax's arithmetic, each later one when one of them has been used.  Left to
// itself the compiler reads each right before its use, to save registers.
constexpr int kAhead = 2;
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

// Two tiles of ROWS rows each (A and B, of one head) from global memory into LDS,
// asynchronously.  Rows past the last one are read from the last one.
template <typename T, int D, int ROWS, int NTH> struct PairLoader {
  using H = HeadRows<T, D>;
  static constexpr int HALF = ROWS * H::CPR;       // chunks of a tile
  static constexpr int N = 2 * HALF / NTH;         // chunks of a thread
  static constexpr int BYTES = 2 * ROWS * H::RB;   // A, then B
  static_assert(2 * HALF % NTH == 0 && HALF % kWave == 0 && (N == 1 || HALF % NTH == 0), "chunks");
  static constexpr int STEP = NTH / H::CPR;                   // rows from one chunk of a thread to its next
  static constexpr int KINDS = STEP % 16 == 0 ? 1 : 16 / STEP;  // keys repeat after 16 rows
  static_assert(NTH % H::CPR == 0 && (N == 1 || ROWS % STEP == 0) && (STEP % 16 == 0 || 16 % STEP == 0), "rows of a thread");
  int row0, chunk[KINDS];  // first row, byte of the chunk
  int wbase;
  __device__ __forceinline__ void init() {
    wbase = __builtin_amdgcn_readfirstlane(threadIdx.x & ~(kWave - 1));
    row0 = threadIdx.x / H::CPR;
#pragma unroll
    for (int c = 0; c < KINDS; ++c) chunk[c] = ((threadIdx.x % H::CPR) ^ H::key(row0 + c * STEP)) << 4;
  }
  // a, b: this head's elements of the tile's first row; as, bs: bytes between rows (< 2^24); last: the last row, from the first
  __device__ __forceinline__ void issue(const void* a, const void* b, int as, int bs, int last, unsigned lds) const {
#pragma unroll
    for (int c = 0; c < N; ++c) {
      // with fewer chunks than threads a thread's only one may be of either tile
      const bool second = N == 1 ? wbase >= HALF : c * NTH >= HALF;
      const int r = min((N == 1 && second ? row0 - ROWS : row0) + c * STEP % ROWS, last);
      stage16(second ? b : a, __umul24(r, second ? bs : as) + chunk[c % KINDS], lds + (wbase + c * NTH) * 16);
    }
  }
};

// A loaded value waited for here.  Else the compiler waits where it is used first, in
// the loop over tiles, and with counts that do not know of the staged loads: each tile
// would wait for the next one's.
template <typename F> __device__ __forceinline__ void settle(F& f) {
  if constexpr (sizeof(F) == 16) {
    u32x4 t = __builtin_bit_cast(u32x4, f);
    asm volatile("" : "+v"(t));
    f = __builtin_bit_cast(F, t);
  } else {
    asm volatile("" : "+v"(f));
  }
}

__device__ __forceinline__ float sum_quads(float v) {  // over lanes l, l ^ 16, l ^ 32, l ^ 48
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float max_quads(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_wave(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += shfl_xor(v, o);
  return v;
}

// What rounding to T takes from v.
template <typename T> __device__ __forceinline__ float lost(float v) { return v - to_f<T>(from_f<T>(v)); }
template <typename T> __device__ __forceinline__ f32x4 lost4(f32x4 v) {
  return f32x4{lost<T>(v[0]), lost<T>(v[1]), lost<T>(v[2]), lost<T>(v[3])};
}

// By the bits: a difference v - v may be fused with the product that v comes from.
__device__ __forceinline__ bool finite1(float v) { return (__float_as_uint(v) & 0x7FFFFFFFu) < 0x7F800000u; }
__device__ __forceinline__ bool finite4(f32x4 v) { return finite1(v[0]) && finite1(v[1]) && finite1(v[2]) && finite1(v[3]); }

// One row of a head over the wave: element e of lane l is dimension e * 64 + l.
template <typename T, int D> struct LaneRow {
  static constexpr int N = (D + kWave - 1) / kWave;
  float v[N];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int d = e * kWave + lane_id();
      v[e] = d < D ? to_f<T>(p[d]) : 0.f;
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = 0.f;
  }
  __device__ __forceinline__ void store(T* p, float f) const {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int d = e * kWave + lane_id();
      if (d < D) p[d] = from_f<T>(v[e] * f);
    }
  }
  __device__ __forceinline__ void store_lost(T* p, float f) const {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int d = e * kWave + lane_id();
      if (d < D) p[d] = from_f<T>(lost<T>(v[e] * f));
    }
  }
  __device__ __forceinline__ void add(float f, const LaneRow& o) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e * kWave + lane_id() < D) v[e] = fmaf(f, o.v[e], v[e]);
  }
  __device__ __forceinline__ float dot(const LaneRow& o) const {
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) t = fmaf(v[e], o.v[e], t);
    return sum_wave(t);
  }
  // every element is NaN: nothing that is added changes it
  __device__ __forceinline__ bool all_nan() const {
    bool all = true;
#pragma unroll
    for (int e = 0; e < N; ++e) all &= e * kWave + lane_id() >= D || v[e] != v[e];
    return __builtin_amdgcn_ballot_w64(!all) == 0;
  }
};

}  // namespace tlf
