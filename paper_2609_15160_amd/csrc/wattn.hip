// Causal attention of ragged rows with a sliding window and sinks, forward: the C
// entry points tlf_attn_ws_bytes and tlf_attn and their kernels.
//
//   s = scale q . k,  o = sum over the visible keys of exp(s - m) v / sum of exp(s - m)
//
// Scores, softmax statistics and sums are float32; the weights exp(s - m) are
// rounded to bf16 as operands of the product with bf16 values (each by 2^-8 of
// itself at most, which the sum over keys averages).  The sum that divides o is of the
// rounded weights, so that o stays a mean of values (error against 64 bits, causal
// over 300 keys with scores of variance 16: 0.0018, with the unrounded sum 0.0023); the
// lse, which the gradients' weights are of, has the sum before the rounding.
// What o loses where it is rounded is kept beside it for the gradients: their delta =
// do . o is subtracted from numbers that are nearly equal to it where few keys have
// most of the weight (gradients' error there 0.0025, from o alone 0.0033).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "tlf.h"
#include "wattn.h"

namespace tlf {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// The row again from the visible keys alone, for rows whose result is not finite:
// in a product of tiles a weight of zero times an infinite or NaN value of a key
// that the query does not see is NaN.  The row sees a key at least.
template <typename T, int D>
__device__ __forceinline__ void slow_row(const WAttnArgs& a, const WSeq& s, int h, int row) {
  const int kvh = h / (a.heads / a.kv_heads), p = row + s.n - s.nq;
  const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)s.k0 * a.ks + kvh * D;
  const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)s.k0 * a.vs + kvh * D;
  LaneRow<T, D> q, x, o;
  q.load(reinterpret_cast<const T*>(a.q) + (int64_t)(s.q0 + row) * a.qs + h * D);
  o.zero();
  const VisibleKeys keys(p, a.window, a.sinks);
  float m = -INFINITY, l = 0.f;
  for (int i = 0; i < keys.count; ++i) {
    x.load(k + (int64_t)keys[i] * a.ks);
    const float t = q.dot(x) * a.scale_log2;
    m = t != t ? t : fmaxf(m, t);
    if (t != t) break;
  }
  for (int i = 0; i < keys.count; ++i) {
    const int64_t j = keys[i];
    x.load(k + j * a.ks);
    const float w = __builtin_amdgcn_exp2f(q.dot(x) * a.scale_log2 - m);
    l += w;
    x.load(v + j * a.vs);
    o.add(w, x);
    if (o.all_nan()) break;
  }
  o.store(reinterpret_cast<T*>(a.out) + (int64_t)(s.q0 + row) * a.os + h * D, 1.f / l);
  if (a.low) o.store_lost(reinterpret_cast<T*>(a.low) + (int64_t)(s.q0 + row) * a.os + h * D, 1.f / l);
  if (a.lse && lane_id() == 0) a.lse[(int64_t)h * a.rows_q + s.q0 + row] = m + log2f(l);
}

// One workgroup: a tile of NW * 32 queries of one head, a wave 32 of them, over the
// visible tiles of BN keys, which all waves share from two places in LDS (one tile
// is used while the next arrives; one barrier a tile).  Tiles of 32 or of 128 keys,
// three places, eight waves and raised priorities around the products were all slower.
//
// 32 keys x 32 queries take 18 products at width 64 (288 clocks of a SIMD's matrix cores;
// 34 and 544 at 128) and 107 other vector instructions of 4 clocks, the 16 exponentials
// among them of 8.  At width 64 their issue bounds it: it takes 75% of the clocks that a
// compute unit has waves in, the matrix cores are busy 38%.  At 128 neither is full (48 and
// 41%): there are two waves on a SIMD, which spend 29% of their time in waits for memory,
// LDS and barriers and 30% waiting to issue.  8 x 4096 rows x 16 heads x 64, window 1024, 4
// sinks: 188-197 us, 640 TFLOP/s of the visible pairs; 4 x 4099 x 16 x 128: 278-284 us, 730
// TFLOP/s.
//
// The softmax base of a query is the largest score of the first tile that it sees a
// key of, or kLeast if that is less (its only key there may be one of little weight):
// weights are exp2(s - base) at once, without a maximum per tile.  Where a
// query's sum has grown past kSumMax the base moves up and the sums are scaled down,
// exactly, by a power of two; o / l does not depend on it.  Within a tile weights, or only
// their sums, may leave float32's range (scores some 120 above the base in base 2; sums of
// weights times small values stay in it), and sums less than kSumMin are of weights near
// its other end (scores of -112 and less, all of them): a row of which a sum or a result is
// not finite, or whose sum is less, is done again by slow_row.  The sum of the rounded
// weights is a product with ones.
template <typename T, int D>
__global__ __launch_bounds__(kTileWaves* kWave, (D == 64 && sizeof(T) == 2 ? 4 : kRoom<T, D>)) void k_wattn(WAttnArgs a) {
  using H = HeadRows<T, D>;
  using O = Opnd<T>;
  typedef typename O::frag Frag;
  constexpr int NW = kTileWaves, QN = 2, QW = 16 * QN, BM = NW * QW, BN = sizeof(T) == 2 ? 64 : 32;
  constexpr int KSTEPS = H::KSTEPS, DT = H::DT, NT = O::TILES;
  constexpr bool kRounds = sizeof(T) == 2;
  constexpr float kSumMax = 0x1p60f, kSumMin = 0x1p-80f, kLeast = -32.f;
  using Loader = PairLoader<T, D, BN, NW * kWave>;
  __shared__ __align__(1024) char lds[2 * Loader::BYTES];

  const int u = xcd_run(blockIdx.x, gridDim.x), h = u / a.slots, slot = u - h * a.slots;
  const int b = seq_of<BM>(a.q_off, a.rows_q, a.batch, slot);
  const WSeq s = load_seq(a, b);
  // a sequence's last tiles see the most keys and come first
  const int tile = (s.nq + BM - 1) / BM - 1 - (slot - slot_of<BM>(a.q_off, a.rows_q, b));
  if (tile < 0 || tile * BM >= s.nq) return;  // offsets that do not ascend may say either
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c16 = lane & 15, g = lane >> 4;
  const int kvh = h / (a.heads / a.kv_heads), off = s.n - s.nq;
  const int p0 = tile * BM + off, p1 = min(tile * BM + BM, s.nq) - 1 + off;  // positions of the tile
  const int r0 = tile * BM + wave * QW;                                      // the wave's first query
  const bool mine = r0 < s.nq;
  const int pw0 = min(r0, s.nq - 1) + off, pw1 = min(r0 + QW, s.nq) - 1 + off;

  int p[QN];
  Frag qf[QN][KSTEPS];
#pragma unroll
  for (int qn = 0; qn < QN; ++qn) {
    const int row = min(r0 + qn * 16 + c16, s.nq - 1);
    p[qn] = row + off;
    const T* src = reinterpret_cast<const T*>(a.q) + (int64_t)(s.q0 + row) * a.qs + h * D + g * H::EPC;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) qf[qn][ks] = *reinterpret_cast<const Frag*>(src + ks * 4 * H::EPC);
  }
#pragma unroll
  for (int qn = 0; qn < QN; ++qn)
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) settle(qf[qn][ks]);
  const unsigned at = H::direct(lane), att = H::transposed(lane);
  f32x4 o[DT][QN];
  float ls[QN], base[QN];  // this lane's part of the sum of weights; the base, -inf: none yet
  f32x4 lr[QN];            // the sum of the rounded weights, in each row
#pragma unroll
  for (int qn = 0; qn < QN; ++qn) {
    base[qn] = -INFINITY;
    ls[qn] = 0.f;
    lr[qn] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt][qn] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool started = false;

  // one operand's rows of keys, from k0 on, row t of the tile whose read addresses are ka (keys) and va (values)
  auto products = [&](int mask, int k0, int t, const unsigned (&ka)[KSTEPS], const unsigned (&va)[DT]) __attribute__((always_inline)) {
    f32x4 sc[QN][NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) sc[qn][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        const Frag kf = H::load(ka[ks], t + nt * 16);
#pragma unroll
        for (int qn = 0; qn < QN; ++qn) sc[qn][nt] = O::mma(kf, qf[qn][ks], sc[qn][nt]);
      }
    }
    if (mask == M_UPPER) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) {
        const int last = p[qn] - k0 - 4 * g;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[qn][nt][r] = last >= nt * 16 + r ? sc[qn][nt][r] : -INFINITY;
      }
    } else if (mask == M_LOWER) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) {
        const int before = p[qn] - k0 - 4 * g - a.window;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[qn][nt][r] = before < nt * 16 + r ? sc[qn][nt][r] : -INFINITY;
      }
    } else if (mask == M_ALL) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int x = k0 + nt * 16 + 4 * g + r, far = reach(x, a.window, a.sinks);
#pragma unroll
          for (int qn = 0; qn < QN; ++qn) sc[qn][nt][r] = sees(p[qn], x, far) ? sc[qn][nt][r] : -INFINITY;
        }
    }
    Frag vf[kAhead];
#pragma unroll
    for (int dt = 0; dt < kAhead && dt < DT; ++dt) vf[dt] = H::load_t(va[dt], t);
    pin();
    if (!started) {
      bool none = false;
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) {
        float mx = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[qn][nt][r]);
        mx = ceilf(max_quads(mx) * a.scale_log2);  // whole numbers: moving it is exact too
        if (base[qn] == -INFINITY && mx != -INFINITY) base[qn] = fmaxf(mx, kLeast);
        none |= base[qn] == -INFINITY;
      }
      started = __builtin_amdgcn_ballot_w64(none) == 0;
    }
#pragma unroll
    for (int qn = 0; qn < QN; ++qn) {
      const float from = started || base[qn] != -INFINITY ? base[qn] : 0.f;  // without a base all weights are 0
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[qn][nt][r] = __builtin_amdgcn_exp2f(fmaf(sc[qn][nt][r], a.scale_log2, -from));
          ls[qn] += sc[qn][nt][r];
        }
    }
    Frag pf[QN];
#pragma unroll
    for (int qn = 0; qn < QN; ++qn) {
      pf[qn] = O::pack(sc[qn]);
      if constexpr (kRounds) lr[qn] = O::mma(O::ones(), pf[qn], lr[qn]);
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) o[dt][qn] = O::mma(vf[dt % kAhead], pf[qn], o[dt][qn]);
      if (dt + kAhead < DT) vf[dt % kAhead] = H::load_t(va[dt + kAhead], t);
      pin();
    }
  };

  auto move_base = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int qn = 0; qn < QN; ++qn) {
      const float sum = sum_quads(ls[qn]);
      const int up = sum > 1.f && sum < INFINITY ? min((int)(__float_as_uint(sum) >> 23) - 127, 100) : 0;
      const float f = __uint_as_float((unsigned)(127 - up) << 23);  // 2^-up
      base[qn] += (float)up;
      ls[qn] *= f;
      lr[qn] *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt][qn] *= f;
    }
  };

  if (s.n > 0 && p1 >= 0) {
    Loader ld;
    ld.init();
    const int first = max(0, max(p0, 0) - a.window + 1) / BN, last = p1 / BN;
    const int sinks = min((min(a.sinks, s.n) + BN - 1) / BN, first), count = sinks + last - first + 1;
    const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)s.k0 * a.ks + kvh * D;
    const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)s.k0 * a.vs + kvh * D;
    const unsigned base = lds_offset(lds);
    const int clear0 = max(pw1, 0) - a.window + 1;  // keys from here on are in the window of all of the wave's queries
    const T *kp = k, *vp = v;  // of the tile that is issued next, and its rows up to the last
    int left = s.n - 1;
    auto issue = [&](int i) __attribute__((always_inline)) {
      if (i == sinks) {
        const int row = first * BN;
        kp = k + row * a.ks;
        vp = v + row * a.vs;
        left = s.n - 1 - row;
      }
      ld.issue(kp, vp, (int)(a.ks * sizeof(T)), (int)(a.vs * sizeof(T)), left, base + (i & 1) * Loader::BYTES);
      kp += BN * a.ks;
      vp += BN * a.vs;
      left -= BN;
    };
    issue(0);
    for (int i = 0; i < count; ++i) {
      wait_barrier<0>();
      if (i + 1 < count) issue(i + 1);
      if (!mine) continue;
      const unsigned kb = base + (i & 1) * Loader::BYTES;
      const int k0 = (i < sinks ? i : first + i - sinks) * BN;
      unsigned ka[KSTEPS], va[DT];
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) ka[ks] = H::step(kb + at, ks);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) va[dt] = H::tile(kb + BN * H::RB + att, dt);
#pragma unroll
      for (int t = 0; t < BN; t += H::ROWS) {
        const bool whole = k0 + t >= clear0 && k0 + t + H::ROWS - 1 <= pw0;
        const int mask = whole ? M_NONE : mask_of(pw0, pw1, k0 + t, k0 + t + H::ROWS - 1, a.window, a.sinks);
        if (mask >= 0) products(mask, k0 + t, t, ka, va);
      }
      if (__builtin_amdgcn_ballot_w64(ls[0] > kSumMax || ls[1] > kSumMax)) move_base();
    }
  }
  if (!mine) return;
#pragma unroll
  for (int qn = 0; qn < QN; ++qn) {
    const int row = r0 + qn * 16 + c16;
    const bool none = p[qn] < 0;  // sees no key: zeros, whatever its weights of zero were multiplied by
    const float sum = sum_quads(ls[qn]), inv = 1.f / (kRounds ? lr[qn][0] : sum);
    bool good = none || (sum >= kSumMin && finite1(sum) && finite1(lr[qn][0]));  // lr: zeros where nothing is rounded
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      o[dt][qn] = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[dt][qn] * inv;
      good &= finite4(o[dt][qn]);
    }
    uint64_t again = __builtin_amdgcn_ballot_w64(!good && row < s.nq);
    again |= again >> 32;
    again = (again | again >> 16) & 0xFFFF;
    if (row < s.nq && !(again >> c16 & 1)) {  // the four lanes of a row alike, which store_pair needs
      T* dst = reinterpret_cast<T*>(a.out) + (int64_t)(s.q0 + row) * a.os + h * D;
      if constexpr (DT >= 2) {
#pragma unroll
        for (int dt = 0; dt < DT; dt += 2) store_pair<T>(dst + dt * 16, o[dt][qn], o[dt + 1][qn], lane);
        if constexpr (kRounds) {
          T* low = reinterpret_cast<T*>(a.low) + (int64_t)(s.q0 + row) * a.os + h * D;
          if (a.low)
#pragma unroll
            for (int dt = 0; dt < DT; dt += 2) store_pair<T>(low + dt * 16, lost4<T>(o[dt][qn]), lost4<T>(o[dt + 1][qn]), lane);
        }
      } else {
        Vec4<T>::store(dst + g * 4, o[0][qn]);
      }
      if (a.lse && g == 0) a.lse[(int64_t)h * a.rows_q + s.q0 + row] = none ? INFINITY : base[qn] + log2f(sum);
    }
    for (; again; again &= again - 1) slow_row<T, D>(a, s, h, r0 + qn * 16 + __builtin_ctzll(again));
  }
}

// Few queries: a workgroup takes one query row and up to 16 of the heads that share
// its keys (the columns of the score products) over one of `splits` ranges of the
// visible keys, its four waves 32 keys each in turn, and adds the waves' sums in
// LDS.  Keys come straight from memory as operands, values through a wave's own LDS
// rows for the transposed read; both of the next turn are on their way while this
// one is used.  The base is the largest score itself, whose weight 1 is not rounded (error
// over 512 keys with scores of variance 16: 0.0018, with whole bases 0.0019; of variance
// 1 0.0023 and 0.0024).  Bound by HBM: every visible key and value is read once:
// 256 rows x 516 keys x 12 heads x 64 72 us, 5.6 TB/s (heads of a row on one XCD; in the
// order of the workgroups 73.3); 2 rows x 49 000 keys x 2 key heads x 128 21 us, 4.7 TB/s.
constexpr int kFewWaves = 4, kFewKeys = 32;
template <typename T, int D> struct FewPart {  // sums of one head over a range
  static constexpr int FLOATS = D + 4;         // o, then m, l, the row's visible keys, l of the rounded weights
};

template <typename T, int D>
__global__ __launch_bounds__(kFewWaves* kWave, (kRoom<T, D>)) void k_wattn_few(WAttnArgs a) {
  using H = HeadRows<T, D>;
  using O = Opnd<T>;
  typedef typename O::frag Frag;
  constexpr int KSTEPS = H::KSTEPS, DT = H::DT, VN = kFewKeys * H::CPR / kWave, NT = kFewKeys / 16;
  constexpr int SUMS = kFewWaves * 16 * (D + 3) * 4, ROWS = kFewWaves * kFewKeys * H::RB;
  __shared__ __align__(1024) char lds[SUMS > ROWS ? SUMS : ROWS];
  const int each = a.heads / a.kv_heads, chunks = (each + 15) / 16;
  const int lin = xcd_run(blockIdx.x, gridDim.x), split = lin % a.splits, unit = lin / a.splits;
  const int gc = unit % chunks, kvh = unit / chunks % a.kv_heads, row = unit / (chunks * a.kv_heads);
  const int h0 = kvh * each + gc * 16, cols = min(each - gc * 16, 16);

  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c16 = lane & 15, g = lane >> 4;
  Frag qf[KSTEPS];
  const T* q = reinterpret_cast<const T*>(a.q) + (int64_t)row * a.qs + (h0 + min(c16, cols - 1)) * D + g * H::EPC;
#pragma unroll
  for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = *reinterpret_cast<const Frag*>(q + ks * 4 * H::EPC);

  // The last sequence that begins at or before the row: with a row of each sequence it is
  // the row's own number, which is tried first (the search costs two trips to memory).
  WSeq s = load_seq(a, min(row, a.batch));
  if (s.q0 > row || row >= s.q0 + s.nq) {
    int b = 0;
    for (int hi = a.batch; hi > b;) {
      const int step = (hi - b + kWave - 1) / kWave, x = b + (lane + 1) * step;
      const bool before = x <= hi && a.q_off[min(x, hi)] <= row;
      b += __builtin_popcountll(__builtin_amdgcn_ballot_w64(before)) * step;
      hi = min(hi, b + step - 1);
    }
    s = load_seq(a, b);
  }
  const int p = row - s.q0 + s.n - s.nq;
  const VisibleKeys keys(p, a.window, a.sinks);
  const int nv = s.n > 0 && (unsigned)(row - s.q0) < (unsigned)s.nq ? keys.count : 0;
  const int per = ((nv + kFewKeys - 1) / kFewKeys + a.splits - 1) / a.splits * kFewKeys;
  const int xa = min(nv, split * per), xb = min(nv, xa + per);  // of the visible keys, sinks first

  const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)s.k0 * a.ks + kvh * D;
  const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)s.k0 * a.vs + kvh * D;
  char* mine = lds + wave * kFewKeys * H::RB;
  const unsigned att = lds_offset(mine) + H::transposed(lane);

  Frag kf[NT][KSTEPS];
  uint4 vf[VN];
  auto load = [&](int x) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const T* src = k + (int64_t)keys[min(x + 16 * t + c16, xb - 1)] * a.ks + g * H::EPC;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) kf[t][ks] = *reinterpret_cast<const Frag*>(src + ks * 4 * H::EPC);
    }
#pragma unroll
    for (int c = 0; c < VN; ++c) {
      const int e = c * kWave + lane;
      vf[c] = *reinterpret_cast<const uint4*>(v + (int64_t)keys[min(x + e / H::CPR, xb - 1)] * a.vs + e % H::CPR * H::EPC);
    }
  };
  f32x4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  f32x4 lr = f32x4{0.f, 0.f, 0.f, 0.f};  // of the rounded weights, in each row
  constexpr int TURN = kFewWaves * kFewKeys;
  int x = xa + wave * kFewKeys;
  if (x < xb) load(x);
  for (; x < xb; x += TURN) {
    f32x4 sc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) sc[t] = O::mma(kf[t][ks], qf[ks], sc[t]);
    }
#pragma unroll
    for (int c = 0; c < VN; ++c) {
      const int e = c * kWave + lane, r = e / H::CPR;
      uint4 w = vf[c];
      if (x + r >= xb) w = make_uint4(0, 0, 0, 0);  // not a key of this range
      *reinterpret_cast<uint4*>(mine + r * H::RB + (((e % H::CPR) ^ H::key(r)) << 4)) = w;
    }
    asm volatile("" ::: "memory");
    if (x + TURN < xb) load(x + TURN);
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (x + t * 16 + 4 * g + r >= xb) sc[t][r] = -INFINITY;
        mx = fmaxf(mx, sc[t][r]);
      }
    mx = fmaxf(m, max_quads(mx) * a.scale_log2);
    const float base = mx == -INFINITY ? 0.f : mx, alpha = __builtin_amdgcn_exp2f(m - base);
    m = mx;
    l *= alpha;
    lr *= alpha;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[t][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][r], a.scale_log2, -base));
        l += sc[t][r];
      }
#pragma unroll
    for (int t = 0; t < NT / O::TILES; ++t) {
      const Frag pf = O::pack(&sc[t * O::TILES]);
      if constexpr (sizeof(T) == 2) lr = O::mma(O::ones(), pf, lr);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = O::mma(H::load_t(H::tile(att, dt), t * H::ROWS), pf, o[dt]);
    }
    asm volatile("" ::: "memory");
  }
  l = sum_quads(l);
  __syncthreads();
  float* os = reinterpret_cast<float*>(lds);  // [wave][column][D], then [wave][column] of m, of l and of lr
  float *ms = os + kFewWaves * 16 * D, *ls = ms + kFewWaves * 16, *rs = ls + kFewWaves * 16;
  float* dst = os + (wave * 16 + c16) * D + 4 * g;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) Vec4<float>::store(dst + dt * 16, o[dt]);
  if (g == 0) {
    ms[wave * 16 + c16] = m;
    ls[wave * 16 + c16] = l;
    rs[wave * 16 + c16] = sizeof(T) == 2 ? lr[0] : l;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < cols * D; e += kFewWaves * kWave) {
    const int c = e / D, d = e % D;
    float top = -INFINITY, sum = 0.f, sumr = 0.f, t = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, ms[w * 16 + c]);
    const float base = top == -INFINITY ? 0.f : top;  // no key of the range, or none with a score
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(ms[w * 16 + c] - base);
      sum += f * ls[w * 16 + c];
      sumr += f * rs[w * 16 + c];
      t += f * os[(w * 16 + c) * D + d];
    }
    if (a.splits > 1) {
      float* part = a.part + ((int64_t)(row * (int64_t)a.heads + h0 + c) * a.splits + split) * FewPart<T, D>::FLOATS;
      part[d] = t;
      if (d == 0) {
        part[D] = top;
        part[D + 1] = sum;
        part[D + 2] = __uint_as_float((unsigned)nv);
        part[D + 3] = sumr;
      }
      continue;
    }
    // without a visible key zeros; visible keys of which none has a score are 0 / 0
    const float o = nv == 0 ? 0.f : t / sumr;
    reinterpret_cast<T*>(a.out)[(int64_t)row * a.os + (h0 + c) * D + d] = from_f<T>(o);
    if (a.low) reinterpret_cast<T*>(a.low)[(int64_t)row * a.os + (h0 + c) * D + d] = from_f<T>(lost<T>(o));
    if (a.lse && d == 0) a.lse[(int64_t)(h0 + c) * a.rows_q + row] = nv == 0 ? INFINITY : top + log2f(sum);
  }
}

// The ranges' sums of one row's head: a workgroup whose threads have four dimensions
// each, so that every D / 4 of them take a range, and the sums of those go through LDS
// in a fixed order (2 rows of 16 heads x 128, 128 ranges: 4 us, most of it the trips to
// memory; a wave each took 79 with 253).
constexpr int kJoinThreads = 512;
template <typename T, int D> __global__ __launch_bounds__(kJoinThreads) void k_wattn_join(WAttnArgs a) {
  constexpr int PER = D / 4, SETS = kJoinThreads / PER, F = FewPart<T, D>::FLOATS;
  __shared__ __align__(16) float sums[SETS][D + 4];
  __shared__ float tops[kJoinThreads / kWave];
  const int row = blockIdx.x / a.heads, h = blockIdx.x % a.heads, set = threadIdx.x / PER, d = threadIdx.x % PER * 4;
  const float* part = a.part + (int64_t)blockIdx.x * a.splits * F;
  float top = -INFINITY;
  for (int k = threadIdx.x; k < a.splits; k += kJoinThreads) top = fmaxf(top, part[(int64_t)k * F + D]);
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) top = fmaxf(top, shfl_xor(top, o));
  if (lane_id() == 0) tops[threadIdx.x / kWave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / kWave; ++w) top = fmaxf(top, tops[w]);
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f, sumr = 0.f;
  f32x4 t = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = set; k < a.splits; k += SETS) {
    const float* s = part + (int64_t)k * F;
    const float f = __builtin_amdgcn_exp2f(s[D] - base);
    sum += f * s[D + 1];
    sumr += f * s[D + 3];
    t += f * Vec4<float>::load(s + d);
  }
  Vec4<float>::store(&sums[set][d], t);
  if (d == 0) {
    sums[set][D] = sum;
    sums[set][D + 1] = sumr;
  }
  __syncthreads();
  if (threadIdx.x >= D) return;
  float all = 0.f, l = 0.f, lr = 0.f;
  for (int k = 0; k < SETS; ++k) {
    all += sums[k][threadIdx.x];
    l += sums[k][D];
    lr += sums[k][D + 1];
  }
  // whether the row has visible keys at all, as k_wattn_few found
  const bool none = __float_as_uint(part[D + 2]) == 0u;
  const float o = none ? 0.f : all / lr;
  reinterpret_cast<T*>(a.out)[(int64_t)row * a.os + h * D + threadIdx.x] = from_f<T>(o);
  if (a.low) reinterpret_cast<T*>(a.low)[(int64_t)row * a.os + h * D + threadIdx.x] = from_f<T>(lost<T>(o));
  if (a.lse && threadIdx.x == 0) a.lse[(int64_t)h * a.rows_q + row] = none ? INFINITY : top + log2f(l);
}

}  // namespace

int wattn_check(const tlf_attn_shape* t) {
  if (!t) return TLF_E_INVALID_ARG;
  if (t->dtype != TLF_DTYPE_F32 && t->dtype != TLF_DTYPE_BF16) return TLF_E_INVALID_ARG;
  if (t->batch < 0 || t->rows_q < 0 || t->rows_k < 0 || t->heads < 1 || t->kv_heads < 1 || t->head_dim < 1 || t->window < 0 ||
      t->sinks < 0 || t->heads % t->kv_heads != 0 || !(t->scale >= TLF_ATTN_MIN_SCALE) || !(t->scale <= TLF_ATTN_MAX_SCALE))
    return TLF_E_INVALID_ARG;
  const int64_t per = t->dtype == TLF_DTYPE_BF16 ? 8 : 4;  // elements of 16 bytes
  for (const int64_t v : {t->q_stride, t->k_stride, t->v_stride, t->o_stride})
    if (v < 0 || v % per != 0) return TLF_E_INVALID_ARG;
  const int64_t wide = (int64_t)t->heads * t->head_dim, kv_wide = (int64_t)t->kv_heads * t->head_dim;
  if (t->q_stride < wide || t->o_stride < wide || t->k_stride < kv_wide || t->v_stride < kv_wide) return TLF_E_INVALID_ARG;
  if (!t->d_q_offsets || !t->d_k_offsets) return TLF_E_INVALID_ARG;
  if (t->head_dim != 64 && t->head_dim != 128 && !(t->head_dim == 16 && t->dtype == TLF_DTYPE_F32)) return TLF_E_UNSUPPORTED;
  for (const int64_t v : {t->q_stride, t->k_stride, t->v_stride, t->o_stride})
    if (v > TLF_ATTN_MAX_STRIDE) return TLF_E_UNSUPPORTED;
  if (t->rows_q > TLF_ATTN_MAX_ROWS || t->rows_k > TLF_ATTN_MAX_ROWS ||
      t->heads > TLF_ATTN_MAX_HEADS || t->sinks > TLF_ATTN_MAX_SINKS || (int64_t)t->rows_q * t->heads > TLF_ATTN_MAX_UNITS ||
      (int64_t)t->rows_k * t->kv_heads > TLF_ATTN_MAX_UNITS || ((int64_t)t->batch + 1) * t->heads > TLF_ATTN_MAX_SEQ_HEADS)
    return TLF_E_UNSUPPORTED;
  return TLF_OK;
}

WAttnArgs wattn_args(const tlf_attn_shape& t) {
  WAttnArgs a{};
  a.q_off = t.d_q_offsets;
  a.k_off = t.d_k_offsets;
  a.k_len = t.d_k_lengths;
  a.qs = t.q_stride;
  a.ks = t.k_stride;
  a.vs = t.v_stride;
  a.os = t.o_stride;
  a.batch = t.batch;
  a.heads = t.heads;
  a.kv_heads = t.kv_heads;
  a.rows_q = t.rows_q;
  a.rows_k = t.rows_k;
  a.window = t.window > 0 ? t.window : INT32_MAX;
  a.sinks = t.window > 0 ? t.sinks : 0;
  a.scale = t.scale;
  a.scale_log2 = t.scale * kLog2e;
  return a;
}

namespace {

// One row for each sequence, or up to eight where the tile kernel would have fewer
// workgroups than there are compute units (12 x 64 heads, us of this kernel and the tile
// kernel: 256 sequences x 100 keys, 1 row each 17 and 22, 2 rows 30 and 23; 64 x 600, 1
// row 26 and 25, 2 rows 38 and 25; 8 x 3000, 2 rows 23 and 64, 8 rows 52 and 64).
bool is_few(const tlf_attn_shape& t) {
  if (t.rows_q <= t.batch) return true;
  return t.rows_q <= 8 * (int64_t)t.batch && (t.rows_q / 128 + (int64_t)t.batch + 1) * t.heads < 256;
}

// Ranges of the keys of a row, for two workgroups on a compute unit, and 256 keys of a
// workgroup at least (with the join, us with one, two and four on a compute unit: 2 rows
// x 65001 keys x 2 key heads x 128 28, 28 and 32; 8 x 4096 x 16 46, 47 and 49; 8 x 4096 x 4
// 19, 19 and 18; 4 x 1500 x 16 16, 17 and 17; 128 keys at least: 30, 47, 19 and 17).
int few_splits(const tlf_attn_shape& t) {
  const int each = t.heads / t.kv_heads;
  const int64_t units = std::max<int64_t>(1, (int64_t)t.rows_q * t.kv_heads * ((each + 15) / 16));
  int64_t keys = t.rows_k / std::max(1, t.batch);
  if (t.window > 0) keys = std::min<int64_t>(keys, (int64_t)t.window + t.sinks);
  return (int)std::max<int64_t>(1, std::min((512 + units - 1) / units, keys / 256));
}

template <typename T, int D> hipError_t launch(const tlf_attn_shape& t, WAttnArgs a, hipStream_t s) {
  if (is_few(t)) {
    a.splits = few_splits(t);
    const int each = t.heads / t.kv_heads;
    const dim3 grid((unsigned)((int64_t)t.rows_q * t.kv_heads * ((each + 15) / 16) * a.splits));
    hipLaunchKernelGGL((k_wattn_few<T, D>), grid, dim3(kFewWaves * kWave), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    hipLaunchKernelGGL((k_wattn_join<T, D>), dim3((unsigned)(t.rows_q * t.heads)), dim3(kJoinThreads), 0, s, a);
    return hipGetLastError();
  }
  a.slots = (int)slots_of<128>(t.rows_q, t.batch);
  hipLaunchKernelGGL((k_wattn<T, D>), dim3((unsigned)(a.slots * t.heads)), dim3(kTileWaves * kWave), 0, s, a);
  return hipGetLastError();
}

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_attn_ws_bytes(const tlf_attn_shape* shape, size_t* ws_bytes) {
  const int st = tlf::wattn_check(shape);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  const int splits = tlf::is_few(*shape) ? tlf::few_splits(*shape) : 1;
  *ws_bytes = splits > 1 ? (size_t)shape->rows_q * shape->heads * splits * (shape->head_dim + 4) * sizeof(float) : 0;
  return TLF_OK;
}

int tlf_attn(const tlf_attn_shape* shape, const void* d_q, const void* d_k, const void* d_v, void* d_o, float* d_lse,
             void* d_o_low, void* d_workspace, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int st = tlf_attn_ws_bytes(shape, &need);
  if (st != TLF_OK) return st;
  if (d_o_low && shape->dtype != TLF_DTYPE_BF16) return TLF_E_INVALID_ARG;
  if (shape->rows_q == 0) return TLF_OK;
  if (!d_q || !d_o || (shape->rows_k > 0 && (!d_k || !d_v)) || (need > 0 && (!d_workspace || ws_bytes < need)))
    return TLF_E_INVALID_ARG;
  for (const void* p : {d_q, d_k, d_v, (const void*)d_o, (const void*)d_o_low, (const void*)d_workspace})
    if (((uintptr_t)p & 15u) != 0) return TLF_E_INVALID_ARG;
  for (const void* p : {(const void*)d_lse, (const void*)shape->d_q_offsets, (const void*)shape->d_k_offsets, (const void*)shape->d_k_lengths})
    if (((uintptr_t)p & 3u) != 0) return TLF_E_INVALID_ARG;
  tlf::WAttnArgs a = tlf::wattn_args(*shape);
  a.q = d_q;
  a.k = d_k;
  a.v = d_v;
  a.out = d_o;
  a.lse = d_lse;
  a.low = d_o_low;
  a.part = (float*)d_workspace;
  const hipStream_t s = (hipStream_t)stream;
  const bool h = shape->dtype == TLF_DTYPE_BF16;
  const hipError_t e = shape->head_dim == 16    ? tlf::launch<float, 16>(*shape, a, s)
                       : shape->head_dim == 64  ? (h ? tlf::launch<bf16, 64>(*shape, a, s) : tlf::launch<float, 64>(*shape, a, s))
                                                : (h ? tlf::launch<bf16, 128>(*shape, a, s) : tlf::launch<float, 128>(*shape, a, s));
  return e == hipSuccess ? TLF_OK : TLF_E_HIP;
}

}  // extern "C"
