// Gradients of the causal attention of ragged rows with a sliding window and sinks:
// the C entry points tlf_attn_grad_ws_bytes and tlf_attn_grad and their kernels.
//
//   P = exp2(scale log2(e) q . k - lse),  dP = do . v,  delta = do . o
//   dS = P (dP - delta),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T do
//
// Two passes, each with its sums in registers and no atomics, so that results are
// the same from call to call: k_wattn_dq owns queries (three products, and delta),
// k_wattn_dkv owns keys (four products).  That the scores and dP are computed twice
// costs less than dS in memory would.  P and dS are rounded to bf16 as operands of
// the next products with bf16 tensors; all else is float32.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "tlf.h"
#include "wattn.h"

namespace tlf {

int wattn_check(const tlf_attn_shape* t);
WAttnArgs wattn_args(const tlf_attn_shape& t);

namespace {

struct GradArgs : WAttnArgs {
  int64_t dqs, dks, dvs;
  int sink_parts;  // ranges of the queries of a sequence's first key tile, where it has sinks, else 0
};

// One query's row again from its visible keys alone (slow_row of the forward pass says why).
template <typename T, int D>
__device__ __forceinline__ void slow_dq(const GradArgs& a, const WSeq& s, int h, int row) {
  const int kvh = h / (a.heads / a.kv_heads), p = row + s.n - s.nq;
  const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)s.k0 * a.ks + kvh * D;
  const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)s.k0 * a.vs + kvh * D;
  LaneRow<T, D> q, d, x, o;
  q.load(reinterpret_cast<const T*>(a.q) + (int64_t)(s.q0 + row) * a.qs + h * D);
  d.load(reinterpret_cast<const T*>(a.dout) + (int64_t)(s.q0 + row) * a.os + h * D);
  x.load(reinterpret_cast<const T*>(a.o) + (int64_t)(s.q0 + row) * a.os + h * D);
  float delta = d.dot(x);
  if (a.low) {
    x.load(reinterpret_cast<const T*>(a.low) + (int64_t)(s.q0 + row) * a.os + h * D);
    delta += d.dot(x);
  }
  const float lse = a.lse[(int64_t)h * a.rows_q + s.q0 + row];
  o.zero();
  const VisibleKeys keys(p, a.window, a.sinks);
  for (int i = 0; i < keys.count; ++i) {
    const int64_t j = keys[i];
    x.load(v + j * a.vs);
    const float dp = d.dot(x);
    x.load(k + j * a.ks);
    o.add(__builtin_amdgcn_exp2f(fmaf(q.dot(x), a.scale_log2, -lse)) * (dp - delta), x);
    if (o.all_nan()) break;
  }
  o.store(reinterpret_cast<T*>(a.dq) + (int64_t)(s.q0 + row) * a.dqs + h * D, a.scale);
}

// One key's rows again from the queries that see it.
template <typename T, int D>
__device__ __forceinline__ void slow_dkv(const GradArgs& a, const WSeq& s, int kvh, int key) {
  const int each = a.heads / a.kv_heads, off = s.n - s.nq;
  LaneRow<T, D> k, v, q, d, dk, dv;
  k.load(reinterpret_cast<const T*>(a.k) + (int64_t)(s.k0 + key) * a.ks + kvh * D);
  v.load(reinterpret_cast<const T*>(a.v) + (int64_t)(s.k0 + key) * a.vs + kvh * D);
  dk.zero();
  dv.zero();
  const int last = key < a.sinks || a.window > s.n - 1 - key ? s.n - 1 : key + a.window - 1;
  for (int h = kvh * each; h < (kvh + 1) * each; ++h)
    for (int j = max(0, key - off); j <= last - off && !(dk.all_nan() && dv.all_nan()); ++j) {
      const int64_t row = s.q0 + j;
      q.load(reinterpret_cast<const T*>(a.q) + row * a.qs + h * D);
      d.load(reinterpret_cast<const T*>(a.dout) + row * a.os + h * D);
      const float w = __builtin_amdgcn_exp2f(fmaf(q.dot(k), a.scale_log2, -a.lse[(int64_t)h * a.rows_q + row]));
      dv.add(w, d);
      dk.add(w * (d.dot(v) + a.ndelta[(int64_t)h * a.rows_q + row]), q);
    }
  dk.store(reinterpret_cast<T*>(a.dk) + (int64_t)(s.k0 + key) * a.dks + kvh * D, a.scale);
  dv.store(reinterpret_cast<T*>(a.dv) + (int64_t)(s.k0 + key) * a.dvs + kvh * D, 1.f);
}

// Tiles, waves and LDS as the forward kernel's (k_wattn).  q and do of the wave's 32
// queries stay in registers; a tile's keys are read as they lie and transposed, its
// values as they lie.  delta is of o with what its rounding took.  dP starts from -delta, so dS = P dP takes one product.
// Neither the issue of vector instructions (100 beside the 24 products of 32 keys x 32
// queries at width 64, the 48 at 128) nor the matrix cores are full: 62 and 42% of the clocks
// that a compute unit has waves in at 64, 42 and 49% at 128; waves spend a third of their
// time in waits and a third waiting to issue.  8 x 4096 x 16 x 64, window 1024: 230-236 us,
// 790 TFLOP/s of three products; 4 x 4099 x 16 x 128: 345-350 us, 880 TFLOP/s.
template <typename T, int D>
__global__ __launch_bounds__(kTileWaves* kWave, (kRoom<T, D>)) void k_wattn_dq(GradArgs a) {
  using H = HeadRows<T, D>;
  using O = Opnd<T>;
  typedef typename O::frag Frag;
  constexpr int NW = kTileWaves, QN = 2, QW = 16 * QN, BM = NW * QW, BN = sizeof(T) == 2 ? 64 : 32;
  constexpr int KSTEPS = H::KSTEPS, DT = H::DT, TL = O::TILES;
  using Loader = PairLoader<T, D, BN, NW * kWave>;
  __shared__ __align__(1024) char lds[2 * Loader::BYTES];

  const int u = xcd_run(blockIdx.x, gridDim.x), h = u / a.slots, slot = u - h * a.slots;
  const int b = seq_of<BM>(a.q_off, a.rows_q, a.batch, slot);
  const WSeq s = load_seq(a, b);
  const int tile = (s.nq + BM - 1) / BM - 1 - (slot - slot_of<BM>(a.q_off, a.rows_q, b));
  if (tile < 0 || tile * BM >= s.nq) return;  // offsets that do not ascend may say either
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c16 = lane & 15, g = lane >> 4;
  const int kvh = h / (a.heads / a.kv_heads), off = s.n - s.nq;
  const int p0 = tile * BM + off, p1 = min(tile * BM + BM, s.nq) - 1 + off;
  const int r0 = tile * BM + wave * QW;
  const bool mine = r0 < s.nq;
  const int pw0 = min(r0, s.nq - 1) + off, pw1 = min(r0 + QW, s.nq) - 1 + off;

  int p[QN];
  Frag qf[QN][KSTEPS], df[QN][KSTEPS];
  float lse[QN], delta[QN];
#pragma unroll
  for (int qn = 0; qn < QN; ++qn) {
    const int row = min(r0 + qn * 16 + c16, s.nq - 1);
    p[qn] = row + off;
    const int64_t at = s.q0 + row, wide = (int64_t)h * D + g * H::EPC;
    const T* q = reinterpret_cast<const T*>(a.q) + at * a.qs + wide;
    const T* d = reinterpret_cast<const T*>(a.dout) + at * a.os + wide;
    const T* o = reinterpret_cast<const T*>(a.o) + at * a.os + wide;
    const T* low = reinterpret_cast<const T*>(a.low ? a.low : a.o) + at * a.os + wide;
    float t = 0.f, tl = 0.f;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      qf[qn][ks] = *reinterpret_cast<const Frag*>(q + ks * 4 * H::EPC);
      df[qn][ks] = *reinterpret_cast<const Frag*>(d + ks * 4 * H::EPC);
      const Frag of = *reinterpret_cast<const Frag*>(o + ks * 4 * H::EPC);
#pragma unroll
      for (int e = 0; e < H::EPC; ++e) t = fmaf((float)df[qn][ks][e], (float)of[e], t);
      if constexpr (sizeof(T) == 2) {  // read in any case: behind a branch it would be one more trip to memory
        const Frag lf = *reinterpret_cast<const Frag*>(low + ks * 4 * H::EPC);
#pragma unroll
        for (int e = 0; e < H::EPC; ++e) tl = fmaf((float)df[qn][ks][e], (float)lf[e], tl);
      }
    }
    delta[qn] = sum_quads(a.low ? t + tl : t);
    lse[qn] = a.lse[(int64_t)h * a.rows_q + at];
    if (g == 0 && r0 + qn * 16 + c16 < s.nq) {  // for k_wattn_dkv, whose products start from them
      a.ndelta[(int64_t)h * a.rows_q + at] = -delta[qn];
      a.nlse[(int64_t)h * a.rows_q + at] = -lse[qn] / a.scale_log2;
    }
  }
#pragma unroll
  for (int qn = 0; qn < QN; ++qn) {
    settle(lse[qn]);
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      settle(qf[qn][ks]);
      settle(df[qn][ks]);
    }
  }
  const unsigned at = H::direct(lane), att = H::transposed(lane);
  f32x4 dq[DT][QN];
#pragma unroll
  for (int qn = 0; qn < QN; ++qn)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dq[dt][qn] = f32x4{0.f, 0.f, 0.f, 0.f};

  // one operand's rows of keys, from k0 on, row t of the tile whose read addresses are ka (keys; values BN rows
  // further) and ta (keys transposed)
  auto products = [&](int mask, int k0, int t, const unsigned (&ka)[KSTEPS], const unsigned (&ta)[DT]) __attribute__((always_inline)) {
    f32x4 sc[QN][TL], dp[QN][TL];
#pragma unroll
    for (int n = 0; n < TL; ++n) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) {
        sc[qn][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        dp[qn][n] = f32x4{-delta[qn], -delta[qn], -delta[qn], -delta[qn]};
      }
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        const Frag kf = H::load(ka[ks], t + n * 16), vf = H::load(ka[ks], BN + t + n * 16);
#pragma unroll
        for (int qn = 0; qn < QN; ++qn) {
          sc[qn][n] = O::mma(kf, qf[qn][ks], sc[qn][n]);
          dp[qn][n] = O::mma(vf, df[qn][ks], dp[qn][n]);
        }
      }
    }
    Frag tk[kAhead];
#pragma unroll
    for (int dt = 0; dt < kAhead && dt < DT; ++dt) tk[dt] = H::load_t(ta[dt], t);
    pin();
    // scores that are not visible are -inf: their weights and their dS are 0
    if (mask == M_UPPER) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) {
        const int last = p[qn] - k0 - 4 * g;
#pragma unroll
        for (int n = 0; n < TL; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[qn][n][r] = last >= n * 16 + r ? sc[qn][n][r] : -INFINITY;
      }
    } else if (mask == M_LOWER) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) {
        const int before = p[qn] - k0 - 4 * g - a.window;
#pragma unroll
        for (int n = 0; n < TL; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[qn][n][r] = before < n * 16 + r ? sc[qn][n][r] : -INFINITY;
      }
    } else if (mask == M_ALL) {
#pragma unroll
      for (int n = 0; n < TL; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int x = k0 + n * 16 + 4 * g + r, far = reach(x, a.window, a.sinks);
#pragma unroll
          for (int qn = 0; qn < QN; ++qn) sc[qn][n][r] = sees(p[qn], x, far) ? sc[qn][n][r] : -INFINITY;
        }
    }
    Frag pf[QN];
#pragma unroll
    for (int qn = 0; qn < QN; ++qn) {
#pragma unroll
      for (int n = 0; n < TL; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) dp[qn][n][r] *= __builtin_amdgcn_exp2f(fmaf(sc[qn][n][r], a.scale_log2, -lse[qn]));
      pf[qn] = O::pack(dp[qn]);
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int qn = 0; qn < QN; ++qn) dq[dt][qn] = O::mma(tk[dt % kAhead], pf[qn], dq[dt][qn]);
      if (dt + kAhead < DT) tk[dt % kAhead] = H::load_t(ta[dt + kAhead], t);
      pin();
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
      unsigned ka[KSTEPS], ta[DT];
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) ka[ks] = H::step(kb + at, ks);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) ta[dt] = H::tile(kb + att, dt);
#pragma unroll
      for (int t = 0; t < BN; t += H::ROWS) {
        const bool whole = k0 + t >= clear0 && k0 + t + H::ROWS - 1 <= pw0;
        const int mask = whole ? M_NONE : mask_of(pw0, pw1, k0 + t, k0 + t + H::ROWS - 1, a.window, a.sinks);
        if (mask >= 0) products(mask, k0 + t, t, ka, ta);
      }
    }
  }
  if (!mine) return;
#pragma unroll
  for (int qn = 0; qn < QN; ++qn) {
    const int row = r0 + qn * 16 + c16;
    bool good = true;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      dq[dt][qn] = p[qn] < 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : dq[dt][qn] * a.scale;  // sees no key: zeros
      good &= finite4(dq[dt][qn]);
    }
    uint64_t again = __builtin_amdgcn_ballot_w64(!good && row < s.nq);
    again |= again >> 32;
    again = (again | again >> 16) & 0xFFFF;
    if (row < s.nq && !(again >> c16 & 1)) {
      T* dst = reinterpret_cast<T*>(a.dq) + (int64_t)(s.q0 + row) * a.dqs + h * D;
      if constexpr (DT >= 2) {
#pragma unroll
        for (int dt = 0; dt < DT; dt += 2) store_pair<T>(dst + dt * 16, dq[dt][qn], dq[dt + 1][qn], lane);
      } else {
        Vec4<T>::store(dst + g * 4, dq[0][qn]);
      }
    }
    for (; again; again &= again - 1) slow_dq<T, D>(a, s, h, r0 + qn * 16 + __builtin_ctzll(again));
  }
}

// Tiles of 16 keys that a wave's registers hold the sums of.
template <typename T, int D> constexpr int key_tiles() { return sizeof(T) == 4 && D == 128 ? 1 : 2; }

// One workgroup: a tile of NW * KN * 16 keys of one key head, whose rows stay in
// registers (each wave KN tiles of 16; the values of 128-wide bf16 heads in LDS), over tiles of BQ queries of every head that
// shares them; q and do, with their lse and delta, which the products of the scores and of dP
// start from, come through two places in LDS.
// A tile's keys are seen by the queries from its first position to the window's end
// behind its last; sinks by all from there: where a first tile has sinks, its queries
// go in `sink_parts` ranges to workgroups of their own, whose sums k_wattn_sinks adds.
// Bound by latency: vector instructions (111 beside the 32 products of 32 keys x 32 queries
// at width 64, 121 beside 64 at 128) take 53 and 38% of the clocks that a compute unit has
// waves in, the matrix cores 43 and 48%; q and do are read twice from LDS, as they lie and
// transposed right before their products, and waves spend 39 and 33% of their time in waits.
// 8 x 4096 x 16 x 64, window 1024: 302-310 us, 780 TFLOP/s of four products; 4 x 4099 x 16 x
// 128: 457-478 us, 860.  Width 64 with two waves on a SIMD and operands read ahead, and tiles of 128
// queries, were slower.
template <typename T, int D>
__global__ __launch_bounds__(kTileWaves* kWave, (sizeof(T) == 4 ? kRoom<T, D> : D == 64 ? 3 : 2)) void k_wattn_dkv(GradArgs a) {
  using H = HeadRows<T, D>;
  using O = Opnd<T>;
  typedef typename O::frag Frag;
  constexpr int NW = kTileWaves, KN = key_tiles<T, D>(), KW = 16 * KN, KT = NW * KW, BQ = sizeof(T) == 2 && D == 64 ? 64 : 32;
  constexpr int KSTEPS = H::KSTEPS, DT = H::DT, TL = O::TILES;
  using Loader = PairLoader<T, D, BQ, NW * kWave>;
  __shared__ __align__(1024) char lds[2 * Loader::BYTES];
  constexpr bool VLDS = sizeof(T) == 2 && D == 128;  // the values' rows in LDS, each wave's own: with them in registers a
                                                      // wave has 16 keys and reads q and do twice as often
  __shared__ __align__(1024) char vrows[VLDS ? KT * H::RB : 16];
  __shared__ __align__(16) float stats[2][2][kWave];  // of each place: nlse, ndelta

  const int sink_blocks = a.batch * a.kv_heads * a.sink_parts;  // sink_parts = 0: first tiles are as others
  int b, kvh, tile, part = 0, parts = 1;
  WSeq s;
  if ((int)blockIdx.x < sink_blocks) {  // the longest first
    part = blockIdx.x % a.sink_parts;
    parts = a.sink_parts;
    kvh = blockIdx.x / a.sink_parts % a.kv_heads;
    b = blockIdx.x / (a.sink_parts * a.kv_heads);
    s = load_seq(a, b);
    tile = 0;
    if (s.n == 0) return;
  } else {
    const int u = xcd_run(blockIdx.x - sink_blocks, gridDim.x - sink_blocks), slot = u % a.slots;
    kvh = u / a.slots;
    b = seq_of<KT>(a.k_off, a.rows_k, a.batch, slot);
    s = load_seq(a, b);
    tile = slot - slot_of<KT>(a.k_off, a.rows_k, b);
    if (tile < 0 || tile * KT >= s.cap || (tile == 0 && sink_blocks > 0 && s.n > 0)) return;
  }
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c16 = lane & 15, g = lane >> 4;
  const int each = a.heads / a.kv_heads, off = s.n - s.nq;
  const int k0 = tile * KT, k1 = min(k0 + KT, s.n) - 1;     // keys of the tile
  const int w0 = k0 + wave * KW, w1 = min(w0 + KW, s.n) - 1;  // of the wave

  Frag kf[KN][KSTEPS], vf[VLDS ? 1 : KN][VLDS ? 1 : KSTEPS];
  const unsigned at = H::direct(lane), att = H::transposed(lane);
  f32x4 dk[DT][KN], dv[DT][KN];
#pragma unroll
  for (int kn = 0; kn < KN; ++kn)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[dt][kn] = dv[dt][kn] = f32x4{0.f, 0.f, 0.f, 0.f};

  // queries [j0, j1] see a key of the tile
  const int last = k0 < a.sinks || a.window > s.n - 1 - k1 ? s.n - 1 : k1 + a.window - 1;
  const int j0 = max(0, k0 - off), j1 = last - off;
  const unsigned va = lds_offset(vrows) + wave * KW * H::RB + at;
  // one operand's rows of queries, from row j on, with read addresses qa and ta (transposed); their do lies BQ rows further
  auto products = [&](int mask, int j, unsigned qa, unsigned ta, const float* stat) __attribute__((always_inline)) {
    f32x4 sc[KN][TL], dp[KN][TL];
#pragma unroll
    for (int n = 0; n < TL; ++n) {
      const f32x4 nlse = Vec4<float>::load(stat + n * 16 + 4 * g), ndelta = Vec4<float>::load(stat + kWave + n * 16 + 4 * g);
#pragma unroll
      for (int kn = 0; kn < KN; ++kn) {
        sc[kn][n] = nlse;
        dp[kn][n] = ndelta;
      }
    }
    if constexpr (VLDS) {
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        Frag v[KN];
#pragma unroll
        for (int kn = 0; kn < KN; ++kn) v[kn] = H::load(H::step(va, ks), kn * 16);
#pragma unroll
        for (int n = 0; n < TL; ++n) {
          const Frag qf = H::load(H::step(qa, ks), n * 16), df = H::load(H::step(qa, ks), BQ + n * 16);
#pragma unroll
          for (int kn = 0; kn < KN; ++kn) {
            sc[kn][n] = O::mma(qf, kf[kn][ks], sc[kn][n]);
            dp[kn][n] = O::mma(df, v[kn], dp[kn][n]);
          }
        }
      }
    } else {
#pragma unroll
      for (int n = 0; n < TL; ++n)
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
          const Frag qf = H::load(H::step(qa, ks), n * 16), df = H::load(H::step(qa, ks), BQ + n * 16);
#pragma unroll
          for (int kn = 0; kn < KN; ++kn) {
            sc[kn][n] = O::mma(qf, kf[kn][ks], sc[kn][n]);
            dp[kn][n] = O::mma(df, vf[kn][ks], dp[kn][n]);
          }
        }
    }
    // scores that are not visible are -inf: their weights and their dS are 0
    if (mask == M_UPPER) {
#pragma unroll
      for (int kn = 0; kn < KN; ++kn) {
        const int first = w0 + kn * 16 + c16 - off - j - 4 * g;
#pragma unroll
        for (int n = 0; n < TL; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[kn][n][r] = first <= n * 16 + r ? sc[kn][n][r] : -INFINITY;
      }
    } else if (mask == M_LOWER) {
#pragma unroll
      for (int kn = 0; kn < KN; ++kn) {
        const int x = w0 + kn * 16 + c16, end = (a.window > s.n - 1 - x ? j1 : min(x + a.window - 1 - off, j1)) - j - 4 * g;
#pragma unroll
        for (int n = 0; n < TL; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[kn][n][r] = end >= n * 16 + r ? sc[kn][n][r] : -INFINITY;
      }
    } else if (mask == M_ALL) {
#pragma unroll
      for (int n = 0; n < TL; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // a row behind the last query stands before every key
          const int q = j + n * 16 + 4 * g + r, at_q = q > j1 ? INT32_MIN / 2 : q + off;
#pragma unroll
          for (int kn = 0; kn < KN; ++kn) {
            const int x = w0 + kn * 16 + c16;
            sc[kn][n][r] = sees(at_q, x, reach(x, a.window, a.sinks)) ? sc[kn][n][r] : -INFINITY;
          }
        }
    }
    Frag pf[KN], sf[KN];
#pragma unroll
    for (int kn = 0; kn < KN; ++kn) {
#pragma unroll
      for (int n = 0; n < TL; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[kn][n][r] = __builtin_amdgcn_exp2f(sc[kn][n][r] * a.scale_log2);
          dp[kn][n][r] *= sc[kn][n][r];
        }
      pf[kn] = O::pack(sc[kn]);
      sf[kn] = O::pack(dp[kn]);
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const Frag df = H::load_t(H::tile(ta, dt), BQ), qf = H::load_t(H::tile(ta, dt), 0);
#pragma unroll
      for (int kn = 0; kn < KN; ++kn) {
        dv[dt][kn] = O::mma(df, pf[kn], dv[dt][kn]);
        dk[dt][kn] = O::mma(qf, sf[kn], dk[dt][kn]);
      }
    }
  };
  if (k0 < s.n && j0 <= j1) {
#pragma unroll
    for (int kn = 0; kn < KN; ++kn) {
      const int64_t row = s.k0 + min(w0 + kn * 16 + c16, s.n - 1);
      const T* k = reinterpret_cast<const T*>(a.k) + row * a.ks + kvh * D + g * H::EPC;
      const T* v = reinterpret_cast<const T*>(a.v) + row * a.vs + kvh * D + g * H::EPC;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        kf[kn][ks] = *reinterpret_cast<const Frag*>(k + ks * 4 * H::EPC);
        const Frag f = *reinterpret_cast<const Frag*>(v + ks * 4 * H::EPC);
        if constexpr (VLDS) *reinterpret_cast<Frag*>(vrows + wave * KW * H::RB + H::step(H::direct(lane), ks) + kn * 16 * H::RB) = f;
        else vf[kn][ks] = f;
      }
    }
#pragma unroll
    for (int kn = 0; kn < KN; ++kn)
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        settle(kf[kn][ks]);
        if constexpr (!VLDS) settle(vf[kn][ks]);
      }
    Loader ld;
    ld.init();
    const int tiles = (j1 - j0 + BQ) / BQ, all = tiles * each;
    const int begin = (int)((int64_t)all * part / parts), end = (int)((int64_t)all * (part + 1) / parts);
    const unsigned base = lds_offset(lds), sbase = lds_offset(stats);
    // the tile that is issued next: of head ih of the group, its first row, where it lies
    int ih = begin / tiles, ij = j0 + begin % tiles * BQ;
    const T *qp, *dp;
    const float *lp, *ep;
    auto at_row = [&]() __attribute__((always_inline)) {
      const int h = kvh * each + ih;
      const int64_t row = s.q0 + ij, stat = (int64_t)h * a.rows_q + row;
      qp = reinterpret_cast<const T*>(a.q) + row * a.qs + h * D;
      dp = reinterpret_cast<const T*>(a.dout) + row * a.os + h * D;
      lp = a.nlse + stat;
      ep = a.ndelta + stat;
    };
    at_row();
    auto issue = [&](int place) __attribute__((always_inline)) {
      const int most = s.nq - 1 - ij;
      ld.issue(qp, dp, (int)(a.qs * sizeof(T)), (int)(a.os * sizeof(T)), most, base + place * Loader::BYTES);
      // 64 values each, of which the tile uses the first BQ
      const unsigned to = sbase + place * (unsigned)sizeof(stats[0]), lane4 = (unsigned)min(lane, most) * 4u;
      if (wave == 0) stage4(lp, lane4, to);
      if (wave == 1) stage4(ep, lane4, to + (unsigned)sizeof(stats[0][0]));
      ij += BQ;
      if (ij <= j1) {
        qp += BQ * a.qs;
        dp += BQ * a.os;
        lp += BQ;
        ep += BQ;
      } else {
        ij = j0;
        ++ih;
        at_row();
      }
    };
    if (begin < end) issue(0);
    // queries that see all of the wave's keys
    const int clear0 = w1 - off, clear1 = w1 < a.sinks || a.window > s.n - 1 - w0 ? j1 : min(j1, w0 + a.window - 1 - off);
    int ut = begin % tiles;  // tile that is used next
    for (int i = begin; i < end; ++i) {
      const int place = (i - begin) & 1;
      wait_barrier<0>();
      if (i + 1 < end) issue(place ^ 1);
      const int j = j0 + ut * BQ;
      if (++ut == tiles) ut = 0;
      if (w0 > w1) continue;
      const unsigned qb = base + place * Loader::BYTES;
#pragma unroll 1
      for (int t = 0; t < BQ; t += H::ROWS) {
        const int ja = j + t, jl = min(ja + H::ROWS - 1, j1);
        if (ja > j1) break;
        int mask = M_NONE;
        if (ja < clear0 || ja + H::ROWS - 1 > clear1) {
          mask = mask_of(ja + off, jl + off, w0, w1, a.window, a.sinks);
          if (jl < ja + H::ROWS - 1 && mask >= 0) mask = (mask & M_UPPER) || w0 < a.sinks ? M_ALL : M_LOWER;  // rows behind j1
        }
        if (mask >= 0) products(mask, ja, qb + t * H::RB + at, qb + t * H::RB + att, &stats[place][0][t]);
      }
    }
  }
  if (parts > 1) {  // [batch][key head][part][key][dk, dv]
    float* dst = a.part + ((int64_t)(b * a.kv_heads + kvh) * parts + part) * KT * 2 * D;
#pragma unroll
    for (int kn = 0; kn < KN; ++kn) {
      float* row = dst + (wave * KW + kn * 16 + c16) * 2 * D + 4 * g;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        Vec4<float>::store(row + dt * 16, dk[dt][kn]);
        Vec4<float>::store(row + D + dt * 16, dv[dt][kn]);
      }
    }
    return;
  }
#pragma unroll
  for (int kn = 0; kn < KN; ++kn) {
    const int key = w0 + kn * 16 + c16;  // from n to cap: room without keys, zeros
    bool good = true;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      if (key >= s.n) dk[dt][kn] = dv[dt][kn] = f32x4{0.f, 0.f, 0.f, 0.f};
      dk[dt][kn] *= a.scale;
      good &= finite4(dk[dt][kn]) && finite4(dv[dt][kn]);
    }
    uint64_t again = __builtin_amdgcn_ballot_w64(!good);
    again |= again >> 32;
    again = (again | again >> 16) & 0xFFFF;
    if (key < s.cap && !(again >> c16 & 1)) {
      T* dkp = reinterpret_cast<T*>(a.dk) + (int64_t)(s.k0 + key) * a.dks + kvh * D;
      T* dvp = reinterpret_cast<T*>(a.dv) + (int64_t)(s.k0 + key) * a.dvs + kvh * D;
      if constexpr (DT >= 2) {
#pragma unroll
        for (int dt = 0; dt < DT; dt += 2) {
          store_pair<T>(dkp + dt * 16, dk[dt][kn], dk[dt + 1][kn], lane);
          store_pair<T>(dvp + dt * 16, dv[dt][kn], dv[dt + 1][kn], lane);
        }
      } else {
        Vec4<T>::store(dkp + g * 4, dk[0][kn]);
        Vec4<T>::store(dvp + g * 4, dv[0][kn]);
      }
    }
    for (; again; again &= again - 1) slow_dkv<T, D>(a, s, kvh, w0 + kn * 16 + __builtin_ctzll(again));
  }
}

// The first tiles' sums over the ranges of their queries: a wave has four keys, whose
// loads it has on their way together (in turn they took four times as long).
constexpr int kSinkKeys = 16;  // of a workgroup
template <typename T, int D, int KT> __global__ __launch_bounds__(256) void k_wattn_sinks(GradArgs a) {
  constexpr int N = (2 * D + kWave - 1) / kWave, BLOCKS = KT / kSinkKeys, KEYS = kSinkKeys / 4;
  const int unit = blockIdx.x / BLOCKS, b = unit / a.kv_heads, kvh = unit % a.kv_heads, lane = lane_id();
  const WSeq s = load_seq(a, b);
  if (s.n == 0) return;  // the tile's own workgroup has written its zeros
  const int key0 = blockIdx.x % BLOCKS * kSinkKeys + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * KEYS;
  const float* src = a.part + ((int64_t)unit * a.sink_parts * KT + key0) * 2 * D + min(lane, 2 * D - 1);
  float t[KEYS][N];
#pragma unroll
  for (int i = 0; i < KEYS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) t[i][e] = 0.f;
#pragma unroll 2
  for (int k = 0; k < a.sink_parts; ++k, src += (int64_t)KT * 2 * D)
#pragma unroll
    for (int i = 0; i < KEYS; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) t[i][e] += src[i * 2 * D + e * kWave];
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    const int key = key0 + i;
    if (key >= s.cap) return;
    T* dk = reinterpret_cast<T*>(a.dk) + (int64_t)(s.k0 + key) * a.dks + kvh * D;
    T* dv = reinterpret_cast<T*>(a.dv) + (int64_t)(s.k0 + key) * a.dvs + kvh * D;
    bool good = true;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (key >= s.n) t[i][e] = 0.f;  // room without keys
      if (e * kWave + lane < D) t[i][e] *= a.scale;
      good &= finite1(t[i][e]);
    }
    if (__builtin_amdgcn_ballot_w64(!good)) {
      slow_dkv<T, D>(a, s, kvh, key);
      continue;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int d = e * kWave + lane;
      if (d < D) dk[d] = from_f<T>(t[i][e]);
      else if (d < 2 * D) dv[d - D] = from_f<T>(t[i][e]);
    }
  }
}

// Ranges of a first tile's queries; 0: there are no sinks.  Its workgroup, which all
// queries of the sequence go through, is started first: it is split where even so it
// would outlast the others, each of which sees the window's queries, on 256 compute
// units with three workgroups each, and into ranges no shorter than theirs (dk and dv
// with the join, us without ranges and with them, 12 x 64 heads, 4 sinks: 8 x 4096 rows,
// window 256 149 and 119 (2 ranges), window 64 149 and 97 (4); 1 x 32768, window 1024
// 1021 and 259 (7); twice as many 125, 101 and 260; 32 x 2048, window 128, which stays
// whole, 172 and in 4 ranges 199).
int sink_parts(const tlf_attn_shape& t) {
  if (t.window <= 0 || t.sinks <= 0 || t.batch <= 0) return 0;
  const int64_t rows = t.rows_q / t.batch, other = std::min<int64_t>((int64_t)t.window + 128, rows);
  const int64_t all = (rows / 128 * other + rows) * t.batch * t.heads, share = std::max<int64_t>({1, other, all / 768});
  return (int)std::max<int64_t>(1, std::min<int64_t>(16, rows * (t.heads / t.kv_heads) / share));
}

int64_t stat_floats(const tlf_attn_shape& t) { return ((int64_t)t.heads * t.rows_q + 3) / 4 * 4; }
int64_t part_floats(const tlf_attn_shape& t) {
  const int parts = sink_parts(t);
  return parts > 1 ? (int64_t)t.batch * t.kv_heads * parts * 128 * 2 * t.head_dim : 0;
}

template <typename T, int D> hipError_t launch(const tlf_attn_shape& t, GradArgs a, hipStream_t s) {
  if (t.rows_q > 0) {
    a.slots = (int)slots_of<128>(t.rows_q, t.batch);
    hipLaunchKernelGGL((k_wattn_dq<T, D>), dim3((unsigned)(a.slots * t.heads)), dim3(kTileWaves * kWave), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (t.rows_k == 0) return hipSuccess;
  constexpr int KT = kTileWaves * key_tiles<T, D>() * 16;
  static_assert(KT >= TLF_ATTN_MAX_SINKS, "sinks lie in a sequence's first tile");
  a.slots = (int)slots_of<KT>(t.rows_k, t.batch);
  a.sink_parts = sink_parts(t);
  const int64_t blocks = ((int64_t)a.slots + (int64_t)a.batch * a.sink_parts) * a.kv_heads;
  hipLaunchKernelGGL((k_wattn_dkv<T, D>), dim3((unsigned)blocks), dim3(kTileWaves * kWave), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.sink_parts <= 1) return e;
  hipLaunchKernelGGL((k_wattn_sinks<T, D, KT>), dim3((unsigned)((int64_t)a.batch * a.kv_heads * (KT / kSinkKeys))), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

}  // namespace tlf

extern "C" {

int tlf_attn_grad_ws_bytes(const tlf_attn_shape* shape, size_t* ws_bytes) {
  const int st = tlf::wattn_check(shape);
  if (st != TLF_OK || !ws_bytes) return st != TLF_OK ? st : TLF_E_INVALID_ARG;
  *ws_bytes = (size_t)(2 * tlf::stat_floats(*shape) + tlf::part_floats(*shape)) * sizeof(float);
  return TLF_OK;
}

int tlf_attn_grad(const tlf_attn_shape* shape, const void* d_do, const void* d_q, const void* d_k, const void* d_v,
                  const void* d_o, const float* d_lse, const void* d_o_low, void* d_dq, int64_t dq_stride, void* d_dk,
                  int64_t dk_stride, void* d_dv, int64_t dv_stride, void* d_workspace, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int st = tlf_attn_grad_ws_bytes(shape, &need);
  if (st != TLF_OK) return st;
  const int64_t per = shape->dtype == TLF_DTYPE_BF16 ? 8 : 4, wide = (int64_t)shape->heads * shape->head_dim;
  const int64_t kv_wide = (int64_t)shape->kv_heads * shape->head_dim;
  if (dq_stride < wide || dk_stride < kv_wide || dv_stride < kv_wide || dq_stride % per || dk_stride % per || dv_stride % per)
    return TLF_E_INVALID_ARG;
  if (std::max({dq_stride, dk_stride, dv_stride}) > TLF_ATTN_MAX_STRIDE) return TLF_E_UNSUPPORTED;
  if (shape->rows_q > 0 && (!d_do || !d_q || !d_o || !d_lse || !d_dq)) return TLF_E_INVALID_ARG;
  if (shape->rows_k > 0 && (!d_k || !d_v || !d_dk || !d_dv)) return TLF_E_INVALID_ARG;
  if (d_o_low && shape->dtype != TLF_DTYPE_BF16) return TLF_E_INVALID_ARG;
  if (need > 0 && (!d_workspace || ws_bytes < need)) return TLF_E_INVALID_ARG;
  for (const void* p : {d_do, d_q, d_k, d_v, d_o, d_o_low, (const void*)d_dq, (const void*)d_dk, (const void*)d_dv, (const void*)d_workspace})
    if (((uintptr_t)p & 15u) != 0) return TLF_E_INVALID_ARG;
  for (const void* p : {(const void*)d_lse, (const void*)shape->d_q_offsets, (const void*)shape->d_k_offsets, (const void*)shape->d_k_lengths})
    if (((uintptr_t)p & 3u) != 0) return TLF_E_INVALID_ARG;
  tlf::GradArgs a{};
  static_cast<tlf::WAttnArgs&>(a) = tlf::wattn_args(*shape);
  a.q = d_q;
  a.k = d_k;
  a.v = d_v;
  a.o = d_o;
  a.dout = d_do;
  a.lse = const_cast<float*>(d_lse);
  a.low = const_cast<void*>(d_o_low);
  a.dq = d_dq;
  a.dk = d_dk;
  a.dv = d_dv;
  a.dqs = dq_stride;
  a.dks = dk_stride;
  a.dvs = dv_stride;
  a.nlse = (float*)d_workspace;
  a.ndelta = a.nlse + tlf::stat_floats(*shape);
  a.part = a.ndelta + tlf::stat_floats(*shape);
  const hipStream_t s = (hipStream_t)stream;
  const bool h = shape->dtype == TLF_DTYPE_BF16;
  const hipError_t e = shape->head_dim == 16    ? tlf::launch<float, 16>(*shape, a, s)
                       : shape->head_dim == 64  ? (h ? tlf::launch<bf16, 64>(*shape, a, s) : tlf::launch<float, 64>(*shape, a, s))
                                                : (h ? tlf::launch<bf16, 128>(*shape, a, s) : tlf::launch<float, 128>(*shape, a, s));
  return e == hipSuccess ? TLF_OK : TLF_E_HIP;
}

}  // extern "C"
