// Dot-product attention forward for bf16 data on v_mfma_f32_32x32x16_bf16, float32
// statistics and accumulators.
//
//     S^T = K Q^T,  a = cap tanh(scale S / cap) - slope |p - j|,  O^T += V^T P^T
//
// A wavefront owns 32 rows, one in each lane (column c of the products): the running
// maximum m and sum l of a row are the lane's own, and P^T goes from the accumulator
// into the second product's operand as it is. K and V come in blocks of 32 keys by
// loads straight into LDS, swizzled row-major; V^T fragments by the transposing LDS read. Head
// dimensions 16 and 32 run as 64 with zeros behind them.
//
//   dot_fwd_kernel   4 wavefronts, 128 rows, which share the blocks: a ring of 4
//                    stages, S(n + 1) formed while P(n) is.
//   dot_few_kernel   32 rows and 4 wavefronts that each take every fourth block (of a
//                    part of the key axis, where there are few rows) through LDS of
//                    their own, added at the end: for few queries, a new token's
//                    above all, where the time is that of reading K and V.
//
// The maximum is raised lazily: P is formed with the present m, and only where a
// row's block sum leaves (0, 2^16] is m raised to the block's maximum and P formed
// again. P is rounded to bf16 for the product with V, whose other operand is bf16: of random
// values each term p v is then off by as much as the output's own rounding takes from it, 0.0024 in
// all (relative norm) for 0.0017; a product of float32 would run at an eighth of the rate. The output
// is divided by the sum of the probabilities as rounded (it is then a weighted mean of V's rows
// whatever the rounding); LSE takes the sum of the unrounded ones.
//
// Bound by the matrix products and the exponentials beside them: B=1 H=32 N=8192 D=128, all
// pairs, 1107 - 1173 us (993 - 937 TFLOP/s from box to box; an 8192^3 product of the library's runs at
// 1173); causal, 16 heads on 4, 296 - 313 us (929 - 878). Where the workgroups do not outnumber the CUs, by the longest row's
// walk: N=4096, 8 heads, a prefix of 1024, 83 us (419 TFLOP/s). dot_few_kernel by the cache: 8 sequences of up to 16384
// keys, 4 heads, 168 MB in 34 us (4.9 TB/s), and 5 us to join the parts.
//
// With a distance bias the blocks are walked from the nearest keys back: the scores fall
// on the way, where forwards every block would raise the maximum (B=1 H=16 Hkv=4 N=8192
// D=128 causal: 451 us forwards, 313 back).
//
// A block whose pairs are all visible has no mask work; blocks without a visible pair
// are not visited (walked 64 at a time, a lane each). A masked pair's probability of
// 0 times an infinity or NaN of V is NaN: rows that it spoilt are formed again by themselves.
#include "dot_mfma.h"

#include "simplicial_layers.h"

#include <algorithm>

namespace sa {
namespace {

constexpr float kPmax = 65536.f;

// A row's running state and the step over one block.
template <int DP, int CAP, bool BIAS>
struct Row {
  static constexpr int NDT = DP / 32;
  f32x16_t acc[NDT];
  float m, l, lr;  // maximum (base 2), sum, sum of the rounded probabilities
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) acc[dt] = f32x16_t{};
    m = -3e38f, l = 0.f, lr = 0.f;  // (finite: m less itself is 0)
  }
  // Probabilities of a block, packed; `masked`: hide(s) sets the scores of pairs that are not
  // visible to -inf; `behind`: all keys are at or before the wavefront's queries.
  template <typename Hide>
  __device__ __forceinline__ void step(f32x16_t& s, const Scores<CAP, BIAS>& score, float dj, bool behind, bool masked, Hide hide,
                                       u32x4_t (&pf)[2]) {
    const bf16x2_t ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
    float mul = score.scale2, less = 0.f;  // scores are mul s - less
    if (BIAS && behind) {
      mul = 1.f, less = score.slope2 * dj;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = score.behind(s[v], v);
    } else if (CAP || BIAS || masked) {
      mul = 1.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = score(s[v], v, dj);
    }
    if (masked) hide(s);
    float lb, lrb;
    auto form = [&]() __attribute__((always_inline)) {
      lb = 0.f, lrb = 0.f;
      const float n = BIAS ? -(m + less) : -m;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = fast_exp2(__builtin_fmaf(s[8 * u + 2 * e], mul, n));
          const float y = fast_exp2(__builtin_fmaf(s[8 * u + 2 * e + 1], mul, n));
          lb += x;
          lb += y;
          const unsigned xy = pack_bf16x2(x, y);
          pf[u][e] = xy;
          lrb = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, xy), ones, lrb, false);
        }
    };
    form();
    if (__builtin_amdgcn_ballot_w64(!(lb <= kPmax)) != 0) {
      // (the scores rounded as their maximum is, not by an fma with the subtraction: past 2^24
      // what is rounded off passes 1)
      if constexpr (!BIAS && CAP != kShortCap) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          float x = s[v] * mul;
          asm("" : "+v"(x));
          s[v] = x;
        }
        mul = 1.f;
      }
      float mx = s[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
      if constexpr (BIAS) mx -= less;  // (the halves' differ)
      mx = fmaxf(m, fmaxf(mx, swap_halves(mx)));
      const float down = fast_exp2(m - mx);
      l *= down, lr *= down;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) acc[dt] *= down;
      m = mx;
      form();
    }
    l += lb, lr += lrb;
  }
  // Both halves' sums; m of a row without a visible key is below any score's.
  __device__ __forceinline__ void finish() {
    l += swap_halves(l);
    lr += swap_halves(lr);
  }
};

// Columns `at` (if d0) and at + 64 (if d1) of O.
__device__ __forceinline__ void write_out(const DotArgs& a, int64_t at, bool d0, float x0, bool d1, float x1) {
  uint16_t *out = static_cast<uint16_t*>(a.out) + at, *lo = static_cast<uint16_t*>(a.out_lo) + at;
  if (d0) out[0] = f32_to_bf16(x0);
  if (d1) out[64] = f32_to_bf16(x1);
  if (a.out_lo && d0) lo[0] = f32_to_bf16(rounded_off(x0));
  if (a.out_lo && d1) lo[64] = f32_to_bf16(rounded_off(x1));
}
// Columns `lane` (if t0) and lane + 64 (if t1) of one row's O by themselves, over its visible keys (LSE is
// not touched by masked pairs), a wavefront's 64 lanes along the columns.
__device__ __forceinline__ void single_row(const DotArgs& a, const DotMask& m, int b, int i, int head, float lse, bool t0, bool t1) {
  const int lane = threadIdx.x & 63, hk = head / a.G, p = m.first + i, dq = m.doc(p);
  const bool d0 = lane < a.D, d1 = lane + 64 < a.D;
  const uint16_t* q = static_cast<const uint16_t*>(a.q) + b * a.qsb + i * a.qsn + head * a.qsh + lane;
  const uint16_t* k = static_cast<const uint16_t*>(a.k) + b * a.ksb + hk * a.ksh + lane;
  const uint16_t* v = static_cast<const uint16_t*>(a.v) + b * a.vsb + hk * a.vsh + lane;
  const float q0 = d0 ? bf16_to_f32(q[0]) : 0.f, q1 = d1 ? bf16_to_f32(q[64]) : 0.f;
  const float slope = a.slopes ? a.slopes[head] : 0.f;
  float o0 = 0.f, o1 = 0.f;
  for (int j = 0; j < m.L; ++j) {
    if (!m.sees(p, j, dq, m.doc(j))) continue;
    const int64_t kj = j * a.ksn, vj = j * a.vsn;
    float s = (d0 ? q0 * bf16_to_f32(k[kj]) : 0.f) + (d1 ? q1 * bf16_to_f32(k[kj + 64]) : 0.f);
    s = sum64(s) * a.scale;
    if (a.cap > 0.f) s = a.cap * tanhf(s / a.cap);
    const float w = fast_exp2((s - slope * static_cast<float>(abs(p - j)) - lse) * kLog2e);
    o0 += d0 ? w * bf16_to_f32(v[vj]) : 0.f;
    o1 += d1 ? w * bf16_to_f32(v[vj + 64]) : 0.f;
    if (__builtin_amdgcn_ballot_w64((t0 && o0 == o0) || (t1 && o1 == o1)) == 0) break;  // all NaN
  }
  write_out(a, ((static_cast<int64_t>(b) * a.Nq + i) * a.H + head) * a.D + lane, t0, o0, t1, o1);
}
// The rows of `bad` (a bit for each of the wavefront's 32), one after another: of row c the columns for
// which t0(c), t1(c) say so.
template <typename T0, typename T1>
__device__ __forceinline__ void single_rows(const DotArgs& a, const DotMask& m, int b, const Lanes& w, float lse, unsigned bad, T0 t0, T1 t1) {
  const int lane = threadIdx.x & 63;
  while (bad) {
    const int c = __builtin_ctz(bad);
    bad &= bad - 1;
    single_row(a, m, b, __builtin_amdgcn_readlane(w.i, c), __builtin_amdgcn_readlane(w.head, c),
               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lse), c)), t0(c) && lane < a.D, t1(c) && lane + 64 < a.D);
  }
}

template <int DP, int CAP, bool BIAS, int GROUPS>
__global__ __launch_bounds__(kThreads* GROUPS, 2) void dot_fwd_kernel(DotArgs a) {
  using T = SwzTile<DP>;
  constexpr int NT = DP / 16, NDT = DP / 32, SPW = T::instrs / kWaves, kStages = 4, kRows = 32 * kWaves;
  static_assert(T::instrs % kWaves == 0, "every wavefront issues as many loads of a tile");
  __shared__ __attribute__((aligned(16))) char kst0[GROUPS * T::bytes], kst1[GROUPS * T::bytes], kst2[GROUPS * T::bytes], kst3[GROUPS * T::bytes];
  __shared__ __attribute__((aligned(16))) char vst0[GROUPS * T::bytes], vst1[GROUPS * T::bytes], vst2[GROUPS * T::bytes], vst3[GROUPS * T::bytes];
  auto kst = [&](auto SC) __attribute__((always_inline)) {
    constexpr int X = decltype(SC)::value;
    return to_lds(X == 0 ? kst0 : X == 1 ? kst1 : X == 2 ? kst2 : kst3);
  };
  auto vst = [&](auto SC) __attribute__((always_inline)) {
    constexpr int X = decltype(SC)::value;
    return to_lds(X == 0 ? vst0 : X == 1 ? vst1 : X == 2 ? vst2 : vst3);
  };
  const int R = a.G * a.Nq, nrb = (R + kRows - 1) / kRows;
  int64_t unit;
  if (!unit_of(static_cast<int64_t>(a.B) * a.Hkv, nrb, unit)) return;
  const int block = nrb - 1 - static_cast<int>(unit % nrb), bh = static_cast<int>(unit / nrb);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane((tid >> 6) % kWaves), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(tid / kThreads) : 0, base = group * T::bytes;
  const DotMask m(a, b);
  const int r0 = block * kRows + 32 * wave;
  const Lanes w(a, m, hk, r0 + c);
  const DotSpan all = rows_span(a, m, block * kRows, kRows), own = rows_span(a, m, min(r0, R - 1), 32);
  const KeysSeen seen(m, w.p);
  const Scores<CAP, BIAS> score(a, w.head);
  const int pos = w.p - 4 * h;
  int lo, hi;
  key_blocks(m, all, lo, hi);
  const bool some = r0 < R;
  auto seq = block_seq<BIAS>(lo, hi, 0, 1, [&](int blk, bool& live, bool& mine, bool& full) {
    const DotSpan k(m, blk * kDotBlock, blk * kDotBlock + kDotBlock - 1);
    live = dot_live(m, all, k);
    mine = some && dot_live(m, own, k);
    full = dot_full(m, own, k);
  });

  // Loads of a tile: wavefront x-th share is 1 KB, lane l the 16-byte chunk at 16 l.
  int kvoff[SPW], vvoff[SPW];
#pragma unroll
  for (int x = 0; x < SPW; ++x) {
    const int p = 64 * (x * kWaves + wave) + lane, row = p / T::CH, ch = (p % T::CH) ^ T::swz(row);
    kvoff[x] = 8 * ch < a.D ? static_cast<int>(row * a.ksn * 2) + 16 * ch : kFar;
    vvoff[x] = 8 * ch < a.D ? static_cast<int>(row * a.vsn * 2) + 16 * ch : kFar;
  }
  const uint16_t* kb = static_cast<const uint16_t*>(a.k) + b * a.ksb + hk * a.ksh;
  const uint16_t* vb = static_cast<const uint16_t*>(a.v) + b * a.vsb + hk * a.vsh;
  // (past the last block: loads of nothing, so that every iteration issues as many)
  auto load_k = [&](lds_char* dst, int blk) __attribute__((always_inline)) {
    const int64_t j0 = max(blk, 0) * kDotBlock;
    const auto r = rows_of(kb + j0 * a.ksn, blk < 0 ? 0 : min(m.L - static_cast<int>(j0), kDotBlock), a.ksn, a.D);
#pragma unroll
    for (int x = 0; x < SPW; ++x) load_lds16(r, dst + base + 1024 * (x * kWaves + wave), kvoff[x]);
  };
  auto load_v = [&](lds_char* dst, int blk) __attribute__((always_inline)) {
    const int64_t j0 = max(blk, 0) * kDotBlock;
    const auto r = rows_of(vb + j0 * a.vsn, blk < 0 ? 0 : min(m.L - static_cast<int>(j0), kDotBlock), a.vsn, a.D);
#pragma unroll
    for (int x = 0; x < SPW; ++x) load_lds16(r, dst + base + 1024 * (x * kWaves + wave), vvoff[x]);
  };
  u32x4_t qf[NT];
  load_row<DP>(qf, q_row(a, w, b), w.valid, a.D, h);
  const Frags<DP> frag(lane, base);
  DotBlock bq[kStages];
  int lead[kStages];  // group 0's block: the groups end together
  auto next = [&](auto SC) __attribute__((always_inline)) {
    constexpr int S = decltype(SC)::value;
    bq[S] = seq.next();
    lead[S] = bq[S].blk;
    if constexpr (GROUPS > 1) {
      const DotBlock other = seq.next();
      if (group) bq[S] = other;
    }
  };
  next(IC<0>{});
  load_k(kst(IC<0>{}), bq[0].blk);
  next(IC<1>{});
  load_k(kst(IC<1>{}), bq[1].blk);
  load_v(vst(IC<0>{}), bq[0].blk);
  next(IC<2>{});
  load_k(kst(IC<2>{}), bq[2].blk);
  load_v(vst(IC<1>{}), bq[1].blk);
  next(IC<3>{});
  load_k(kst(IC<3>{}), bq[3].blk);
  load_v(vst(IC<2>{}), bq[2].blk);

  Row<DP, CAP, BIAS> row;
  row.clear();
  f32x16_t sc[2];
  u32x4_t kf[NT];
  auto products = [&](f32x16_t& dst) __attribute__((always_inline)) {
    dst = mfma32(kf[0], qf[0], f32x16_t{});
#pragma unroll
    for (int t = 1; t < NT; ++t) dst = mfma32(kf[t], qf[t], dst);
  };
  wait_vmcnt<5 * SPW>();  // K(0), K(1)
  lds_barrier_tracked();
#pragma unroll
  for (int t = 0; t < NT; ++t) kf[t] = frag.row(kst(IC<0>{}), t);
  __builtin_amdgcn_sched_barrier(0);
  products(sc[0]);
#pragma unroll
  for (int t = 0; t < NT; ++t) kf[t] = frag.row(kst(IC<1>{}), t);

  // Iteration n: S(n + 1) and P(n), O += P V(n). K(n + 2) and V(n) have to be in LDS: of the loads
  // issued after them V(n + 1), K(n + 3) and V(n + 2) may be in flight.
  auto iteration = [&](auto SC) __attribute__((always_inline)) {
    constexpr int S = decltype(SC)::value, cur = S & 1, nxt = cur ^ 1;
    const DotBlock at = bq[S];
    if (lead[S] < 0) return false;
    const Frags<DP> f = frag.fresh();
    wait_vmcnt<3 * SPW>();
    lds_barrier_tracked();
    next(IC<S>{});
    load_k(kst(IC<S>{}), bq[S].blk);                            // K(n) was read in iteration n - 2
    load_v(vst(IC<(S + 3) % kStages>{}), bq[(S + 3) % kStages].blk);  // V(n - 1) in iteration n - 1
    if (at.mine) {
      u32x4_t vf[2][NDT];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) vf[u][dt] = f.tr(vst(IC<S>{}), dt, u);
      __builtin_amdgcn_s_setprio(1);
      products(sc[nxt]);
      u32x4_t pf[2];
      const int j0 = at.blk * kDotBlock;
      row.step(sc[cur], score, static_cast<float>(pos - j0), BIAS && j0 + 31 <= own.p0, !at.full,
               [&](f32x16_t& s) __attribute__((always_inline)) {
                 each_pair(m, seen, c, h, [&](int x) { return j0 + x; }, [&](int v, bool see) { s[v] = see ? s[v] : -kInf; });
               },
               pf);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) row.acc[dt] = mfma32(vf[u][dt], pf[u], row.acc[dt]);
      __builtin_amdgcn_s_setprio(0);
    } else {
      products(sc[nxt]);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) kf[t] = f.row(kst(IC<(S + 2) % kStages>{}), t);
    return true;
  };
  while (iteration(IC<0>{}) && iteration(IC<1>{}) && iteration(IC<2>{}) && iteration(IC<3>{})) {
  }
  wait_vmcnt<0>();
  row.finish();
  if constexpr (GROUPS > 1) {
    // The second group's states into the first's, through the ring's LDS (a stage's array a wavefront).
    __shared__ float stat[3][kWaves][32];
    float* buf = reinterpret_cast<float*>(wave == 0 ? kst0 : wave == 1 ? kst1 : wave == 2 ? kst2 : kst3) + lane;
    __syncthreads();
    if (group) {
      if (h == 0) stat[0][wave][c] = row.m, stat[1][wave][c] = row.l, stat[2][wave][c] = row.lr;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) buf[64 * (16 * dt + v)] = row.acc[dt][v];
    }
    __syncthreads();
    if (group) return;
    const float om = stat[0][wave][c], top = fmaxf(row.m, om), x = fast_exp2(row.m - top), y = fast_exp2(om - top);
    row.m = top;
    row.l = x * row.l + y * stat[1][wave][c];
    row.lr = x * row.lr + y * stat[2][wave][c];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) row.acc[dt][v] = x * row.acc[dt][v] + y * buf[64 * (16 * dt + v)];
  }
  const bool empty = row.l == 0.f;
  const float inv = empty ? 0.f : 1.f / row.lr;
  const float lse = empty ? -kInf : row.m * kLn2 + logf(row.l);
  const float check = not_finite(row.acc);
  const unsigned bad = has_mask(a) ? rows_where(w.valid && fabsf(row.l) < kInf && check != check) : 0;
  if (w.valid) {
    const int64_t o = ((static_cast<int64_t>(b) * a.Nq + w.i) * a.H + w.head) * a.D + 4 * h;
    store_row<DP>(static_cast<uint16_t*>(a.out) + o, row.acc, inv, a.D);
    if (a.out_lo) store_row_lo<DP>(static_cast<uint16_t*>(a.out_lo) + o, row.acc, inv, a.D);
    if (h == 0) a.lse[(static_cast<int64_t>(b) * a.H + w.head) * a.Nq + w.i] = lse;
  }
  if (__builtin_expect(bad != 0, 0) && keys_spoil(a, m, own, vb, a.vsn)) {
    const NanColumns<NDT> nan(row.acc);
    wait_vmcnt<0>();  // (the rows are written)
    single_rows(a, m, b, w, lse, bad, [&](int x) { return nan.template at<0>(x); }, [&](int x) { return nan.template at<1>(x); });
  }
}

template <int DP, int CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 1) void dot_few_kernel(DotArgs a) {
  using T = SwzTile<DP>;
  constexpr int NT = DP / 16, NDT = DP / 32, SPW = T::instrs;
  __shared__ __attribute__((aligned(16))) char kst0[kWaves * T::bytes], kst1[kWaves * T::bytes];
  __shared__ __attribute__((aligned(16))) char vst0[kWaves * T::bytes], vst1[kWaves * T::bytes];
  __shared__ float stat[3][kWaves][32];
  auto kst = [&](auto SC) __attribute__((always_inline)) { return to_lds(decltype(SC)::value == 0 ? kst0 : kst1); };
  auto vst = [&](auto SC) __attribute__((always_inline)) { return to_lds(decltype(SC)::value == 0 ? vst0 : vst1); };
  const int R = a.G * a.Nq, nrb = (R + 31) / 32;
  int64_t unit;
  if (!unit_of(static_cast<int64_t>(a.B) * a.Hkv, static_cast<int64_t>(nrb) * a.nsplit, unit)) return;
  const int part = static_cast<int>(unit % a.nsplit);
  unit /= a.nsplit;
  const int block = nrb - 1 - static_cast<int>(unit % nrb), bh = static_cast<int>(unit / nrb);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const DotMask m(a, b);
  const Lanes w(a, m, hk, block * 32 + c);
  const DotSpan own = rows_span(a, m, block * 32, 32);
  const KeysSeen seen(m, w.p);
  const Scores<CAP, BIAS> score(a, w.head);
  const int pos = w.p - 4 * h;
  int lo, hi;
  key_blocks(m, own, lo, hi);
  auto seq = block_seq<BIAS>(lo, hi, part * kWaves + wave, kWaves * a.nsplit, [&](int blk, bool& live, bool& mine, bool& full) {
    const DotSpan k(m, blk * kDotBlock, blk * kDotBlock + kDotBlock - 1);
    live = dot_live(m, own, k);
    mine = live;
    full = dot_full(m, own, k);
  });
  int kvoff[SPW], vvoff[SPW];
#pragma unroll
  for (int x = 0; x < SPW; ++x) {
    const int p = 64 * x + lane, row = p / T::CH, ch = (p % T::CH) ^ T::swz(row);
    kvoff[x] = 8 * ch < a.D ? static_cast<int>(row * a.ksn * 2) + 16 * ch : kFar;
    vvoff[x] = 8 * ch < a.D ? static_cast<int>(row * a.vsn * 2) + 16 * ch : kFar;
  }
  const uint16_t* kb = static_cast<const uint16_t*>(a.k) + b * a.ksb + hk * a.ksh;
  const uint16_t* vb = static_cast<const uint16_t*>(a.v) + b * a.vsb + hk * a.vsh;
  auto load = [&](auto SC, int blk) __attribute__((always_inline)) {
    const int64_t j0 = max(blk, 0) * kDotBlock;
    const int n = blk < 0 ? 0 : min(m.L - static_cast<int>(j0), kDotBlock);
    const auto rk = rows_of(kb + j0 * a.ksn, n, a.ksn, a.D), rv = rows_of(vb + j0 * a.vsn, n, a.vsn, a.D);
#pragma unroll
    for (int x = 0; x < SPW; ++x) load_lds16(rk, kst(SC) + wave * T::bytes + 1024 * x, kvoff[x]);
#pragma unroll
    for (int x = 0; x < SPW; ++x) load_lds16(rv, vst(SC) + wave * T::bytes + 1024 * x, vvoff[x]);
  };
  u32x4_t qf[NT];
  load_row<DP>(qf, q_row(a, w, b), w.valid, a.D, h);
  const Frags<DP> frag(lane, wave * T::bytes);
  DotBlock bq[2];
  bq[0] = seq.next();
  load(IC<0>{}, bq[0].blk);
  bq[1] = seq.next();
  load(IC<1>{}, bq[1].blk);
  Row<DP, CAP, BIAS> row;
  row.clear();
  // (the wavefronts' blocks are their own: no barriers)
  auto iteration = [&](auto SC) __attribute__((always_inline)) {
    constexpr int S = decltype(SC)::value;
    const DotBlock at = bq[S];
    if (at.blk < 0) return false;
    const Frags<DP> f = frag.fresh();
    wait_vmcnt<2 * SPW>();
    asm volatile("" ::: "memory");
    f32x16_t s = mfma32(f.row(kst(SC), 0), qf[0], f32x16_t{});
#pragma unroll
    for (int t = 1; t < NT; ++t) s = mfma32(f.row(kst(SC), t), qf[t], s);
    u32x4_t vf[2][NDT];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) vf[u][dt] = f.tr(vst(SC), dt, u);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // the stage is read: its next block may come
    asm volatile("" ::: "memory");
    bq[S] = seq.next();
    load(SC, bq[S].blk);
    u32x4_t pf[2];
    const int j0 = at.blk * kDotBlock;
    row.step(s, score, static_cast<float>(pos - j0), BIAS && j0 + 31 <= own.p0, !at.full,
             [&](f32x16_t& s) __attribute__((always_inline)) {
               each_pair(m, seen, c, h, [&](int x) { return j0 + x; }, [&](int v, bool see) { s[v] = see ? s[v] : -kInf; });
             },
             pf);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) row.acc[dt] = mfma32(vf[u][dt], pf[u], row.acc[dt]);
    return true;
  };
  while (iteration(IC<0>{}) && iteration(IC<1>{})) {
  }
  wait_vmcnt<0>();
  row.finish();
  // The wavefronts' states joined: their accumulators, scaled to the common maximum, through
  // the tiles' LDS (one array a tile, 4 KB a wavefront).
  auto joined = [&](int dt) { return reinterpret_cast<float*>(dt == 0 ? kst0 : dt == 1 ? kst1 : dt == 2 ? vst0 : vst1) + lane; };
  if (h == 0) stat[0][wave][c] = row.m, stat[1][wave][c] = row.l, stat[2][wave][c] = row.lr;
  __syncthreads();
  float top = stat[0][0][c];
#pragma unroll
  for (int x = 1; x < kWaves; ++x) top = fmaxf(top, stat[0][x][c]);
  float l = 0.f, lr = 0.f;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    const float f = fast_exp2(stat[0][x][c] - top);
    l += f * stat[1][x][c];
    lr += f * stat[2][x][c];
  }
  const float down = fast_exp2(row.m - top);
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
    float* x = joined(dt) + wave * 1024;
#pragma unroll
    for (int v = 0; v < 16; ++v) x[64 * v] = row.acc[dt][v] * down;
  }
  __syncthreads();
  const bool empty = l == 0.f;
  const float inv = a.nsplit > 1 ? 1.f : empty ? 0.f : 1.f / lr;
  const int64_t rr = static_cast<int64_t>(bh) * R + block * 32 + c;
  float* pr = a.part + (rr * a.nsplit + part) * a.D + 4 * h;
  const int64_t o = ((static_cast<int64_t>(b) * a.Nq + w.i) * a.H + w.head) * a.D + 4 * h;
  uint16_t *out = static_cast<uint16_t*>(a.out) + o, *olo = static_cast<uint16_t*>(a.out_lo) + o;
  float check = 0.f;
  const float lse = empty ? -kInf : top * kLn2 + logf(l);
  // Each wavefront takes quad `wave` of every tile.
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
    const float* x = joined(dt);
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = 0.f;
#pragma unroll
      for (int z = 0; z < kWaves; ++z) y[e] += x[z * 1024 + 64 * (4 * wave + e)];
      check += y[e] * 0.f;
      y[e] *= inv;
    }
    if (w.valid && 32 * dt + 8 * wave < a.D) {
      if (a.nsplit > 1)
        *reinterpret_cast<u32x4_t*>(pr + 32 * dt + 8 * wave) =
            u32x4_t{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
      else
        *reinterpret_cast<u32x2_t*>(out + 32 * dt + 8 * wave) = u32x2_t{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
      if (a.nsplit == 1 && a.out_lo)
        *reinterpret_cast<u32x2_t*>(olo + 32 * dt + 8 * wave) = u32x2_t{pack_bf16x2(rounded_off(y[0]), rounded_off(y[1])),
                                                                        pack_bf16x2(rounded_off(y[2]), rounded_off(y[3]))};
    }
  }
  if (wave == 0 && h == 0 && w.valid) {
    if (a.nsplit > 1) {
      float* st = a.part + static_cast<int64_t>(a.B) * a.H * a.Nq * a.nsplit * a.D + (rr * a.nsplit + part) * 3;
      st[0] = l == 0.f ? -kInf : top, st[1] = l, st[2] = lr;
    } else {
      a.lse[(static_cast<int64_t>(b) * a.H + w.head) * a.Nq + w.i] = lse;
    }
  }
  if (a.nsplit > 1 || !has_mask(a)) return;
  // (a row is not finite if any wavefront's columns of it are not)
  __shared__ unsigned flags[kWaves];
  const unsigned x = rows_where(w.valid && fabsf(l) < kInf && check != check);
  if (lane == 0) flags[wave] = x;
  __syncthreads();
  const unsigned bad = __builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3]);
  if (wave == 0 && bad && keys_spoil(a, m, own, vb, a.vsn))
    single_rows(a, m, b, w, lse, bad, [](int) { return true; }, [](int) { return true; });
}

// Joins the parts of a row: one workgroup, its wavefronts taking every fourth part.
__global__ __launch_bounds__(kThreads) void dot_join_kernel(DotArgs a) {
  const int64_t all = static_cast<int64_t>(a.B) * a.H * a.Nq, r = blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float* st = a.part + all * a.nsplit * a.D + r * a.nsplit * 3;
  const float* rows = a.part + r * a.nsplit * a.D + lane;
  const bool d0 = lane < a.D, d1 = lane + 64 < a.D;
  float top = -kInf;
  for (int s = lane; s < a.nsplit; s += 64) top = fmaxf(top, st[3 * s]);
  top = reduce32(top, [](float x, float y) { return fmaxf(x, y); });
  top = fmaxf(top, swap_halves(top));
  const float base = top == -kInf ? 0.f : top;
  float l = 0.f, lr = 0.f, x0 = 0.f, x1 = 0.f;
  for (int s0 = 0; s0 < a.nsplit; s0 += 64) {
    const int s = s0 + lane;
    const float f = s < a.nsplit ? fast_exp2(st[3 * s] - base) : 0.f;
    l += s < a.nsplit ? f * st[3 * s + 1] : 0.f;
    lr += s < a.nsplit ? f * st[3 * s + 2] : 0.f;
    const int n = min(a.nsplit - s0, 64);
    for (int i = wave; i < n; i += kWaves) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i));
      const float* p = rows + static_cast<int64_t>(s0 + i) * a.D;
      x0 += d0 ? w * p[0] : 0.f;
      x1 += d1 ? w * p[64] : 0.f;
    }
  }
  __shared__ float sums[2][kWaves][64];
  sums[0][wave][lane] = x0, sums[1][wave][lane] = x1;
  __syncthreads();
  if (wave) return;
  x0 = ((sums[0][0][lane] + sums[0][1][lane]) + sums[0][2][lane]) + sums[0][3][lane];
  x1 = ((sums[1][0][lane] + sums[1][1][lane]) + sums[1][2][lane]) + sums[1][3][lane];
  l = sum64(l), lr = sum64(lr);
  const int64_t rh = static_cast<int64_t>(a.G) * a.Nq;
  const int bh = static_cast<int>(r / rh), rr = static_cast<int>(r - bh * rh), i = rr / a.G;
  const int b = bh / a.Hkv, head = (bh - b * a.Hkv) * a.G + rr - i * a.G;
  const float lse = l == 0.f ? -kInf : top * kLn2 + logf(l);
  if (lane == 0) a.lse[(static_cast<int64_t>(b) * a.H + head) * a.Nq + i] = lse;
  const float inv = l == 0.f ? 0.f : 1.f / lr;
  write_out(a, ((static_cast<int64_t>(b) * a.Nq + i) * a.H + head) * a.D + lane, d0, x0 * inv, d1, x1 * inv);
  const bool n0 = d0 && x0 != x0, n1 = d1 && x1 != x1;
  if (has_mask(a) && fabsf(l) < kInf && __builtin_amdgcn_ballot_w64(n0 || n1) != 0) {
    const DotMask m(a, b);
    const uint16_t* vb = static_cast<const uint16_t*>(a.v) + b * a.vsb + head / a.G * a.vsh;
    if (keys_spoil(a, m, rows_span(a, m, rr / 32 * 32, 32), vb, a.vsn)) single_row(a, m, b, i, head, lse, n0, n1);
  }
}

template <int DP, int CAP, bool BIAS>
hipError_t launch(const DotArgs& a, hipStream_t st) {
  const int64_t R = static_cast<int64_t>(a.G) * a.Nq, heads = static_cast<int64_t>(a.B) * a.Hkv;
  if (a.nsplit <= 0) {
    if (a.nsplit == 0)
      dot_fwd_kernel<DP, CAP, BIAS, 1><<<unit_grid(heads, (R + 127) / 128), kThreads, 0, st>>>(a);
    else
      dot_fwd_kernel<DP, CAP, BIAS, 2><<<unit_grid(heads, (R + 127) / 128), 2 * kThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  dot_few_kernel<DP, CAP, BIAS><<<unit_grid(heads, ((R + 31) / 32) * a.nsplit), kThreads, 0, st>>>(a);
  if (a.nsplit > 1) dot_join_kernel<<<static_cast<unsigned>(heads * R), kThreads, 0, st>>>(a);
  return hipGetLastError();
}
template <int DP>
hipError_t launch(const DotArgs& a, hipStream_t st) {
  return with_cap(a.cap, [&](auto cap) {
    constexpr int CAP = decltype(cap)::value;
    return a.slopes ? launch<DP, CAP, true>(a, st) : launch<DP, CAP, false>(a, st);
  });
}

}  // namespace

hipError_t dot_fwd_bf16(const DotArgs& a, hipStream_t st) { return a.D <= 64 ? launch<64>(a, st) : launch<128>(a, st); }

}  // namespace sa
