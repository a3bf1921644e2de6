// Dot-product attention backward for bf16 data on v_mfma_f32_32x32x16_bf16, float32
// sums.
//
//     P = exp(a - LSE),  dS = P (dO V^T - Delta) (1 - tanh^2)
//     dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// Two kernels without atomics. The query side owns rows: S^T = K Q^T and dP^T = V dO^T
// put one row in each lane, dQ^T += K^T dS^T; it also forms Delta = <dO, O> and leaves
// what the key side needs of a block of 32 rows (Stat) in the workspace. The key side
// owns keys: S = Q K^T, dP = dO V^T with one key in each lane, dV^T += dO^T P and
// dK^T += Q^T dS over all rows of the head's group, which sums the gradients of a
// shared head in float32. 7 matrix products where 5 would do with S and dP formed
// once, against atomics or partial sums of dQ for every block of keys.
//
// As in the forward, a workgroup's 4 wavefronts own 32 rows (keys) each and share the
// blocks of the other side through a ring in LDS, or (PRIV, where there are few rows
// or keys) own the same 32 and take every fourth block through LDS of their own, their
// sums added at the end in a fixed order.
//
// Bound by the products and, on the key side, by registers (K, V, dK and dV of 32 keys a
// wavefront): B=1 H=32 N=8192 D=128, all pairs, query side 1.53 - 1.56 ms (1.6 TFLOP, 1080 - 1054 TFLOP/s), key
// side 2.4 - 2.6 ms (2.2 TFLOP, 910 - 850 TFLOP/s); three documents with a cap, 16 heads on 4: 401 and 508 + 66 us.
//
// P and dS are rounded to bf16 for their products, as the operands are (which puts gradients of random
// values off by 0.0024, relative norm, where rounding them alone takes 0.0017); everything
// else is float32. Rows or keys whose sums met an infinity or NaN of a masked pair are
// formed again by themselves (dot_mfma.h).
#include "dot_mfma.h"

namespace sa {
namespace {

// What the key side reads of a block of 32 rows: LSE in base 2 (+inf: a row without a
// key or none, whose probabilities are 0), Delta, the distance bias's slope in base 2 and the
// query less the block's first.
struct Stat {
  float lse2[32], delta[32], slope2[32], query[32];
};
__device__ __forceinline__ Stat* stats_of(const DotArgs& a, int bh) {
  const int nrb = (a.G * a.Nq + 31) / 32;
  return reinterpret_cast<Stat*>(a.delta) + static_cast<int64_t>(bh) * nrb;
}

// Base-2 score and the cap's derivative.
template <int CAP, bool BIAS>
__device__ __forceinline__ float score_of(const Scores<CAP, BIAS>& c, float s, float slope2, float dj, float less, float& dcap) {
  float x;
  if constexpr (CAP)
    x = c.capped(s, dcap) - less;
  else
    x = __builtin_fmaf(s, c.scale2, -less);
  if constexpr (BIAS) x = __builtin_fmaf(-slope2, fabsf(dj), x);
  return x;
}

// Columns `lane` (if t0) and lane + 64 (if t1) of dQ of one row by themselves.
__device__ __forceinline__ void single_row(const DotArgs& a, const DotMask& m, int b, int i, int head, float lse, float delta, bool t0, bool t1) {
  const int lane = threadIdx.x & 63, hk = head / a.G, p = m.first + i, dq = m.doc(p);
  const bool d0 = lane < a.D, d1 = lane + 64 < a.D;
  const int64_t at = ((static_cast<int64_t>(b) * a.Nq + i) * a.H + head) * a.D + lane;
  const uint16_t* q = static_cast<const uint16_t*>(a.q) + b * a.qsb + i * a.qsn + head * a.qsh + lane;
  const uint16_t* g = static_cast<const uint16_t*>(a.dout) + at;
  const uint16_t* k = static_cast<const uint16_t*>(a.k) + b * a.ksb + hk * a.ksh + lane;
  const uint16_t* v = static_cast<const uint16_t*>(a.v) + b * a.vsb + hk * a.vsh + lane;
  const float q0 = d0 ? bf16_to_f32(q[0]) : 0.f, q1 = d1 ? bf16_to_f32(q[64]) : 0.f;
  const float g0 = d0 ? bf16_to_f32(g[0]) : 0.f, g1 = d1 ? bf16_to_f32(g[64]) : 0.f;
  const float slope = a.slopes ? a.slopes[head] : 0.f;
  float o0 = 0.f, o1 = 0.f;
  for (int j = 0; j < m.L; ++j) {
    if (!m.sees(p, j, dq, m.doc(j))) continue;
    const int64_t kj = j * a.ksn, vj = j * a.vsn;
    const float k0 = d0 ? bf16_to_f32(k[kj]) : 0.f, k1 = d1 ? bf16_to_f32(k[kj + 64]) : 0.f;
    float s = sum64(q0 * k0 + q1 * k1) * a.scale, dcap = 1.f;
    const float dp = sum64((d0 ? g0 * bf16_to_f32(v[vj]) : 0.f) + (d1 ? g1 * bf16_to_f32(v[vj + 64]) : 0.f));
    if (a.cap > 0.f) {
      const float t = tanhf(s / a.cap);
      s = a.cap * t;
      dcap = 1.f - t * t;
    }
    const float w = fast_exp2((s - slope * static_cast<float>(abs(p - j)) - lse) * kLog2e) * (dp - delta) * dcap * a.scale;
    o0 += w * k0;
    o1 += w * k1;
    if (__builtin_amdgcn_ballot_w64((t0 && o0 == o0) || (t1 && o1 == o1)) == 0) break;  // all NaN
  }
  uint16_t* out = static_cast<uint16_t*>(a.dq) + at;
  if (t0) out[0] = f32_to_bf16(o0);
  if (t1) out[64] = f32_to_bf16(o1);
}
// The same of dK (k0, k1) and dV (v0, v1) of one key.
struct KeyColumns {
  bool k0, k1, v0, v1;
};
__device__ __forceinline__ void single_key(const DotArgs& a, const DotMask& m, int b, int hk, int j, KeyColumns t) {
  const int lane = threadIdx.x & 63, dk = m.doc(j);
  const bool d0 = lane < a.D, d1 = lane + 64 < a.D;
  const uint16_t* k = static_cast<const uint16_t*>(a.k) + b * a.ksb + j * a.ksn + hk * a.ksh + lane;
  const uint16_t* v = static_cast<const uint16_t*>(a.v) + b * a.vsb + j * a.vsn + hk * a.vsh + lane;
  const float k0 = d0 ? bf16_to_f32(k[0]) : 0.f, k1 = d1 ? bf16_to_f32(k[64]) : 0.f;
  const float v0 = d0 ? bf16_to_f32(v[0]) : 0.f, v1 = d1 ? bf16_to_f32(v[64]) : 0.f;
  const Stat* stats = stats_of(a, b * a.Hkv + hk);
  float x0 = 0.f, x1 = 0.f, y0 = 0.f, y1 = 0.f;
  for (int i = max(-m.first, 0); i < a.Nq; ++i) {
    const int p = m.first + i;
    if (!m.sees(p, j, m.doc(p), dk)) continue;
    for (int gr = 0; gr < a.G; ++gr) {
      const int head = hk * a.G + gr, r = i * a.G + gr;
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + b * a.qsb + i * a.qsn + head * a.qsh + lane;
      const uint16_t* g = static_cast<const uint16_t*>(a.dout) + ((static_cast<int64_t>(b) * a.Nq + i) * a.H + head) * a.D + lane;
      const float q0 = d0 ? bf16_to_f32(q[0]) : 0.f, q1 = d1 ? bf16_to_f32(q[64]) : 0.f;
      const float g0 = d0 ? bf16_to_f32(g[0]) : 0.f, g1 = d1 ? bf16_to_f32(g[64]) : 0.f;
      float s = sum64(q0 * k0 + q1 * k1) * a.scale, dcap = 1.f;
      const float dp = sum64(g0 * v0 + g1 * v1);
      if (a.cap > 0.f) {
        const float t = tanhf(s / a.cap);
        s = a.cap * t;
        dcap = 1.f - t * t;
      }
      const Stat& st = stats[r >> 5];
      const float w = fast_exp2((s - (a.slopes ? a.slopes[head] : 0.f) * static_cast<float>(abs(p - j))) * kLog2e - st.lse2[r & 31]);
      const float ds = w * (dp - st.delta[r & 31]) * dcap * a.scale;
      x0 += ds * q0;
      x1 += ds * q1;
      y0 += w * g0;
      y1 += w * g1;
    }
    if (__builtin_amdgcn_ballot_w64((t.k0 && x0 == x0) || (t.k1 && x1 == x1) || (t.v0 && y0 == y0) || (t.v1 && y1 == y1)) == 0) break;
  }
  const int64_t at = ((static_cast<int64_t>(b) * a.Nk + j) * a.Hkv + hk) * a.D + lane;
  if (t.k0) static_cast<uint16_t*>(a.dk)[at] = f32_to_bf16(x0);
  if (t.k1) static_cast<uint16_t*>(a.dk)[at + 64] = f32_to_bf16(x1);
  if (t.v0) static_cast<uint16_t*>(a.dv)[at] = f32_to_bf16(y0);
  if (t.v1) static_cast<uint16_t*>(a.dv)[at + 64] = f32_to_bf16(y1);
}

// LDS arrays of the ring: W copies of NS stages of two tensors' tiles, every stage its own
// array (so that the wait for one stage's loads is not for the others').
#define SA_DOT_RING(W, NS)                                                                                  \
  __shared__ __attribute__((aligned(16))) char xst0[(W)*T::bytes], xst1[(W)*T::bytes], yst0[(W)*T::bytes],  \
      yst1[(W)*T::bytes], xst2[NS > 2 ? (W)*T::bytes : 16], xst3[NS > 2 ? (W)*T::bytes : 16],               \
      yst2[NS > 2 ? (W)*T::bytes : 16], yst3[NS > 2 ? (W)*T::bytes : 16];                                   \
  auto xst = [&](auto SC) __attribute__((always_inline)) {                                                  \
    constexpr int X = decltype(SC)::value;                                                                  \
    return to_lds(X == 0 ? xst0 : X == 1 ? xst1 : X == 2 ? xst2 : xst3);                                    \
  };                                                                                                        \
  auto yst = [&](auto SC) __attribute__((always_inline)) {                                                  \
    constexpr int X = decltype(SC)::value;                                                                  \
    return to_lds(X == 0 ? yst0 : X == 1 ? yst1 : X == 2 ? yst2 : yst3);                                    \
  }

// The second group's accumulators into the first's, through LDS: 64 floats a register.
template <int NDT>
__device__ __forceinline__ void leave(const f32x16_t (&acc)[NDT], float* buf) {
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) buf[64 * (16 * dt + v)] = acc[dt][v];
}
template <int NDT>
__device__ __forceinline__ void take(f32x16_t (&acc)[NDT], const float* buf) {
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[dt][v] += buf[64 * (16 * dt + v)];
}

// Adds the wavefronts' accumulator tiles in order, through one LDS array of 16 KB each:
// wavefront w ends with quad w (columns 8 w + 4 h .. + 3) of every tile in y.
template <int NDT, typename Buf>
__device__ __forceinline__ void add_waves(const f32x16_t (&acc)[NDT], float (&y)[NDT][4], Buf buf, int wave, int lane) {
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) buf(dt)[wave * 1024 + 64 * v + lane] = acc[dt][v];
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[dt][e] = 0.f;
#pragma unroll
      for (int z = 0; z < kWaves; ++z) y[dt][e] += buf(dt)[z * 1024 + 64 * (4 * wave + e) + lane];
    }
  __syncthreads();
}
template <int NDT>
__device__ __forceinline__ float store_quads(uint16_t* p, const float (&y)[NDT][4], float mul, int wave, int D) {
  float check = 0.f;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
#pragma unroll
    for (int e = 0; e < 4; ++e) check += y[dt][e] * 0.f;
    if (p && 32 * dt + 8 * wave < D)
      *reinterpret_cast<u32x2_t*>(p + 32 * dt + 8 * wave) = u32x2_t{pack_bf16x2(y[dt][0] * mul, y[dt][1] * mul), pack_bf16x2(y[dt][2] * mul, y[dt][3] * mul)};
  }
  return check;
}

// ---- query side ----
template <int DP, int CAP, bool BIAS, bool PRIV, int GROUPS>
__global__ __launch_bounds__(kThreads* GROUPS, PRIV ? 1 : 2) void dot_dq_kernel(DotArgs a) {
  using T = SwzTile<DP>;
  constexpr int NT = DP / 16, NDT = DP / 32, SPW = PRIV ? T::instrs : T::instrs / kWaves, kRows = PRIV ? 32 : 32 * kWaves;
  constexpr int NS = PRIV ? 2 : 4;
  SA_DOT_RING(PRIV ? kWaves : GROUPS, NS);
  const int R = a.G * a.Nq, nrb = (R + kRows - 1) / kRows;
  int64_t unit;
  if (!unit_of(static_cast<int64_t>(a.B) * a.Hkv, nrb, unit)) return;
  const int block = nrb - 1 - static_cast<int>(unit % nrb), bh = static_cast<int>(unit / nrb);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane((tid >> 6) % kWaves), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(tid / kThreads) : 0, base = (PRIV ? wave : group) * T::bytes;
  const DotMask m(a, b);
  const int r0 = block * kRows + (PRIV ? 0 : 32 * wave);
  const Lanes w(a, m, hk, r0 + c);
  const DotSpan all = rows_span(a, m, block * kRows, kRows), own = rows_span(a, m, min(r0, R - 1), 32);
  const KeysSeen seen(m, w.p);
  const int pos = w.p - 4 * h;
  const Scores<CAP, BIAS> score(a, w.head);
  int lo, hi;
  key_blocks(m, all, lo, hi);
  const bool some = r0 < R;
  auto seq = block_seq(lo, hi, PRIV ? wave : 0, PRIV ? kWaves : 1, [&](int blk, bool& live, bool& mine, bool& full) {
    const DotSpan k(m, blk * kDotBlock, blk * kDotBlock + kDotBlock - 1);
    live = dot_live(m, all, k);
    mine = some && dot_live(m, own, k);
    full = dot_full(m, own, k);
  });
  int kvoff[SPW], vvoff[SPW];
#pragma unroll
  for (int x = 0; x < SPW; ++x) {
    const int p = 64 * (PRIV ? x : x * kWaves + wave) + lane, row = p / T::CH, ch = (p % T::CH) ^ T::swz(row);
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
    for (int x = 0; x < SPW; ++x) load_lds16(rk, xst(SC) + base + 1024 * (PRIV ? x : x * kWaves + wave), kvoff[x]);
#pragma unroll
    for (int x = 0; x < SPW; ++x) load_lds16(rv, yst(SC) + base + 1024 * (PRIV ? x : x * kWaves + wave), vvoff[x]);
  };
  // This row's q, dO and Delta.
  u32x4_t qf[NT], gf[NT];
  const int64_t orow = ((static_cast<int64_t>(b) * a.Nq + w.i) * a.H + w.head) * a.D;
  load_row<DP>(qf, q_row(a, w, b), w.valid, a.D, h);
  load_row<DP>(gf, static_cast<const uint16_t*>(a.dout) + orow, w.valid, a.D, h);
  float delta = 0.f;
  for (int part = 0; part < (a.out_lo_in ? 2 : 1); ++part) {
    u32x4_t of[NT];
    load_row<DP>(of, static_cast<const uint16_t*>(part ? a.out_lo_in : a.out_in) + orow, w.valid, a.D, h);
    f32x16_t x = mfma32(of[0], gf[0], f32x16_t{});
#pragma unroll
    for (int t = 1; t < NT; ++t) x = mfma32(of[t], gf[t], x);
    delta += diagonal(x, c, h);
  }
  const float lse = w.valid ? a.lse[(static_cast<int64_t>(b) * a.H + w.head) * a.Nq + w.i] : -kInf;
  const float lse2 = lse == -kInf ? kInf : lse * kLog2e;
  if (h == 0 && some && group == 0 && (!PRIV || wave == 0)) {
    Stat& st = stats_of(a, bh)[r0 / 32];
    st.lse2[c] = lse2;
    st.delta[c] = w.valid ? delta : 0.f;
    st.slope2[c] = score.slope2;
    st.query[c] = static_cast<float>(w.i - div_group(r0, a));
  }
  const Frags<DP> frag(lane, base);
  DotBlock bq[NS];
  int lead[NS];  // group 0's block: the groups end together
  auto next = [&](auto SC) __attribute__((always_inline)) {
    constexpr int S = decltype(SC)::value;
    bq[S] = seq.next();
    lead[S] = bq[S].blk;
    if constexpr (GROUPS > 1) {
      const DotBlock other = seq.next();
      if (group) bq[S] = other;
    }
    load(SC, bq[S].blk);
  };
  next(IC<0>{});
  next(IC<1>{});
  if constexpr (!PRIV) next(IC<2>{});
  f32x16_t acc[NDT] = {};
  auto iteration = [&](auto SC) __attribute__((always_inline)) {
    constexpr int S = decltype(SC)::value;
    const DotBlock at = bq[S];
    if (lead[S] < 0) return false;
    const Frags<DP> f = frag.fresh();
    if constexpr (PRIV) {
      wait_vmcnt<2 * SPW>();
      asm volatile("" ::: "memory");
    } else {
      wait_vmcnt<4 * SPW>();
      lds_barrier_tracked();
      next(IC<(S + 3) % NS>{});
    }
    if (at.mine) {
      f32x16_t s = mfma32(f.row(xst(SC), 0), qf[0], f32x16_t{}), dp = mfma32(f.row(yst(SC), 0), gf[0], f32x16_t{});
#pragma unroll
      for (int t = 1; t < NT; ++t) {
        s = mfma32(f.row(xst(SC), t), qf[t], s);
        dp = mfma32(f.row(yst(SC), t), gf[t], dp);
      }
      const int j0 = at.blk * kDotBlock;
      const float dj = static_cast<float>(pos - j0);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float dcap = 1.f;
        const float x = score_of(score, s[v], score.slope2, dj - static_cast<float>(8 * (v >> 2) + (v & 3)), lse2, dcap);
        s[v] = fast_exp2(x) * (dp[v] - delta);
        if constexpr (CAP) s[v] *= dcap;
      }
      if (!at.full)
        each_pair(m, seen, c, h, [&](int x) { return j0 + x; }, [&](int v, bool see) { s[v] = see ? s[v] : 0.f; });
      const float* sv = reinterpret_cast<const float*>(&s);
      u32x4_t pf[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) pf[u] = pack_frag(sv, u);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) acc[dt] = mfma32(f.tr(xst(SC), dt, u), pf[u], acc[dt]);
    }
    if constexpr (PRIV) {
      __builtin_amdgcn_s_waitcnt(0xC07F);  // the stage is read: its next block may come
      asm volatile("" ::: "memory");
      next(SC);
    }
    return true;
  };
  if constexpr (PRIV) {
    while (iteration(IC<0>{}) && iteration(IC<1>{})) {
    }
  } else {
    while (iteration(IC<0>{}) && iteration(IC<1>{}) && iteration(IC<2>{}) && iteration(IC<3>{})) {
    }
  }
  wait_vmcnt<0>();
  if constexpr (GROUPS > 1) {
    float* buf = reinterpret_cast<float*>(wave == 0 ? xst0 : wave == 1 ? xst1 : wave == 2 ? xst2 : xst3) + lane;
    __syncthreads();
    if (group) leave(acc, buf);
    __syncthreads();
    if (group) return;
    take(acc, buf);
  }
  uint16_t* dst = static_cast<uint16_t*>(a.dq) + orow + 4 * h;
  unsigned bad = 0;  // rows that a masked pair may have spoilt
  const bool masks = has_mask(a);
  if constexpr (PRIV) {
    __shared__ unsigned flags[kWaves];
    float y[NDT][4];
    __syncthreads();
    add_waves(acc, y, [&](int dt) { return reinterpret_cast<float*>(dt == 0 ? xst0 : dt == 1 ? xst1 : dt == 2 ? yst0 : yst1); }, wave, lane);
    const float check = store_quads(w.valid ? dst : nullptr, y, a.scale, wave, a.D);
    const unsigned x = rows_where(masks && w.valid && check != check);
    if (lane == 0) flags[wave] = x;
    __syncthreads();
    if (wave == 0) bad = __builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3]);
  } else {
    const float check = not_finite(acc);
    bad = rows_where(masks && w.valid && check != check);
    if (w.valid) store_row<DP>(dst, acc, a.scale, a.D);
  }
  if (bad == 0 || !keys_spoil(a, m, own, kb, a.ksn)) return;
  const NanColumns<NDT> nan(acc);  // (PRIV: the wavefront's own part's)
  wait_vmcnt<0>();                 // (the rows are written)
  while (bad) {
    const int x = __builtin_ctz(bad);
    bad &= bad - 1;
    single_row(a, m, b, __builtin_amdgcn_readlane(w.i, x), __builtin_amdgcn_readlane(w.head, x),
               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lse), x)),
               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(delta), x)), lane < a.D && (PRIV || nan.template at<0>(x)),
               lane + 64 < a.D && (PRIV || nan.template at<1>(x)));
  }
}

// ---- key side ----
template <int DP, int CAP, bool BIAS, bool PRIV, int GROUPS>
__global__ __launch_bounds__(kThreads* GROUPS, PRIV ? 1 : 2) void dot_dkv_kernel(DotArgs a) {
  using T = SwzTile<DP>;
  constexpr int NT = DP / 16, NDT = DP / 32, SPW = PRIV ? T::instrs : T::instrs / kWaves, kKeys = PRIV ? 32 : 32 * kWaves;
  constexpr int NS = PRIV ? 2 : 4, kInfo = BIAS ? 512 : 256, LPB = 2 * SPW + (BIAS ? 2 : 1);  // loads of a block
  SA_DOT_RING(PRIV ? kWaves : GROUPS, NS);
  constexpr int kCopies = PRIV ? kWaves : GROUPS;
  __shared__ __attribute__((aligned(16))) char info0[kCopies * kInfo], info1[kCopies * kInfo], info2[NS > 2 ? kCopies * kInfo : 16],
      info3[NS > 2 ? kCopies * kInfo : 16];
  const int R = a.G * a.Nq, nkb = (a.Nk + kKeys - 1) / kKeys;
  int64_t unit;
  if (!unit_of(static_cast<int64_t>(a.B) * a.Hkv, static_cast<int64_t>(nkb) * a.ks, unit)) return;
  const int part = static_cast<int>(unit % a.ks);
  unit /= a.ks;
  const int block = static_cast<int>(unit % nkb), bh = static_cast<int>(unit / nkb);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane((tid >> 6) % kWaves), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(tid / kThreads) : 0, base = (PRIV ? wave : group) * T::bytes;
  const DotMask m(a, b);
  auto ist = [&](auto SC) __attribute__((always_inline)) {
    constexpr int X = decltype(SC)::value;
    return to_lds(X == 0 ? info0 : X == 1 ? info1 : X == 2 ? info2 : info3) + base / T::bytes * kInfo;
  };
  const int j0 = block * kKeys + (PRIV ? 0 : 32 * wave), j = j0 + c;
  const DotSpan all(m, block * kKeys, block * kKeys + kKeys - 1), own(m, j0, j0 + 31);
  const Scores<CAP, false> score(a, 0);
  int lo, hi;
  row_blocks(m, all, a.G, R, lo, hi);
  const bool some = j0 < m.L;
  auto seq = block_seq(lo, hi, PRIV ? wave : part, PRIV ? kWaves : a.ks, [&](int blk, bool& live, bool& mine, bool& full) {
    const DotSpan q(m, m.first + div_group(blk * 32, a), m.first + div_group(min(blk * 32 + 32, R) - 1, a));
    live = dot_live(m, q, all);
    mine = some && dot_live(m, q, own);
    full = dot_full(m, q, own);
  });
  // What depends on the lane alone is formed anew in every block: the accumulators and
  // the keys' operands leave no registers for it, and a reload from scratch memory would
  // wait for the block loads issued before it.
  auto lane_anew = [&]() __attribute__((always_inline)) {
    int x = lane;
    asm volatile("" : "+v"(x));
    return x;
  };
  const uint16_t* qb = static_cast<const uint16_t*>(a.q) + b * a.qsb;
  const uint16_t* gb = static_cast<const uint16_t*>(a.dout) + static_cast<int64_t>(b) * a.Nq * a.H * a.D;
  const Stat* stats = stats_of(a, bh);
  const int64_t gsn = static_cast<int64_t>(a.H) * a.D;
  const int qsn2 = static_cast<int>(a.qsn * 2), qsh2 = static_cast<int>(a.qsh * 2), gsn2 = static_cast<int>(gsn * 2);
  auto load = [&](auto SC, int blk) __attribute__((always_inline)) {
    const int i0 = div_group(max(blk, 0) * 32, a), n = blk < 0 ? 0 : min(a.Nq - i0, 33);
    const auto rq = rows_of(qb + i0 * a.qsn, n, a.qsn, (a.H - 1) * a.qsh + a.D), rg = rows_of(gb + i0 * gsn, n, gsn, gsn);
    const auto rs = make_rsrc(stats + max(blk, 0), blk < 0 ? 0 : sizeof(Stat));
    const int ln = lane_anew();
    // Rows of q and dO: the chunk of row 32 blk + p / CH that this lane brings.
#pragma unroll
    for (int x = 0; x < SPW; ++x) {
      const int at = PRIV ? x : x * kWaves + wave, p = 64 * at + ln, row = p / T::CH, ch = (p % T::CH) ^ T::swz(row);
      const int r = max(blk, 0) * 32 + row, i = div_group(r, a), head = hk * a.G + r - i * a.G;
      const bool in = r < R && 8 * ch < a.D;
      load_lds16(rq, xst(SC) + base + 1024 * at, in ? (i - i0) * qsn2 + head * qsh2 + 16 * ch : kFar);
      load_lds16(rg, yst(SC) + base + 1024 * at, in ? (i - i0) * gsn2 + head * a.D * 2 + 16 * ch : kFar);
    }
    // (every wavefront brings the same numbers)
    load_lds4(rs, ist(SC), ln * 4);
    if constexpr (BIAS) load_lds4(rs, ist(SC) + 256, 256 + ln * 4);
  };
  const bool key = j < m.L;
  u32x4_t kf[NT], vf[NT];
  load_row<DP>(kf, static_cast<const uint16_t*>(a.k) + b * a.ksb + (key ? j : 0) * a.ksn + hk * a.ksh, key, a.D, h);
  load_row<DP>(vf, static_cast<const uint16_t*>(a.v) + b * a.vsb + (key ? j : 0) * a.vsn + hk * a.vsh, key, a.D, h);
  const Frags<DP> frag(lane, base);
  DotBlock bq[NS];
  int lead[NS];  // group 0's block: the groups end together
  auto next = [&](auto SC) __attribute__((always_inline)) {
    constexpr int S = decltype(SC)::value;
    bq[S] = seq.next();
    lead[S] = bq[S].blk;
    if constexpr (GROUPS > 1) {
      const DotBlock other = seq.next();
      if (group) bq[S] = other;
    }
    load(SC, bq[S].blk);
  };
  next(IC<0>{});
  next(IC<1>{});
  if constexpr (!PRIV) next(IC<2>{});
  f32x16_t acck[NDT] = {}, accv[NDT] = {};
  auto iteration = [&](auto SC) __attribute__((always_inline)) {
    constexpr int S = decltype(SC)::value;
    const DotBlock at = bq[S];
    if (lead[S] < 0) return false;
    const Frags<DP> f = frag.fresh();
    if constexpr (PRIV) {
      wait_vmcnt<LPB>();
      asm volatile("" ::: "memory");
    } else {
      wait_vmcnt<2 * LPB>();
      lds_barrier_tracked();
      next(IC<(S + 3) % NS>{});
    }
    if (at.mine) {
      const int ln = lane_anew(), jn = j0 + (ln & 31);
      // Bit v: whether the pair of accumulator register v is visible (before the products,
      // where registers are free; rows past the last one have probabilities of 0 as they are).
      unsigned seen = 0;
      auto position = [&](int x) { return m.first + div_group(at.blk * 32 + x, a); };
      if (!at.full) {
        const QueriesSeeing sees(m, jn);
        if constexpr (DP == 64)
          each_pair(m, sees, ln & 31, ln >> 5, position, [&](int v, bool see) { seen |= static_cast<unsigned>(see) << v; });
        else  // (unrolled it spills: 3029 us for 2527 at B=1 H=32 N=8192 D=128, all pairs)
          seen = pairs_seen(m, sees, ln & 31, ln >> 5, position);
      }
      f32x16_t s = mfma32(f.row(xst(SC), 0), kf[0], f32x16_t{}), dp = mfma32(f.row(yst(SC), 0), vf[0], f32x16_t{});
#pragma unroll
      for (int t = 1; t < NT; ++t) {
        s = mfma32(f.row(xst(SC), t), kf[t], s);
        dp = mfma32(f.row(yst(SC), t), vf[t], dp);
      }
      const lds_char* info = ist(SC) + 16 * (ln >> 5);
      const float dj = static_cast<float>(m.first + div_group(at.blk * 32, a) - jn);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4_t lse2 = lds_ld<f32x4_t>(info + 32 * q), delta = lds_ld<f32x4_t>(info + 128 + 32 * q);
        f32x4_t slope2 = {}, query = {};
        if constexpr (BIAS) slope2 = lds_ld<f32x4_t>(info + 256 + 32 * q), query = lds_ld<f32x4_t>(info + 384 + 32 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float dcap = 1.f, x = score_of(score, s[4 * q + e], 0.f, 0.f, lse2[e], dcap);
          if constexpr (BIAS) x = __builtin_fmaf(-slope2[e], fabsf(query[e] + dj), x);
          const float p = fast_exp2(x);
          s[4 * q + e] = p;
          dp[4 * q + e] = p * (dp[4 * q + e] - delta[e]);
          if constexpr (CAP) dp[4 * q + e] *= dcap;
        }
      }
      u32x4_t pf[2], df[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        pf[u] = pack_frag(reinterpret_cast<const float*>(&s), u);
        df[u] = pack_frag(reinterpret_cast<const float*>(&dp), u);
      }
      if (!at.full) {  // masked pairs out of the packed values (fewer registers than before packing)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = 8 * u + 2 * e, lo = __builtin_amdgcn_sbfe(seen, v, 1), hi = __builtin_amdgcn_sbfe(seen, v + 1, 1);
            const unsigned keep = (lo & 0xffffu) | (hi & 0xffff0000u);
            pf[u][e] &= keep;
            df[u][e] &= keep;
          }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          accv[dt] = mfma32(f.tr(yst(SC), dt, u), pf[u], accv[dt]);
          acck[dt] = mfma32(f.tr(xst(SC), dt, u), df[u], acck[dt]);
        }
    }
    if constexpr (PRIV) {
      __builtin_amdgcn_s_waitcnt(0xC07F);  // the stage is read: its next block may come
      asm volatile("" ::: "memory");
      next(SC);
    }
    return true;
  };
  if constexpr (PRIV) {
    while (iteration(IC<0>{}) && iteration(IC<1>{})) {
    }
  } else {
    while (iteration(IC<0>{}) && iteration(IC<1>{}) && iteration(IC<2>{}) && iteration(IC<3>{})) {
    }
  }
  wait_vmcnt<0>();
  if constexpr (GROUPS > 1) {
    float* bk = reinterpret_cast<float*>(wave == 0 ? xst0 : wave == 1 ? xst1 : wave == 2 ? xst2 : xst3) + lane;
    float* bv = reinterpret_cast<float*>(wave == 0 ? yst0 : wave == 1 ? yst1 : wave == 2 ? yst2 : yst3) + lane;
    __syncthreads();
    if (group) leave(acck, bk), leave(accv, bv);
    __syncthreads();
    if (group) return;
    take(acck, bk);
    take(accv, bv);
  }
  // Keys behind the filled length have no visible pair: zeros, whatever their masked pairs' products are.
  if (!key) {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) acck[dt] = f32x16_t{}, accv[dt] = f32x16_t{};
  }
  const bool out = j < a.Nk;
  if (!PRIV && a.ks > 1) {  // partial sums, added by dot_keys_kernel
    if (!out) return;
    const int64_t n = static_cast<int64_t>(a.B) * a.Hkv * a.Nk * a.D;
    float* p = a.part + 2 * part * n + (static_cast<int64_t>(bh) * a.Nk + j) * a.D + 4 * h;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (32 * dt + 8 * q < a.D) {
          *reinterpret_cast<f32x4_t*>(p + 32 * dt + 8 * q) = f32x4_t{acck[dt][4 * q], acck[dt][4 * q + 1], acck[dt][4 * q + 2], acck[dt][4 * q + 3]};
          *reinterpret_cast<f32x4_t*>(p + n + 32 * dt + 8 * q) = f32x4_t{accv[dt][4 * q], accv[dt][4 * q + 1], accv[dt][4 * q + 2], accv[dt][4 * q + 3]};
        }
    return;
  }
  const int64_t at = ((static_cast<int64_t>(b) * a.Nk + (out ? j : 0)) * a.Hkv + hk) * a.D + 4 * h;
  uint16_t *pk = static_cast<uint16_t*>(a.dk) + at, *pv = static_cast<uint16_t*>(a.dv) + at;
  unsigned bad = 0;  // keys, as the rows of the query side
  const bool masks = has_mask(a);
  if constexpr (PRIV) {
    __shared__ unsigned flags[kWaves];
    auto buf = [&](int dt) { return reinterpret_cast<float*>(dt == 0 ? xst0 : dt == 1 ? xst1 : dt == 2 ? yst0 : yst1); };
    float y[NDT][4];
    __syncthreads();
    add_waves(acck, y, buf, wave, lane);
    float check = store_quads(out ? pk : nullptr, y, a.scale, wave, a.D);
    add_waves(accv, y, buf, wave, lane);
    check += store_quads(out ? pv : nullptr, y, 1.f, wave, a.D);
    const unsigned x = rows_where(masks && key && check != check);
    if (lane == 0) flags[wave] = x;
    __syncthreads();
    if (wave == 0) bad = __builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3]);
  } else {
    const float check = not_finite(acck) + not_finite(accv);
    bad = rows_where(masks && key && check != check);
    if (out) {
      store_row<DP>(pk, acck, a.scale, a.D);
      store_row<DP>(pv, accv, 1.f, a.D);
    }
  }
  if (bad == 0 || !queries_spoil(a, m, own, b, hk)) return;
  const NanColumns<NDT> nank(acck), nanv(accv);  // (PRIV: the wavefront's own part's)
  wait_vmcnt<0>();                               // (the keys are written)
  while (bad) {
    const int x = __builtin_ctz(bad);
    bad &= bad - 1;
    const bool d0 = lane < a.D, d1 = lane + 64 < a.D;
    single_key(a, m, b, hk, j0 + x,
               KeyColumns{d0 && (PRIV || nank.template at<0>(x)), d1 && (PRIV || nank.template at<1>(x)), d0 && (PRIV || nanv.template at<0>(x)),
                          d1 && (PRIV || nanv.template at<1>(x))});
  }
}

// dK and dV from the partial sums of a.ks workgroups, a wavefront a key.
__global__ __launch_bounds__(kThreads) void dot_keys_kernel(DotArgs a) {
  const int64_t keys = static_cast<int64_t>(a.B) * a.Hkv * a.Nk, at = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (at >= keys) return;
  const bool d0 = lane < a.D, d1 = lane + 64 < a.D;
  const int64_t n = keys * a.D;
  const float* p = a.part + at * a.D + lane;
  float x0 = 0.f, x1 = 0.f, y0 = 0.f, y1 = 0.f;
  for (int s = 0; s < a.ks; ++s, p += 2 * n) {
    if (d0) x0 += p[0], y0 += p[n];
    if (d1) x1 += p[64], y1 += p[n + 64];
  }
  const int bh = static_cast<int>(at / a.Nk), j = static_cast<int>(at - static_cast<int64_t>(bh) * a.Nk), b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int64_t o = ((static_cast<int64_t>(b) * a.Nk + j) * a.Hkv + hk) * a.D + lane;
  uint16_t *pk = static_cast<uint16_t*>(a.dk) + o, *pv = static_cast<uint16_t*>(a.dv) + o;
  if (d0) pk[0] = f32_to_bf16(x0 * a.scale), pv[0] = f32_to_bf16(y0);
  if (d1) pk[64] = f32_to_bf16(x1 * a.scale), pv[64] = f32_to_bf16(y1);
  const KeyColumns nan{d0 && x0 != x0, d1 && x1 != x1, d0 && y0 != y0, d1 && y1 != y1};
  if (has_mask(a) && __builtin_amdgcn_ballot_w64(nan.k0 || nan.k1 || nan.v0 || nan.v1) != 0) {
    const DotMask m(a, b);
    const int first = j & ~(kDotBlock - 1);
    if (j < m.L && queries_spoil(a, m, DotSpan(m, first, first + kDotBlock - 1), b, hk)) single_key(a, m, b, hk, j, nan);
  }
}

template <int DP, int CAP, bool BIAS>
hipError_t launch(const DotArgs& a, hipStream_t st) {
  const int64_t R = static_cast<int64_t>(a.G) * a.Nq, heads = static_cast<int64_t>(a.B) * a.Hkv;
  const unsigned wide = unit_grid(heads, (R + 127) / 128);
  if (a.nsplit > 0)
    dot_dq_kernel<DP, CAP, BIAS, true, 1><<<unit_grid(heads, (R + 31) / 32), kThreads, 0, st>>>(a);
  else if (a.nsplit == 0)
    dot_dq_kernel<DP, CAP, BIAS, false, 1><<<wide, kThreads, 0, st>>>(a);
  else
    dot_dq_kernel<DP, CAP, BIAS, false, 2><<<wide, 2 * kThreads, 0, st>>>(a);
  const unsigned keys = unit_grid(heads, (a.Nk + 127) / 128 * static_cast<int64_t>(a.ks));
  if (a.kside > 0)
    dot_dkv_kernel<DP, CAP, BIAS, true, 1><<<unit_grid(heads, (a.Nk + 31) / 32), kThreads, 0, st>>>(a);
  else if (a.kside == 0)
    dot_dkv_kernel<DP, CAP, BIAS, false, 1><<<keys, kThreads, 0, st>>>(a);
  else
    dot_dkv_kernel<DP, CAP, BIAS, false, 2><<<keys, 2 * kThreads, 0, st>>>(a);
  if (a.ks > 1) dot_keys_kernel<<<static_cast<unsigned>((heads * a.Nk + kWaves - 1) / kWaves), kThreads, 0, st>>>(a);
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

hipError_t dot_bwd_bf16(const DotArgs& a, hipStream_t st) { return a.D <= 64 ? launch<64>(a, st) : launch<128>(a, st); }

}  // namespace sa
