// What the bf16 dot-product attention kernels share: tiles of 32 rows in LDS and their
// fragments, scores, and the order of the workgroups.
#pragma once

#include "dot_common.h"

#include "simplicial_layers.h"

#include <algorithm>

namespace sa {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kFar = 0x7fffffff;

template <int X>
using IC = std::integral_constant<int, X>;

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);
}

// `n` positions from `p` on, `sn` elements apart, rows of `more` elements.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const uint16_t* p, int n, int64_t sn, int64_t more) {
  const int64_t bytes = n > 0 ? ((n - 1) * sn + more) * 2 : 0;
  return make_rsrc(p, static_cast<unsigned>(bytes < kFar ? bytes : kFar));
}

// How scores are capped. 1 - 2 / (exp(2 x) + 1) is tanh to 2^-23 absolutely, the score then to
// cap 2^-22: up to kCapShort 1/8 of the rounding of P to bf16. Larger caps, whose scores
// mostly lie where tanh is near its argument, take tanhf (B=1 H=16 Hkv=4 N=8192 D=128
// causal, cap 0 / 50 / 2000: forward 313 / 384 / 467 us, backward 1041 / 1229 / 1799).
enum Cap { kNoCap, kShortCap, kLargeCap };
constexpr float kCapShort = 1024.f;

// What scores need beside the products, in base 2: a = mul s without cap and bias.
template <int CAP, bool BIAS>
struct Scores {
  float scale2, to_cap, cap2, slope2;
  float ramp[BIAS ? 16 : 1];  // the bias over a block's keys: slope2 times key 8 (v / 4) + v % 4
  __device__ __forceinline__ Scores(const DotArgs& a, int head)
      : scale2(a.scale * kLog2e), to_cap(CAP == kShortCap ? 2.f * kLog2e * a.scale / a.cap : CAP ? a.scale / a.cap : 0.f),
        cap2(a.cap * kLog2e), slope2(BIAS ? a.slopes[head] * kLog2e : 0.f) {
    if constexpr (BIAS) {
#pragma unroll
      for (int v = 0; v < 16; ++v) ramp[v] = slope2 * static_cast<float>(8 * (v >> 2) + (v & 3));
    }
  }
  // Without the bias; 1 - tanh^2 of the cap.
  __device__ __forceinline__ float capped(float s, float& dcap) const {
    if constexpr (CAP == kShortCap) {
      const float u = __builtin_amdgcn_rcpf(fast_exp2(s * to_cap) + 1.f);  // tanh = 1 - 2 u
      dcap = 4.f * (u - u * u);
      return cap2 - 2.f * cap2 * u;
    } else if constexpr (CAP == kLargeCap) {
      const float t = tanhf(s * to_cap);
      dcap = 1.f - t * t;
      return cap2 * t;
    } else {
      dcap = 1.f;
      return s * scale2;
    }
  }
  // dj: position less the block's first key (of the lane's half).
  __device__ __forceinline__ float operator()(float s, int v, float dj) const {
    float dcap, x = capped(s, dcap);
    if constexpr (BIAS) x = __builtin_fmaf(-slope2, fabsf(dj - static_cast<float>(8 * (v >> 2) + (v & 3))), x);
    return x;
  }
  // The same plus slope2 dj, for a block whose keys are all at or before the query: no
  // distance to form for each.
  __device__ __forceinline__ float behind(float s, int v) const {
    float dcap;
    if constexpr (CAP) return capped(s, dcap) + (BIAS ? ramp[v] : 0.f);
    return __builtin_fmaf(s, scale2, BIAS ? ramp[v] : 0.f);
  }
};
template <typename F>
hipError_t with_cap(float cap, F f) {
  return cap > kCapShort ? f(IC<kLargeCap>{}) : cap > 0.f ? f(IC<kShortCap>{}) : f(IC<kNoCap>{});
}

// The 32 rows of a wavefront, one a lane.
struct Lanes {
  int i, head, p;
  bool valid;
  __device__ __forceinline__ Lanes(const DotArgs& a, const DotMask& m, int hk, int r) {
    valid = r < a.G * a.Nq;
    const int rr = valid ? r : 0;
    i = div_group(rr, a);
    head = hk * a.G + rr - i * a.G;
    p = valid ? m.first + i : -1;
  }
};
__device__ __forceinline__ DotSpan rows_span(const DotArgs& a, const DotMask& m, int r0, int n) {
  return DotSpan(m, m.first + r0 / a.G, m.first + (min(r0 + n, a.G * a.Nq) - 1) / a.G);
}

// A row (of D columns from p on; none: zeros) as a product's operand.
template <int DP>
__device__ __forceinline__ void load_row(u32x4_t (&f)[DP / 16], const uint16_t* p, bool valid, int D, int h) {
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) f[t] = valid && 16 * t + 8 * h < D ? ldg128(p + 16 * t + 8 * h) : u32x4_t{0, 0, 0, 0};
}
__device__ __forceinline__ const uint16_t* q_row(const DotArgs& a, const Lanes& w, int b) {
  return static_cast<const uint16_t*>(a.q) + b * a.qsb + w.i * a.qsn + w.head * a.qsh;
}

// Writes an accumulator's row c times `mul`: 4 consecutive columns of each quad, from
// p on (already + 4 h).
template <int DP>
__device__ __forceinline__ void store_row(uint16_t* p, const f32x16_t (&acc)[DP / 32], float mul, int D) {
#pragma unroll
  for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (32 * dt + 8 * q < D)
        *reinterpret_cast<u32x2_t*>(p + 32 * dt + 8 * q) =
            u32x2_t{pack_bf16x2(acc[dt][4 * q] * mul, acc[dt][4 * q + 1] * mul), pack_bf16x2(acc[dt][4 * q + 2] * mul, acc[dt][4 * q + 3] * mul)};
}
// What rounding to bf16 takes from x (not a number's: nothing).
__device__ __forceinline__ float rounded_off(float x) {
  const float d = x - bf16_to_f32(f32_to_bf16(x));
  return d == d ? d : 0.f;
}
template <int DP>
__device__ __forceinline__ void store_row_lo(uint16_t* p, const f32x16_t (&acc)[DP / 32], float mul, int D) {
#pragma unroll
  for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (32 * dt + 8 * q < D)
        *reinterpret_cast<u32x2_t*>(p + 32 * dt + 8 * q) =
            u32x2_t{pack_bf16x2(rounded_off(acc[dt][4 * q] * mul), rounded_off(acc[dt][4 * q + 1] * mul)),
                    pack_bf16x2(rounded_off(acc[dt][4 * q + 2] * mul), rounded_off(acc[dt][4 * q + 3] * mul))};
}
// NaN if any of a lane's accumulators is an infinity or NaN, else 0.
template <int NDT>
__device__ __forceinline__ float not_finite(const f32x16_t (&acc)[NDT]) {
  float x = 0.f;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) x += acc[dt][v] * 0.f;
  return x;
}
// The rows (bits 0 .. 31) for which either half's lane says so.
__device__ __forceinline__ unsigned rows_where(bool x) {
  const unsigned long long b = __builtin_amdgcn_ballot_w64(x);
  return static_cast<unsigned>(b) | static_cast<unsigned>(b >> 32);
}

// A masked pair's weight of 0 times an infinity or NaN of the tile it is multiplied with is NaN:
// where a row (key) with masks comes out so, the tiles of its wavefront's blocks with masked pairs are
// looked over, and only if one of them holds such a value are its columns that are NaN formed again,
// over the visible pairs alone. (Values that are visible are none's fault: B=1 H=16 Hkv=4 N=4096 D=128
// causal with an infinity in the first row of V 0.16 ms, without 0.12; forming every such row again 100.)
template <typename Row>
__device__ __forceinline__ bool rows_not_finite(int n, int D, Row row) {
  const int per = D / 8;  // 16-byte chunks of a row
  bool bad = false;
  for (int at = threadIdx.x & 63; at < n * per; at += 64) {
    const u32x4_t x = ldg128(row(at / per) + 8 * (at % per));
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
  }
  return __builtin_amdgcn_ballot_w64(bad) != 0;
}
// Of k or v (a head's rows from x on, sn apart), for the 32 rows of span q.
__device__ __forceinline__ bool keys_spoil(const DotArgs& a, const DotMask& m, const DotSpan& q, const uint16_t* x, int64_t sn) {
  int lo, hi;
  key_blocks(m, q, lo, hi);
  bool bad = false;
  walk_blocks(
      lo, hi, 0, 1,
      [&](int blk, bool& live, bool& full) {
        const DotSpan k(m, blk * kDotBlock, blk * kDotBlock + kDotBlock - 1);
        live = dot_live(m, q, k) && !dot_full(m, q, k);
        full = false;
      },
      [&](int blk, bool) {
        const int j0 = blk * kDotBlock;
        if (!bad) bad = rows_not_finite(min(m.L - j0, kDotBlock), a.D, [&](int r) { return x + (j0 + r) * sn; });
      });
  return bad;
}
// Of q and dO, for the 32 keys of span k.
__device__ __forceinline__ bool queries_spoil(const DotArgs& a, const DotMask& m, const DotSpan& k, int b, int hk) {
  const int R = a.G * a.Nq;
  int lo, hi;
  row_blocks(m, k, a.G, R, lo, hi);
  bool bad = false;
  walk_blocks(
      lo, hi, 0, 1,
      [&](int blk, bool& live, bool& full) {
        const DotSpan q(m, m.first + div_group(blk * 32, a), m.first + div_group(min(blk * 32 + 32, R) - 1, a));
        live = dot_live(m, q, k) && !dot_full(m, q, k);
        full = false;
      },
      [&](int blk, bool) {
        const int r0 = blk * kDotBlock, n = min(R - r0, kDotBlock);
        auto at = [&](const void* x, int r, int64_t sb, int64_t sn, int64_t sh) {
          const int i = div_group(r0 + r, a);
          return static_cast<const uint16_t*>(x) + b * sb + i * sn + (hk * a.G + r0 + r - i * a.G) * sh;
        };
        if (!bad) bad = rows_not_finite(n, a.D, [&](int r) { return at(a.q, r, a.qsb, a.qsn, a.qsh); });
        const int64_t sn = static_cast<int64_t>(a.H) * a.D;
        if (!bad) bad = rows_not_finite(n, a.D, [&](int r) { return at(a.dout, r, a.Nq * sn, sn, a.D); });
      });
  return bad;
}
// Which columns of the wavefront's 32 rows are NaN in an accumulator, a bit for each of a lane's.
template <int NDT>
struct NanColumns {
  unsigned w[NDT / 2];
  __device__ __forceinline__ explicit NanColumns(const f32x16_t (&acc)[NDT]) {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
      if (dt % 2 == 0) w[dt / 2] = 0;
#pragma unroll
      for (int v = 0; v < 16; ++v) w[dt / 2] |= static_cast<unsigned>(acc[dt][v] != acc[dt][v]) << (16 * (dt % 2) + v);
    }
  }
  // Column (lane + 64 K) of row x.
  template <int K>
  __device__ __forceinline__ bool at(int x) const {
    if constexpr (K >= NDT / 2) return false;
    else {
      const int d = threadIdx.x & 63, v = 4 * ((d & 31) >> 3) + (d & 3);
      const unsigned lo = __builtin_amdgcn_readlane(w[K], x), hi = __builtin_amdgcn_readlane(w[K], x + 32);
      return (((d & 4) ? hi : lo) >> (16 * (d >> 5) + v)) & 1;
    }
  }
};

__device__ __forceinline__ bool has_mask(const DotArgs& a) { return a.causal || a.window || a.prefix || a.docs || a.lens; }

// A tile's fragments. Row fragment t of lane (h, c) is chunk 2 t + h of row c, at slot
// (2 t + h) ^ swz(c): the offset of t = 0 with 32 t exclusive-or'ed in. A transposed
// fragment's two reads are at rows r and r + 8 (whose swz differ by 2), columns 32 dt
// on: one offset with 64 dt, and with 32 besides, exclusive-or'ed in. So two registers
// hold them all; fresh() is called once a block and keeps them from being expanded
// into sixteen that live through the loop.
template <int DP>
struct Frags {
  using T = SwzTile<DP>;
  int ko, vo;
  __device__ __forceinline__ Frags(int lane, int base) {
    const int c = lane & 31, h = lane >> 5, grp = lane >> 4, sl = lane & 15;
    ko = base + T::off(c, h);
    const int col = 16 * (grp & 1) + 4 * (sl & 3);
    vo = base + T::off(4 * (grp >> 1) + (sl >> 2), col >> 3) + (col & 7) * 2;
  }
  __device__ __forceinline__ Frags fresh() const {
    Frags f = *this;
    asm volatile("" : "+v"(f.ko), "+v"(f.vo));
    return f;
  }
  __device__ __forceinline__ u32x4_t row(const lds_char* tile, int t) const { return lds_ld<u32x4_t>(tile + (ko ^ (32 * t))); }
  __device__ __forceinline__ u32x4_t tr(const lds_char* tile, int dt, int u) const {
    const lds_char* p = tile + 2 * DP * 16 * u;
    const u32x2_t x = lds_tr16(p + (vo ^ (64 * dt))), y = lds_tr16(p + 16 * DP + (vo ^ (64 * dt) ^ 32));
    return u32x4_t{x[0], x[1], y[0], y[1]};
  }
};

}  // namespace
}  // namespace sa
