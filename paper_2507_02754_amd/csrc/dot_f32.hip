// Dot-product attention in float32 arithmetic on the gfx950 matrix cores
// (v_mfma_f32_32x32x2_f32).
//
//     s = scale q k;  a = cap tanh(s / cap) - slope |p - j|;  O = softmax(a) v
//     dA = P (dO v - Delta);  dS = dA (1 - tanh^2);  dq = scale dS k, ...
//
// A workgroup owns 32 rows (forward, dq) or 32 keys (dk, dv) of one K-side head; its
// wavefronts (4 or 8) take every 4th or 8th block of 32 keys (rows) that holds a visible pair
// and add their sums at the end in a fixed order. A block's products S^T = K Q^T put
// one row in each lane, so the softmax statistics are the lane's own and the
// probabilities go into the next product's operand as they are. Matrix operands come
// from L1 / L2 straight into registers: at 1/16 of the bf16 rate the products, not
// the loads, take the time.
//
// Measured, B=1 H=4 N=2000 D=64 causal with a prefix of 200: forward 42 us, dq 71, dk and dv
// 115, 32 TFLOP/s of the 7.2 GFLOP that forward and backward need (a large product of the
// library's runs at 154). With 252 workgroups of rows and of keys, the longest one's walk of
// dependent products is the time, on the key side with 107 registers spilled (both row operands and a
// column operand at once). One token over 8 caches of up to 16384 keys, 4 heads of 128: 121 us (2.8 TB/s) and 13
// to join; N=3000 H=8 D=128: 277 us forward, 852 backward (67 and 54 TFLOP/s).
//
// Each block's products start from zero and are added to the running sums, so that
// sums over a long axis round once per 32 terms. Operand layouts as in f32.hip: a row
// operand's float4 t holds columns 8 t + 4 h .. + 3 of row c; product v of a
// transposed one contracts rows acc_row(v, 0) and acc_row(v, 1).
//
// A block with masked pairs whose products come out infinite or NaN is added again
// term by term without the masked pairs: their probability of 0 times such a value
// is not 0.
#include "dot_common.h"

#include "simplicial_layers.h"

#include <algorithm>

namespace sa {
namespace {

// Wavefronts of a backward workgroup: two for each SIMD where their registers allow it
// (one takes the other's load latency).
template <int D>
constexpr int kWavesOf = D <= 64 ? 8 : 4;
constexpr int kFar = 0x7fffffff;  // an offset past every buffer's end

__device__ __forceinline__ f32x16_t mfma_f32(float a, float b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
struct F4 {
  float x[4];
};
__device__ __forceinline__ F4 ld4(__amdgpu_buffer_rsrc_t r, int off) {
  const u32x4_t a = ldbuf128(r, off);
  return F4{{__uint_as_float(a[0]), __uint_as_float(a[1]), __uint_as_float(a[2]), __uint_as_float(a[3])}};
}
__device__ __forceinline__ float ld1(__amdgpu_buffer_rsrc_t r, int off) { return __uint_as_float(ldbuf32(r, off)); }
__device__ __forceinline__ void st4(float* p, const float* x) {
  *reinterpret_cast<u32x4_t*>(p) = u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

template <int D>
struct Geo {
  static constexpr int NF = D / 8;                 // float4s of a row operand per lane
  static constexpr int NDT = D < 32 ? 1 : D / 32;  // accumulator tiles over the columns
  static constexpr int NV = D < 32 ? 8 : 16;       // accumulator registers that hold a column
};

// `n` positions from `p` on, `sn` elements apart, whose rows reach `more` elements past
// the last position: the buffer that a block's loads go through (what lies
// behind it loads as zeros).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const float* p, int n, int64_t sn, int64_t more) {
  const int64_t bytes = n > 0 ? ((n - 1) * sn + more) * static_cast<int64_t>(sizeof(float)) : 0;
  return make_rsrc(p, static_cast<unsigned>(bytes < kFar ? bytes : kFar));
}
// One row in every lane: its float4s of columns 8 t + 4 h.
template <int D>
struct RowOp {
  F4 f[Geo<D>::NF];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int off, int h) {
#pragma unroll
    for (int t = 0; t < Geo<D>::NF; ++t)
      f[t] = ld4(r, off == kFar ? kFar : off + (8 * t + 4 * h) * 4);
  }
};
// a's rows times b's rows, contracted over the columns, in two chains added at the end
// (the rounding of one chain of D is the largest error of a score).
template <int D>
__device__ __forceinline__ f32x16_t row_product(const RowOp<D>& a, const RowOp<D>& b) {
  f32x16_t x = {}, y = {};
#pragma unroll
  for (int t = 0; t < Geo<D>::NF / 2; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x = mfma_f32(a.f[t].x[e], b.f[t].x[e], x);
      y = mfma_f32(a.f[t + Geo<D>::NF / 2].x[e], b.f[t + Geo<D>::NF / 2].x[e], y);
    }
#pragma unroll
  for (int v = 0; v < 16; ++v) x[v] += y[v];
  return x;
}

// The block's 32 rows by columns: lane (h, c) holds column 32 dt + c of rows acc_row(v, h).
// off(x) is row x's byte offset in the buffer.
template <int D>
struct ColOp {
  float x[Geo<D>::NDT][16];
  template <typename Off>
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, Off off, int c, int h) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int o = off(acc_row(v, h));
#pragma unroll
      for (int dt = 0; dt < Geo<D>::NDT; ++dt) {
        x[dt][v] = ld1(r, o == kFar ? kFar : o + (32 * dt + (D < 32 ? c & (D - 1) : c)) * 4);
        if (D < 32 && c >= D) x[dt][v] = 0.f;
      }
    }
  }
};
// Adds the sum of the block's rows x weighted with w (accumulator order). `masked`: pairs of
// bit v of `seen` zero are left out where the products are not finite.
template <int D, typename Off>
__device__ __forceinline__ void weighted_rows(f32x16_t (&acc)[Geo<D>::NDT], const float* w, const ColOp<D>& cols,
                                              __amdgpu_buffer_rsrc_t r, Off off, int c, int h, bool masked, unsigned seen, float* scratch) {
  constexpr int S = 4;
#pragma unroll
  for (int dt = 0; dt < Geo<D>::NDT; ++dt) {
    f32x16_t u = {};
#pragma unroll
    for (int v = 0; v < 16; ++v) u = mfma_f32(cols.x[dt][v], w[v], u);
    if (masked) {
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) sum += u[v];
      if (__builtin_amdgcn_ballot_w64(!(fabsf(sum) < kInf)) != 0) {
        u = f32x16_t{};
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          scratch[acc_row(v, h) * 33 + c] = (seen >> v) & 1 ? w[v] : __builtin_nanf("");
          // (whether the pair is visible beside it: NaN may be a weight)
          reinterpret_cast<unsigned*>(scratch)[32 * 33 + acc_row(v, h) * 33 + c] = (seen >> v) & 1;
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int x = 0; x < 32; ++x) {
          const float wx = scratch[x * 33 + c];
          const bool use = reinterpret_cast<unsigned*>(scratch)[32 * 33 + x * 33 + c] != 0;
          const int o = off(x);
#pragma unroll
          for (int vq = 0; vq < Geo<D>::NV / 4; ++vq) {
            const F4 y = ld4(r, o == kFar ? kFar : o + (32 * dt + 8 * vq + 4 * h) * S);
#pragma unroll
            for (int e = 0; e < 4; ++e) u[4 * vq + e] += use ? wx * y.x[e] : 0.f;
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[dt][v] += u[v];
  }
}
constexpr int kScratch = 2 * 32 * 33;

// Score a of a product s, and its derivative by the cap, 1 - tanh^2.
struct Score {
  float scale, cap, inv_cap;
  __device__ __forceinline__ explicit Score(const DotArgs& a) : scale(a.scale), cap(a.cap), inv_cap(a.cap > 0.f ? 1.f / a.cap : 0.f) {}
  __device__ __forceinline__ float operator()(float s, float slope, int distance, float& dcap) const {
    float x = s * scale;
    dcap = 1.f;
    if (cap > 0.f) {
      const float t = tanhf(x * inv_cap);
      x = cap * t;
      dcap = 1.f - t * t;
    }
    return x - slope * static_cast<float>(distance);
  }
};

// Adds the wavefronts' accumulators in order: afterwards wavefront w holds the sum's
// tile w, if there is one (the others' are left as they were). `lds`: kWaves NDT 1024 floats.
template <int kWaves, int NDT>
__device__ __forceinline__ void add_waves(f32x16_t (&acc)[NDT], float* lds, int wave, int lane) {
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) lds[((wave * NDT + dt) * 16 + v) * 64 + lane] = acc[dt][v];
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
    if (dt % kWaves != wave) continue;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) x += lds[((w * NDT + dt) * 16 + v) * 64 + lane];
      acc[dt][v] = x;
    }
  }
  __syncthreads();
}

// The 32 rows of a workgroup (forward and dq): row c of every lane.
struct Rows {
  int i0, i, head, p;  // first query; the lane's query, query head and position (-1: no row)
  bool valid;
  DotSpan span;
  __device__ __forceinline__ Rows(const DotArgs& a, const DotMask& m, int hk, int block, int c)
      : span(m, m.first + block * kDotBlock / a.G, m.first + (min(block * kDotBlock + kDotBlock, a.G * a.Nq) - 1) / a.G) {
    const int r = block * kDotBlock + c;
    valid = r < a.G * a.Nq;
    i0 = block * kDotBlock / a.G;
    i = r / a.G;
    head = hk * a.G + r - i * a.G;
    p = valid ? m.first + i : -1;
  }
};

template <int D>
__global__ __launch_bounds__(256, D <= 64 ? 2 : 1) void dot_fwd_f32_kernel(DotArgs a) {
  constexpr int NDT = Geo<D>::NDT, S = 4, kWaves = 4;
  __shared__ float lds[kWaves * NDT * 1024 > kWaves * kScratch ? kWaves * NDT * 1024 : kWaves * kScratch];
  __shared__ float stat[2][kWaves][32];
  const int nrb = (a.G * a.Nq + kDotBlock - 1) / kDotBlock;
  int64_t unit;
  if (!unit_of(static_cast<int64_t>(a.B) * a.Hkv, static_cast<int64_t>(nrb) * a.nsplit, unit)) return;
  const int part = static_cast<int>(unit % a.nsplit);
  unit /= a.nsplit;
  const int block = nrb - 1 - static_cast<int>(unit % nrb), bh = static_cast<int>(unit / nrb);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const DotMask m(a, b);
  const Rows row(a, m, hk, block, c);
  const KeysSeen sees(m, row.p);
  const float slope = a.slopes ? a.slopes[row.valid ? row.head : 0] : 0.f;
  const Score score(a);
  RowOp<D> q;
  {
    const auto r = rows_of(static_cast<const float*>(a.q) + b * a.qsb + row.i0 * a.qsn, a.Nq - row.i0, a.qsn, (a.H - 1) * a.qsh + D);
    q.load(r, row.valid ? static_cast<int>(((row.i - row.i0) * a.qsn + row.head * a.qsh) * S) : kFar, h);
  }
  const float* kb = static_cast<const float*>(a.k) + b * a.ksb + hk * a.ksh;
  const float* vb = static_cast<const float*>(a.v) + b * a.vsb + hk * a.vsh;
  f32x16_t acc[NDT] = {};
  float mx = -kInf, l = 0.f;
  int lo, hi;
  key_blocks(m, row.span, lo, hi);
  walk_blocks(
      lo, hi, part * kWaves + wave, kWaves * a.nsplit,
      [&](int blk, bool& live, bool& full) {
        const DotSpan k(m, blk * kDotBlock, blk * kDotBlock + kDotBlock - 1);
        live = dot_live(m, row.span, k);
        full = dot_full(m, row.span, k);
      },
      [&](int blk, bool full) {
        const int j0 = blk * kDotBlock;
        RowOp<D> k;
        k.load(rows_of(kb + j0 * a.ksn, m.L - j0, a.ksn, D), static_cast<int>(c * a.ksn * S), h);
        const auto rv = rows_of(vb + j0 * a.vsn, m.L - j0, a.vsn, D);
        auto voff = [&](int y) { return static_cast<int>(y * a.vsn * S); };
        ColOp<D> vt;  // (on its way while the scores are formed)
        vt.load(rv, voff, c, h);
        __builtin_amdgcn_sched_barrier(0);
        const f32x16_t s = row_product(k, q);
        float x[16], top = -kInf;
        unsigned seen = 0;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int j = j0 + acc_row(v, h);
          float unused;
          x[v] = score(s[v], slope, abs(row.p - j), unused);
        }
        if (!full)
          each_pair(m, sees, c, h, [&](int y) { return j0 + y; }, [&](int v, bool see) {
            seen |= static_cast<unsigned>(see) << v;
            x[v] = see ? x[v] : -kInf;
          });
#pragma unroll
        for (int v = 0; v < 16; ++v) top = fmaxf(top, x[v]);
        top = fmaxf(mx, fmaxf(top, swap_halves(top)));
        const float base = top == -kInf ? 0.f : top, down = fast_exp2((mx - base) * kLog2e);
        mx = top;
        l *= down;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          x[v] = fast_exp2((x[v] - base) * kLog2e);
          l += x[v];
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[dt][v] *= down;
        weighted_rows<D>(acc, x, vt, rv, voff, c, h, !full, seen, lds + wave * kScratch);
      });
  l += swap_halves(l);
  if (h == 0) stat[0][wave][c] = mx, stat[1][wave][c] = l;
  __syncthreads();
  float top = -kInf;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[0][w][c]);
  const float base = top == -kInf ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += stat[1][w][c] * fast_exp2((stat[0][w][c] - base) * kLog2e);
  const float down = fast_exp2((mx - base) * kLog2e);
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[dt][v] *= down;
  add_waves<kWaves>(acc, lds, wave, lane);
  if (!row.valid) return;
  const float scale = a.nsplit > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
  const int64_t r = static_cast<int64_t>(bh) * a.G * a.Nq + block * kDotBlock + c;
  float* pr = a.part + (r * a.nsplit + part) * D;
  float* out = static_cast<float*>(a.out) + ((static_cast<int64_t>(b) * a.Nq + row.i) * a.H + row.head) * D;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
    if (dt % kWaves != wave) continue;
#pragma unroll
    for (int vq = 0; vq < Geo<D>::NV / 4; ++vq) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = scale == 0.f ? 0.f : acc[dt][4 * vq + e] * scale;
      if (a.nsplit > 1)
        st4(pr + 32 * dt + 8 * vq + 4 * h, y);
      else
        st4(out + 32 * dt + 8 * vq + 4 * h, y);
    }
  }
  if (wave == 0 && h == 0) {
    if (a.nsplit > 1) {
      float* st = a.part + static_cast<int64_t>(a.B) * a.H * a.Nq * a.nsplit * D + (r * a.nsplit + part) * 2;
      st[0] = top, st[1] = sum;
    } else {
      a.lse[(static_cast<int64_t>(b) * a.H + row.head) * a.Nq + row.i] = sum == 0.f ? -kInf : top + logf(sum);
    }
  }
}

// Joins the parts of a row: one thread a column.
__global__ void dot_join_kernel(DotArgs a) {
  const int rows = blockDim.x / a.D;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * rows + threadIdx.x / a.D, all = static_cast<int64_t>(a.B) * a.H * a.Nq;
  const int d = threadIdx.x % a.D;
  if (r >= all) return;
  const float* st = a.part + all * a.nsplit * a.D + r * a.nsplit * 2;
  float top = -kInf;
  for (int s = 0; s < a.nsplit; ++s) top = fmaxf(top, st[2 * s]);
  const float base = top == -kInf ? 0.f : top;
  float l = 0.f, x = 0.f;
  for (int s = 0; s < a.nsplit; ++s) {
    const float w = fast_exp2((st[2 * s] - base) * kLog2e);
    l += w * st[2 * s + 1];
    // (a part without a visible key holds zeros)
    x += w * a.part[(r * a.nsplit + s) * a.D + d];
  }
  const int64_t rh = static_cast<int64_t>(a.G) * a.Nq;
  const int bh = static_cast<int>(r / rh), rr = static_cast<int>(r - bh * rh), i = rr / a.G;
  const int b = bh / a.Hkv, head = (bh - b * a.Hkv) * a.G + rr - i * a.G;
  const float y = l == 0.f ? 0.f : x / l;
  float* out = static_cast<float*>(a.out) + ((static_cast<int64_t>(b) * a.Nq + i) * a.H + head) * a.D + d;
  *out = y;
  if (d == 0) a.lse[(static_cast<int64_t>(b) * a.H + head) * a.Nq + i] = l == 0.f ? -kInf : top + logf(l);
}

// Probability of a score; of a row without a key: 0.
__device__ __forceinline__ float prob(float x, float lse) { return lse == -kInf ? 0.f : fast_exp2((x - lse) * kLog2e); }

template <int D>
__global__ __launch_bounds__(64 * kWavesOf<D>, D <= 64 ? 2 : 1) void dot_dq_f32_kernel(DotArgs a) {
  constexpr int NDT = Geo<D>::NDT, S = 4, kWaves = kWavesOf<D>;
  __shared__ float lds[kWaves * NDT * 1024 > kWaves * kScratch ? kWaves * NDT * 1024 : kWaves * kScratch];
  const int nrb = (a.G * a.Nq + kDotBlock - 1) / kDotBlock;
  int64_t unit;
  if (!unit_of(static_cast<int64_t>(a.B) * a.Hkv, nrb, unit)) return;
  const int block = nrb - 1 - static_cast<int>(unit % nrb), bh = static_cast<int>(unit / nrb);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const DotMask m(a, b);
  const Rows row(a, m, hk, block, c);
  const KeysSeen sees(m, row.p);
  const float slope = a.slopes ? a.slopes[row.valid ? row.head : 0] : 0.f;
  const Score score(a);
  RowOp<D> q, g;
  float delta = 0.f;
  const int64_t orow = static_cast<int64_t>(a.H) * D;
  const int off = row.valid ? static_cast<int>(((row.i - row.i0) * orow + row.head * D) * S) : kFar;
  {
    const auto r = rows_of(static_cast<const float*>(a.q) + b * a.qsb + row.i0 * a.qsn, a.Nq - row.i0, a.qsn, (a.H - 1) * a.qsh + D);
    q.load(r, row.valid ? static_cast<int>(((row.i - row.i0) * a.qsn + row.head * a.qsh) * S) : kFar, h);
    const int64_t at = (static_cast<int64_t>(b) * a.Nq + row.i0) * orow;
    g.load(rows_of(static_cast<const float*>(a.dout) + at, a.Nq - row.i0, orow, orow), off, h);
    RowOp<D> o;
    o.load(rows_of(static_cast<const float*>(a.out_in) + at, a.Nq - row.i0, orow, orow), off, h);
    delta = diagonal(row_product(o, g), c, h);
  }
  const int64_t srow = row.valid ? (static_cast<int64_t>(b) * a.H + row.head) * a.Nq + row.i : 0;
  const float lse = row.valid ? a.lse[srow] : -kInf;
  if (row.valid && wave == 0 && h == 0) a.delta[srow] = delta;
  const float* kb = static_cast<const float*>(a.k) + b * a.ksb + hk * a.ksh;
  const float* vb = static_cast<const float*>(a.v) + b * a.vsb + hk * a.vsh;
  f32x16_t acc[NDT] = {};
  int lo, hi;
  key_blocks(m, row.span, lo, hi);
  walk_blocks(
      lo, hi, wave, kWaves,
      [&](int blk, bool& live, bool& full) {
        const DotSpan k(m, blk * kDotBlock, blk * kDotBlock + kDotBlock - 1);
        live = dot_live(m, row.span, k);
        full = dot_full(m, row.span, k);
      },
      [&](int blk, bool full) {
        const int j0 = blk * kDotBlock;
        const auto rk = rows_of(kb + j0 * a.ksn, m.L - j0, a.ksn, D);
        auto koff = [&](int y) { return static_cast<int>(y * a.ksn * S); };
        // At head_dim 128, with one wavefront a SIMD and registers to spare, operands are loaded a
        // product ahead (527 -> 372 us at B=1 H=8 N=3000; at 64 it spills, 73 -> 78 us at H=4 N=2000).
        constexpr bool kAhead = D > 64;
        const auto rv = rows_of(vb + j0 * a.vsn, m.L - j0, a.vsn, D);
        const int voff = static_cast<int>(c * a.vsn * S);
        RowOp<D> k, v;
        ColOp<D> kt;
        k.load(rk, koff(c), h);
        if constexpr (kAhead) {
          v.load(rv, voff, h);
          __builtin_amdgcn_sched_barrier(0);
        }
        const f32x16_t s = row_product(k, q);
        if constexpr (kAhead) {
          kt.load(rk, koff, c, h);
          __builtin_amdgcn_sched_barrier(0);
        } else {
          v.load(rv, voff, h);
        }
        const f32x16_t dp = row_product(v, g);
        if constexpr (!kAhead) kt.load(rk, koff, c, h);
        float x[16];
        unsigned seen = 0;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int j = j0 + acc_row(v, h);
          float dcap;
          const float p = prob(score(s[v], slope, abs(row.p - j), dcap), lse);
          x[v] = p * (dp[v] - delta) * dcap * a.scale;
        }
        if (!full)
          each_pair(m, sees, c, h, [&](int y) { return j0 + y; }, [&](int v, bool see) {
            seen |= static_cast<unsigned>(see) << v;
            x[v] = see ? x[v] : 0.f;
          });
        weighted_rows<D>(acc, x, kt, rk, koff, c, h, !full, seen, lds + wave * kScratch);
      });
  __syncthreads();
  add_waves<kWaves>(acc, lds, wave, lane);
  if (!row.valid) return;
  float* dst = static_cast<float*>(a.dq) + ((static_cast<int64_t>(b) * a.Nq + row.i) * a.H + row.head) * D;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
    if (dt % kWaves != wave) continue;
#pragma unroll
    for (int vq = 0; vq < Geo<D>::NV / 4; ++vq) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = acc[dt][4 * vq + e];
      st4(dst + 32 * dt + 8 * vq + 4 * h, y);
    }
  }
}

// What a row block's 32 rows are, one wavefront's copy in LDS.
struct RowInfo {
  int p[32], qoff[32], goff[32];
  float lse[32], delta[32], slope[32];
};

template <int D>
__global__ __launch_bounds__(64 * kWavesOf<D>, D <= 64 ? 2 : 1) void dot_dkv_f32_kernel(DotArgs a) {
  constexpr int NDT = Geo<D>::NDT, S = 4, kWaves = kWavesOf<D>;
  __shared__ float lds[kWaves * NDT * 1024 > kWaves * kScratch ? kWaves * NDT * 1024 : kWaves * kScratch];
  __shared__ RowInfo infos[kWaves];
  const int nkb = (a.Nk + kDotBlock - 1) / kDotBlock;
  int64_t unit;
  if (!unit_of(static_cast<int64_t>(a.B) * a.Hkv, nkb, unit)) return;
  const int block = static_cast<int>(unit % nkb), bh = static_cast<int>(unit / nkb);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const DotMask m(a, b);
  const Score score(a);
  RowInfo& info = infos[wave];
  const int j0 = block * kDotBlock, j = j0 + c, R = a.G * a.Nq;
  const DotSpan span(m, j0, j0 + kDotBlock - 1);
  const QueriesSeeing sees(m, j);
  RowOp<D> k, v;
  k.load(rows_of(static_cast<const float*>(a.k) + b * a.ksb + hk * a.ksh + j0 * a.ksn, m.L - j0, a.ksn, D), static_cast<int>(c * a.ksn * S), h);
  v.load(rows_of(static_cast<const float*>(a.v) + b * a.vsb + hk * a.vsh + j0 * a.vsn, m.L - j0, a.vsn, D), static_cast<int>(c * a.vsn * S), h);
  const float* qb = static_cast<const float*>(a.q) + b * a.qsb;
  const int64_t orow = static_cast<int64_t>(a.H) * D;
  f32x16_t acck[NDT] = {}, accv[NDT] = {};
  int lo, hi;
  row_blocks(m, span, a.G, R, lo, hi);
  walk_blocks(
      lo, hi, wave, kWaves,
      [&](int blk, bool& live, bool& full) {
        const int r1 = min(blk * kDotBlock + kDotBlock, R) - 1;
        const DotSpan q(m, m.first + blk * kDotBlock / a.G, m.first + r1 / a.G);
        live = dot_live(m, q, span);
        full = dot_full(m, q, span);
      },
      [&](int blk, bool full) {
        const int r = blk * kDotBlock + c, i0 = blk * kDotBlock / a.G, i = r / a.G, head = hk * a.G + r - i * a.G;
        const bool valid = r < R;
        const int p = valid ? m.first + i : -1;
        const int64_t srow = valid ? (static_cast<int64_t>(b) * a.H + head) * a.Nq + i : 0;
        const int qoff = valid ? static_cast<int>(((i - i0) * a.qsn + head * a.qsh) * S) : kFar;
        const int goff = valid ? static_cast<int>(((i - i0) * orow + head * D) * S) : kFar;
        if (h == 0) {
          info.p[c] = p;
          info.qoff[c] = qoff;
          info.goff[c] = goff;
          info.lse[c] = valid ? a.lse[srow] : -kInf;
          info.delta[c] = valid ? a.delta[srow] : 0.f;
          info.slope[c] = a.slopes && valid ? a.slopes[head] : 0.f;
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_wave_barrier();
        const auto rq = rows_of(qb + i0 * a.qsn, a.Nq - i0, a.qsn, (a.H - 1) * a.qsh + D);
        const auto rg = rows_of(static_cast<const float*>(a.dout) + (static_cast<int64_t>(b) * a.Nq + i0) * orow, a.Nq - i0, orow, orow);
        auto qat = [&](int y) { return info.qoff[y]; };
        auto gat = [&](int y) { return info.goff[y]; };
        RowOp<D> q, g;
        q.load(rq, qoff, h);
        g.load(rg, goff, h);
        __builtin_amdgcn_sched_barrier(0);
        const f32x16_t s = row_product(q, k);
        ColOp<D> t;
        t.load(rg, gat, c, h);
        __builtin_amdgcn_sched_barrier(0);
        const f32x16_t dp = row_product(g, v);
        float x[16], w[16];
        unsigned seen = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int y = acc_row(e, h);
          float dcap;
          w[e] = prob(score(s[e], info.slope[y], abs(info.p[y] - j), dcap), info.lse[y]);
          x[e] = w[e] * (dp[e] - info.delta[y]) * dcap * a.scale;
        }
        if (!full)
          each_pair(m, sees, c, h, [&](int y) { return info.p[y]; }, [&](int e, bool see) {
            seen |= static_cast<unsigned>(see) << e;
            w[e] = see ? w[e] : 0.f;
            x[e] = see ? x[e] : 0.f;
          });
        // (rows past the last query load as zeros, with probabilities of 0)
        weighted_rows<D>(accv, w, t, rg, gat, c, h, !full, seen, lds + wave * kScratch);
        t.load(rq, qat, c, h);
        weighted_rows<D>(acck, x, t, rq, qat, c, h, !full, seen, lds + wave * kScratch);
        __builtin_amdgcn_wave_barrier();
      });
  __syncthreads();
  add_waves<kWaves>(accv, lds, wave, lane);
  add_waves<kWaves>(acck, lds, wave, lane);
  if (j >= a.Nk) return;
  const int64_t at = ((static_cast<int64_t>(b) * a.Nk + j) * a.Hkv + hk) * D;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) {
    if (dt % kWaves != wave) continue;
#pragma unroll
    for (int vq = 0; vq < Geo<D>::NV / 4; ++vq) {
      float y[4], z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = acck[dt][4 * vq + e], z[e] = accv[dt][4 * vq + e];
      st4(static_cast<float*>(a.dk) + at + 32 * dt + 8 * vq + 4 * h, y);
      st4(static_cast<float*>(a.dv) + at + 32 * dt + 8 * vq + 4 * h, z);
    }
  }
}

// Smallest and largest document number of 32 positions (DotArgs::ranges), one thread each.
__global__ void dot_ranges_kernel(const int* docs, int2* ranges, int B, int Nk) {
  const int blocks = (Nk + kDotBlock - 1) / kDotBlock;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (at >= static_cast<int64_t>(B) * blocks) return;
  const int b = static_cast<int>(at / blocks), j0 = static_cast<int>(at - static_cast<int64_t>(b) * blocks) * kDotBlock;
  const int* d = docs + static_cast<int64_t>(b) * Nk;
  int lo = 0x7fffffff, hi = -1;
  bool pad = false;
  for (int j = j0; j < min(j0 + kDotBlock, Nk); ++j) {
    pad |= d[j] < 0;
    lo = d[j] < 0 ? lo : min(lo, d[j]), hi = max(hi, d[j]);
  }
  ranges[at] = make_int2(pad ? ~lo : lo, hi);
}

template <int D>
hipError_t launch_fwd(const DotArgs& a, hipStream_t st) {
  const int64_t nrb = (static_cast<int64_t>(a.G) * a.Nq + kDotBlock - 1) / kDotBlock;
  dot_fwd_f32_kernel<D><<<unit_grid(static_cast<int64_t>(a.B) * a.Hkv, nrb * a.nsplit), 256, 0, st>>>(a);
  if (a.nsplit > 1) {
    const int64_t rows = static_cast<int64_t>(a.B) * a.H * a.Nq;
    dot_join_kernel<<<static_cast<unsigned>((rows + 256 / D - 1) / (256 / D)), 256, 0, st>>>(a);
  }
  return hipGetLastError();
}
template <int D>
hipError_t launch_bwd(const DotArgs& a, hipStream_t st) {
  const int64_t nrb = (static_cast<int64_t>(a.G) * a.Nq + kDotBlock - 1) / kDotBlock;
  const int64_t nkb = (a.Nk + kDotBlock - 1) / kDotBlock;
  dot_dq_f32_kernel<D><<<unit_grid(static_cast<int64_t>(a.B) * a.Hkv, nrb), 64 * kWavesOf<D>, 0, st>>>(a);
  dot_dkv_f32_kernel<D><<<unit_grid(static_cast<int64_t>(a.B) * a.Hkv, nkb), 64 * kWavesOf<D>, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch(const DotArgs& a, bool backward, hipStream_t st) {
  switch (a.D) {
    case 16: return backward ? launch_bwd<16>(a, st) : launch_fwd<16>(a, st);
    case 32: return backward ? launch_bwd<32>(a, st) : launch_fwd<32>(a, st);
    case 64: return backward ? launch_bwd<64>(a, st) : launch_fwd<64>(a, st);
    default: return backward ? launch_bwd<128>(a, st) : launch_fwd<128>(a, st);
  }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace

hipError_t dot_ranges(const DotArgs& a, int2* ranges, hipStream_t st) {
  const int64_t n = static_cast<int64_t>(a.B) * ((a.Nk + kDotBlock - 1) / kDotBlock);
  dot_ranges_kernel<<<static_cast<unsigned>((n + 63) / 64), 64, 0, st>>>(a.docs, ranges, a.B, a.Nk);
  return hipGetLastError();
}

// How the bf16 kernels' workgroups own `units` blocks of 128 rows (or keys) of all heads:
// 0 whole blocks of 128, a wavefront 32 each; -1 the same with two groups of wavefronts
// that share the other side's blocks; 1 blocks of 32, their wavefronts sharing the other
// side. Whole blocks move the fewest bytes, but where there are few of them the time is
// that of the longest one. Measured, forward us of 0 / -1 / 1 (causal): D = 128, units 2048
// 1120 / 1231 / 1825 (all pairs), 1024: 300 / 344 / 519, 512: 135 / 105 / 160, 256: 113 / 84 / 84 and
// 36 / 32 / 42, 128: 61 / 48 / 31; D = 64 (twice the workgroups of 32 fit a CU), 1024: 235 / 266 / 234 and
// 128 / 151 / 140, 512: 98 / 79 / 73, 128: 47 / 37 / 17. With documents,
// whose lengths the device alone knows, a block at the end of one is masked along its whole walk, which two
// groups halve: that gains where few heads have long sequences. Means of four draws of 1 / 3 / 16 random documents
// and padding, -1 to 0: units 768 of 1 x 12288, 8 heads (96 blocks a head) 0.66 / 0.76 / 0.93, of 1 x 6144, 16 heads on 4 (192)
// 0.68 / 0.73 / 1.08; 1024 of 1 x 8192, 16 on 4 (256) 0.79 / 0.82 / 1.10, with a cap 0.98 / 0.93 / 1.12, of 1 x 16384, 8 heads (128)
// 0.78 / 0.89 / 1.02, with a cap 0.94 / 1.01 / 1.08, of 1 x 8192, 16 heads (64) 0.98 / 0.97 / 1.15, with a cap 1.06 / 1.03 / 1.18,
// of 2 x 4096 (32) 1.00 / 1.07 / 1.20, 8 x 1024 (8) 1.25 / 1.29 / 1.45; 1280 of 1 x 10240, 16 on 4 0.94 / 0.92 / 1.05, with a cap 1.19 /
// 1.05 / 1.06; 1536 of 1 x 12288, 16 on 4 1.07 / 0.95 / 1.12; 2048 of 1 x 16384, 16 on 4 1.13 / 1.03 / 1.17.
int rows_form(int64_t units, int64_t heads, int64_t D, bool docs) {
  if (D <= 64) return units < 640 ? 1 : 0;
  if (units <= 160) return 1;
  return units < 768 || (docs && units < 1152 && units >= 96 * heads) ? -1 : 0;
}

DotPlan dot_fwd_plan(int64_t B, int64_t Nq, int64_t Nk, int64_t H, int64_t Hkv, int64_t D, int causal, int window, bool docs,
                     int dtype) {
  DotPlan p = {};
  const bool bf16 = dtype == SA_DTYPE_BF16;
  const int64_t R = H / Hkv * Nq;
  p.nsplit = bf16 ? rows_form(B * Hkv * ((R + 127) / 128), B * Hkv, D, docs) : 1;
  if (p.nsplit == 1) {
    // Keys a row block walks: the parts take 256 of them at least.
    const int64_t units = B * Hkv * ((R + kDotBlock - 1) / kDotBlock);
    const int64_t keys = window && causal ? std::min<int64_t>(Nk, int64_t(window) + Nq) : Nk;
    p.nsplit = static_cast<int>(std::max<int64_t>(1, std::min((bf16 ? 512 : 1024) / units, keys / 256)));
  }
  p.ranges_off = 0;
  p.part_off = docs ? up256(static_cast<size_t>(B) * ((Nk + kDotBlock - 1) / kDotBlock) * sizeof(int2)) : 0;
  p.bytes = p.part_off + (p.nsplit > 1 ? static_cast<size_t>(B) * H * Nq * p.nsplit * (D + 3) * sizeof(float) : 0);
  return p;
}
DotPlan dot_bwd_plan(int64_t B, int64_t Nq, int64_t Nk, int64_t H, int64_t Hkv, int64_t D, int causal, int window, bool docs,
                     int dtype) {
  DotPlan p = {};
  const int64_t R = H / Hkv * Nq, rows = B * Hkv * ((R + 127) / 128), keys = B * Hkv * ((Nk + 127) / 128);
  // Rows that a block of 128 keys sees (keys before a prefix, which a plan does not know of, all).
  const int64_t seen = window > 0 ? std::min(R, H / Hkv * ((causal ? 1 : 2) * int64_t(window) + 128)) : R;
  const bool bf16 = dtype == SA_DTYPE_BF16;
  p.nsplit = p.kside = p.ks = 1;
  if (bf16) {
    p.nsplit = rows_form(rows, B * Hkv, D, docs);
    // The key side: as the rows where a block of keys sees few of them; else `ks` workgroups for a
    // block of 128 keys, their float32 sums added afterwards, up to about 1024 in all; with
    // documents, which make some key blocks' rows many, and more than 16384 rows 2048 (means of four draws of 1 / 2 / 3 /
    // 6 / 16 random documents, keys 256 (units of 128), ks 8 to 4: R = 65536 1.02 / 0.76 / 0.78 / 0.83 / 0.85, 32768 of three shapes
    // 1.04 - 1.05 / 0.81 - 0.84 / 0.78 - 0.86 / 0.89 - 0.92 / 0.95 - 0.99, 16384 1.11 / 0.97 / 0.87 / 1.00 / 1.06, 8192 1.21 / 1.00 /
    // 1.01 / 1.04 / 1.13).
    // Backward us of (0, ks 1) / (-1, 1) / 1 / (0, ks 2) / 4 / 8 at D = 128, causal: keys 1024, R = 8192
    // 1039 / 1080 / 1807 / 1079 / 1201 / 1479; 512, 4096: 391 / 328 / 535 / 333 / 407 / 556; 256, 4096: 355 / 271 / 308 /
    // 260 / 231 / 318; 256, 32768: 2430 / 1668 / 1721 / 1411 / 996 / 1042; 32, 8192: 565 / 373 / 211 / 313 / 189 / 130;
    // 256, 1024: 119 / 99 / 127 / 113 / 126 / 209; 96, 1500: 135 / 105 / 78 / 104 / 85 / 96; 64, 2048: 166 / 123 / 87 / 120 /
    // 93 / 86. With a window (rows of a block of keys given): keys 256, 1024 rows 162 / 138 / - / 144 / 169 / 259; 256,
    // 640: 92 / 82 / - / 95 / 118 / 202; 256, 8704: 791 / 580 / - / 544 / 540 / 596; 128, 1536: 189 / 147 / 125 / 141 /
    // 120 / 142; D = 64, 256, 1024: 106 / 90 / 78 / 95 / 104 / 119; 376, 640: 84 / 96 / 91 / 91 / 108 / 141.
    if (D <= 64 ? keys < 640 && seen <= 8192 : keys <= 128 && seen <= 2048)
      p.kside = 1;
    else if (keys >= 768)
      p.kside = 0;
    else if (seen <= 2048 || keys >= 384)
      p.kside = -1;
    else
      p.kside = 0, p.ks = static_cast<int>(std::max<int64_t>(2, std::min<int64_t>(8, (docs && seen > 16384 ? 2048 : 1024) / keys)));
  }
  p.ranges_off = 0;
  p.delta_off = docs ? up256(static_cast<size_t>(B) * ((Nk + kDotBlock - 1) / kDotBlock) * sizeof(int2)) : 0;
  // Delta, or for every 32 rows what the bf16 kernels keep of them (dot_bwd.hip)
  p.part_off = up256(p.delta_off + (bf16 ? static_cast<size_t>(B) * Hkv * ((R + 31) / 32) * 512 : static_cast<size_t>(B) * H * Nq * sizeof(float)));
  p.bytes = p.part_off + (p.ks > 1 ? static_cast<size_t>(p.ks) * 2 * B * Hkv * Nk * D * sizeof(float) : 0);
  return p;
}

hipError_t dot_fwd_f32(const DotArgs& a, hipStream_t st) { return launch(a, false, st); }
hipError_t dot_bwd_f32(const DotArgs& a, hipStream_t st) { return launch(a, true, st); }

}  // namespace sa
