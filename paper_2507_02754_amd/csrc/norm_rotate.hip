// RMS norm of every head's row and its position rotation, forward and backward,
// of up to three tensors (q, k, k') in one launch.
//
//     u = x r w, r = (mean x^2 + eps)^-1/2;  y = R(p) u
//     g = R(-p) dy;  dw = sum g x r;  dx = r (g w - x r^2 mean(g w x))
//
// R(p) turns component pairs by position * frequency. Bound by memory: every
// row is read once and written once (backward: x and dy read).
//
// D / 16 lanes hold a row, 16 elements each, in two runs of 8 (16-byte loads of
// bf16). In the half layout the runs of a rotated lane are i .. i + 7 and nfreq + i
// .. , so that both elements of a pair are in one lane; in the other layouts they
// are 16 consecutive elements. A chunk of the axis layout may reach into the next
// lane: its neighbour element comes by a shuffle. A lane group takes one position
// and a share of its heads, so that the sines and cosines (float64 product and
// reduction to a fraction of a turn, then float32) are formed once for all of them.
//
// Measured, bf16 (a large copy runs at 5.2 TB/s): two tensors of B=2 N=8192 H=8 D=128, half layout
// with norm and weights, forward 31 us (134 MB, 4.3 TB/s), backward 44 + 4 us (201 MB, 4.2 TB/s);
// pairs 34 and 46 + 4; float32 60 and 95 + 5 (4.5 and 4.1 TB/s);
// axis layout, 24 heads of 6001 positions in three tensors, 21 - 22 and 30 - 31 us (74 and 111 MB, 3.5 - 3.3 and 3.7 - 3.6 TB/s:
// the shuffles and selects of chunks that cross lanes, as 3 does not divide 16); one token of 4 sequences 6 us, a
// launch's latency and the float64 angles.
#include "layers_internal.h"
#include "mfma_common.h"

#include "simplicial_layers.h"

#include <algorithm>

namespace sa {
namespace {

constexpr int kRThreads = 256;

template <typename T>
struct Run8;
template <>
struct Run8<uint16_t> {
  u32x4_t a;
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = bf16_lo(a[i]), f[2 * i + 1] = bf16_hi(a[i]);
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  }
};
template <>
struct Run8<float> {
  u32x4_t a, b;
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(a[i]), f[4 + i] = __uint_as_float(b[i]);
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(f[i]), b[i] = __float_as_uint(f[4 + i]);
  }
};
template <typename T>
__device__ __forceinline__ Run8<T> ld_run(const T* p) {
  return *reinterpret_cast<const Run8<T>*>(p);
}

__device__ __forceinline__ float ld_w(const void* w, int wdtype, int d) {
  return wdtype == SA_DTYPE_F32 ? static_cast<const float*>(w)[d] : bf16_to_f32(static_cast<const uint16_t*>(w)[d]);
}

// Sum over the LPR consecutive lanes of a row; every one gets it.
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  if constexpr (LPR >= 2) x += dpp_f<0xB1>(x);
  if constexpr (LPR >= 4) x += dpp_f<0x4E>(x);
  if constexpr (LPR >= 8) x += dpp_f<0x141>(x);
  return x;
}

// First element of the lane's runs; `rot` (half layout): whether they are a pair's.
template <int LAYOUT>
struct Runs {
  int a, b;
  bool rot;
  __device__ __forceinline__ Runs(int r, int nfreq) {
    if constexpr (LAYOUT == SA_ROTATE_HALF) {
      const int lanes = nfreq >> 3;
      rot = r < lanes;
      a = rot ? 8 * r : 2 * nfreq + 16 * (r - lanes);
      b = rot ? nfreq + a : a + 8;
    } else {
      a = 16 * r;
      b = a + 8;
      rot = true;
    }
  }
};

// cos and sin of the lane's elements at one position. Half and pairs: of its
// eight pairs. Axis: per element, the sine with the sign it takes, both for a
// turn forwards.
template <int LAYOUT>
struct Turn {
  static constexpr int N = LAYOUT == SA_ROTATE_AXIS ? 16 : 8;
  float c[N], s[N];
  __device__ __forceinline__ static void one(double p, double t, float& c, float& s) {
    const double x = p * t;
    // (a fraction of a turn in [-0.5, 0.5], then in half turns)
    sincospif(2.f * static_cast<float>(x - rint(x)), &s, &c);
  }
  __device__ __forceinline__ Turn(const RotArgs& args, const double* turns, int r, double p) {
    const int nfreq = args.nfreq;
    if constexpr (LAYOUT != SA_ROTATE_AXIS) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = 8 * r + e;
        c[e] = 1.f, s[e] = 0.f;
        if (i < nfreq) one(p, turns[i], c[e], s[e]);
      }
    } else {
      const int l0 = 16 * r / 3, m0 = (16 * r) % 3;
      float cc[7], ss[7];
#pragma unroll
      for (int e = 0; e < 6; ++e) {
        cc[e] = 1.f, ss[e] = 0.f;
        if (l0 + e < nfreq) one(p, turns[l0 + e], cc[e], ss[e]);
      }
      cc[6] = 1.f, ss[6] = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const bool up = m0 + e % 3 >= 3;  // this element is in the chunk after e / 3
        const int m = up ? m0 + e % 3 - 3 : m0 + e % 3;
        const float x = up ? cc[e / 3 + 1] : cc[e / 3], y = up ? ss[e / 3 + 1] : ss[e / 3];
        c[e] = m == 2 ? 1.f : x;
        s[e] = m == 2 ? 0.f : m == 0 ? -y : y;
      }
    }
  }
};

// The argument's frequencies as memory (the lanes read different ones; as an
// array of the argument they would be copied to scratch memory). The arguments
// begin with the RotArgs.
__device__ __forceinline__ const double* arg_turns() {
  return (const double*)((const char*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(RotArgs, turns));
}

// Turns the lane's 16 elements in place: forwards (INV false) or back. Elements of
// no pair are not touched, whatever their neighbours hold.
template <int LAYOUT, int LPR, bool INV>
__device__ __forceinline__ void turn_row(float* u, const Turn<LAYOUT>& t, const Runs<LAYOUT>& runs, int r, int nfreq) {
  if constexpr (LAYOUT == SA_ROTATE_HALF) {
    if (runs.rot) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = u[e], b = u[8 + e], s = INV ? -t.s[e] : t.s[e];
        u[e] = a * t.c[e] - b * s;
        u[8 + e] = b * t.c[e] + a * s;
      }
    }
  } else if constexpr (LAYOUT == SA_ROTATE_PAIRS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = u[2 * e], b = u[2 * e + 1], s = INV ? -t.s[e] : t.s[e];
      const bool in = 8 * r + e < nfreq;
      u[2 * e] = in ? a * t.c[e] - b * s : a;
      u[2 * e + 1] = in ? b * t.c[e] + a * s : b;
    }
  } else {
    const int m0 = (16 * r) % 3;
    float before = 0.f, after = 0.f;  // the neighbours' elements
    if constexpr (LPR > 1) {
      before = __shfl_up(u[15], 1, LPR);
      after = __shfl_down(u[0], 1, LPR);
    }
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int m = m0 + e % 3 >= 3 ? m0 + e % 3 - 3 : m0 + e % 3;
      const float prev = e ? u[e - 1] : before, next = e < 15 ? u[e + 1] : after;
      const bool in = m < 2 && (16 * r + e) / 3 < nfreq;
      const float s = INV ? -t.s[e] : t.s[e];
      y[e] = in ? u[e] * t.c[e] + s * (m == 0 ? next : prev) : u[e];
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) u[e] = y[e];
  }
}

// What a lane group works on: position (b, n) and heads sub, sub + n, ... of one tensor, whose
// heads n groups share.
struct Share {
  int t, sub, n;
  __device__ __forceinline__ Share(const RotArgs& a, int s) {
    const int n0 = a.shares[0], n1 = a.shares[1];
    t = s < n0 ? 0 : s < n0 + n1 ? 1 : 2;
    sub = t == 0 ? s : t == 1 ? s - n0 : s - n0 - n1;
    n = t == 0 ? n0 : t == 1 ? n1 : a.shares[2];
  }
};
template <typename P>
__device__ __forceinline__ P pick(P const (&p)[kRotTensors], int t) {
  return t == 0 ? p[0] : t == 1 ? p[1] : p[2];
}
__device__ __forceinline__ float inv_rms(float sum, const RotArgs& a) {
  const float ms = sum / static_cast<float>(a.D) + a.eps;
  return ms > 0.f ? 1.f / sqrtf(ms) : ms == 0.f ? 0.f : ms;  // (NaN stays NaN)
}

// The weight's 16 elements of the lane (ones without one).
template <int LAYOUT>
__device__ __forceinline__ void lane_weight(float* w, const void* p, const RotArgs& a, const Runs<LAYOUT>& runs) {
#pragma unroll
  for (int e = 0; e < 16; ++e) w[e] = p ? ld_w(p, a.wdtype, (e < 8 ? runs.a : runs.b - 8) + e) : 1.f;
}

template <typename T, int LPR, int LAYOUT>
__global__ __launch_bounds__(kRThreads) void rotate_fwd_kernel(RotArgs a) {
  const double* turns = arg_turns();
  const int groups = a.shares[0] + a.shares[1] + a.shares[2];  // of a position
  const int64_t group = (static_cast<int64_t>(blockIdx.x) * kRThreads + threadIdx.x) / LPR;
  const int r = threadIdx.x % LPR;
  const int64_t bn = group / groups;
  if (bn >= static_cast<int64_t>(a.B) * a.N) return;
  const Share sh(a, static_cast<int>(group - bn * groups));
  const int b = static_cast<int>(bn / a.N), n = static_cast<int>(bn - static_cast<int64_t>(b) * a.N);
  const Runs<LAYOUT> runs(r, a.nfreq);
  const int64_t p = a.pos ? a.pos[b * a.pos_stride + n] : a.start + n;
  const Turn<LAYOUT> turn(a, turns, r, static_cast<double>(p));
  const int heads = pick(a.heads, sh.t);
  const int64_t step = pick(a.sh, sh.t);
  const T* x = static_cast<const T*>(pick(a.x, sh.t)) + b * pick(a.sb, sh.t) + n * pick(a.sn, sh.t);
  T* y = static_cast<T*>(pick(a.y, sh.t)) + bn * heads * a.D;
  float w[16];
  lane_weight(w, a.norm ? pick(a.w, sh.t) : nullptr, a, runs);
  for (int h = sh.sub; h < heads; h += sh.n) {
    float u[16];
    ld_run(x + h * step + runs.a).get(u);
    ld_run(x + h * step + runs.b).get(u + 8);
    if (a.norm) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += u[e] * u[e];
      const float inv = inv_rms(row_sum<LPR>(sum), a);
#pragma unroll
      for (int e = 0; e < 16; ++e) u[e] = u[e] * inv * w[e];
    }
    turn_row<LAYOUT, LPR, false>(u, turn, runs, r, a.nfreq);
    Run8<T> o;
    o.set(u);
    *reinterpret_cast<Run8<T>*>(y + h * a.D + runs.a) = o;
    o.set(u + 8);
    *reinterpret_cast<Run8<T>*>(y + h * a.D + runs.b) = o;
  }
}

// Backward. With a weight's gradient asked for (DW) the lane groups stride over the
// positions (the grid is a multiple of a position's groups, so that each keeps its
// tensor) and every workgroup leaves one partial sum per tensor in `part` ([workgroup,
// tensor, D]), which rotate_dw_kernel adds in order.
template <typename T, int LPR, int LAYOUT, bool DW>
__global__ __launch_bounds__(kRThreads) void rotate_bwd_kernel(RotArgs a, float* part) {
  const double* turns = arg_turns();
  const int groups = a.shares[0] + a.shares[1] + a.shares[2];
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kRThreads + threadIdx.x) / LPR;
  const int64_t all = static_cast<int64_t>(a.B) * a.N;
  const int64_t step = DW ? static_cast<int64_t>(gridDim.x) * (kRThreads / LPR) / groups : all;
  const int r = threadIdx.x % LPR;
  const Runs<LAYOUT> runs(r, a.nfreq);
  const Share sh(a, static_cast<int>(first % groups));
  const int heads = pick(a.heads, sh.t);
  const int64_t hstep = pick(a.sh, sh.t);
  float w[16];
  lane_weight(w, a.norm ? pick(a.w, sh.t) : nullptr, a, runs);
  float acc[DW ? 16 : 1] = {};
  for (int64_t bn = first / groups; bn < all; bn += step) {
    const int b = static_cast<int>(bn / a.N), n = static_cast<int>(bn - static_cast<int64_t>(b) * a.N);
    const int64_t p = a.pos ? a.pos[b * a.pos_stride + n] : a.start + n;
    const Turn<LAYOUT> turn(a, turns, r, static_cast<double>(p));
    const T* x = static_cast<const T*>(pick(a.x, sh.t)) + b * pick(a.sb, sh.t) + n * pick(a.sn, sh.t);
    const T* dy = static_cast<const T*>(pick(a.dy, sh.t)) + bn * heads * a.D;
    T* dx = static_cast<T*>(pick(a.y, sh.t)) + bn * heads * a.D;
    for (int h = sh.sub; h < heads; h += sh.n) {
      float g[16], u[16];
      const Run8<T> ga = ld_run(dy + h * a.D + runs.a), gb = ld_run(dy + h * a.D + runs.b);
      const Run8<T> xa = ld_run(x + h * hstep + runs.a), xb = ld_run(x + h * hstep + runs.b);
      ga.get(g);
      gb.get(g + 8);
      turn_row<LAYOUT, LPR, true>(g, turn, runs, r, a.nfreq);
      if (a.norm) {
        xa.get(u);
        xb.get(u + 8);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += u[e] * u[e];
        const float inv = inv_rms(row_sum<LPR>(sum), a);
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          u[e] *= inv;  // x r
          if constexpr (DW) acc[e] += g[e] * u[e];
          g[e] *= w[e];
          dot += g[e] * u[e];
        }
        dot = row_sum<LPR>(dot) / static_cast<float>(a.D);
#pragma unroll
        for (int e = 0; e < 16; ++e) g[e] = inv * (g[e] - u[e] * dot);
      }
      Run8<T> z;
      z.set(g);
      *reinterpret_cast<Run8<T>*>(dx + h * a.D + runs.a) = z;
      z.set(g + 8);
      *reinterpret_cast<Run8<T>*>(dx + h * a.D + runs.b) = z;
    }
  }
  if constexpr (DW) {
    constexpr int kGroups = kRThreads / LPR;
    __shared__ float red[kRThreads * 17];
#pragma unroll
    for (int e = 0; e < 16; ++e) red[threadIdx.x * 17 + e] = acc[e];
    __syncthreads();
    const int64_t g0 = static_cast<int64_t>(blockIdx.x) * kGroups;
    for (int at = threadIdx.x; at < a.count * 16 * LPR; at += kRThreads) {
      const int t = at / (16 * LPR), lane = at / 16 % LPR, e = at % 16;
      float x = 0.f;
      for (int g = 0; g < kGroups; ++g)
        if (Share(a, static_cast<int>((g0 + g) % groups)).t == t) x += red[(g * LPR + lane) * 17 + e];
      const Runs<LAYOUT> of(lane, a.nfreq);
      part[(static_cast<int64_t>(blockIdx.x) * a.count + t) * a.D + (e < 8 ? of.a : of.b - 8) + e] = x;
    }
  }
}

// dweight: 16 columns of one tensor a workgroup, 64 threads a column.
constexpr int kDwThreads = 1024;
__global__ __launch_bounds__(kDwThreads) void rotate_dw_kernel(RotArgs a, const float* part, int blocks) {
  const int per = a.D / 16, t = blockIdx.x / per, d = blockIdx.x % per * 16 + threadIdx.x % 16, row = threadIdx.x / 16;
  void* dw = pick(a.dw, t);
  if (!dw) return;
  float x = 0.f;
#pragma unroll 4
  for (int i = row; i < blocks; i += kDwThreads / 16) x += part[(static_cast<int64_t>(i) * a.count + t) * a.D + d];
  __shared__ float red[kDwThreads / 16][17];
  red[row][threadIdx.x % 16] = x;
  __syncthreads();
  if (row) return;
  x = 0.f;
  for (int i = 0; i < kDwThreads / 16; ++i) x += red[i][threadIdx.x];
  if (a.wdtype == SA_DTYPE_F32)
    static_cast<float*>(dw)[d] = x;
  else
    static_cast<uint16_t*>(dw)[d] = f32_to_bf16(x);
}

constexpr int kRotBlocks = 1024;        // workgroups of a backward with weights, at most
constexpr int64_t kRotLanes = 1 << 19;  // lanes that fill the chip (256 CUs x 2048)

// Groups that share a tensor's heads at a position: few, so that sines and cosines are
// formed for as many heads as possible, but enough for all positions to fill the chip.
// Returns their sum.
int share_heads(RotArgs& a, int lpr) {
  int all = 0, sum = 0;
  for (int t = 0; t < a.count; ++t) all += a.heads[t];
  const int64_t positions = static_cast<int64_t>(a.B) * a.N, want = std::min<int64_t>({all, kRotBlocks / 2, (kRotLanes + positions * lpr - 1) / (positions * lpr)});
  for (int t = 0; t < kRotTensors; ++t) {
    a.shares[t] = t < a.count ? static_cast<int>(std::max<int64_t>(1, want * a.heads[t] / all)) : 0;
    sum += a.shares[t];
  }
  return sum;
}

template <typename T, int LPR, int LAYOUT>
hipError_t launch_rotate(RotArgs a, bool backward, float* part, hipStream_t st) {
  const int groups = share_heads(a, LPR);
  const unsigned blocks = static_cast<unsigned>((static_cast<int64_t>(a.B) * a.N * groups * LPR + kRThreads - 1) / kRThreads);
  if (!backward) {
    rotate_fwd_kernel<T, LPR, LAYOUT><<<blocks, kRThreads, 0, st>>>(a);
  } else if (!part) {
    rotate_bwd_kernel<T, LPR, LAYOUT, false><<<blocks, kRThreads, 0, st>>>(a, nullptr);
  } else {
    const int nb = std::max(1, static_cast<int>(std::min<unsigned>(blocks, kRotBlocks)) / groups) * groups;  // <= kRotBlocks
    rotate_bwd_kernel<T, LPR, LAYOUT, true><<<nb, kRThreads, 0, st>>>(a, part);
    rotate_dw_kernel<<<a.count * (a.D / 16), kDwThreads, 0, st>>>(a, part, nb);
  }
  return hipGetLastError();
}
template <typename T, int LPR>
hipError_t launch_layout(const RotArgs& a, bool backward, float* part, hipStream_t st) {
  switch (a.layout) {
    case SA_ROTATE_HALF: return launch_rotate<T, LPR, SA_ROTATE_HALF>(a, backward, part, st);
    case SA_ROTATE_PAIRS: return launch_rotate<T, LPR, SA_ROTATE_PAIRS>(a, backward, part, st);
    default: return launch_rotate<T, LPR, SA_ROTATE_AXIS>(a, backward, part, st);
  }
}
template <typename T>
hipError_t launch_dim(const RotArgs& a, bool backward, float* part, hipStream_t st) {
  switch (a.D) {
    case 16: return launch_layout<T, 1>(a, backward, part, st);
    case 32: return launch_layout<T, 2>(a, backward, part, st);
    case 64: return launch_layout<T, 4>(a, backward, part, st);
    default: return launch_layout<T, 8>(a, backward, part, st);
  }
}
hipError_t launch(const RotArgs& a, bool backward, float* part, hipStream_t st) {
  return a.dtype == SA_DTYPE_F32 ? launch_dim<float>(a, backward, part, st) : launch_dim<uint16_t>(a, backward, part, st);
}

}  // namespace

hipError_t rotate_fwd(const RotArgs& a, hipStream_t st) { return launch(a, false, nullptr, st); }

size_t rotate_bwd_bytes(int count, int64_t D) { return static_cast<size_t>(kRotBlocks) * count * D * sizeof(float); }
hipError_t rotate_bwd(const RotArgs& a, float* part, hipStream_t st) { return launch(a, true, part, st); }

}  // namespace sa
