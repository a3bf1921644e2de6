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

// What a lane group works on: position (b, n) and heads s, s + hsplit, ... of all
// tensors' heads in a row. Tensor and head of a flat head index.
struct Which {
  int t, h;
};
__device__ __forceinline__ Which which(const RotArgs& a, int f) {
  const int h0 = a.heads[0], h1 = a.count > 1 ? a.heads[1] : 0;
  return f < h0 ? Which{0, f} : f < h0 + h1 ? Which{1, f - h0} : Which{2, f - h0 - h1};
}
template <typename P>
__device__ __forceinline__ P pick(P const (&p)[kRotTensors], int t) {
  return t == 0 ? p[0] : t == 1 ? p[1] : p[2];
}
__device__ __forceinline__ int all_heads(const RotArgs& a) {
  return a.heads[0] + (a.count > 1 ? a.heads[1] : 0) + (a.count > 2 ? a.heads[2] : 0);
}
__device__ __forceinline__ float inv_rms(float sum, const RotArgs& a) {
  const float ms = sum / static_cast<float>(a.D) + a.eps;
  return ms > 0.f ? 1.f / sqrtf(ms) : ms == 0.f ? 0.f : ms;  // (NaN stays NaN)
}

template <typename T, int LPR, int LAYOUT>
__global__ __launch_bounds__(kRThreads) void rotate_fwd_kernel(RotArgs a, int hsplit) {
  const double* turns = arg_turns();
  const int64_t group = (static_cast<int64_t>(blockIdx.x) * kRThreads + threadIdx.x) / LPR;
  const int r = threadIdx.x % LPR;
  const int64_t bn = group / hsplit;
  if (bn >= static_cast<int64_t>(a.B) * a.N) return;
  const int s = static_cast<int>(group - bn * hsplit);
  const int b = static_cast<int>(bn / a.N), n = static_cast<int>(bn - static_cast<int64_t>(b) * a.N);
  const Runs<LAYOUT> runs(r, a.nfreq);
  const int64_t p = a.pos ? a.pos[b * a.pos_stride + n] : a.start + n;
  const Turn<LAYOUT> turn(a, turns, r, static_cast<double>(p));
  const int H = all_heads(a);
  for (int f = s; f < H; f += hsplit) {
    const Which w = which(a, f);
    const T* x = static_cast<const T*>(pick(a.x, w.t)) + b * pick(a.sb, w.t) + n * pick(a.sn, w.t) + w.h * pick(a.sh, w.t);
    float u[16];
    ld_run(x + runs.a).get(u);
    ld_run(x + runs.b).get(u + 8);
    if (a.norm) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += u[e] * u[e];
      const float inv = inv_rms(row_sum<LPR>(sum), a);
      const void* wt = pick(a.w, w.t);
#pragma unroll
      for (int e = 0; e < 16; ++e) u[e] *= inv;
      if (wt) {
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] *= ld_w(wt, a.wdtype, (e < 8 ? runs.a : runs.b - 8) + e);
      }
    }
    turn_row<LAYOUT, LPR, false>(u, turn, runs, r, a.nfreq);
    const int hs = w.t == 0 ? a.heads[0] : w.t == 1 ? a.heads[1] : a.heads[2];
    T* y = static_cast<T*>(pick(a.y, w.t)) + (bn * hs + w.h) * a.D;
    Run8<T> o;
    o.set(u);
    *reinterpret_cast<Run8<T>*>(y + runs.a) = o;
    o.set(u + 8);
    *reinterpret_cast<Run8<T>*>(y + runs.b) = o;
  }
}

// Backward. With a weight's gradient asked for (DW) the lane groups stride over the
// positions and every workgroup leaves one partial sum per tensor in `part`
// ([workgroup, tensor, D]), which rotate_dw_kernel adds in order.
template <typename T, int LPR, int LAYOUT, bool DW>
__global__ __launch_bounds__(kRThreads) void rotate_bwd_kernel(RotArgs a, int hsplit, float* part) {
  const double* turns = arg_turns();
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kRThreads + threadIdx.x) / LPR;
  const int64_t groups = static_cast<int64_t>(a.B) * a.N * hsplit;
  const int64_t step = DW ? static_cast<int64_t>(gridDim.x) * (kRThreads / LPR) : groups;
  const int r = threadIdx.x % LPR;
  const Runs<LAYOUT> runs(r, a.nfreq);
  const int H = all_heads(a);
  float acc[DW ? kRotTensors : 1][16] = {};
  for (int64_t group = first; group < groups; group += step) {
    const int64_t bn = group / hsplit;
    const int s = static_cast<int>(group - bn * hsplit);
    const int b = static_cast<int>(bn / a.N), n = static_cast<int>(bn - static_cast<int64_t>(b) * a.N);
    const int64_t p = a.pos ? a.pos[b * a.pos_stride + n] : a.start + n;
    const Turn<LAYOUT> turn(a, turns, r, static_cast<double>(p));
    for (int f = s; f < H; f += hsplit) {
      const Which w = which(a, f);
      const int hs = w.t == 0 ? a.heads[0] : w.t == 1 ? a.heads[1] : a.heads[2];
      const int64_t o = (bn * hs + w.h) * a.D;
      const T* dy = static_cast<const T*>(pick(a.dy, w.t)) + o;
      float g[16];
      ld_run(dy + runs.a).get(g);
      ld_run(dy + runs.b).get(g + 8);
      turn_row<LAYOUT, LPR, true>(g, turn, runs, r, a.nfreq);
      if (a.norm) {
        const T* x = static_cast<const T*>(pick(a.x, w.t)) + b * pick(a.sb, w.t) + n * pick(a.sn, w.t) + w.h * pick(a.sh, w.t);
        float u[16];
        ld_run(x + runs.a).get(u);
        ld_run(x + runs.b).get(u + 8);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += u[e] * u[e];
        const float inv = inv_rms(row_sum<LPR>(sum), a);
        // u: x r from here on
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] *= inv;
        if constexpr (DW) {
#pragma unroll
          for (int t = 0; t < kRotTensors; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][e] += w.t == t ? g[e] * u[e] : 0.f;
        }
        const void* wt = pick(a.w, w.t);
        if (wt) {
#pragma unroll
          for (int e = 0; e < 16; ++e) g[e] *= ld_w(wt, a.wdtype, (e < 8 ? runs.a : runs.b - 8) + e);
        }
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) dot += g[e] * u[e];
        dot = row_sum<LPR>(dot) / static_cast<float>(a.D);
#pragma unroll
        for (int e = 0; e < 16; ++e) g[e] = inv * (g[e] - u[e] * dot);
      }
      T* dx = static_cast<T*>(pick(a.y, w.t)) + o;
      Run8<T> z;
      z.set(g);
      *reinterpret_cast<Run8<T>*>(dx + runs.a) = z;
      z.set(g + 8);
      *reinterpret_cast<Run8<T>*>(dx + runs.b) = z;
    }
  }
  if constexpr (DW) {
    __shared__ float red[kRThreads * 17];
#pragma unroll
    for (int t = 0; t < kRotTensors; ++t) {
      if (t >= a.count) break;
#pragma unroll
      for (int e = 0; e < 16; ++e) red[threadIdx.x * 17 + e] = acc[t][e];
      __syncthreads();
      if (threadIdx.x < 16 * LPR) {
        const int lane = threadIdx.x / 16, e = threadIdx.x % 16;
        float x = 0.f;
        for (int g = 0; g < kRThreads / LPR; ++g) x += red[(g * LPR + lane) * 17 + e];
        const Runs<LAYOUT> of(lane, a.nfreq);
        part[(static_cast<int64_t>(blockIdx.x) * a.count + t) * a.D + (e < 8 ? of.a : of.b - 8) + e] = x;
      }
      __syncthreads();
    }
  }
}

// dweight: 16 columns of one tensor a workgroup, 16 threads a column.
__global__ __launch_bounds__(kRThreads) void rotate_dw_kernel(RotArgs a, const float* part, int blocks) {
  const int per = a.D / 16, t = blockIdx.x / per, d = blockIdx.x % per * 16 + threadIdx.x % 16, row = threadIdx.x / 16;
  void* dw = pick(a.dw, t);
  if (!dw) return;
  float x = 0.f;
  for (int i = row; i < blocks; i += 16) x += part[(static_cast<int64_t>(i) * a.count + t) * a.D + d];
  __shared__ float red[16][17];
  red[row][threadIdx.x % 16] = x;
  __syncthreads();
  if (row) return;
  x = 0.f;
  for (int i = 0; i < 16; ++i) x += red[i][threadIdx.x];
  if (a.wdtype == SA_DTYPE_F32)
    static_cast<float*>(dw)[d] = x;
  else
    static_cast<uint16_t*>(dw)[d] = f32_to_bf16(x);
}

constexpr int64_t kRotBlocks = 1024;  // workgroups of a backward with weights
constexpr int64_t kRotLanes = 1 << 19;  // lanes that fill the chip (256 CUs x 2048)

// Groups that share a position's heads: as few as fill the chip, so that sines and
// cosines are formed for as many heads as possible.
int head_split(int64_t positions, int lpr, int heads) {
  int s = 1;
  while (s < heads && positions * lpr * s < kRotLanes) s *= 2;
  return std::min(s, heads);
}
int heads_of(const RotArgs& a) {
  int h = 0;
  for (int t = 0; t < a.count; ++t) h += a.heads[t];
  return h;
}
int64_t rot_blocks(int64_t positions, int lpr, int hsplit) {
  return (positions * hsplit * lpr + kRThreads - 1) / kRThreads;
}

template <typename T, int LPR, int LAYOUT>
hipError_t launch_rotate(const RotArgs& a, bool backward, float* part, hipStream_t st) {
  const int64_t positions = static_cast<int64_t>(a.B) * a.N;
  const int hs = head_split(positions, LPR, heads_of(a));
  const int64_t blocks = rot_blocks(positions, LPR, hs);
  if (!backward) {
    rotate_fwd_kernel<T, LPR, LAYOUT><<<static_cast<unsigned>(blocks), kRThreads, 0, st>>>(a, hs);
  } else if (!part) {
    rotate_bwd_kernel<T, LPR, LAYOUT, false><<<static_cast<unsigned>(blocks), kRThreads, 0, st>>>(a, hs, nullptr);
  } else {
    const int nb = static_cast<int>(std::min(blocks, kRotBlocks));
    rotate_bwd_kernel<T, LPR, LAYOUT, true><<<nb, kRThreads, 0, st>>>(a, hs, part);
    rotate_dw_kernel<<<a.count * (a.D / 16), kRThreads, 0, st>>>(a, part, nb);
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

// (an upper bound over the head counts)
size_t rotate_bwd_bytes(int count, int64_t B, int64_t N, int64_t D) {
  (void)B, (void)N;
  return static_cast<size_t>(kRotBlocks) * count * D * sizeof(float);
}
hipError_t rotate_bwd(const RotArgs& a, float* part, hipStream_t st) { return launch(a, true, part, st); }

}  // namespace sa
