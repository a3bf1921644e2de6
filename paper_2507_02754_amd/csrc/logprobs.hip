// Log probabilities of given tokens, entropy and top alternatives of rows of
// logits, and their gradient.
//
//     m = max x, l = sum e^(x - m), t = sum e^(x - m) (x - m)
//     lse = m + log l;  logprob = x[target] - lse;  entropy = log l - t / l
//     dx_j = p_j (d_lse - d_logprob - d_entropy (log p_j + entropy)) + d_logprob [j = target]
//
// Bound by memory: the forward reads every logit once, the backward reads it and
// writes its gradient. A workgroup holds its slice of a row in registers (16-byte
// chunks), so that the maximum is known before the first exponential and the top
// tokens are found without a second read. A row longer than a workgroup holds, or
// one of few rows, is cut into slices, joined by a second small kernel.
// Measured (bf16): 8192 rows of 65536 forward 208 us (5.2 TB/s, the rate of a large copy),
// gradient 348 us (2.1 GB, 6.2 TB/s); 4096 rows of 65536 in float32 the same, 204 and 350 us; 2047
// rows of 32000 with their top 5, 39 - 42 us (3.3 - 3.1 TB/s: a row's read, exponentials and search follow one
// another, three workgroups of 512 threads a CU, and nothing of the next row is on its way meanwhile);
// 8 rows of 50001 with their top 8, 7 + 6 us (two launches' latency).
//
// The top tokens: the K-th largest of the lanes' maxima in any wavefront is no
// larger than the K-th largest logit, so everything at or above the largest such
// value contains the top K. It is collected in LDS (some ten times K values of
// ordinary rows) and ranked by counting; where ties or sorted rows make it
// overflow, the tokens are picked one after another, each from the whole slice. Values are
// compared as whole numbers that order like them (NaN first), with the token in
// the lower half, the lowest first: the order of collection does not matter.
#include "layers_internal.h"
#include "mfma_common.h"

#include "simplicial_layers.h"

#include <algorithm>

namespace sa {
namespace {

constexpr int kCand = 1024;    // candidates held in LDS
constexpr int kMaxSlices = 64; // of a row: one lane each in the joining kernel
constexpr float kFloor = -1000.f;  // below any log probability whose exponential is not 0

__device__ __forceinline__ float value(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float value(float x) { return x; }
template <typename T>
constexpr int kEpc = 16 / static_cast<int>(sizeof(T));  // elements of a chunk

template <typename T>
__device__ __forceinline__ float chunk_at(const u32x4_t& c, int e) {
  if constexpr (sizeof(T) == 2)
    return (e & 1) ? bf16_hi(c[e >> 1]) : bf16_lo(c[e >> 1]);
  else
    return __uint_as_float(c[e]);
}
// The chunk, its unpacked values not known from an earlier use: a chunk's values are
// formed anew in each pass instead of staying in registers between passes.
__device__ __forceinline__ u32x4_t anew(u32x4_t c) {
  asm volatile("" : "+v"(c));
  return c;
}
// -inf in every element
template <typename T>
__device__ __forceinline__ u32x4_t empty_chunk() {
  const unsigned u = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
  return u32x4_t{u, u, u, u};
}
// Chunk of elements j .. j + kEpc - 1 of a row of V (16-byte aligned where it lies
// inside the row); elements outside are -inf.
template <typename T>
__device__ __forceinline__ u32x4_t load_chunk(const T* row, int64_t j, int64_t V) {
  if (j >= 0 && j + kEpc<T> <= V) return *reinterpret_cast<const u32x4_t*>(row + j);
  u32x4_t c = empty_chunk<T>();
#pragma unroll
  for (int e = 0; e < kEpc<T>; ++e)
    if (j + e >= 0 && j + e < V) {
      if constexpr (sizeof(T) == 2) {
        const unsigned x = row[j + e];
        c[e >> 1] = (e & 1) ? (c[e >> 1] & 0xffffu) | (x << 16) : (c[e >> 1] & 0xffff0000u) | x;
      } else {
        c[e] = __float_as_uint(row[j + e]);
      }
    }
  return c;
}
// Elements of a row before its first 16-byte boundary, counted back to the one
// before: the row's chunks start at element -lead.
template <typename T>
__device__ __forceinline__ int row_lead(const T* row) {
  return static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / static_cast<int>(sizeof(T));
}

// Whole numbers in the order of the values; NaN is the largest, 0 is none's.
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned u = __float_as_uint(x + 0.f);  // (-0 as 0)
  if (x != x) return 0xffffffffu;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) {
  if (k == 0xffffffffu) return __builtin_nanf("");
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}
typedef unsigned long long u64;
__device__ __forceinline__ u64 pack_key(unsigned key, unsigned token) { return (static_cast<u64>(key) << 32) | (0xffffffffu - token); }
__device__ __forceinline__ unsigned key_token(u64 x) { return 0xffffffffu - static_cast<unsigned>(x); }

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ u64 wave_max(u64 x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const u64 y = __shfl_xor(x, o);
    x = y > x ? y : x;
  }
  return x;
}

// What a slice leaves for the joining kernel, followed by its `top` best.
struct Part {
  float m, l, t, pad;
};
__device__ __forceinline__ size_t part_stride(int top) { return sizeof(Part) + static_cast<size_t>(top) * sizeof(u64); }

// Outputs of one row from its m, l and t (one thread), and what the top tokens' need:
// log probabilities as (x - m) - log l, which no size of the logits makes less exact.
struct RowNorm {
  float m, log_l;
  __device__ __forceinline__ float operator()(float x) const { return m == -__builtin_inff() ? m : (x - m) - log_l; }
};
template <typename T>
__device__ __forceinline__ RowNorm finish_row(const LogprobArgs& a, int64_t row, float m, float l, float t) {
  const bool none = m == -__builtin_inff() && l == 0.f;
  const float log_l = none ? 0.f : logf(l);
  // (a row with NaN: l, not its maximum, says so)
  const RowNorm norm = {l != l ? l : m, log_l};
  const int64_t y = a.targets[row];
  float lp = 0.f;
  if (y >= a.V) lp = __builtin_nanf("");
  if (y >= 0 && y < a.V) lp = norm(value(static_cast<const T*>(a.x)[row * a.stride + y]));
  a.logprob[row] = lp;
  a.entropy[row] = none ? 0.f : log_l - t / l;
  const float lse = none ? m : m + log_l;
  a.lse[row] = lse;
  if (a.lse_lo) {  // (exact where both are finite, whichever is larger)
    const float lo = (m - (lse - (lse - m))) + (log_l - (lse - m));
    a.lse_lo[row] = lo == lo ? lo : 0.f;
  }
  return norm;
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, int64_t row, int k, u64 x, RowNorm norm) {
  a.top_logprob[row * a.top + k] = norm(key_value(static_cast<unsigned>(x >> 32)));
  a.top_index[row * a.top + k] = key_token(x);
}

// One slice of one row: chunks slice * per .. of the row, NC a thread.
template <typename T, int NC, bool TOP>
__global__ __launch_bounds__(1024) void logprobs_kernel(LogprobArgs a, int slices, int per, char* parts) {
  constexpr int E = kEpc<T>;
  __shared__ float red[3][16];
  __shared__ RowNorm row_norm;
  const int tid = threadIdx.x, nt = blockDim.x, wave = tid >> 6, waves = nt >> 6, lane = tid & 63;
  const int64_t row = blockIdx.x / static_cast<unsigned>(slices);
  const int slice = blockIdx.x % static_cast<unsigned>(slices);
  const T* x = static_cast<const T*>(a.x) + row * a.stride;
  const int lead = row_lead(x);
  u32x4_t c[NC];
  // (the row's elements of the slice: [from, to) counted from the boundary)
  const int64_t q0 = static_cast<int64_t>(slice) * per;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int q = i * nt + tid;
    c[i] = q < per ? load_chunk(x, (q0 + q) * E - lead, a.V) : empty_chunk<T>();
  }
  float mine = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const u32x4_t y = anew(c[i]);
#pragma unroll
    for (int e = 0; e < E; ++e) mine = fmaxf(mine, chunk_at<T>(y, e));
  }
  float m = wave_max(mine);
  if (lane == 0) red[0][wave] = m;
  __syncthreads();
  for (int w = 0; w < waves; ++w) m = fmaxf(m, red[0][w]);
  const float base = m == -__builtin_inff() ? 0.f : m;
  float l = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const u32x4_t y = anew(c[i]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = chunk_at<T>(y, e) - base, p = fast_exp2(d * kLog2e);
      l += p;
      t += p * fmaxf(d, kFloor);  // (a token without probability: 0)
    }
  }
  l = wave_sum(l);
  t = wave_sum(t);
  if (lane == 0) red[1][wave] = l, red[2][wave] = t;
  __syncthreads();
  l = 0.f, t = 0.f;
  for (int w = 0; w < waves; ++w) l += red[1][w], t += red[2][w];
  char* part = parts + (row * slices + slice) * part_stride(a.top);
  if (tid == 0) {
    if (slices == 1)
      row_norm = finish_row<T>(a, row, m, l, t);
    else
      *reinterpret_cast<Part*>(part) = Part{m, l, t, 0.f};
  }
  if constexpr (TOP) {
    __shared__ unsigned red_key[16];
    __shared__ int found;
    __shared__ u64 cand[kCand];
    __shared__ u64 best[16];
    const int K = a.top;
    // Element e of chunk i as a whole number with its token; 0 outside the row.
    auto packed = [&](u32x4_t y, int i, int e) __attribute__((always_inline)) -> u64 {
      int q = tid;
      asm volatile("" : "+v"(q));
      q += i * nt;
      const int64_t j = (q0 + q) * E + e - lead;
      if (q >= per || j < 0 || j >= a.V) return 0;
      return pack_key(order_key(chunk_at<T>(y, e)), static_cast<unsigned>(j));
    };
    const unsigned top = order_key(mine);
    // The K-th largest of the lanes', from the highest bit down, its last 12 bits left 0 (a count
    // over the wavefront for each bit: 42 us where ranking every lane among the 64 took 48, 2047 rows
    // of 32000 bf16, K = 5).
    unsigned kth = 0;
#pragma unroll
    for (int bit = 31; bit >= 12; --bit) {
      const unsigned with = kth | (1u << bit);
      if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(top >= with)) >= K) kth = with;
    }
    if (lane == 0) red_key[wave] = kth;
    if (tid == 0) found = 0;
    __syncthreads();
    unsigned least = 0x007fffffu;  // (-inf)
    for (int w = 0; w < waves; ++w) least = max(least, red_key[w]);
    const float from = key_value(least);
    const bool nan = l != l;
    if (!(mine < from) || nan) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const u32x4_t y = anew(c[i]);
        float most = chunk_at<T>(y, 0);
#pragma unroll
        for (int e = 1; e < E; ++e) most = fmaxf(most, chunk_at<T>(y, e));
        if (most < from && !nan) continue;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!(chunk_at<T>(y, e) < from)) {  // (NaN is collected)
            const u64 v = packed(y, i, e);
            if (v) {
              const int at = atomicAdd(&found, 1);
              if (at < kCand) cand[at] = v;
            }
          }
      }
    }
    __syncthreads();
    const int n = found;
    auto put = [&](int k, u64 v) {
      if (slices == 1)
        write_top(a, row, k, v, row_norm);
      else
        reinterpret_cast<u64*>(part + sizeof(Part))[k] = v;
    };
    if (n <= kCand) {
      for (int i = tid; i < n; i += nt) {
        const u64 v = cand[i];
        int before = 0;
        for (int o = 0; o < n; ++o) before += cand[o] > v;
        if (before < K) put(before, v);
      }
      // (a slice with fewer tokens than `top`)
      for (int k = n + tid; k < K; k += nt) put(k, 0);
    } else {
      u64 last = ~0ull;
      for (int k = 0; k < K; ++k) {
        u64 v = 0;
#pragma unroll 1
        for (int i = 0; i * nt + tid < per; ++i) {  // (rare: the logits are read again)
          const u32x4_t y = load_chunk(x, (q0 + i * nt + tid) * E - lead, a.V);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const u64 o = packed(y, i, e);
            if (o < last && o > v) v = o;
          }
        }
        v = wave_max(v);
        __syncthreads();
        if (lane == 0) best[wave] = v;
        __syncthreads();
        for (int w = 0; w < waves; ++w) v = best[w] > v ? best[w] : v;
        last = v;
        if (tid == 0) put(k, v);
      }
    }
  }
}

// Joins the slices of a row: one wavefront a row, one lane a slice.
template <typename T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobArgs a, int slices, const char* parts) {
  const int lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= a.R) return;
  const char* part = parts + (row * slices + lane) * part_stride(a.top);
  const bool have = lane < slices;
  const Part p = have ? *reinterpret_cast<const Part*>(part) : Part{-__builtin_inff(), 0.f, 0.f, 0.f};
  const float m = wave_max(p.m), base = m == -__builtin_inff() ? 0.f : m;
  const float d = p.m - base, s = fast_exp2(d * kLog2e);
  const float l = wave_sum(p.l * s), t = wave_sum(s * (p.t + fmaxf(d, kFloor) * p.l));
  RowNorm norm = {};
  if (lane == 0) norm = finish_row<T>(a, row, m, l, t);
  const u64* list = reinterpret_cast<const u64*>(part + sizeof(Part));
  int next = 0;
  u64 v = have && a.top ? list[0] : 0;
  for (int k = 0; k < a.top; ++k) {
    const u64 best = wave_max(v);
    if (v == best && have) {
      ++next;
      v = next < a.top ? list[next] : 0;
    }
    if (lane == 0) write_top(a, row, k, best, norm);
  }
}

// Gradient: chunks of one row, aligned to where they are written.
template <typename T>
__global__ __launch_bounds__(256) void logprobs_bwd_kernel(LogprobGrad a, int slices, int per) {
  constexpr int E = kEpc<T>;
  const int64_t row = blockIdx.x / static_cast<unsigned>(slices);
  const int slice = blockIdx.x % static_cast<unsigned>(slices);
  const T* x = static_cast<const T*>(a.x) + row * a.stride;
  T* dx = static_cast<T*>(a.dx) + row * a.V;
  const int lead = row_lead(dx);
  const bool together = row_lead(x) == lead;
  // (x - lse is exact for the largest logits, so that no constant added to a row makes p less so)
  const float lse = a.lse[row], lo = a.lse_lo ? a.lse_lo[row] : 0.f, h = a.entropy[row];
  const float gh = a.d_entropy ? a.d_entropy[row] : 0.f;
  const int64_t y = a.targets[row];
  float glp = a.d_logprob && y >= 0 ? a.d_logprob[row] : 0.f;
  if (y >= a.V && a.d_logprob) glp = __builtin_nanf("");
  const float g = (a.d_lse ? a.d_lse[row] : 0.f) - glp;
  const bool none = lse == -__builtin_inff();
  const int64_t end = static_cast<int64_t>(slice + 1) * per;
  for (int64_t q = static_cast<int64_t>(slice) * per + threadIdx.x; q < end; q += blockDim.x) {
    const int64_t j = q * E - lead;
    if (j >= a.V) break;
    const bool whole = j >= 0 && j + E <= a.V;
    u32x4_t c = empty_chunk<T>();
    if (together) {
      c = load_chunk(x, j, a.V);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (j + e >= 0 && j + e < a.V) {
          if constexpr (sizeof(T) == 2)
            c[e >> 1] = (e & 1) ? (c[e >> 1] & 0xffffu) | (static_cast<unsigned>(x[j + e]) << 16)
                                : (c[e >> 1] & 0xffff0000u) | x[j + e];
          else
            c[e] = __float_as_uint(x[j + e]);
        }
    }
    float o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float lp = (chunk_at<T>(c, e) - lse) - lo, p = fast_exp2(lp * kLog2e);
      float v = p * (g - gh * (fmaxf(lp, kFloor) + h));
      if (j + e == y) v += glp;
      o[e] = none ? 0.f : v;
    }
    if (whole) {
      u32x4_t z;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2)
          z[i] = pack_bf16x2(o[2 * i], o[2 * i + 1]);
        else
          z[i] = __float_as_uint(o[i]);
      }
      *reinterpret_cast<u32x4_t*>(dx + j) = z;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (j + e >= 0 && j + e < a.V) {
          if constexpr (sizeof(T) == 2)
            dx[j + e] = f32_to_bf16(o[e]);
          else
            dx[j + e] = o[e];
        }
    }
  }
}

// Slices of a row, their chunks, threads and chunks a thread.
struct Cut {
  int slices, per, threads, nc;
};
Cut cut_rows(int64_t R, int64_t V, int epc, bool aligned) {
  // (a row that is not aligned may begin and end inside a chunk)
  const int64_t chunks = aligned ? (V + epc - 1) / epc : V / epc + 2;
  // A workgroup holds 16 chunks a thread, and more of smaller ones overlap better: rows of
  // more than 4096 chunks are cut into slices of 2048, 8 for each of 256 threads (8192 rows
  // of 65536 bf16 in 1 / 2 / 4 / 8 slices: 218 / 205 / 197 / 199 us; 4096 rows of 32000 in 1 / 2 / 4:
  // 57.1 / 57.5 / 56.8). Fewer rows than workgroups that fill the chip are cut further,
  // down to 256 chunks (4 KiB) a slice.
  int64_t s = chunks <= 4096 ? 1 : std::min<int64_t>((chunks + 2047) / 2048, kMaxSlices);
  if (R * s < 512) s = std::max(s, std::min<int64_t>({(512 + R - 1) / R, chunks / 256, kMaxSlices}));
  Cut c;
  c.slices = static_cast<int>(s);
  c.per = static_cast<int>((chunks + s - 1) / s);
  c.nc = 2;
  while (c.nc < 8 && c.per > 256 * c.nc) c.nc *= 2;
  if (c.per > 1024 * 8) c.nc = 16;
  c.threads = ((c.per + c.nc - 1) / c.nc + 63) / 64 * 64;
  return c;
}

// The same of the gradient: slices of about 1024 chunks.
Cut cut_grad(int64_t V, int epc) {
  const int64_t chunks = V / epc + 2;
  Cut c = {};
  c.slices = static_cast<int>((chunks + 1023) / 1024);
  c.per = static_cast<int>((chunks + c.slices - 1) / c.slices);
  c.threads = std::min(256, (c.per + 63) / 64 * 64);
  return c;
}

template <typename T, bool TOP>
void launch_fwd(const LogprobArgs& a, const Cut& c, char* parts, hipStream_t st) {
  const unsigned grid = static_cast<unsigned>(a.R * c.slices);
  switch (c.nc) {
    case 2: logprobs_kernel<T, 2, TOP><<<grid, c.threads, 0, st>>>(a, c.slices, c.per, parts); break;
    case 4: logprobs_kernel<T, 4, TOP><<<grid, c.threads, 0, st>>>(a, c.slices, c.per, parts); break;
    case 8: logprobs_kernel<T, 8, TOP><<<grid, c.threads, 0, st>>>(a, c.slices, c.per, parts); break;
    default: logprobs_kernel<T, 16, TOP><<<grid, c.threads, 0, st>>>(a, c.slices, c.per, parts); break;
  }
}
template <typename T>
hipError_t fwd(const LogprobArgs& a, char* parts, hipStream_t st) {
  const Cut c = cut_rows(a.R, a.V, kEpc<T>, reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.stride % kEpc<T> == 0);
  if (a.top)
    launch_fwd<T, true>(a, c, parts, st);
  else
    launch_fwd<T, false>(a, c, parts, st);
  if (c.slices > 1) logprobs_join_kernel<T><<<static_cast<unsigned>((a.R + 3) / 4), 256, 0, st>>>(a, c.slices, parts);
  return hipGetLastError();
}

}  // namespace

bool logprobs_fit(int64_t R, int64_t V, int dtype) {
  if (R >= int64_t(1) << 26) return false;
  const int epc = dtype == SA_DTYPE_F32 ? 4 : 8;
  int64_t most = 0;  // threads of a row
  for (const Cut& c : {cut_rows(R, V, epc, true), cut_rows(R, V, epc, false), cut_grad(V, epc)})
    most = std::max(most, static_cast<int64_t>(c.slices) * c.threads);
  return R <= 0xffffffffll / most;
}
size_t logprobs_fwd_bytes(int64_t R, int64_t V, int top, int dtype) {
  // (rows that are not aligned may take a slice more)
  const int epc = dtype == SA_DTYPE_F32 ? 4 : 8;
  const int s = std::max(cut_rows(R, V, epc, true).slices, cut_rows(R, V, epc, false).slices);
  return s == 1 ? 0 : static_cast<size_t>(R) * s * (sizeof(Part) + top * sizeof(u64));
}
hipError_t logprobs_fwd(const LogprobArgs& a, void* workspace, hipStream_t st) {
  char* parts = static_cast<char*>(workspace);
  return a.dtype == SA_DTYPE_F32 ? fwd<float>(a, parts, st) : fwd<uint16_t>(a, parts, st);
}

hipError_t logprobs_bwd(const LogprobGrad& a, hipStream_t st) {
  const int epc = a.dtype == SA_DTYPE_F32 ? 4 : 8;
  const Cut c = cut_grad(a.V, epc);
  const unsigned grid = static_cast<unsigned>(a.R * c.slices);
  if (a.dtype == SA_DTYPE_F32)
    logprobs_bwd_kernel<float><<<grid, c.threads, 0, st>>>(a, c.slices, c.per);
  else
    logprobs_bwd_kernel<uint16_t><<<grid, c.threads, 0, st>>>(a, c.slices, c.per);
  return hipGetLastError();
}

}  // namespace sa
