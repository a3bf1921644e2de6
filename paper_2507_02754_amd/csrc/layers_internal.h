// Internal declarations of the operators of include/simplicial_layers.h (host
// launchers; layers_api.hip validates their arguments and maps their errors).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sa {

// ---- norm_rotate.hip ----
constexpr int kRotTensors = 3;
constexpr int kRotFreqs = 64;
struct RotArgs {
  const void* x[kRotTensors];
  const void* w[kRotTensors];   // [D] or null
  const void* dy[kRotTensors];  // backward
  void* y[kRotTensors];         // forward: y, backward: dx
  void* dw[kRotTensors];        // backward: [D] or null
  int64_t sb[kRotTensors], sn[kRotTensors], sh[kRotTensors];
  int heads[kRotTensors], shares[kRotTensors];
  int count;
  const int64_t* pos;
  int64_t pos_stride, start;
  int B, N, D, norm, nfreq, layout, dtype, wdtype;
  float eps;
  double turns[kRotFreqs];  // turns per position: freqs / 2 pi
};
hipError_t rotate_fwd(const RotArgs& a, hipStream_t st);
size_t rotate_bwd_bytes(int count, int64_t D);
hipError_t rotate_bwd(const RotArgs& a, float* part, hipStream_t st);

// ---- logprobs.hip ----
struct LogprobArgs {
  const void* x;
  const int64_t* targets;
  float *logprob, *entropy, *lse, *top_logprob;
  float* lse_lo;  // what rounding took from lse, or null
  int64_t* top_index;
  int64_t R, V, stride;
  int top, dtype;
};
// Whether the launches hold less than 2^32 threads.
bool logprobs_fit(int64_t R, int64_t V, int dtype);
size_t logprobs_fwd_bytes(int64_t R, int64_t V, int top, int dtype);
hipError_t logprobs_fwd(const LogprobArgs& a, void* workspace, hipStream_t st);
struct LogprobGrad {
  const void* x;
  const int64_t* targets;
  const float *lse, *lse_lo, *entropy, *d_logprob, *d_entropy, *d_lse;  // lse_lo: or null
  void* dx;
  int64_t R, V, stride;
  int dtype;
};
hipError_t logprobs_bwd(const LogprobGrad& a, hipStream_t st);

// ---- dot_f32.hip, dot_fwd.hip, dot_bwd.hip ----
// Dot-product attention. A K-side head's rows are its G = H / Hkv query heads at
// every position, r = G i + g: one position's heads share their keys.
struct DotArgs {
  const void *q, *k, *v, *dout;
  const void *out_in, *out_lo_in;  // backward: O, and what its rounding took or null
  void *out, *out_lo;
  float* lse;  // forward: written, backward: read
  void *dq, *dk, *dv;
  int64_t qsb, qsn, qsh, ksb, ksn, ksh, vsb, vsn, vsh;
  int B, Nq, Nk, H, Hkv, D, G;
  unsigned magic;  // of the division by G (dot_common.h)
  int shift;
  float scale, cap;
  int causal, window;  // window 0: none
  const float* slopes;
  const int* docs;
  const int* prefix;
  const int* lens;
  // Smallest and largest document number of every 32 positions, [B, ceil(Nk / 32)], padding apart: with
  // padding among them the complement of the smallest (2^31 - 1 and -1 where there is none).
  const int2* ranges;
  float* delta;  // backward: Delta [B, H, Nq] (bf16: what dot_bwd.hip keeps of the rows)
  // Workgroups over rows. Forward: parts of the key axis that workgroups of 32 rows take; bf16
  // also 0: workgroups of 128 rows, -1: of 128 rows with two groups of wavefronts.
  int nsplit;
  // bf16 backward: likewise over keys (1, 0 or -1), and workgroups that share a block of
  // keys, each a part of the rows (not with 1).
  int kside, ks;
  float* part;   // partial results of nsplit or ks > 1
  int dtype;
};
struct DotPlan {
  int nsplit, kside, ks;
  size_t ranges_off, delta_off, part_off, bytes;
};
DotPlan dot_fwd_plan(int64_t B, int64_t Nq, int64_t Nk, int64_t H, int64_t Hkv, int64_t D, int causal, int window,
                     bool docs, int dtype);
DotPlan dot_bwd_plan(int64_t B, int64_t Nq, int64_t Nk, int64_t H, int64_t Hkv, int64_t D, int causal, int window,
                     bool docs, int dtype);
hipError_t dot_ranges(const DotArgs& a, int2* ranges, hipStream_t st);
hipError_t dot_fwd_f32(const DotArgs& a, hipStream_t st);
hipError_t dot_bwd_f32(const DotArgs& a, hipStream_t st);
hipError_t dot_fwd_bf16(const DotArgs& a, hipStream_t st);
hipError_t dot_bwd_bf16(const DotArgs& a, hipStream_t st);

}  // namespace sa
