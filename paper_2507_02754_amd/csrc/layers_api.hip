// C-ABI entry points of include/simplicial_layers.h: argument validation (host
// only, before any HIP call) and error mapping.
#include "simplicial_layers.h"

#include <limits.h>
#include <math.h>

#include <initializer_list>

#include "layers_internal.h"

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Pointers that may not be null, 16-byte aligned as all of the library's.
bool good(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!p || !aligned(p, 16)) return false;
  return true;
}
bool good_or_null(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!aligned(p, 4)) return false;
  return true;
}
int to_status(hipError_t e) { return e == hipSuccess ? SA_OK : SA_ERR_HIP; }
int element_size(int32_t dtype) { return dtype == SA_DTYPE_F32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == SA_DTYPE_F32 || dtype == SA_DTYPE_BF16; }
bool known_dim(int64_t D) { return D == 16 || D == 32 || D == 64 || D == 128; }

// a * b * c within `most` (all positive).
bool product_fits(int64_t a, int64_t b, int64_t c, int64_t most) { return a <= most / b && a * b <= most / c; }

constexpr int64_t kElements = int64_t(1) << 40;  // of a tensor

// A view's strides: not negative, its rows 16-byte aligned.
bool good_stride(int64_t s, int32_t dtype) { return s >= 0 && s <= kElements && s * element_size(dtype) % 16 == 0; }

// ---- norm and rotation ----

int check_rotate(int32_t count, const void* const* x, const int64_t* strides, const int32_t* heads,
                 const int64_t* positions, int64_t pos_stride, int64_t B, int64_t N, int64_t D, int32_t norm,
                 float eps, int32_t layout, const double* freqs, int32_t nfreq, int32_t dtype, int32_t wdtype,
                 const void* const* weight) {
  if (count < 1 || count > SA_ROTATE_MAX || !x || !strides || !heads) return SA_ERR_INVALID;
  if (B <= 0 || N <= 0 || D <= 0 || B > INT_MAX || N > INT_MAX || !product_fits(B, N, 1, INT_MAX)) return SA_ERR_INVALID;
  if (!known(dtype) || !known(wdtype) || !known_dim(D)) return SA_ERR_UNSUPPORTED;
  int64_t all = 0;
  for (int t = 0; t < count; ++t) {
    if (!good({x[t]}) || heads[t] < 1) return SA_ERR_INVALID;
    for (int i = 0; i < 3; ++i)
      if (!good_stride(strides[3 * t + i], dtype)) return SA_ERR_INVALID;
    if (weight && weight[t] && (!norm || !aligned(weight[t], 4))) return SA_ERR_INVALID;
    all += heads[t];
  }
  // A launch holds less than 2^32 threads (D / 16 a position and tensor), a position 2^31
  // elements, a tensor 2^40.
  if (all > INT_MAX / D || !product_fits(B * N, D / 16, count, 0xffffff00) || !product_fits(B * N, all, D, kElements)) return SA_ERR_INVALID;
  if (!aligned(positions, 8) || pos_stride < 0 || (positions && pos_stride != 0 && pos_stride < N)) return SA_ERR_INVALID;
  if (norm && !(isfinite(eps) && eps >= 0.f)) return SA_ERR_INVALID;
  if (layout != SA_ROTATE_HALF && layout != SA_ROTATE_PAIRS && layout != SA_ROTATE_AXIS) return SA_ERR_INVALID;
  if (nfreq < 0 || nfreq > (layout == SA_ROTATE_AXIS ? D / 3 : D / 2) || (nfreq && !freqs)) return SA_ERR_INVALID;
  if (layout == SA_ROTATE_HALF && nfreq % 8 != 0) return SA_ERR_UNSUPPORTED;
  for (int i = 0; i < nfreq; ++i)
    if (!isfinite(freqs[i])) return SA_ERR_INVALID;
  return SA_OK;
}

sa::RotArgs rotate_args(int32_t count, const void* const* x, const int64_t* strides, const void* const* weight,
                        const int32_t* heads, const int64_t* positions, int64_t pos_stride, int64_t start, int64_t B,
                        int64_t N, int64_t D, int32_t norm, float eps, int32_t layout, const double* freqs,
                        int32_t nfreq, int32_t dtype, int32_t wdtype) {
  sa::RotArgs a = {};
  for (int t = 0; t < count; ++t) {
    a.x[t] = x[t];
    a.w[t] = weight ? weight[t] : nullptr;
    a.sb[t] = strides[3 * t], a.sn[t] = strides[3 * t + 1], a.sh[t] = strides[3 * t + 2];
    a.heads[t] = heads[t];
  }
  a.count = count;
  a.pos = positions, a.pos_stride = pos_stride, a.start = start;
  a.B = static_cast<int>(B), a.N = static_cast<int>(N), a.D = static_cast<int>(D);
  a.norm = norm != 0, a.eps = eps, a.layout = layout, a.nfreq = nfreq, a.dtype = dtype, a.wdtype = wdtype;
  for (int i = 0; i < nfreq; ++i) a.turns[i] = freqs[i] * 0.15915494309189533577;  // 1 / 2 pi
  return a;
}

// ---- dot-product attention ----

int check_dot(int64_t B, int64_t Nq, int64_t Nk, int64_t H, int64_t Hkv, int64_t D, int32_t window, int32_t dtype) {
  if (B <= 0 || Nq <= 0 || Nk <= 0 || H <= 0 || Hkv <= 0 || D <= 0 || Nq > Nk || window < 0) return SA_ERR_INVALID;
  if (Hkv > H || H % Hkv != 0) return SA_ERR_INVALID;
  // Rows of a sequence and positions are 32-bit numbers, and a launch holds less than
  // 2^32 threads, up to 512 for each block of 32 rows or keys (and up to 7 blocks of none).
  const int64_t rows = int64_t(1) << 30, blocks = (int64_t(1) << 23) - 8;
  if (Nk > rows || B > rows || H > rows || !product_fits(H / Hkv, Nk, 1, rows)) return SA_ERR_INVALID;
  if (!product_fits(B, Hkv, (H / Hkv * Nk + 31) / 32, blocks)) return SA_ERR_INVALID;
  if (!known(dtype) || !known_dim(D)) return SA_ERR_UNSUPPORTED;
  return SA_OK;
}
// A block of 32 rows is read through 32-bit offsets: its positions and all heads
// within 2^31 bytes.
bool block_fits(int64_t sn, int64_t sh, int64_t heads, int64_t D, int32_t dtype) {
  const int64_t most = (int64_t(1) << 31) / element_size(dtype);
  return sn < most / 64 && sh < most / 4 && 33 * sn + (heads - 1) * sh + D < most && (heads - 1) <= most / (sh ? sh : 1);
}

// Scale and cap whose quotients and base-2 products, as the kernels form them in float32, neither
// overflow (an infinity times a score of 0 is NaN) nor lose digits.
bool good_scores(float scale, float cap) {
  const float log2e = 1.4426950408889634f;
  if (!isfinite(scale * log2e) || !isfinite(cap * log2e) || cap < 0.f) return false;
  return cap == 0.f || (isnormal(1.f / cap) && isfinite(2.f * log2e * scale / cap) && (scale == 0.f || isnormal(scale / cap)));
}

struct DotCall {
  int64_t B, Nq, Nk, H, Hkv, D, st[9];
  float scale, softcap;
  int32_t causal, window;
  const float* slopes;
  const int32_t *documents, *prefix, *k_lens;
  int32_t dtype;
};
int check_dot_call(const DotCall& c) {
  const int rc = check_dot(c.B, c.Nq, c.Nk, c.H, c.Hkv, c.D, c.window, c.dtype);
  if (rc != SA_OK) return rc;
  if (!good_scores(c.scale, c.softcap)) return SA_ERR_INVALID;
  for (int64_t s : c.st)
    if (!good_stride(s, c.dtype)) return SA_ERR_INVALID;
  if (!block_fits(c.st[1], c.st[2], c.H, c.D, c.dtype) || !block_fits(c.st[4], c.st[5], 1, c.D, c.dtype) ||
      !block_fits(c.st[7], c.st[8], 1, c.D, c.dtype) || !block_fits(c.H * c.D, c.D, c.H, c.D, c.dtype))
    return SA_ERR_UNSUPPORTED;
  return good_or_null({c.slopes, c.documents, c.prefix, c.k_lens}) ? SA_OK : SA_ERR_INVALID;
}
sa::DotArgs dot_args(const DotCall& c, const void* q, const void* k, const void* v) {
  sa::DotArgs a = {};
  a.q = q, a.k = k, a.v = v;
  a.qsb = c.st[0], a.qsn = c.st[1], a.qsh = c.st[2];
  a.ksb = c.st[3], a.ksn = c.st[4], a.ksh = c.st[5];
  a.vsb = c.st[6], a.vsn = c.st[7], a.vsh = c.st[8];
  a.B = static_cast<int>(c.B), a.Nq = static_cast<int>(c.Nq), a.Nk = static_cast<int>(c.Nk), a.H = static_cast<int>(c.H);
  a.Hkv = static_cast<int>(c.Hkv), a.D = static_cast<int>(c.D), a.G = a.H / a.Hkv;
  if (a.G > 1) {
    int l = 0;
    while ((int64_t(1) << l) < a.G) ++l;
    a.magic = static_cast<unsigned>((uint64_t(1) << (31 + l)) / static_cast<uint64_t>(a.G) + 1);
    a.shift = l - 1;
  }
  a.scale = c.scale, a.cap = c.softcap, a.causal = c.causal != 0;
  a.window = c.window >= c.Nk ? 0 : c.window;  // (no distance reaches Nk)
  a.slopes = c.slopes, a.docs = c.documents, a.prefix = c.prefix, a.lens = c.k_lens;
  a.dtype = c.dtype;
  return a;
}

}  // namespace

extern "C" {

int simplicial_norm_rotate_fwd(int32_t count, const void* const* x, const int64_t* strides,
                               const void* const* weight, void* const* y, const int32_t* heads,
                               const int64_t* positions, int64_t pos_stride, int64_t start, int64_t B,
                               int64_t N, int64_t D, int32_t norm, float eps, int32_t layout,
                               const double* freqs, int32_t nfreq, int32_t dtype, int32_t wdtype,
                               void* stream) {
  const int rc = check_rotate(count, x, strides, heads, positions, pos_stride, B, N, D, norm, eps, layout, freqs,
                              nfreq, dtype, wdtype, weight);
  if (rc != SA_OK) return rc;
  if (!y) return SA_ERR_INVALID;
  sa::RotArgs a = rotate_args(count, x, strides, weight, heads, positions, pos_stride, start, B, N, D, norm, eps,
                              layout, freqs, nfreq, dtype, wdtype);
  for (int t = 0; t < count; ++t) {
    if (!good({y[t]})) return SA_ERR_INVALID;
    a.y[t] = y[t];
  }
  return to_status(sa::rotate_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t simplicial_norm_rotate_bwd_workspace_size(int32_t count, int64_t B, int64_t N, int64_t D) {
  if (count < 1 || count > SA_ROTATE_MAX || B <= 0 || N <= 0 || !known_dim(D)) return 0;
  return sa::rotate_bwd_bytes(count, D);
}

int simplicial_norm_rotate_bwd(int32_t count, const void* const* x, const int64_t* strides,
                               const void* const* weight, const void* const* dy, void* const* dx,
                               void* const* dweight, const int32_t* heads, const int64_t* positions,
                               int64_t pos_stride, int64_t start, void* workspace,
                               size_t workspace_bytes, int64_t B, int64_t N, int64_t D, int32_t norm,
                               float eps, int32_t layout, const double* freqs, int32_t nfreq,
                               int32_t dtype, int32_t wdtype, void* stream) {
  const int rc = check_rotate(count, x, strides, heads, positions, pos_stride, B, N, D, norm, eps, layout, freqs,
                              nfreq, dtype, wdtype, weight);
  if (rc != SA_OK) return rc;
  if (!dy || !dx) return SA_ERR_INVALID;
  sa::RotArgs a = rotate_args(count, x, strides, weight, heads, positions, pos_stride, start, B, N, D, norm, eps,
                              layout, freqs, nfreq, dtype, wdtype);
  bool dw = false;
  for (int t = 0; t < count; ++t) {
    if (!good({dy[t], dx[t]})) return SA_ERR_INVALID;
    a.dy[t] = dy[t];
    a.y[t] = dx[t];
    a.dw[t] = dweight ? dweight[t] : nullptr;
    if (a.dw[t] && (!norm || !aligned(a.dw[t], 4))) return SA_ERR_INVALID;
    dw = dw || a.dw[t];
  }
  if (dw) {
    if (!good({workspace})) return SA_ERR_INVALID;
    if (workspace_bytes < sa::rotate_bwd_bytes(count, D)) return SA_ERR_WORKSPACE;
  }
  return to_status(sa::rotate_bwd(a, dw ? static_cast<float*>(workspace) : nullptr, static_cast<hipStream_t>(stream)));
}

size_t simplicial_dot_attn_fwd_workspace_size(int64_t B, int64_t Nq, int64_t Nk, int64_t H,
                                              int64_t Hkv, int64_t D, int32_t causal, int32_t window,
                                              int32_t has_documents, int32_t dtype) {
  if (check_dot(B, Nq, Nk, H, Hkv, D, window, dtype) != SA_OK) return 0;
  return sa::dot_fwd_plan(B, Nq, Nk, H, Hkv, D, causal, window, has_documents != 0, dtype).bytes;
}

int simplicial_dot_attn_fwd(const void* q, const void* k, const void* v, void* out, void* out_lo,
                            float* lse, void* workspace, size_t workspace_bytes, int64_t B, int64_t Nq, int64_t Nk,
                            int64_t H, int64_t Hkv, int64_t D, int64_t q_sb, int64_t q_sn, int64_t q_sh,
                            int64_t k_sb, int64_t k_sn, int64_t k_sh, int64_t v_sb, int64_t v_sn,
                            int64_t v_sh, float scale, float softcap, int32_t causal, int32_t window,
                            const float* slopes, const int32_t* documents, const int32_t* prefix,
                            const int32_t* k_lens, int32_t dtype, void* stream) {
  const DotCall c = {B, Nq, Nk, H, Hkv, D, {q_sb, q_sn, q_sh, k_sb, k_sn, k_sh, v_sb, v_sn, v_sh}, scale, softcap,
                     causal, window, slopes, documents, prefix, k_lens, dtype};
  if (!good({q, k, v, out, lse})) return SA_ERR_INVALID;
  const int rc = check_dot_call(c);
  if (rc != SA_OK) return rc;
  if (!aligned(out_lo, 16) || (out_lo && dtype != SA_DTYPE_BF16)) return SA_ERR_INVALID;
  const sa::DotPlan p = sa::dot_fwd_plan(B, Nq, Nk, H, Hkv, D, causal, window, documents != nullptr, dtype);
  if (p.bytes && !good({workspace})) return SA_ERR_INVALID;
  if (workspace_bytes < p.bytes) return SA_ERR_WORKSPACE;
  sa::DotArgs a = dot_args(c, q, k, v);
  a.out = out, a.out_lo = out_lo, a.lse = lse;
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  a.nsplit = p.nsplit;
  a.part = reinterpret_cast<float*>(ws + p.part_off);
  if (documents) {
    int2* ranges = reinterpret_cast<int2*>(ws + p.ranges_off);
    const int r = to_status(sa::dot_ranges(a, ranges, st));
    if (r != SA_OK) return r;
    a.ranges = ranges;
  }
  return to_status(dtype == SA_DTYPE_BF16 ? sa::dot_fwd_bf16(a, st) : sa::dot_fwd_f32(a, st));
}

size_t simplicial_dot_attn_bwd_workspace_size(int64_t B, int64_t Nq, int64_t Nk, int64_t H,
                                              int64_t Hkv, int64_t D, int32_t causal, int32_t window,
                                              int32_t has_documents, int32_t dtype) {
  if (check_dot(B, Nq, Nk, H, Hkv, D, window, dtype) != SA_OK) return 0;
  return sa::dot_bwd_plan(B, Nq, Nk, H, Hkv, D, causal, window, has_documents != 0, dtype).bytes;
}

int simplicial_dot_attn_bwd(const void* q, const void* k, const void* v, const void* out,
                            const void* out_lo, const void* dout, const float* lse, void* dq, void* dk, void* dv,
                            void* workspace, size_t workspace_bytes, int64_t B, int64_t Nq, int64_t Nk,
                            int64_t H, int64_t Hkv, int64_t D, int64_t q_sb, int64_t q_sn, int64_t q_sh,
                            int64_t k_sb, int64_t k_sn, int64_t k_sh, int64_t v_sb, int64_t v_sn,
                            int64_t v_sh, float scale, float softcap, int32_t causal, int32_t window,
                            const float* slopes, const int32_t* documents, const int32_t* prefix,
                            const int32_t* k_lens, int32_t dtype, void* stream) {
  const DotCall c = {B, Nq, Nk, H, Hkv, D, {q_sb, q_sn, q_sh, k_sb, k_sn, k_sh, v_sb, v_sn, v_sh}, scale, softcap,
                     causal, window, slopes, documents, prefix, k_lens, dtype};
  if (!good({q, k, v, out, dout, lse, dq, dk, dv, workspace})) return SA_ERR_INVALID;
  const int rc = check_dot_call(c);
  if (rc != SA_OK) return rc;
  if (!aligned(out_lo, 16) || (out_lo && dtype != SA_DTYPE_BF16)) return SA_ERR_INVALID;
  const sa::DotPlan p = sa::dot_bwd_plan(B, Nq, Nk, H, Hkv, D, causal, window, documents != nullptr, dtype);
  if (workspace_bytes < p.bytes) return SA_ERR_WORKSPACE;
  sa::DotArgs a = dot_args(c, q, k, v);
  a.out_in = out, a.out_lo_in = out_lo, a.dout = dout, a.lse = const_cast<float*>(lse);
  a.dq = dq, a.dk = dk, a.dv = dv;
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  a.delta = reinterpret_cast<float*>(ws + p.delta_off);
  a.part = reinterpret_cast<float*>(ws + p.part_off);
  if (documents) {
    int2* ranges = reinterpret_cast<int2*>(ws + p.ranges_off);
    const int r = to_status(sa::dot_ranges(a, ranges, st));
    if (r != SA_OK) return r;
    a.ranges = ranges;
  }
  a.nsplit = p.nsplit, a.kside = p.kside, a.ks = p.ks;
  return to_status(dtype == SA_DTYPE_BF16 ? sa::dot_bwd_bf16(a, st) : sa::dot_bwd_f32(a, st));
}

static constexpr int64_t kMostTokens = 4000000;  // that 64 slices of a row hold

// The low parts behind lse, if the dtype asks for them (and the dtype without that).
static float* lse_lo(const float* lse, int64_t R, int32_t& dtype) {
  if (dtype < 0 || !(dtype & SA_LOGPROBS_LSE_LO)) return nullptr;
  dtype &= ~SA_LOGPROBS_LSE_LO;
  return const_cast<float*>(lse) + R;
}

static int check_logprobs(const void* logits, const int64_t* targets, int64_t R, int64_t V, int64_t row_stride,
                          int32_t dtype) {
  if (R <= 0 || V <= 0 || row_stride < V || row_stride > kElements) return SA_ERR_INVALID;
  if (!known(dtype)) return SA_ERR_UNSUPPORTED;
  if (!logits || !aligned(logits, element_size(dtype)) || !targets || !aligned(targets, 8)) return SA_ERR_INVALID;
  if (V > kMostTokens) return SA_ERR_UNSUPPORTED;
  return sa::logprobs_fit(R, V, dtype) ? SA_OK : SA_ERR_INVALID;
}

size_t simplicial_logprobs_fwd_workspace_size(int64_t R, int64_t V, int32_t top, int32_t dtype) {
  lse_lo(nullptr, 0, dtype);
  if (R <= 0 || V <= 0 || V > kMostTokens || !known(dtype) || !sa::logprobs_fit(R, V, dtype) || top < 0 || top > SA_LOGPROBS_MAX_TOP || top > V) return 0;
  return sa::logprobs_fwd_bytes(R, V, top, dtype);
}

int simplicial_logprobs_fwd(const void* logits, const int64_t* targets, float* logprob,
                            float* entropy, float* lse, float* top_logprob, int64_t* top_index,
                            void* workspace, size_t workspace_bytes, int64_t R, int64_t V,
                            int64_t row_stride, int32_t top, int32_t dtype, void* stream) {
  float* const lo = lse_lo(lse, R, dtype);
  const int rc = check_logprobs(logits, targets, R, V, row_stride, dtype);
  if (rc != SA_OK) return rc;
  if (top < 0 || top > SA_LOGPROBS_MAX_TOP || top > V) return SA_ERR_INVALID;
  if (!logprob || !entropy || !lse || !good_or_null({logprob, entropy, lse, top_logprob}) || !aligned(top_index, 8)) return SA_ERR_INVALID;
  if (top && (!top_logprob || !top_index)) return SA_ERR_INVALID;
  const size_t need = sa::logprobs_fwd_bytes(R, V, top, dtype);
  if (need && !good({workspace})) return SA_ERR_INVALID;
  if (workspace_bytes < need) return SA_ERR_WORKSPACE;
  const sa::LogprobArgs a = {logits, targets, logprob, entropy, lse, top_logprob, lo, top_index, R, V, row_stride, top, dtype};
  return to_status(sa::logprobs_fwd(a, workspace, static_cast<hipStream_t>(stream)));
}

int simplicial_logprobs_bwd(const void* logits, const int64_t* targets, const float* lse,
                            const float* entropy, const float* d_logprob, const float* d_entropy,
                            const float* d_lse, void* dlogits, int64_t R, int64_t V,
                            int64_t row_stride, int32_t dtype, void* stream) {
  const float* const lo = lse_lo(lse, R, dtype);
  const int rc = check_logprobs(logits, targets, R, V, row_stride, dtype);
  if (rc != SA_OK) return rc;
  if (!lse || !entropy || !good({dlogits}) || !good_or_null({lse, entropy, d_logprob, d_entropy, d_lse})) return SA_ERR_INVALID;
  const sa::LogprobGrad a = {logits, targets, lse, lo, entropy, d_logprob, d_entropy, d_lse, dlogits, R, V, row_stride, dtype};
  return to_status(sa::logprobs_bwd(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
