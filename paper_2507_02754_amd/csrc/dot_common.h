// What the dot-product attention kernels share: which keys a query sees, for a
// single pair and for a block of 32 rows by 32 keys, and the walk over the blocks
// that hold a visible pair.
//
// A row is r = G i + g: query head g of the K-side head's group at query i, at
// position p = L - Nq + i of the L keys.
#pragma once

#include "layers_internal.h"
#include "mfma_common.h"

namespace sa {

constexpr float kInf = __builtin_inff();
constexpr int kDotBlock = 32;

// One sequence's mask.
struct DotMask {
  int L, first;  // keys; position of query 0
  int prefix, causal, window;
  const int* docs;  // of this sequence, or null
  const int2* ranges;
  __device__ __forceinline__ DotMask(const DotArgs& a, int b) {
    L = a.lens ? min(max(a.lens[b], 0), a.Nk) : a.Nk;
    first = L - a.Nq;
    prefix = a.prefix ? min(a.prefix[b], L) : 0;
    causal = a.causal;
    window = a.window;
    docs = a.docs ? a.docs + static_cast<int64_t>(b) * a.Nk : nullptr;
    ranges = a.docs ? a.ranges + static_cast<int64_t>(b) * ((a.Nk + kDotBlock - 1) / kDotBlock) : nullptr;
  }
  __device__ __forceinline__ int doc(int p) const { return docs && p >= 0 && p < L ? docs[p] : 0; }
  // Whether the query at p (p < 0: none) sees key j; document numbers dq, dk.
  __device__ __forceinline__ bool sees(int p, int j, int dq, int dk) const {
    const bool near = (!causal || j <= p) && (window == 0 || abs(p - j) < window);
    return (near || j < prefix) && j < L && p >= 0 && (!docs || (dq == dk && dk >= 0));
  }
};

// Positions p0 .. p1 of a block's rows or of its keys, the range of their document numbers and
// whether padding is among them. Padding has no part in the range: with its negative number a block
// at the end of the last document would span, and walk, all documents (N=8192, 16 heads on 4, D=128,
// causal, documents of 2876, 2182 and 2762, forward 413 us, so 207).
struct DotSpan {
  int p0, p1, dmin, dmax;
  int pad;  // negative: with padding
  __device__ __forceinline__ DotSpan(const DotMask& m, int lo, int hi) : p0(lo), p1(hi), dmin(0), dmax(0), pad(0) {
    if (m.docs && hi >= 0 && lo < m.L) {
      const int last = min(hi, m.L - 1) / kDotBlock;
      const int2 r = m.ranges[max(lo, 0) / kDotBlock];
      dmin = max(r.x, ~r.x), dmax = r.y, pad = r.x;
      for (int t = max(lo, 0) / kDotBlock + 1; t <= last; ++t) {
        const int2 s = m.ranges[t];
        dmin = min(dmin, max(s.x, ~s.x)), dmax = max(dmax, s.y);
        pad |= s.x;
      }
    }
  }
};
// Whether any (live), or every (full) query of q sees any / every key of k. live may
// be true, and full false, of a block for which they need not be.
__device__ __forceinline__ bool dot_live(const DotMask& m, const DotSpan& q, const DotSpan& k) {
  const bool near = (!m.causal || k.p0 <= q.p1) &&
                    (m.window == 0 || (k.p1 > max(q.p0, 0) - m.window && (m.causal || k.p0 < q.p1 + m.window)));
  return (near || k.p0 < m.prefix) && k.p0 < m.L && q.p1 >= 0 &&
         (!m.docs || (k.dmax >= 0 && q.dmax >= k.dmin && k.dmax >= q.dmin));
}
__device__ __forceinline__ bool dot_full(const DotMask& m, const DotSpan& q, const DotSpan& k) {
  const bool near = (!m.causal || k.p1 <= q.p0) &&
                    (m.window == 0 || (q.p1 - k.p0 < m.window && (m.causal || k.p1 - q.p0 < m.window)));
  return (near || k.p1 < m.prefix) && k.p1 < m.L && q.p0 >= 0 &&
         (!m.docs || (k.dmin == k.dmax && q.dmin == q.dmax && k.dmin == q.dmin && (k.pad | q.pad) >= 0));
}
// Key blocks that any of the rows may see: [lo, hi).
__device__ __forceinline__ void key_blocks(const DotMask& m, const DotSpan& q, int& lo, int& hi) {
  const int from = m.window && m.prefix <= 0 ? max(max(q.p0, 0) - m.window + 1, 0) : 0;
  const int to = m.causal ? min(max(q.p1 + 1, m.prefix), m.L) : m.L;
  lo = from / kDotBlock;
  hi = q.p1 < 0 ? lo : (to + kDotBlock - 1) / kDotBlock;
}
// Row blocks that may see any of the keys (G rows a position, R rows): [lo, hi).
__device__ __forceinline__ void row_blocks(const DotMask& m, const DotSpan& k, int G, int R, int& lo, int& hi) {
  const bool all = k.p0 < m.prefix;
  int from = max(-m.first, 0), to = R / G;  // queries
  if (!all && m.causal) from = max(from, k.p0 - m.first);
  if (!all && m.window) {
    to = static_cast<int>(min(static_cast<int64_t>(to), static_cast<int64_t>(k.p1) + m.window - m.first));
    if (!m.causal) from = max(from, k.p0 - m.window + 1 - m.first);
  }
  lo = static_cast<int>(static_cast<int64_t>(from) * G / kDotBlock);
  hi = k.p0 >= m.L || to <= from ? lo : static_cast<int>((static_cast<int64_t>(to) * G + kDotBlock - 1) / kDotBlock);
}

// The keys j that a query at p sees, as ranges: a0 <= j < a0 + n or j < pre, and of its
// document; a query that sees nothing has n = pre = 0.
struct KeysSeen {
  int a0, pre, doc;
  unsigned n;
  __device__ __forceinline__ KeysSeen(const DotMask& m, int p) : a0(0), pre(0), doc(m.doc(p)), n(0) {
    if (p < 0 || doc < 0) return;
    a0 = m.window ? max(p - m.window + 1, 0) : 0;
    const int end = m.causal ? p + 1 : m.window ? static_cast<int>(min(static_cast<int64_t>(p) + m.window, static_cast<int64_t>(m.L))) : m.L;
    n = static_cast<unsigned>(max(min(end, m.L) - a0, 0));
    pre = m.prefix;
  }
  __device__ __forceinline__ bool operator()(int j) const { return (static_cast<unsigned>(j - a0) < n) | (j < pre); }
};
// The positions p of the queries that see key j, likewise: b0 <= p < b0 + n.
struct QueriesSeeing {
  int b0, doc;
  unsigned n;
  __device__ __forceinline__ QueriesSeeing(const DotMask& m, int j) : b0(0), doc(m.doc(j)), n(0) {
    if (j >= m.L || doc < 0) return;
    n = 0x7fffffff;
    if (j < m.prefix) return;
    b0 = m.causal ? j : m.window ? max(j - m.window + 1, 0) : 0;
    if (m.window) n = static_cast<unsigned>(j - b0 + m.window);
  }
  __device__ __forceinline__ bool operator()(int p) const { return static_cast<unsigned>(p - b0) < n; }
};
// Calls f(v, visible) for the accumulator registers of a block whose 32 rows (keys or
// queries) are at position at(x), x = 0 .. 31, against the lane's own query or key `seen`.
// Document numbers are loaded once, a lane each, and read across lanes.
template <typename Seen, typename At, typename F>
__device__ __forceinline__ void each_pair(const DotMask& m, const Seen& seen, int c, int h, At at, F f) {
  if (m.docs) {
    const int mine = m.doc(at(c));
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int lo = __builtin_amdgcn_readlane(mine, acc_row(v, 0)), hi = __builtin_amdgcn_readlane(mine, acc_row(v, 1));
      f(v, seen(at(acc_row(v, h))) & ((h ? hi : lo) == seen.doc));
    }
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v) f(v, seen(at(acc_row(v, h))));
  }
}

// The same as bits v, in a loop that takes few registers.
template <typename Seen, typename At>
__device__ __forceinline__ unsigned pairs_seen(const DotMask& m, const Seen& seen, int c, int h, At at) {
  const int mine = m.docs ? m.doc(at(c)) : 0;
  unsigned bits = 0;
#pragma unroll 1
  for (int v = 0; v < 16; ++v) {
    bool see = seen(at(acc_row(v, h)));
    if (m.docs) {
      const int lo = __builtin_amdgcn_readlane(mine, acc_row(v, 0)), hi = __builtin_amdgcn_readlane(mine, acc_row(v, 1));
      see = see & ((h ? hi : lo) == seen.doc);
    }
    bits |= static_cast<unsigned>(see) << v;
  }
  return bits;
}

// Walks the blocks lo + off, lo + off + step, .. < hi that are live: 64 at a time are
// looked at, one a lane. test(block, live, full) and body(block, full), all wavefront-uniform
// but for test's block.
template <typename Test, typename Body>
__device__ __forceinline__ void walk_blocks(int lo, int hi, int off, int step, Test test, Body body) {
  const int lane = threadIdx.x & 63;
  const int count = lo + off < hi ? (hi - lo - off + step - 1) / step : 0;
  for (int n0 = 0; n0 < count; n0 += 64) {
    bool live = false, full = false;
    if (n0 + lane < count) test(lo + off + (n0 + lane) * step, live, full);
    unsigned long long todo = __builtin_amdgcn_ballot_w64(live);
    const unsigned long long whole = __builtin_amdgcn_ballot_w64(full);
    while (todo) {
      const int i = __builtin_ctzll(todo);
      todo &= todo - 1;
      body(lo + off + (n0 + i) * step, static_cast<bool>((whole >> i) & 1));
    }
  }
}

// The same walk as a sequence that a pipelined loop asks for its next block, ahead of
// the one it works on. test(block, live, mine, full): a block that is `live` comes up;
// `mine` and `full` are given with it (as when the blocks are a workgroup's and the
// wavefront's own rows see none, or all, of the block's pairs). blk < 0: no more.
struct DotBlock {
  int blk;
  bool mine, full;
};
// Blocks lo + off, lo + off + step, .. < hi, or (BACK) hi - 1 - off, hi - 1 - off - step, .. >= lo.
template <bool BACK, typename Test>
struct BlockSeq {
  Test test;
  int first, count, step, n0;
  unsigned long long todo, mine, full;
  __device__ __forceinline__ BlockSeq(int lo, int hi, int off, int by, Test t)
      : test(t), first(BACK ? hi - 1 - off : lo + off), count(lo + off < hi ? (hi - lo - off + by - 1) / by : 0), step(BACK ? -by : by),
        n0(-64), todo(0), mine(0), full(0) {}
  __device__ __forceinline__ DotBlock next() {
    while (todo == 0) {
      n0 += 64;
      if (n0 >= count) {
        n0 = count;  // (stays at the end)
        return DotBlock{-1, false, false};
      }
      const int lane = threadIdx.x & 63;
      bool l = false, w = false, f = false;
      if (n0 + lane < count) test(first + (n0 + lane) * step, l, w, f);
      todo = __builtin_amdgcn_ballot_w64(l);
      mine = __builtin_amdgcn_ballot_w64(w);
      full = __builtin_amdgcn_ballot_w64(f);
    }
    const int i = __builtin_ctzll(todo);
    todo &= todo - 1;
    return DotBlock{first + (n0 + i) * step, static_cast<bool>((mine >> i) & 1), static_cast<bool>((full >> i) & 1)};
  }
};
template <bool BACK = false, typename Test>
__device__ __forceinline__ BlockSeq<BACK, Test> block_seq(int lo, int hi, int off, int step, Test t) {
  return BlockSeq<BACK, Test>(lo, hi, off, step, t);
}

// Workgroup order. Workgroups go to the 8 XCDs in turn. `heads` (sequence, K-side head) pairs of
// `per` units each: gcd(heads, 8) groups of XCDs take an equal share of the heads, so that
// a head's keys stay in few L2s, and the XCDs of a group take its units in turn, so that
// long and short ones (the first and last rows of a causal sequence) spread evenly: a
// contiguous run for each XCD instead left half of them with the short rows.
__device__ __forceinline__ bool unit_of(int64_t heads, int64_t per, int64_t& unit) {
  const int groups = heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1, share = 8 / groups;
  const int x = blockIdx.x & 7, group = x / share;
  const int64_t all = heads / groups * per, k = static_cast<int64_t>(blockIdx.x >> 3) * share + x % share;
  unit = group * all + k;
  return k < all;
}
inline unsigned unit_grid(int64_t heads, int64_t per) {
  const int64_t groups = heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1, share = 8 / groups;
  return static_cast<unsigned>((heads / groups * per + share - 1) / share * 8);
}

// r / G for 0 <= r < 2^31, as a product with magic = floor(2^(31 + l) / G) + 1, l =
// ceil(log2 G), and a shift (G = 1: r).
__device__ __forceinline__ int div_group(int r, const DotArgs& a) {
  return a.G == 1 ? r : static_cast<int>(__umulhi(static_cast<unsigned>(r), a.magic) >> a.shift);
}

// Element (c, c) of an accumulator tile, in both of lane c's halves. Delta = <dO, O> is taken
// from such a product, not from a sum of the lane's own: where a row sees one key alone, O is
// V's row and Delta then dP to the bit, and its dS of 0 comes out as 0.
__device__ __forceinline__ float diagonal(const f32x16_t& x, int c, int h) {
  float y = 0.f;
#pragma unroll
  for (int v = 0; v < 16; ++v) y = acc_row(v, h) == c ? x[v] : y;
  return y + swap_halves(y);
}

// Sum over the wavefront; every lane gets it.
__device__ __forceinline__ float sum64(float x) {
  x = reduce32(x, [](float p, float q) { return p + q; });
  return x + swap_halves(x);
}

}  // namespace sa
