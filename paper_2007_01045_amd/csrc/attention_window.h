// Attention of the visible pairs only, forward and backward: the kernels of attention_window.hip (a window and sinks, sequences of
// equal stride: what is described here) and of attention_docs.hip (runs from arrays, capped and lowered logits).
//   query i sees key j of its sequence where  j < len  and  (not causal or j <= i)  and  (W = 0 or |i - j| < W or j < S)
//   -- a window of W positions, and the first S keys for every query.  A query heads share Ak key heads, A / Ak
//   neighbouring ones each.  ctx = softmax(scale q k^T) v over the visible keys, lse = log2 of the sum of 2^(scale2 q k)
//   (-infinity and ctx = 0 for rows at and behind len: they see nothing),  delta = rowsum(dctx o ctx),
//   dv = P^T dctx,  dS = P o (dP - delta),  dq = scale dS k,  dk = scale dS^T q, dk and dv summed over the sharing heads.
//
// The orientation is that of attention.hip: a wave owns 32 query rows (forward, dq) or 32 key rows (dk, dv), 64-row blocks of the
// other side stream through a ring in LDS, the accumulator's lane index is the row the wave owns.  What is visible to a row
// is one run of the other side's rows, and for queries the sinks besides: [lo, hi) and [0, S).  So a workgroup walks the
// blocks that hold sinks and then the blocks of its rows' runs, skips in each wave what none of its 32 rows sees, and compares
// element by element only in blocks that some row sees in part.  Bound by the chain MFMA -> exponentials -> MFMA like the kernels
// without a window; the work is that of the visible blocks.
//
// dk and dv of a key: the query blocks that see it, for each of the sharing heads, one walk.  Where the walks are longer than
// others (keys among the sinks: every query sees them) or too few to fill the chip, a walk is cut into parts (make_plan); each
// part leaves fp32 sums in the workspace, and a second kernel adds them in ascending order: no atomics, the same bits every time.
//
// bf16: P and dS are rounded once, to bf16, as operands of their products; logits, statistics, dP and all sums are fp32.  Outputs are then
// off by 0.0019 to 0.0020 (ctx) and 0.0024 (dq, dk, dv) in the 2-norm, where their own rounding alone leaves 0.0017; operands of 24 bits, three of
// bf16 each as in attention.hip, would triple the second products' MFMAs.
//
// Rows at and behind len may hold anything: their q, k, v and dctx are never used (they read as zeros, past the buffer's records),
// and their outputs are zeros.
#pragma once
#include <algorithm>
#include <type_traits>

#include "attention_tile.h"
#include "walk_parts.h"

namespace dapple {

// Workgroups go round robin to the eight XCDs, each with an L2 of its own: XCD x takes the x-th eighth of the range, so that
// tiles of one head, and heads that share keys, find each other's rows there.
__device__ __forceinline__ unsigned spread(unsigned id, unsigned n) {
  const unsigned per = n / 8;
  return id < per * 8 ? (id & 7) * per + (id >> 3) : id;
}

// Sequence and head of the u-th of all, n heads to a sequence: the heads of a sequence one after the other; where the sequences
// have lengths of their own, the sequences of a head, so that each XCD gets some of every length (4 sequences of 1987 rows
// and less, 16 heads of 64, window 256: forward 45 -> 42 us, backward 114 -> 103).
__device__ __forceinline__ void unit_of(const AttnWinArgs& a, int u, int n, int& bi, int& head) {
  bi = a.lens ? u % a.b : u / n;
  head = a.lens ? u / a.b : u % n;
}

template <int M>
__device__ __forceinline__ int len_of(const AttnWinArgs& a, int bi) {
  if (M == MASK_SPANS) return min(max(a.spans[4L * a.s], 0), a.s);
  return a.lens ? min(max(a.lens[bi], 0), a.s) : a.s;
}

// MASK_SPANS: the runs come from arrays (doc_spans), of key_lo, key_hi, query_lo and query_hi, none of which ever falls from row to row (behind
// the last document all are its end: a row there may stand for the last one, and no index waits for the length)
__device__ __forceinline__ int span_of(const AttnWinArgs& a, int which, int i) {
  return min(max(a.spans[(long)which * a.s + min(i, a.s - 1)], 0), a.s);
}
// the last of n rows from row i on that may be asked for
template <int M>
__device__ __forceinline__ int last_row(const AttnWinArgs& a, int i, int n, int len) { return min(i + n, M == MASK_SPANS ? a.s : len) - 1; }
// keys that query i sees: [lo, hi) and [0, min(S, hi))
template <int M>
__device__ __forceinline__ int key_lo(const AttnWinArgs& a, int i) {
  if (M == MASK_SPANS) return span_of(a, 0, i);
  return a.W ? max(0, i - a.W + 1) : 0;
}
template <int M>
__device__ __forceinline__ int key_hi(const AttnWinArgs& a, int i, int len) {
  if (M == MASK_SPANS) return min(len, span_of(a, 1, i));
  return min(len, a.causal ? i + 1 : a.W ? max(i + a.W, a.S) : len);   // (W < s and S <= s, below 2^27)
}
// queries that see key j: [lo, hi)
template <int M>
__device__ __forceinline__ int query_lo(const AttnWinArgs& a, int j) {
  if (M == MASK_SPANS) return span_of(a, 2, j);
  return a.causal ? j : a.W && j >= a.S ? max(0, j - a.W + 1) : 0;
}
template <int M>
__device__ __forceinline__ int query_hi(const AttnWinArgs& a, int j, int len) {
  if (M == MASK_SPANS) return min(len, span_of(a, 3, j));
  return a.W && j >= a.S ? min(len, j + a.W) : len;
}
// whether key j is a sink: every query sees it
template <int M>
__device__ __forceinline__ bool is_sink(const AttnWinArgs& a, int j) { return M == MASK_WINDOW && a.W && j < a.S; }

// The logit, in log2 units, of a product `raw`: unit t - slope2 |distance|, where t is raw, or its cap:
//   t = tanh(x), x = raw scale / cap, unit = cap log2(e);   d logit / d raw = (1 - t^2) scale log2(e).
// Backward, whose results are rounded to bf16: tanh(x) = 1 - 2 / (1 + e^2x), off by an ulp or two of 1 whatever x: two instructions of four times
// the others' time.  Us, 4 documents of 2048 rows, both directions, cap 50, products up to about 30 / four times that and more: 16
// heads of 128 on 4 554 / 558, of 64 352 / 358; a polynomial where all products of a wave's block are small, and there alone, took 547 / 691 and
// 353 / 463.  Forward, whose lse is fp32 and, where few keys are seen, hardly more than a logit: with e = e^-2|x|, tanh |x| = (1 - e) / (1 + e), where
// only e's own rounding counts against 1 (by 2^-25) and the others against tanh x.  Documents of one row, random q and k of 64, cap 50: lse off by 4.6e-7 in the
// 2-norm, 2.3e-6 by the backward's form.  It costs two instructions more, us: 191 where that took 181 (128 wide), 134 / 123 (64).  A polynomial
// below |x| = 1/16 besides, for relative precision down to 0, took 211 and 154, and 185 and 123 for the rows that see fewer than 8 keys alone, but 33
// where this takes 31 (30 before) on 200 documents of 40 rows.
constexpr bool capped(int S) { return S == SCORE_CAP || S == SCORE_BOTH; }
constexpr bool sloped(int S) { return S == SCORE_SLOPE || S == SCORE_BOTH; }
template <int S>
struct Score {
  float unit, slope2, bend, bend2;   // slope2: -slope log2(e); bend: scale / cap; bend2 = 2 bend log2(e)
  __device__ __forceinline__ Score(const AttnWinArgs& a, float scale2) : unit(capped(S) ? a.cap2 : scale2), slope2(0.f), bend(a.bend), bend2(a.bend * (2.f * LOG2E)) {}
  __device__ __forceinline__ void head(const AttnWinArgs& a, int h) {
    if (sloped(S)) slope2 = a.slopes ? a.slopes[h] * -LOG2E : 0.f;
  }
  __device__ __forceinline__ float of(float raw) const {   // t
    return capped(S) ? fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(raw * bend2)), 1.f) : raw;
  }
  __device__ __forceinline__ float of_fwd(float raw) const {
    if (!capped(S)) return raw;
    const float a = raw * bend2, e = __builtin_amdgcn_exp2f(-fabsf(a));
    return copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), a);
  }
  template <bool FWD = false, typename V>
  __device__ __forceinline__ void cap(V& raw) const {
#pragma unroll
    for (int v = 0; v < 16; ++v) raw[v] = FWD ? of_fwd(raw[v]) : of(raw[v]);
  }
  // the logit less l; far: the rows' distance, of either sign
  __device__ __forceinline__ float less(float t, float far, float l) const {
    const float s = fmaf(t, unit, -l);
    return sloped(S) ? fmaf(slope2, fabsf(far), s) : s;
  }
  __device__ __forceinline__ float derivative(float t) const { return capped(S) ? fmaf(-t, t, 1.f) : 1.f; }
  // With slopes: the logits of a block of the other side's rows r0 + 8 (v >> 2) + (v & 3) (4 h is in r0) against the lane's row, less what is
  // returned, which is the same for all of them: on one side of the rows the bias is linear, and a constant for each v.  row0: the wave's
  // first row, b0: the block's (both the same for the wave)
  template <typename V>
  __device__ __forceinline__ float block(const V& t, float (&o)[16], int row, int r0, int row0, int b0) const {
    if (b0 + 31 <= row0) {
#pragma unroll
      for (int v = 0; v < 16; ++v) o[v] = fmaf(t[v], unit, -(float)(8 * (v >> 2) + (v & 3)) * slope2);
      return (float)(row - r0) * slope2;
    }
    if (b0 >= row0 + 31) {
#pragma unroll
      for (int v = 0; v < 16; ++v) o[v] = fmaf(t[v], unit, (float)(8 * (v >> 2) + (v & 3)) * slope2);
      return (float)(r0 - row) * slope2;
    }
    const float x = (float)(row - r0);
#pragma unroll
    for (int v = 0; v < 16; ++v) o[v] = less(t[v], x - (8 * (v >> 2) + (v & 3)), 0.f);
    return 0.f;
  }
  // fp32: tanh of full precision, and no cap at all at run time (bend 0).  t: for derivative()
  __device__ __forceinline__ float less32(float raw, float scale2, float far, float l, float& t) const {
    t = 0.f;
    float s = raw * scale2;
    if (bend > 0.f) {
      t = tanhf(raw * bend);
      s = unit * t;
    }
    return fmaf(slope2, fabsf(far), s) - l;
  }
};

// The blocks of BLK keys that the queries q0 .. q1 of a workgroup see: `first` ones of the sinks, then from lo on, n in all
template <int M>
struct KeyWalk {
  int first, lo, n;
  // the queries' runs begin at key `begin` and end before `end`; any: whether there are queries at all
  __device__ __forceinline__ KeyWalk(const AttnWinArgs& a, int begin, int end, bool any, int blk) {
    lo = begin / blk;
    first = M == MASK_WINDOW && a.W ? min((a.S + blk - 1) / blk, lo) : 0;
    n = any ? first + (end + blk - 1) / blk - lo : 0;
  }
  __device__ __forceinline__ int block(int t) const { return t < first ? t : lo + t - first; }
};
// What the R queries of a wave from row0 on see, what the n of its workgroup from t0 on do, and the documents' length.  Of MASK_SPANS in two
// loads, a row's ends and the rest to a lane each, that wait for nothing and are waited for once: one by one, each had to wait for the last
// (8192 rows of 16 heads, forward: 2 % less at widths 64 and 128).  For what sees a wave's keys (KeyRows) it gave nothing and took 1 to 3 % at width 64.
template <int M, int R>
struct WaveRows {
  int len, lo, hi;                        // the lane's row's run; hi = 0 behind the last
  int lo_min, lo_max, hi_min, hi_max;     // of the wave's rows: the least and the greatest beginning and end of a run
  int walk_lo, walk_hi;                   // of the workgroup's rows: where the first run begins, the last ends
  __device__ __forceinline__ WaveRows(const AttnWinArgs& a, int bi, int row0, int t0, int n, int lane) {
    const int row = row0 + (lane & (R - 1));
    if constexpr (M == MASK_SPANS) {
      const int end = a.s - 1, x = lane & 3;
      const long at = (lane / R & 1) * (long)a.s + min(row, end);
      const long of = x == 2 ? 4L * a.s : x % 2 * (long)a.s + min(x ? t0 + n - 1 : t0, end);
      const int own = min(max(a.spans[at], 0), a.s), rest = min(max(a.spans[of], 0), a.s);
      len = __builtin_amdgcn_readlane(rest, 2);
      walk_lo = __builtin_amdgcn_readlane(rest, 0);
      walk_hi = min(len, __builtin_amdgcn_readlane(rest, 1));
      lo_min = __builtin_amdgcn_readlane(own, 0);
      lo_max = __builtin_amdgcn_readlane(own, R - 1);
      hi_min = min(len, __builtin_amdgcn_readlane(own, R));
      hi_max = min(len, __builtin_amdgcn_readlane(own, 2 * R - 1));
      if constexpr (R == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap((unsigned)own, (unsigned)own, false, false);
        lo = (int)r[0];
        hi = (int)r[1];
      } else {
        lo = __shfl(own, lane & (R - 1), 64);
        hi = __shfl(own, R + (lane & (R - 1)), 64);
      }
      hi = row < len ? min(len, hi) : 0;
    } else {
      len = len_of<M>(a, bi);
      const int qb = min(row0 + R, len) - 1;   // the wave's last row
      lo = key_lo<M>(a, row), hi = row < len ? key_hi<M>(a, row, len) : 0;
      lo_min = key_lo<M>(a, row0), lo_max = key_lo<M>(a, qb);
      hi_min = row0 + R - 1 < len ? key_hi<M>(a, row0, len) : 0, hi_max = key_hi<M>(a, qb, len);
      walk_lo = key_lo<M>(a, t0), walk_hi = key_hi<M>(a, min(t0 + n, len) - 1, len);
    }
  }
};
// whether a wave's rows, whose runs begin at lo_min and end at hi_max, see any of keys k0 .. k1
template <int M>
__device__ __forceinline__ bool any_seen(const AttnWinArgs& a, int k0, int k1, int lo_min, int hi_max) {
  return k0 < hi_max && (k1 >= lo_min || (M == MASK_WINDOW && k0 < a.S));
}
template <int M>
__device__ __forceinline__ bool sees(const AttnWinArgs& a, int j, int lo, int hi) { return j < hi && (j >= lo || (M == MASK_WINDOW && j < a.S)); }

// x[v] = hidden where a lane's row does not see element v of a 32-row accumulator block that begins at row r0 of the other side:
// rows r0 + 8 (v >> 2) + 4 h + (v & 3), the row's run [lo, hi), and [0, S) besides.  In an instruction or two per bound: the bounds
// are taken relative to the lane's first row, and one that lies outside the block for all rows of the wave is not compared
// (below: some row's run begins inside; above: some row's ends inside).
template <bool SINKS>
__device__ __forceinline__ void hide(float (&x)[16], float hidden, int r0, int h, int lo, int hi, int S, bool below, bool above) {
  const int l = lo - r0 - 4 * h, u = hi - r0 - 4 * h, s = S - r0 - 4 * h;
  if (above) {
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 8 * (v >> 2) + (v & 3) < u ? x[v] : hidden;
  }
  if (!below) return;
  if (SINKS && S > r0) {
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 8 * (v >> 2) + (v & 3) >= l || 8 * (v >> 2) + (v & 3) < s ? x[v] : hidden;
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 8 * (v >> 2) + (v & 3) >= l ? x[v] : hidden;
  }
}

// Workgroup id's head and its place among that head's.  Of g heads' greatest common divisor with the eight XCDs: 8 / g XCDs share heads / g heads,
// which take turns.  A launch has heads_grid() workgroups, some of them with a place past the last.
__host__ __device__ inline int heads_gcd(int heads) { return heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1; }
__host__ __device__ inline unsigned heads_grid(int heads, long places) {
  const int g = heads_gcd(heads), xcds = 8 / g;
  return (unsigned)((places * (heads / g) + xcds - 1) / xcds * 8);
}
__device__ __forceinline__ void by_heads(unsigned id, int heads, int& head, int& place) {
  const unsigned g = heads_gcd(heads), each = (unsigned)heads / g, x = id & 7, turn = (id >> 3) * (8 / g) + x / g;
  head = (x % g) * each + turn % each;
  place = turn / each;
}

// The query tile of workgroup id of n.  MASK_WINDOW: the last tiles first (causal: they have the longest walks).
// MASK_SPANS: likewise, all heads by turns.  RANKED: where the workgroups do not all run at once, the longest walks first: a long one that
// begins last would be what the launch ends with.  Each wave ranks the tiles itself, up to 64 groups of neighbours, one to a lane, by the walk
// of a group's last row.  That is for dq, whose workgroups follow those of dk and dv; a forward whose long walks share the units from the start
// is slower.  Us ranked / as they lie, packed documents of 3, 6 and 12 (6, 8, 14; 3, 6, 7), gradient: 8192 rows of 16 heads of 128 749 / 778, 409 / 412,
// 253 / 287; 6001 rows of 16 heads of 64 180 / 178, 114 / 115, 89 / 100; fp32, 1554 rows of 12 heads 101 / 98, 88 / 93, 85 / 85.  Forward: 291 / 258, 149 /
// 145, 95 / 97; 104 / 95, 65 / 61, 56 / 54; 49 / 44, 44 / 43, 40 / 34.
template <int M, bool RANKED>
struct QueryTask {
  int tile, bi, hh;
  bool run = true;
  __device__ __forceinline__ QueryTask(const AttnWinArgs& a, unsigned id, unsigned n, int q_tiles, int rows, int lane) {
    if constexpr (M == MASK_WINDOW) {
      id = spread(id, n);
      tile = q_tiles - 1 - id % q_tiles;
      unit_of(a, id / q_tiles, a.A, bi, hh);
      return;
    }
    int rank;
    by_heads(id, a.A, hh, rank);
    bi = 0;
    tile = q_tiles - 1 - rank;
    run = rank < q_tiles;
    if (!RANKED || n <= 256 || !run) return;
    const int group = (q_tiles + 63) / 64, groups = (q_tiles + group - 1) / group, first = lane * group, last = min(first + group, q_tiles) - 1;
    int walk = -1;
    if (lane < groups) {
      const int row = min((last + 1) * rows, a.s) - 1;
      walk = max(span_of(a, 1, row) - span_of(a, 0, last * rows), 0);
    }
    int before = 0;   // tiles of the groups that come before the lane's
    for (int g = 0; g < groups; ++g) {
      const int other = __builtin_amdgcn_readlane(walk, g);
      if (other > walk || (other == walk && g > lane)) before += g == groups - 1 ? q_tiles - g * group : group;
    }
    const unsigned long long mine = __ballot(lane < groups && rank >= before && rank < before + last - first + 1);
    const int at = __builtin_ctzll(mine);
    tile = __builtin_amdgcn_readlane(last, at) - (rank - __builtin_amdgcn_readlane(before, at));
  }
};

// A workgroup of the dk, dv launch: KT keys of a key head, and a part of their walk over the sharing heads' query blocks
template <int M>
struct KeyTask {
  int bi, kv, k0, len, qlo, nq, n0, n1, slot;   // blocks of the walk [n0, n1): head n / nq, block qlo + n % nq; slot < 0: no parts
  bool run;
  __device__ __forceinline__ KeyTask() {}
  __device__ __forceinline__ void span(const AttnWinArgs& a, int kt, int blk) {
    const int k1 = last_row<M>(a, k0, kt, len);
    qlo = nq = 0;
    if (k0 >= len) return;
    const bool sink = is_sink<M>(a, k0);   // the walk of the tile's first key has the lower end of all, its last key's the upper,
                                         // but a sink's is everything
    qlo = (sink && !a.causal ? 0 : query_lo<M>(a, k0)) / blk;
    nq = ((sink ? len : query_hi<M>(a, k1, len)) + blk - 1) / blk - qlo;
    if (M == MASK_SPANS) nq = max(nq, 0);
  }
  // t: the workgroup of n
  __device__ __forceinline__ KeyTask(const AttnWinArgs& a, unsigned t, unsigned n, int kt, int blk) {
    const WinPlan& p = a.plan;
    if constexpr (M == MASK_SPANS) {
      int rank;
      by_heads(t, a.Ak, kv, rank);
      bi = 0;
      slot = -1;
      n0 = n1 = 0;
      run = rank < a.table[0];
      if (!run) return;
      const int32_t* const e = a.table + 4 + 4L * rank;   // tile, the part's blocks, slot
      k0 = e[0] * kt;
      len = len_of<M>(a, bi);
      span(a, kt, blk);
      n0 = e[1];
      n1 = e[2];
      if (e[3] >= 0) slot = kv * p.slots + e[3];
      return;
    }
    init(a, spread(t, n), kt, blk);
  }
  __device__ __forceinline__ void init(const AttnWinArgs& a, unsigned t, int kt, int blk) {
    const WinPlan& p = a.plan;
    const int sinks = p.sink_tiles * p.sink_parts, per = sinks + (p.key_tiles - p.sink_tiles) * p.parts;
    const int head = t / per, r = t % per;
    unit_of(a, head, a.Ak, bi, kv);
    const bool sink = r < sinks;
    const int parts = sink ? p.sink_parts : p.parts, u = sink ? r : r - sinks;
    const int tile = u / parts + (sink ? 0 : p.sink_tiles), part = u % parts;
    k0 = tile * kt;
    len = len_of<M>(a, bi);
    span(a, kt, blk);
    const int all = nq * (a.A / a.Ak), steps = sink ? p.sink_steps : p.steps;
    n0 = parts > 1 ? min(all, part * steps) : 0;
    n1 = parts > 1 ? min(all, n0 + steps) : all;
    slot = parts > 1 ? head * p.slots + (sink || p.sink_parts == 1 ? 0 : sinks) + u : -1;
    run = parts == 1 || n0 < n1;
  }
};

// What sees the R keys of a wave from row0 on: of the lane's key, and the least and the greatest beginning and end of the wave's
template <int M, int R>
struct KeyRows {
  int lo, hi, lo_min, lo_max, hi_min, hi_max;
  __device__ __forceinline__ KeyRows(const AttnWinArgs& a, int row0, int len, int lane) {
    const int krow = row0 + (lane & (R - 1)), kb = last_row<M>(a, row0, R, len);
    lo = query_lo<M>(a, krow), hi = krow < len ? query_hi<M>(a, krow, len) : 0;
    const bool sink = is_sink<M>(a, row0);
    lo_min = sink && !a.causal ? 0 : query_lo<M>(a, row0), lo_max = query_lo<M>(a, kb);
    hi_max = sink ? len : query_hi<M>(a, kb, len);
    hi_min = row0 + R - 1 < len ? query_hi<M>(a, sink ? min(kb, a.S) : row0, len) : 0;
  }
};

// ------------------------------------------------------------------ bf16
template <int D, int NW, bool STATS>
using WinRing = Ring<D, NW, D == 128 ? 2 : 3, STATS>;

// o: accumulators of 32 rows (lane & 31) x D columns; D = 128 in two halves, which the ring's LDS has room for
template <int D>
__device__ __forceinline__ void store_rows(unsigned char* sm, int wave, const f32x16* o, float f, bf16* C, float* C32, long ld, int rows, int d, int lane) {
  constexpr int NDB = D / 32 < 2 ? D / 32 : 2;
  float* const S = (float*)(sm + wave * OutTile<NDB>::BYTES);
#pragma unroll
  for (int c = 0; c < D / 32; c += NDB)
    OutTile<NDB>::store(S, o + c, f, C + 32 * c, C32 ? C32 + 32 * c : nullptr, ld, rows, d - 32 * c, lane);
}

// NW: waves per workgroup (4, or 2 where the grid is small), each with 32 query rows
template <int M, int S, int D, int NW>
__global__ __launch_bounds__(64 * NW, D <= 64 ? 3 : 2) void attn_win_fwd(AttnWinArgs a, float scale2) {
  constexpr int NKK = D / 16, NDB = D / 32;
  typedef WinRing<D, NW, false> R;
  extern __shared__ __attribute__((aligned(1024))) unsigned char asm_[];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q_tiles = (a.s + 32 * NW - 1) / (32 * NW);
  const QueryTask<M, false> task(a, blockIdx.x, gridDim.x, q_tiles, 32 * NW, lane);
  if (!task.run) return;
  const int tile = task.tile, bi = task.bi, hh = task.hh;
  Score<S> sc(a, scale2);
  sc.head(a, hh);
  const int kv = hh / (a.A / a.Ak);
  const int q0 = tile * 32 * NW, row0 = q0 + wave * 32, qrow = row0 + (lane & 31);
  const WaveRows<M, 32> seen(a, bi, row0, q0, 32 * NW, lane);
  const int len = seen.len, d = a.d, lo = seen.lo, hi = seen.hi, lo_min = seen.lo_min, lo_max = seen.lo_max, hi_min = seen.hi_min, hi_max = seen.hi_max;
  const long r0 = (long)bi * a.s;
  const bf16 *Q = (const bf16*)a.q + r0 * a.ldq + hh * d, *K = (const bf16*)a.k + r0 * a.ldk + kv * d, *V = (const bf16*)a.v + r0 * a.ldv + kv * d;
  const bool qok = qrow < len;
  const KeyWalk<M> walk(a, seen.walk_lo, seen.walk_hi, q0 < len, 64);
  bf16x8 qf[NKK];
#pragma unroll
  for (int kk = 0; kk < NKK; ++kk) qf[kk] = frag_global<true>(Q, qrow, qok, a.ldq, kk, lane, d);
  R ring;
  ring.init(wave < NW / 2 ? K : V, wave < NW / 2 ? a.ldk : a.ldv, len, d, wave, lane, [](int) { return (const float*)nullptr; });
  int asked = 0;
  auto ask = [&](int stage) __attribute__((always_inline)) {
    if (asked == walk.first) ring.seek(walk.lo, len, 0, 0);
    if (asked >= walk.n) ring.stop();   // past the last block: reads nothing
    ring.request(stage, lane);
    ++asked;
  };
#pragma unroll
  for (int t = 0; t < R::NS - 1; ++t) ask(t);
  __builtin_amdgcn_s_waitcnt(0x0F70);   // (once, with the ring's first blocks: below, the counts are the ring's alone)

  float m = -3e38f, l = 0.f;   // (finite: a row that has seen nothing yet keeps m - m = 0)
  f32x16 o[NDB];  // rows d = 32 dblk + 8 blk + 4 h + e, column = the lane's query
#pragma unroll
  for (int db = 0; db < NDB; ++db) o[db] = zero16();

  int stage = 0;
  for (int t = 0; t < walk.n; ++t) {
    R::wait();
    ask(stage == 0 ? R::NS - 1 : stage - 1);
    const bf16 *Ks = (const bf16*)(asm_ + stage * R::STAGE), *Vs = (const bf16*)((const unsigned char*)Ks + R::Y_OFF);
    stage = stage + 1 == R::NS ? 0 : stage + 1;
    const int k0 = walk.block(t) * 64;
    if (row0 >= len) continue;
    if (!any_seen<M>(a, k0, k0 + 63, lo_min, hi_max)) continue;
    float p[2][16], shift[2] = {0.f, 0.f};   // (with slopes: logits less their shift)
    float mx = -INFINITY;
    // (all LDS reads of a phase before its first MFMA: see attn_fwd_mfma)
    bf16x8 kf[2][NKK], vf[4][NDB];
    constexpr bool WHOLE = D <= 64;
    if (WHOLE) {
#pragma unroll
      for (int kb2 = 0; kb2 < 2; ++kb2)
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) kf[kb2][kk] = frag_rows<D>(Ks, kb2 * 32, kk, lane);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int kb2 = 0; kb2 < 2; ++kb2) {
      if (!WHOLE) {
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) kf[kb2][kk] = frag_rows<D>(Ks, kb2 * 32, kk, lane);
        __builtin_amdgcn_sched_barrier(0);
      }
      f32x16 sa = zero16();  // rows: key 32 kb2 + 8 blk + 4 h + e, column: query
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) sa = MFMA(kf[kb2][kk], qf[kk], sa);
      sc.template cap<true>(sa);
      if constexpr (sloped(S)) {
        const int b0 = k0 + 32 * kb2;
        shift[kb2] = sc.block(sa, p[kb2], qrow, b0 + 4 * h, row0, b0);
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) p[kb2][v] = sa[v];
      }
    }
#pragma unroll
    for (int kb2 = 0; kb2 < 2; ++kb2) hide<M == MASK_WINDOW>(p[kb2], -INFINITY, k0 + kb2 * 32, h, lo, hi, a.S, lo_max > k0 + kb2 * 32, hi_min < k0 + kb2 * 32 + 32);
    if constexpr (!sloped(S)) {
#pragma unroll
      for (int kb2 = 0; kb2 < 2; ++kb2)
#pragma unroll
        for (int v = 0; v < 16; ++v) mx = fmaxf(mx, p[kb2][v]);
    } else {
      float m1 = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, p[0][v]);
#pragma unroll
      for (int v = 0; v < 16; ++v) m1 = fmaxf(m1, p[1][v]);
      mx = fmaxf(mx + shift[0], m1 + shift[1]);
    }
    if (WHOLE) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int db = 0; db < NDB; ++db) vf[ks][db] = frag_cols<D>(Vs, db * 32, ks * 16, lane);
      __builtin_amdgcn_sched_barrier(0);
    }
    // (what the row's sums are relative to follows its maximum only when that is 2^8 above: seldom after a walk's first block.  The
    // probabilities keep their relative precision and the fp32 sums have room for it.  16 heads of 64, 4 x 1987 rows 42.2 -> 39.5 us,
    // 16 of 128, 8192 rows 114 -> 107)
    const float top = sloped(S) ? halves_max(mx) : halves_max(mx) * sc.unit, mn = top > m + 8.f ? top : m;
    const float alpha = __builtin_amdgcn_exp2f(m - mn);
    float rs = 0.f;
#pragma unroll
    for (int kb2 = 0; kb2 < 2; ++kb2)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        // (the bare v_exp_f32: a probability below 2^-126 may be zero, it is rounded to bf16)
        p[kb2][v] = __builtin_amdgcn_exp2f(sloped(S) ? p[kb2][v] + (shift[kb2] - mn) : fmaf(p[kb2][v], sc.unit, -mn));
        rs += p[kb2][v];
      }
    l = l * alpha + halves_sum(rs);
    m = mn;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const bf16x8 pf = acc_to_operand(p[ks >> 1], ks & 1);
      if (!WHOLE) {
#pragma unroll
        for (int db = 0; db < NDB; ++db) vf[ks][db] = frag_cols<D>(Vs, db * 32, ks * 16, lane);
      }
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db] = MFMA(vf[ks][db], pf, o[db]);
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);   // the ring's last requests (they read nothing) before the wave may end
  __syncthreads();                      // every wave is done with the ring
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  if (!qok) {   // (not 0 times what an infinite v may have made of them)
#pragma unroll
    for (int db = 0; db < NDB; ++db) o[db] = zero16();
  }
  const long o0 = (r0 + row0) * a.ldc + hh * d;
  store_rows<D>(asm_, wave, o, inv, (bf16*)a.ctx + o0, a.ctx32 ? a.ctx32 + o0 : nullptr, a.ldc, a.s - row0, d, lane);
  if (qrow < a.s && h == 0) a.lse[((long)bi * a.A + hh) * a.s + qrow] = l > 0.f ? m + log2f(l) : -INFINITY;
}

// the sums of a part of a walk, in the accumulators' own order
template <int D, int NW>
__device__ __forceinline__ void store_part(const AttnWinArgs& a, int slot, int wave, const f32x16* dk, const f32x16* dv, int lane) {
  float* const P = a.partial + (long)slot * 2 * 32 * NW * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {
      const int u = (((wave * (D / 32) + db) * 4 + blk) * 64 + lane) * 4;
      *(f32x4*)(P + u) = f32x4{dk[db][4 * blk], dk[db][4 * blk + 1], dk[db][4 * blk + 2], dk[db][4 * blk + 3]};
      *(f32x4*)(P + 32 * NW * D + u) = f32x4{dv[db][4 * blk], dv[db][4 * blk + 1], dv[db][4 * blk + 2], dv[db][4 * blk + 3]};
    }
}

// dk, dv of 32 keys a wave; query blocks of 64 stream through LDS with their lse and delta
template <int M, int S, int D, int NW, typename R>
__device__ __forceinline__ void win_dkdv(const AttnWinArgs& a, unsigned task, unsigned tasks, float scale2, float scale, unsigned char* sm) {
  constexpr int NKK = D / 16, NDB = D / 32;
  const KeyTask<M> w(a, task, tasks, 32 * NW, 64);
  if (!w.run) return;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = w.len, d = a.d, h0 = w.kv * (a.A / a.Ak);
  const long r0 = (long)w.bi * a.s;
  const bf16 *Q = (const bf16*)a.q + r0 * a.ldq + h0 * d, *G = (const bf16*)a.dctx + r0 * a.lddc + h0 * d;
  const bf16 *K = (const bf16*)a.k + r0 * a.ldk + w.kv * d, *V = (const bf16*)a.v + r0 * a.ldv + w.kv * d;
  const float *lse = a.lse + ((long)w.bi * a.A + h0) * a.s, *delta = a.delta + ((long)w.bi * a.A + h0) * a.s;
  const int row0 = w.k0 + wave * 32, krow = row0 + (lane & 31);
  const bool kok = krow < len;
  const KeyRows<M, 32> seen(a, row0, len, lane);
  const int lo = seen.lo, hi = seen.hi, lo_min = seen.lo_min, lo_max = seen.lo_max, hi_min = seen.hi_min, hi_max = seen.hi_max;

  bf16x8 kf[NKK], vf[NKK];
#pragma unroll
  for (int kk = 0; kk < NKK; ++kk) {
    kf[kk] = frag_global<true>(K, krow, kok, a.ldk, kk, lane, d);
    vf[kk] = frag_global<true>(V, krow, kok, a.ldv, kk, lane, d);
  }
  f32x16 dv[NDB], dk[NDB];  // rows d, column = the lane's key
#pragma unroll
  for (int db = 0; db < NDB; ++db) dv[db] = dk[db] = zero16();
  R ring;
  const bool first = wave < NW / 2;
  // (a query beyond the last: zero rows, lse and delta 0, and not visible)
  ring.init(first ? Q : G, first ? a.ldq : a.lddc, len, d, wave, lane, [&](int r) { return r == 0 ? lse : (r == 1 ? delta : nullptr); });
  int asked = w.n0, ahead = w.nq ? w.n0 / w.nq : 0, aq = w.nq ? w.n0 % w.nq : 0;   // the next block to request: head, block
  bool jump = true;
  auto ask = [&](int stage) __attribute__((always_inline)) {
    if (jump) ring.seek(w.qlo + aq, len, ahead * d * 2, (long)ahead * a.s * 4);
    if (asked >= w.n1) ring.stop();
    ring.request(stage, lane);
    ++asked;
    jump = ++aq == w.nq;
    if (jump) {
      aq = 0;
      ++ahead;
    }
  };
#pragma unroll
  for (int t = 0; t < R::NS - 1; ++t) ask(t);
  __builtin_amdgcn_s_waitcnt(0x0F70);   // (as in attn_win_fwd)

  Score<S> sc(a, scale2);
  int stage = 0, qblk = w.nq ? w.n0 % w.nq : 0, qhead = h0 + (w.nq ? w.n0 / w.nq : 0);
  sc.head(a, min(qhead, a.A - 1));
  for (int n = w.n0; n < w.n1; ++n) {
    R::wait();
    ask(stage == 0 ? R::NS - 1 : stage - 1);
    const bf16 *Qs = (const bf16*)(sm + stage * R::STAGE), *Gs = (const bf16*)((const unsigned char*)Qs + R::Y_OFF);
    const float *Ls = (const float*)((const unsigned char*)Qs + R::S_OFF), *Ds = Ls + 64;
    stage = stage + 1 == R::NS ? 0 : stage + 1;
    const int i0 = (w.qlo + qblk) * 64;
    if (sloped(S) && qblk == 0) sc.head(a, min(qhead, a.A - 1));
    qblk = qblk + 1 == w.nq ? 0 : qblk + 1;
    qhead += qblk == 0;
    if (row0 >= len) continue;
#pragma unroll
    for (int qb2 = 0; qb2 < 2; ++qb2) {
      const int j0 = i0 + qb2 * 32;
      if (j0 >= hi_max || j0 + 31 < lo_min) continue;
      // (all LDS reads of a phase before its first MFMA, see attn_fwd_mfma)
      bf16x8 qf[NKK], gf[NKK], gc[2][NDB], qc[2][NDB];
      f32x4 L4[4], D4[4];
      f32x16 sa = zero16(), dp;  // rows: query 32 qb2 + 8 blk + 4 h + e, column: key
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        qf[kk] = frag_rows<D>(Qs, qb2 * 32, kk, lane);
        gf[kk] = frag_rows<D>(Gs, qb2 * 32, kk, lane);
      }
#pragma unroll
      for (int blk = 0; blk < 4; ++blk) {
        L4[blk] = *(const f32x4*)(Ls + qb2 * 32 + 8 * blk + 4 * h);
        D4[blk] = *(const f32x4*)(Ds + qb2 * 32 + 8 * blk + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * blk + e] = D4[blk][e];   // (the product adds to -delta)
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        sa = MFMA(qf[kk], kf[kk], sa);
        dp = MFMA(gf[kk], vf[kk], dp);
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          gc[ks][db] = frag_cols<D>(Gs, db * 32, qb2 * 32 + ks * 16, lane);
          qc[ks][db] = frag_cols<D>(Qs, db * 32, qb2 * 32 + ks * 16, lane);
        }
      __builtin_amdgcn_sched_barrier(0);
      float p[16], ds[16];
      sc.cap(sa);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        p[v] = __builtin_amdgcn_exp2f(sc.less(sa[v], (float)(krow - j0 - 4 * h) - (8 * (v >> 2) + (v & 3)), L4[v >> 2][v & 3]));
        ds[v] = dp[v] * p[v];
        if (capped(S)) ds[v] *= sc.derivative(sa[v]);
      }
      hide<false>(p, 0.f, j0, h, lo, hi, 0, lo_max > j0, hi_min < j0 + 32);
      hide<false>(ds, 0.f, j0, h, lo, hi, 0, lo_max > j0, hi_min < j0 + 32);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 pf = acc_to_operand(p, ks), dsf = acc_to_operand(ds, ks);
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          dv[db] = MFMA(gc[ks][db], pf, dv[db]);
          dk[db] = MFMA(qc[ks][db], dsf, dk[db]);
        }
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);
  if (w.slot >= 0) {
    store_part<D, NW>(a, w.slot, wave, dk, dv, lane);
    return;
  }
  __syncthreads();
  store_rows<D>(sm, wave, dk, scale, (bf16*)a.dk + (r0 + row0) * a.lddk + w.kv * d, nullptr, a.lddk, a.s - row0, d, lane);
  store_rows<D>(sm, wave, dv, 1.f, (bf16*)a.dv + (r0 + row0) * a.lddv + w.kv * d, nullptr, a.lddv, a.s - row0, d, lane);
}

// dq of 32 queries a wave; key blocks of 64 stream through LDS
template <int M, int S, int D, int NW, typename R>
__device__ __forceinline__ void win_dq(const AttnWinArgs& a, unsigned id, unsigned ids, float scale2, float scale, unsigned char* sm) {
  constexpr int NKK = D / 16, NDB = D / 32;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q_tiles = (a.s + 32 * NW - 1) / (32 * NW);
  const QueryTask<M, true> task(a, id, ids, q_tiles, 32 * NW, lane);
  if (!task.run) return;
  const int tile = task.tile, bi = task.bi, hh = task.hh;
  Score<S> sc(a, scale2);
  sc.head(a, hh);
  const int kv = hh / (a.A / a.Ak);
  const int q0 = tile * 32 * NW, row0 = q0 + wave * 32, qrow = row0 + (lane & 31);
  const WaveRows<M, 32> seen(a, bi, row0, q0, 32 * NW, lane);
  const int len = seen.len, d = a.d, lo = seen.lo, hi = seen.hi, lo_min = seen.lo_min, lo_max = seen.lo_max, hi_min = seen.hi_min, hi_max = seen.hi_max;
  const long r0 = (long)bi * a.s;
  const bf16 *Q = (const bf16*)a.q + r0 * a.ldq + hh * d, *G = (const bf16*)a.dctx + r0 * a.lddc + hh * d;
  const bf16 *K = (const bf16*)a.k + r0 * a.ldk + kv * d, *V = (const bf16*)a.v + r0 * a.ldv + kv * d;
  const bool qok = qrow < len;
  const KeyWalk<M> walk(a, seen.walk_lo, seen.walk_hi, q0 < len, 64);
  const long st = ((long)bi * a.A + hh) * a.s + qrow;
  const float Lq = qok ? a.lse[st] : 0.f, Dq = qok ? a.delta[st] : 0.f;
  bf16x8 qf[NKK], gf[NKK];
#pragma unroll
  for (int kk = 0; kk < NKK; ++kk) {
    qf[kk] = frag_global<true>(Q, qrow, qok, a.ldq, kk, lane, d);
    gf[kk] = frag_global<true>(G, qrow, qok, a.lddc, kk, lane, d);
  }
  constexpr bool ADDS = D <= 64;   // the product dctx v adds to -delta (D = 128: no registers for it)
  f32x16 dp0;
#pragma unroll
  for (int v = 0; v < 16; ++v) dp0[v] = ADDS ? Dq : 0.f;
  f32x16 dq[NDB];  // rows d, column = the lane's query
#pragma unroll
  for (int db = 0; db < NDB; ++db) dq[db] = zero16();
  R ring;
  ring.init(wave < NW / 2 ? K : V, wave < NW / 2 ? a.ldk : a.ldv, len, d, wave, lane, [](int) { return (const float*)nullptr; });   // (the statistics' loads read nothing)
  int asked = 0;
  auto ask = [&](int stage) __attribute__((always_inline)) {
    if (asked == walk.first) ring.seek(walk.lo, len, 0, 0);
    if (asked >= walk.n) ring.stop();
    ring.request(stage, lane);
    ++asked;
  };
#pragma unroll
  for (int t = 0; t < R::NS - 1; ++t) ask(t);
  __builtin_amdgcn_s_waitcnt(0x0F70);   // (as in attn_win_fwd)

  int stage = 0;
  for (int t = 0; t < walk.n; ++t) {
    R::wait();
    ask(stage == 0 ? R::NS - 1 : stage - 1);
    const bf16 *Ks = (const bf16*)(sm + stage * R::STAGE), *Vs = (const bf16*)((const unsigned char*)Ks + R::Y_OFF);
    stage = stage + 1 == R::NS ? 0 : stage + 1;
    const int k0 = walk.block(t) * 64;
    if (row0 >= len) continue;
#pragma unroll
    for (int kb2 = 0; kb2 < 2; ++kb2) {
      const int j0 = k0 + kb2 * 32;
      if (!any_seen<M>(a, j0, j0 + 31, lo_min, hi_max)) continue;
      // (all LDS reads of a phase before its first MFMA, see attn_fwd_mfma; D = 128 in halves, for registers)
      constexpr int KB = D == 128 ? NKK / 2 : NKK, KS = D == 128 ? 1 : 2;
      bf16x8 kr[KB], vr[KB], kc[KS][NDB];
      f32x16 sa = zero16(), dp = dp0;  // rows: key 32 kb2 + 8 blk + 4 h + e, column: query
#pragma unroll
      for (int k8 = 0; k8 < NKK; k8 += KB) {
#pragma unroll
        for (int kk = 0; kk < KB; ++kk) {
          kr[kk] = frag_rows<D>(Ks, kb2 * 32, k8 + kk, lane);
          vr[kk] = frag_rows<D>(Vs, kb2 * 32, k8 + kk, lane);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < KB; ++kk) {
          sa = MFMA(kr[kk], qf[k8 + kk], sa);
          dp = MFMA(vr[kk], gf[k8 + kk], dp);
        }
        if (D == 128) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int db = 0; db < NDB; ++db) kc[ks][db] = frag_cols<D>(Ks, db * 32, kb2 * 32 + ks * 16, lane);
      __builtin_amdgcn_sched_barrier(0);
      float ds[16];
      sc.cap(sa);
      if constexpr (S == SCORE_SLOPE) {
        const float c = sc.block(sa, ds, qrow, j0 + 4 * h, row0, j0) - Lq;
#pragma unroll
        for (int v = 0; v < 16; ++v) ds[v] = __builtin_amdgcn_exp2f(ds[v] + c) * (ADDS ? dp[v] : dp[v] + Dq);
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          ds[v] = __builtin_amdgcn_exp2f(sc.less(sa[v], (float)(qrow - j0 - 4 * h) - (8 * (v >> 2) + (v & 3)), Lq)) * (ADDS ? dp[v] : dp[v] + Dq);
          if (capped(S)) ds[v] *= sc.derivative(sa[v]);
        }
      }
      hide<M == MASK_WINDOW>(ds, 0.f, j0, h, lo, hi, a.S, lo_max > j0, hi_min < j0 + 32);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 dsf = acc_to_operand(ds, ks);
        if (ks >= KS) {
#pragma unroll
          for (int db = 0; db < NDB; ++db) kc[0][db] = frag_cols<D>(Ks, db * 32, kb2 * 32 + ks * 16, lane);
        }
#pragma unroll
        for (int db = 0; db < NDB; ++db) dq[db] = MFMA(kc[ks < KS ? ks : 0][db], dsf, dq[db]);
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  if (!qok) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) dq[db] = zero16();
  }
  store_rows<D>(sm, wave, dq, scale, (bf16*)a.dq + (r0 + row0) * a.lddq + hh * d, nullptr, a.lddq, a.s - row0, d, lane);
}

// Both kinds of workgroups in one launch, dk and dv first: they share a compute unit and fill each other's waits (as in attention.hip).
// D <= 64
template <int M, int S, int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_win_bwd(AttnWinArgs a, float scale2, float scale) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char asm_[];
  typedef WinRing<D, NW, true> R;
  const unsigned nk = a.plan.key_tasks;
  if (blockIdx.x < nk) win_dkdv<M, S, D, NW, R>(a, blockIdx.x, nk, scale2, scale, asm_);
  else win_dq<M, S, D, NW, R>(a, blockIdx.x - nk, gridDim.x - nk, scale2, scale, asm_);
}

// dk and dv of 128 keys at D = 128.  A wave that does all four products holds 128 registers of sums, 64 of keys and values and 32 of
// the products before the exponentials, and is alone on its SIMD: its chain of MFMA -> exponentials -> MFMA waits for itself.  So the
// chain is cut in two: waves 0-3 own 32 keys each, make S and dP of 32 queries (a step) and leave P and dS in LDS, as the operands
// they are; waves 4-7, a step behind, hold the sums of the same keys and add dctx^T P and Q^T dS to them.  One of each on a SIMD.  Waves
// 0-3 make the next step's S and dP between the exponentials of the current one.  Either kind reads its next fragments behind the
// MFMAs that used the last ones.
// Waves 0-3 do step i between barriers i and i + 1, waves 4-7 between i + 1 and i + 2.  Blocks of 32 queries lie in a ring of seven:
// block i + 2 has landed at barrier i, behind which its first fragments are read, and there block i + 5 is requested, into the place of
// block i - 2, whose last fragments were read before.
// 8192 rows, 16 heads on 4, window 1024: with waves that do all four products, one to a SIMD, dk, dv and dq took 432 us with the joining of
// parts, 343 so.  A step takes 2100 clocks, 1024 of them MFMAs on each SIMD; LDS is asked for 208 KB in it (1660 clocks at 128 bytes).
// A lane's LDS addresses of fragments (frag_rows, frag_cols) in a block of 64 x 128: all that depends on the lane, kept in a few
// registers; the block's place is added once a step, rows and the matrix are an instruction's immediate offset.
struct RowsAt {
  unsigned a[8];
  __device__ __forceinline__ explicit RowsAt(int lane) {
    const int r = lane & 31;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) a[kk] = r * 256 + (((kk * 2 + (lane >> 5)) ^ aswz<128>(r)) << 4);
  }
  // AT: rows' and the matrix's bytes
  template <int AT>
  __device__ __forceinline__ bf16x8 get(const unsigned char* sm, unsigned block, int kk) const {
    return *(const bf16x8*)(sm + (a[kk] + block) + AT);
  }
};
struct ColsAt {
  unsigned a[4][2];
  __device__ __forceinline__ explicit ColsAt(int lane) {
    const int i16 = lane & 15, r = 4 * (lane >> 5) + (i16 >> 2), c = 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int k = 0; k < 2; ++k) a[db][k] = (r + 8 * k) * 256 + ((((db * 32 + c) >> 3) ^ aswz<128>(r + 8 * k)) << 4) + (c & 7) * 2;
  }
  template <int AT>
  __device__ __forceinline__ bf16x8 get(const unsigned char* sm, unsigned block, int db) const {
    return join8(lds_read_tr16((const bf16*)(sm + (a[db][0] + block) + AT)), lds_read_tr16((const bf16*)(sm + (a[db][1] + block) + AT)));
  }
};
constexpr int PAIR_X = 4 * 4 * 1024;   // P and dS of a step: per wave two operands each of 16 bytes a lane
typedef Ring<128, 8, 7, true, 32> PairRing;
typedef Ring<128, 8, 4, true> PairDqRing;
constexpr int PAIR_BYTES = PairRing::BYTES + 2 * PAIR_X;
static_assert(PAIR_BYTES <= 160 * 1024 && PairDqRing::BYTES <= PAIR_BYTES && 8 * OutTile<2>::BYTES <= PairRing::BYTES,
              "LDS of a compute unit; the output's staging lies where the ring was");

template <int M, int S>
__device__ __forceinline__ void win_dkdv_pair(const AttnWinArgs& a, unsigned task, unsigned tasks, float scale2, float scale, unsigned char* sm) {
  constexpr int D = 128, NKK = 8, NDB = 4;
  typedef PairRing R;
  const KeyTask<M> w(a, task, tasks, 128, 32);
  if (!w.run) return;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), own = wave & 3;   // which 32 of the keys
  const int len = w.len, d = a.d, h0 = w.kv * (a.A / a.Ak);
  const long r0 = (long)w.bi * a.s;
  const bf16 *Q = (const bf16*)a.q + r0 * a.ldq + h0 * d, *G = (const bf16*)a.dctx + r0 * a.lddc + h0 * d;
  const float *lse = a.lse + ((long)w.bi * a.A + h0) * a.s, *delta = a.delta + ((long)w.bi * a.A + h0) * a.s;
  const int row0 = w.k0 + own * 32, krow = row0 + (lane & 31);
  const bool kok = krow < len;
  const KeyRows<M, 32> seen(a, row0, len, lane);
  const int lo_min = seen.lo_min, lo_max = seen.lo_max, hi_min = seen.hi_min, hi_max = row0 < len ? seen.hi_max : 0;
  unsigned char* const X = sm + R::BYTES + own * 4096 + lane * 16;

  R ring;
  const bool first = wave < 4;
  ring.init(first ? Q : G, first ? a.ldq : a.lddc, len, d, wave, lane, [&](int r) { return r == 0 ? lse : (r == 1 ? delta : nullptr); });
  int asked = w.n0, ahead = w.nq ? w.n0 / w.nq : 0, aq = w.nq ? w.n0 % w.nq : 0, slot = 0;   // the next block to request: head, block
  bool jump = true;
  auto ask = [&]() __attribute__((always_inline)) {
    if (jump) ring.seek(w.qlo + aq, len, ahead * d * 2, (long)ahead * a.s * 4);
    if (asked >= w.n1) ring.stop();
    ring.request(slot, lane);
    slot = slot == R::NS - 1 ? 0 : slot + 1;
    ++asked;
    jump = ++aq == w.nq;
    if (jump) {
      aq = 0;
      ++ahead;
    }
  };
  auto barrier = []() __attribute__((always_inline)) { R::wait<-3 * R::LOADS>(); };   // all but the two newest blocks have landed
  int stage = 0;
  if (first) {
    Score<S> sc(a, scale2);
    int qblk = w.nq ? w.n0 % w.nq : 0, qhead = h0 + (w.nq ? w.n0 / w.nq : 0);
    sc.head(a, min(qhead, a.A - 1));
    const bf16 *K = (const bf16*)a.k + r0 * a.ldk + w.kv * d, *V = (const bf16*)a.v + r0 * a.ldv + w.kv * d;
    const int lo = seen.lo, hi = seen.hi;
    constexpr int FD = 4;
    bf16x8 kf[NKK], vf[NKK], qf[FD], gf[FD];   // (qf, gf: FD k-steps' fragments, read so many ahead of their use)
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      kf[kk] = frag_global<true>(K, krow, kok, a.ldk, kk, lane, d);
      vf[kk] = frag_global<true>(V, krow, kok, a.ldv, kk, lane, d);
    }
    for (int t = 0; t < R::NS - 2; ++t) ask();
    __builtin_amdgcn_s_waitcnt(0x0F70);   // (as in attn_win_fwd)
    barrier();
    __builtin_amdgcn_s_setprio(2);   // (their products first: the exponentials then run beside the other wave's)
    const RowsAt fr(lane);
    // k-step kk of the fragments' block at `at` (kk < 8), or kk - 8 of the one at `next`
    auto fetch = [&](int kk, unsigned at, unsigned next) __attribute__((always_inline)) {
      qf[kk & (FD - 1)] = fr.get<0>(sm, kk < 8 ? at : next, kk & 7);
      gf[kk & (FD - 1)] = fr.get<R::Y_OFF>(sm, kk < 8 ? at : next, kk & 7);
    };
    auto slot_after = [](int t) { return t == R::NS - 1 ? 0 : t + 1; };
    // sa, dp: S and dP of the current step (rows: query 8 blk + 4 h + e of its block, column: key); sn, dn: of the next one, made
    // meanwhile: two MFMAs and two elements' exponentials by turns
    enum { HIDDEN, WHOLE, PART };
    auto step = [&](auto MODE, const f32x16& sa, const f32x16& dp, f32x16& sn, f32x16& dn, unsigned cur, unsigned at, unsigned next, unsigned char* x,
                    int j0) __attribute__((always_inline)) {
      constexpr int mode = decltype(MODE)::value;
      const float *Ls = (const float*)(sm + cur + R::S_OFF) + 4 * h, *Ds = Ls + 64;
      const int l = lo - j0 - 4 * h, u = hi - j0 - 4 * h;
      f32x4 L4[4], D4[4];
      if constexpr (mode != HIDDEN) {
#pragma unroll
        for (int blk = 0; blk < 4; ++blk) {
          L4[blk] = *(const f32x4*)(Ls + 8 * blk);
          D4[blk] = *(const f32x4*)(Ds + 8 * blk);
        }
      }
      sn = dn = zero16();
      float p[16], ds[16];
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        sn = MFMA(qf[kk & (FD - 1)], kf[kk], sn);
        dn = MFMA(gf[kk & (FD - 1)], vf[kk], dn);
        fetch(kk + FD, at, next);
        if constexpr (mode != HIDDEN) {
#pragma unroll
          for (int v = 2 * kk; v < 2 * kk + 2; ++v) {
            const float t = sc.of(sa[v]);
            p[v] = __builtin_amdgcn_exp2f(sc.less(t, (float)(krow - j0 - 4 * h) - (8 * (v >> 2) + (v & 3)), L4[v >> 2][v & 3]));
            ds[v] = (dp[v] + D4[v >> 2][v & 3]) * p[v];
            if (capped(S)) ds[v] *= sc.derivative(t);
            if constexpr (mode == PART) {
              const bool in = 8 * (v >> 2) + (v & 3) >= l && 8 * (v >> 2) + (v & 3) < u;
              p[v] = in ? p[v] : 0.f;
              ds[v] = in ? ds[v] : 0.f;
            }
          }
        }
        if (kk % 4 == 3) {
          const int ks = kk / 4;
          if constexpr (mode == HIDDEN) {   // (zeros: a branch round the other waves' products would move their sums between registers)
            *(f32x4*)(x + ks * 1024) = *(f32x4*)(x + (2 + ks) * 1024) = f32x4{0.f, 0.f, 0.f, 0.f};
          } else {
            *(bf16x8*)(x + ks * 1024) = acc_to_operand(p, ks);
            *(bf16x8*)(x + (2 + ks) * 1024) = acc_to_operand(ds, ks);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    typedef std::integral_constant<int, HIDDEN> Hidden;
    typedef std::integral_constant<int, WHOLE> Whole;
    typedef std::integral_constant<int, PART> Part;
    f32x16 s0, d0, s1, d1;
    int cur = 0, at = 1;   // places of the current step's block and the next one's
    {
#pragma unroll
      for (int kk = 0; kk < FD; ++kk) fetch(kk, 0, 0);
      s0 = d0 = zero16();
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        s0 = MFMA(qf[kk & (FD - 1)], kf[kk], s0);
        d0 = MFMA(gf[kk & (FD - 1)], vf[kk], d0);
        fetch(kk + FD, 0, R::STAGE);
      }
    }
    int n = w.n0;
    auto one = [&](const f32x16& sa, const f32x16& dp, f32x16& sn, f32x16& dn) __attribute__((always_inline)) {
      const int after = slot_after(at), j0 = (w.qlo + qblk) * 32;
      if (sloped(S) && qblk == 0) sc.head(a, min(qhead, a.A - 1));
      qblk = qblk + 1 == w.nq ? 0 : qblk + 1;
      qhead += qblk == 0;
      unsigned char* const x = X + (n & 1) * PAIR_X;
      barrier();
      ask();
      const unsigned c = cur * R::STAGE, f = at * R::STAGE, g = after * R::STAGE;
      if (j0 >= hi_max || j0 + 31 < lo_min) step(Hidden{}, sa, dp, sn, dn, c, f, g, x, j0);   // none of the wave's keys is seen
      else if (lo_max > j0 || hi_min < j0 + 32) step(Part{}, sa, dp, sn, dn, c, f, g, x, j0);
      else step(Whole{}, sa, dp, sn, dn, c, f, g, x, j0);
      cur = at;
      at = after;
      return ++n < w.n1;
    };
    if (n < w.n1)
      while (one(s0, d0, s1, d1) && one(s1, d1, s0, d0)) {}
    barrier();                            // (the last step of waves 4-7)
    __builtin_amdgcn_s_waitcnt(0x0F70);   // the last requests (they read nothing) before the wave may end
    __syncthreads();
    return;
  }
  f32x16 dv[NDB], dk[NDB];  // rows d, column = the lane's key
#pragma unroll
  for (int db = 0; db < NDB; ++db) dv[db] = dk[db] = zero16();
  for (int t = 0; t < R::NS - 2; ++t) ask();
  barrier();
  const ColsAt fc(lane);
  bf16x8 gc[NDB], qc[NDB];   // (of 16 queries, read that many MFMAs ahead of their use)
#pragma unroll
  for (int db = 0; db < NDB; ++db) {
    gc[db] = fc.get<R::Y_OFF>(sm, 0, db);
    qc[db] = fc.get<0>(sm, 0, db);
  }
  barrier();   // 0
  ask();
  for (int n = w.n0; n < w.n1; ++n) {
    const unsigned at = stage * R::STAGE;
    stage = stage == R::NS - 1 ? 0 : stage + 1;
    const unsigned next = stage * R::STAGE;
    const unsigned char* const x = X + (n & 1) * PAIR_X;
    barrier();   // n + 1
    ask();
    bf16x8 pf[2], dsf[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      pf[ks] = *(const bf16x8*)(x + ks * 1024);
      dsf[ks] = *(const bf16x8*)(x + (2 + ks) * 1024);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        dv[db] = MFMA(gc[db], pf[ks], dv[db]);
        dk[db] = MFMA(qc[db], dsf[ks], dk[db]);
        // the step's second 16 queries, the next step's first
        gc[db] = ks ? fc.get<R::Y_OFF>(sm, next, db) : fc.get<R::Y_OFF + 16 * 256>(sm, at, db);
        qc[db] = ks ? fc.get<0>(sm, next, db) : fc.get<16 * 256>(sm, at, db);
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
  if (w.slot >= 0) {
    store_part<D, 4>(a, w.slot, own, dk, dv, lane);
    return;
  }
  store_rows<D>(sm, own, dk, scale, (bf16*)a.dk + (r0 + row0) * a.lddk + w.kv * d, nullptr, a.lddk, a.s - row0, d, lane);
  store_rows<D>(sm, own, dv, 1.f, (bf16*)a.dv + (r0 + row0) * a.lddv + w.kv * d, nullptr, a.lddv, a.s - row0, d, lane);
}

// D = 128: dk and dv, and behind them the workgroups of dq, 256 queries each (none, where those are few: attn_win_dq)
template <int M, int S>
__global__ __launch_bounds__(512, 2) void attn_win_bwd_pair(AttnWinArgs a, float scale2, float scale) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char asm_[];
  const unsigned nk = a.plan.key_tasks;
  if (blockIdx.x < nk) win_dkdv_pair<M, S>(a, blockIdx.x, nk, scale2, scale, asm_);
  else win_dq<M, S, 128, 8, PairDqRing>(a, blockIdx.x - nk, gridDim.x - nk, scale2, scale, asm_);
}
template <int M, int S, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_win_dq(AttnWinArgs a, float scale2, float scale) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char asm_[];
  win_dq<M, S, 128, NW, WinRing<128, NW, true>>(a, blockIdx.x, gridDim.x, scale2, scale, asm_);
}

// ------------------------------------------------------------------ fp32 (see attention_f32.hip)
// RG: waves of a group, NG: groups.  A wave is a chain of MFMAs, exponentials and MFMAs, and the tiles of a micro-batch seldom give a SIMD
// more than one; so two groups share a tile, take the blocks of its walk by turns, and add what they have at the end.  Us forward
// and backward with one group of four waves, two of four, two of two: 2 x 777 rows, 12 heads of 64 on 6, window 200 111, 110, 101;
// 2 x 2048 rows, 16 heads, no window 940, 879, 914.
template <int D, int RG, int NG>
struct F32Lds {
  static constexpr int BLK = BR * (D + 8), STAT = 2 * BR;          // floats: a block; the statistics of one
  static constexpr int FLOATS = NG * (2 * BLK + STAT);
  // the second group's sums (n floats of a lane; n at most 2 D / 4)
  static_assert(NG == 1 || 64 * RG * (D / 2) <= FLOATS, "the sums lie where the blocks were");
};
// max and sum over the four lanes of one owned row (16 apart), in all of them: rows of 16 lanes change places, then half waves, without
// a trip through the LDS crossbar
__device__ __forceinline__ float groups_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return halves_max(fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])));
}
__device__ __forceinline__ float groups_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return halves_sum(__builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]));
}

template <int M, int S, int D, int RG, int NG>
__global__ __launch_bounds__(64 * RG * NG) void attn_win_fwd_f32(AttnWinArgs a, float scale2) {
  constexpr int NK = D / 16;
  extern __shared__ __attribute__((aligned(16))) float fsm[];
  const int tid = threadIdx.x & (64 * RG - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = lane >> 4;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * RG));
  float *const Ks = fsm + group * 2 * F32Lds<D, RG, NG>::BLK, *const Vs = Ks + F32Lds<D, RG, NG>::BLK;
  const int q_tiles = (a.s + 16 * RG - 1) / (16 * RG);
  const QueryTask<M, false> task(a, blockIdx.x, gridDim.x, q_tiles, 16 * RG, lane);
  if (!task.run) return;
  const int tile = task.tile, bi = task.bi, hh = task.hh;
  Score<S> sc(a, scale2);
  sc.head(a, hh);
  const int kv = hh / (a.A / a.Ak), q0 = tile * 16 * RG, row0 = q0 + wave * 16, qrow = row0 + (lane & 15);
  const WaveRows<M, 16> seen(a, bi, row0, q0, 16 * RG, lane);
  const int len = seen.len, d = a.d, lo = seen.lo, hi = seen.hi, lo_min = seen.lo_min, hi_max = seen.hi_max;
  const long r0 = (long)bi * a.s;
  const float *Q = (const float*)a.q + r0 * a.ldq + hh * d, *K = (const float*)a.k + r0 * a.ldk + kv * d, *V = (const float*)a.v + r0 * a.ldv + kv * d;
  const bool qok = qrow < len;
  const KeyWalk<M> walk(a, seen.walk_lo, seen.walk_hi, q0 < len, BR);
  f32x4 qf[NK];
  own_row<D>(Q + (long)qrow * a.ldq, qok, d, lane, qf);
  F32Block<D, 64 * RG> kb, vb;
  auto load = [&](int t) {
    const int k0 = walk.block(t) * BR;
    kb.load(K + (long)k0 * a.ldk, a.ldk, tid, len - k0, d);
    vb.load(V + (long)k0 * a.ldv, a.ldv, tid, len - k0, d);
  };
  __builtin_amdgcn_s_waitcnt(0x0F70);   // (the wave's own rows: waited for in the loop, the next block would be too)
  if (group < walk.n) load(group);
  float m = -3e38f, l = 0.f;
  f32x4 o[NK];   // rows d = 16 i + 4 g4 + e, column = the lane's query
#pragma unroll
  for (int i = 0; i < NK; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int n = group; n - group < walk.n; n += NG) {   // (both groups pass the same barriers)
    __syncthreads();
    kb.store(Ks, tid);
    vb.store(Vs, tid);
    __syncthreads();
    if (n + NG < walk.n) load(n + NG);
    if (n >= walk.n) continue;
    const int k0 = walk.block(n) * BR;
    if (row0 >= len || !any_seen<M>(a, k0, k0 + BR - 1, lo_min, hi_max)) continue;
    // All LDS reads of a phase before its first MFMA, the values' before the exponentials: read where they are used, each one was waited
    // for, 120 clocks to two MFMAs of 32 (36.9 -> 34.9 us for 2 x 777 rows, 12 heads of 64, window 200).
    f32x4 p[2], kf[2][NK];
    float mx = -INFINITY, vf[2][4][NK];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) kf[t][kk] = frow<D>(Ks, 16 * t, kk, lane);
    __builtin_amdgcn_sched_barrier(0);
    p[0] = p[1] = f32x4{0.f, 0.f, 0.f, 0.f};   // rows: key k0 + 16 t + 4 g4 + e, column: query
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < 2; ++t) p[t] = MFMA4(kf[t][kk][e], qf[kk][e], p[t]);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < NK; ++i) vf[t][e][i] = fcol<D>(Vs, 16 * i, 16 * t, e, lane);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float bent;
        const float x = S == SCORE_PLAIN ? p[t][e] * scale2 : sc.less32(p[t][e], scale2, (float)(qrow - k0 - 16 * t - 4 * g4 - e), 0.f, bent);
        p[t][e] = sees<M>(a, k0 + 16 * t + 4 * g4 + e, lo, hi) ? x : -INFINITY;
        mx = fmaxf(mx, p[t][e]);
      }
    // (a maximum that moves seldom, as in attn_win_fwd)
    const float top = groups_max(mx), mn = top > m + 8.f ? top : m, alpha = __builtin_amdgcn_exp2f(m - mn);
    float rs = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[t][e] = __builtin_amdgcn_exp2f(p[t][e] - mn);   // (the bare v_exp_f32: below 2^-126 of the row's largest it may be zero)
        rs += p[t][e];
      }
    l = l * alpha + groups_sum(rs);
    m = mn;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {
#pragma unroll
      for (int i = 0; i < NK; ++i) o[i] *= alpha;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < NK; ++i) o[i] = MFMA4(vf[t][e][i], p[t][e], o[i]);
  }
  if constexpr (NG == 2) {   // the second group's maximum, sum and o, of the same rows
    __syncthreads();
    if (group == 1) {
      fsm[tid] = m;
      fsm[64 * RG + tid] = l;
#pragma unroll
      for (int i = 0; i < NK; ++i) *(f32x4*)(fsm + 128 * RG + (i * 64 * RG + tid) * 4) = o[i];
    }
    __syncthreads();
    if (group == 1) return;
    const float m1 = fsm[tid], l1 = fsm[64 * RG + tid], mn = fmaxf(m, m1), f0 = exp2f(m - mn), f1 = exp2f(m1 - mn);
    l = l * f0 + l1 * f1;
    m = mn;
#pragma unroll
    for (int i = 0; i < NK; ++i) o[i] = o[i] * f0 + *(const f32x4*)(fsm + 128 * RG + (i * 64 * RG + tid) * 4) * f1;
  }
  if (qrow < a.s) {
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    const long at = (r0 + qrow) * a.ldc + hh * d;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int col = 16 * i + 4 * g4;
      if (col < d) {
        const f32x4 v = qok ? o[i] * inv : f32x4{0.f, 0.f, 0.f, 0.f};
        *(f32x4*)((float*)a.ctx + at + col) = v;
        if (a.ctx32) *(f32x4*)(a.ctx32 + at + col) = v;
      }
    }
    if (g4 == 0) a.lse[((long)bi * a.A + hh) * a.s + qrow] = l > 0.f ? m + log2f(l) : -INFINITY;
  }
}

// the second group's sums are added to the first's (which alone goes on: true)
template <int RG, int NG, int N>
__device__ __forceinline__ bool join_groups(f32x4 (&x)[N], float* fsm, int group, int tid) {
  if constexpr (NG == 2) {
    __syncthreads();
    if (group == 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) *(f32x4*)(fsm + (i * 64 * RG + tid) * 4) = x[i];
    }
    __syncthreads();
    if (group == 1) return false;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += *(const f32x4*)(fsm + (i * 64 * RG + tid) * 4);
  }
  return true;
}

template <int M, int S, int D, int RG, int NG>
__device__ __forceinline__ void win_dq_f32(const AttnWinArgs& a, unsigned id, unsigned ids, float scale2, float scale, float* fsm) {
  constexpr int NK = D / 16;
  const int tid = threadIdx.x & (64 * RG - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = lane >> 4;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * RG));
  float *const Ks = fsm + group * 2 * F32Lds<D, RG, NG>::BLK, *const Vs = Ks + F32Lds<D, RG, NG>::BLK;
  const int q_tiles = (a.s + 16 * RG - 1) / (16 * RG);
  const QueryTask<M, true> task(a, id, ids, q_tiles, 16 * RG, lane);
  if (!task.run) return;
  const int tile = task.tile, bi = task.bi, hh = task.hh;
  Score<S> sc(a, scale2);
  sc.head(a, hh);
  const int kv = hh / (a.A / a.Ak), q0 = tile * 16 * RG, row0 = q0 + wave * 16, qrow = row0 + (lane & 15);
  const WaveRows<M, 16> seen(a, bi, row0, q0, 16 * RG, lane);
  const int len = seen.len, d = a.d, lo = seen.lo, hi = seen.hi, lo_min = seen.lo_min, hi_max = seen.hi_max;
  const long r0 = (long)bi * a.s;
  const float *K = (const float*)a.k + r0 * a.ldk + kv * d, *V = (const float*)a.v + r0 * a.ldv + kv * d;
  const bool qok = qrow < len;
  const KeyWalk<M> walk(a, seen.walk_lo, seen.walk_hi, q0 < len, BR);
  f32x4 qf[NK], gf[NK];
  own_row<D>((const float*)a.q + (r0 + qrow) * a.ldq + hh * d, qok, d, lane, qf);
  own_row<D>((const float*)a.dctx + (r0 + qrow) * a.lddc + hh * d, qok, d, lane, gf);
  const long st = ((long)bi * a.A + hh) * a.s + qrow;
  const float Lq = qok ? a.lse[st] : 0.f, Dq = qok ? a.delta[st] : 0.f;
  f32x4 dq[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i) dq[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  F32Block<D, 64 * RG> kb, vb;
  auto load = [&](int t) {
    const int k0 = walk.block(t) * BR;
    kb.load(K + (long)k0 * a.ldk, a.ldk, tid, len - k0, d);
    vb.load(V + (long)k0 * a.ldv, a.ldv, tid, len - k0, d);
  };
  __builtin_amdgcn_s_waitcnt(0x0F70);   // (as in attn_win_fwd_f32)
  if (group < walk.n) load(group);
  for (int n = group; n - group < walk.n; n += NG) {   // (both groups pass the same barriers)
    __syncthreads();
    kb.store(Ks, tid);
    vb.store(Vs, tid);
    __syncthreads();
    if (n + NG < walk.n) load(n + NG);
    if (n >= walk.n) continue;
    const int k0 = walk.block(n) * BR;
    if (row0 >= len) continue;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (!any_seen<M>(a, k0 + 16 * t, k0 + 16 * t + 15, lo_min, hi_max)) continue;
      f32x4 s{0.f, 0.f, 0.f, 0.f}, dp{0.f, 0.f, 0.f, 0.f}, kf[NK], vf[NK];   // (reads first: see attn_win_fwd_f32)
      float kc[4][NK], ds[4];
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        kf[kk] = frow<D>(Ks, 16 * t, kk, lane);
        vf[kk] = frow<D>(Vs, 16 * t, kk, lane);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s = MFMA4(kf[kk][e], qf[kk][e], s);
          dp = MFMA4(vf[kk][e], gf[kk][e], dp);
        }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < NK; ++i) kc[e][i] = fcol<D>(Ks, 16 * i, 16 * t, e, lane);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float bent = 0.f;
        const float x = S == SCORE_PLAIN ? s[e] * scale2 - Lq : sc.less32(s[e], scale2, (float)(qrow - k0 - 16 * t - 4 * g4 - e), Lq, bent);
        ds[e] = __builtin_amdgcn_exp2f(x) * (dp[e] + Dq);
        if (capped(S)) ds[e] *= sc.derivative(bent);
        if (!sees<M>(a, k0 + 16 * t + 4 * g4 + e, lo, hi)) ds[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < NK; ++i) dq[i] = MFMA4(kc[e][i], ds[e], dq[i]);
    }
  }
  if (!join_groups<RG, NG>(dq, fsm, group, tid)) return;
  if (qrow < a.s) {
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int col = 16 * i + 4 * g4;
      if (col < d) *(f32x4*)((float*)a.dq + (r0 + qrow) * a.lddq + hh * d + col) = qok ? dq[i] * scale : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
}

template <int M, int S, int D, int RG, int NG>
__device__ __forceinline__ void win_dkdv_f32(const AttnWinArgs& a, unsigned task, unsigned tasks, float scale2, float scale, float* fsm) {
  constexpr int NK = D / 16;
  const KeyTask<M> w(a, task, tasks, 16 * RG, BR);
  if (!w.run) return;
  const int tid = threadIdx.x & (64 * RG - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = lane >> 4;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * RG));
  float *const Qs = fsm + group * 2 * F32Lds<D, RG, NG>::BLK, *const Gs = Qs + F32Lds<D, RG, NG>::BLK;
  float *const Ls = fsm + NG * 2 * F32Lds<D, RG, NG>::BLK + group * F32Lds<D, RG, NG>::STAT, *const Ds = Ls + BR;
  const int len = w.len, d = a.d, h0 = w.kv * (a.A / a.Ak);
  const long r0 = (long)w.bi * a.s;
  const float *Q = (const float*)a.q + r0 * a.ldq + h0 * d, *G = (const float*)a.dctx + r0 * a.lddc + h0 * d;
  const float *lse = a.lse + ((long)w.bi * a.A + h0) * a.s, *delta = a.delta + ((long)w.bi * a.A + h0) * a.s;
  const int row0 = w.k0 + wave * 16, krow = row0 + (lane & 15);
  const bool kok = krow < len;
  const KeyRows<M, 16> seen(a, row0, len, lane);
  const int lo = seen.lo, hi = seen.hi, lo_min = seen.lo_min, hi_max = seen.hi_max;
  f32x4 kf[NK], vf[NK], sum[2 * NK];   // sums: dk, dv
  f32x4 *const dk = sum, *const dv = sum + NK;
  own_row<D>((const float*)a.k + (r0 + krow) * a.ldk + w.kv * d, kok, d, lane, kf);
  own_row<D>((const float*)a.v + (r0 + krow) * a.ldv + w.kv * d, kok, d, lane, vf);
#pragma unroll
  for (int i = 0; i < NK; ++i) dk[i] = dv[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  Score<S> sc(a, scale2);
  F32Block<D, 64 * RG> qb, gb;
  float L = 0.f, De = 0.f;
  auto load = [&](int n) {
    const int hd = n / w.nq, i0 = (w.qlo + n % w.nq) * BR;
    qb.load(Q + (long)i0 * a.ldq + hd * d, a.ldq, tid, len - i0, d);
    gb.load(G + (long)i0 * a.lddc + hd * d, a.lddc, tid, len - i0, d);
    const bool in = tid < BR && i0 + tid < len;
    L = in ? lse[(long)hd * a.s + i0 + tid] : 0.f;
    De = in ? delta[(long)hd * a.s + i0 + tid] : 0.f;
  };
  __builtin_amdgcn_s_waitcnt(0x0F70);   // (as in attn_win_fwd_f32)
  if (w.n0 + group < w.n1) load(w.n0 + group);
  for (int n = w.n0 + group; n - group < w.n1; n += NG) {   // (both groups pass the same barriers)
    __syncthreads();
    qb.store(Qs, tid);
    gb.store(Gs, tid);
    if (tid < BR) {
      Ls[tid] = L;
      Ds[tid] = De;
    }
    __syncthreads();
    if (n + NG < w.n1) load(n + NG);
    if (row0 >= len || n >= w.n1) continue;
    const int i0 = (w.qlo + n % w.nq) * BR;
    sc.head(a, h0 + n / w.nq);
#pragma unroll
    for (int t = 0; t < 2; ++t) {   // rows: query i0 + 16 t + 4 g4 + e, column: key
      if (i0 + 16 * t >= hi_max || i0 + 16 * t + 15 < lo_min) continue;
      f32x4 s{0.f, 0.f, 0.f, 0.f}, dp{0.f, 0.f, 0.f, 0.f}, qf[NK], gf[NK];   // (reads first: see attn_win_fwd_f32)
      float gc[4][NK], qc[4][NK], p[4], ds[4];
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        qf[kk] = frow<D>(Qs, 16 * t, kk, lane);
        gf[kk] = frow<D>(Gs, 16 * t, kk, lane);
      }
      const f32x4 L4 = *(const f32x4*)(Ls + 16 * t + 4 * g4), D4 = *(const f32x4*)(Ds + 16 * t + 4 * g4);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s = MFMA4(qf[kk][e], kf[kk][e], s);
          dp = MFMA4(gf[kk][e], vf[kk][e], dp);
        }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          gc[e][c] = fcol<D>(Gs, 16 * c, 16 * t, e, lane);
          qc[e][c] = fcol<D>(Qs, 16 * c, 16 * t, e, lane);
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + 16 * t + 4 * g4 + e;
        const bool ok = i >= lo && i < hi;
        float bent = 0.f;
        const float x = S == SCORE_PLAIN ? s[e] * scale2 - L4[e] : sc.less32(s[e], scale2, (float)(krow - i), L4[e], bent);
        p[e] = ok ? __builtin_amdgcn_exp2f(x) : 0.f;
        ds[e] = ok ? p[e] * (dp[e] + D4[e]) : 0.f;
        if (capped(S)) ds[e] *= sc.derivative(bent);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          dv[c] = MFMA4(gc[e][c], p[e], dv[c]);
          dk[c] = MFMA4(qc[e][c], ds[e], dk[c]);
        }
    }
  }
  if (!join_groups<RG, NG>(sum, fsm, group, tid)) return;
  if (w.slot >= 0) {
    float* const P = a.partial + (long)w.slot * 2 * 16 * RG * D;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      *(f32x4*)(P + ((wave * NK + i) * 64 + lane) * 4) = dk[i];
      *(f32x4*)(P + 16 * RG * D + ((wave * NK + i) * 64 + lane) * 4) = dv[i];
    }
    return;
  }
  if (krow < a.s) {
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int col = 16 * i + 4 * g4;
      if (col < d) {
        *(f32x4*)((float*)a.dk + (r0 + krow) * a.lddk + w.kv * d + col) = dk[i] * scale;
        *(f32x4*)((float*)a.dv + (r0 + krow) * a.lddv + w.kv * d + col) = dv[i];
      }
    }
  }
}

template <int M, int S, int D, int RG, int NG>
__global__ __launch_bounds__(64 * RG * NG) void attn_win_bwd_f32(AttnWinArgs a, float scale2, float scale) {
  extern __shared__ __attribute__((aligned(16))) float fsm[];
  const unsigned nk = a.plan.key_tasks;
  if (blockIdx.x < nk) win_dkdv_f32<M, S, D, RG, NG>(a, blockIdx.x, nk, scale2, scale, fsm);
  else win_dq_f32<M, S, D, RG, NG>(a, blockIdx.x - nk, gridDim.x - nk, scale2, scale, fsm);
}

// ------------------------------------------------------------------ both types
// MASK_SPANS: the walks' lengths are known on the device alone, and so is how they are cut: into parts no longer than a unit's share of all of
// them.  table: {tasks, cut tiles, -, -}, then tasks of four words (tile, first and last block of the part, slot of its sums or
// -1), the longest first, then cut tiles of four (tile, first slot, parts, -); per key head, for all have the same.  One workgroup writes it.  The
// order among tasks of about one length and the slots' numbers may differ from call to call, but no sum goes by them.
// A walk longer than the share has at most twice its length over the share parts: no more than 2 units of them in all.
template <int M>
__device__ __forceinline__ void docs_plan(const AttnWinArgs& a) {
  constexpr int NB = 64;
  __shared__ unsigned long long all;
  __shared__ int count[NB], slots, cuts;
  const WinPlan& p = a.plan;
  const int tid = threadIdx.x, G = a.A / a.Ak;
  KeyTask<M> w;
  w.len = len_of<M>(a, 0);
  auto walk = [&](int tile) {
    w.k0 = tile * p.kt;
    w.span(a, p.kt, p.blk);
    return w.nq * G;   // (below 2^23: A times blocks of 32 rows is)
  };
  if (tid == 0) all = 0, slots = cuts = 0;
  if (tid < NB) count[tid] = 0;
  __syncthreads();
  const int first = tid < p.key_tiles ? walk(tid) : 0;   // (of most calls, all)
  auto length = [&](int t) { return t == tid ? first : walk(t); };
  unsigned long long mine = 0;
  for (int t = tid; t < p.key_tiles; t += 256) mine += length(t);
  atomicAdd(&all, mine);
  __syncthreads();
  const int steps = walk_share(all, a.Ak, p.units, p.min_steps);
  auto parts_of = [&](int n) { return walk_parts(n, steps); };
  auto bucket = [&](int n) { return NB - 1 - min(NB - 1, (int)((long)n * NB / (steps + 1))); };
  for (int t = tid; t < p.key_tiles; t += 256) {
    const int n = length(t), parts = parts_of(n);
    atomicAdd(&count[bucket((n + parts - 1) / parts)], parts);
  }
  __syncthreads();
  if (tid < NB) {   // (one wave)
    int at = count[tid];
    const int own = at;
#pragma unroll
    for (int o = 1; o < NB; o <<= 1) {
      const int v = __shfl_up(at, o, 64);
      if (tid >= o) at += v;
    }
    count[tid] = at - own;
    if (tid == NB - 1) a.table[0] = at;
  }
  __syncthreads();
  for (int t = tid; t < p.key_tiles; t += 256) {
    const int n = length(t), parts = parts_of(n), per = (n + parts - 1) / parts, at = atomicAdd(&count[bucket(per)], parts);
    int slot = -1;
    if (parts > 1) {
      slot = atomicAdd(&slots, parts);
      int32_t* const e = a.table + 4 + 4L * p.max_tasks + 4L * atomicAdd(&cuts, 1);
      e[0] = t, e[1] = slot, e[2] = parts, e[3] = 0;
    }
    for (int i = 0; i < parts; ++i) {
      int32_t* const e = a.table + 4 + 4L * (at + i);
      e[0] = t, e[1] = min(n, i * per), e[2] = min(n, (i + 1) * per), e[3] = slot < 0 ? -1 : slot + i;
    }
  }
  __syncthreads();
  if (tid == 0) a.table[1] = cuts;
}

// -delta [b, A, s]: 16 lanes per head, V columns each, four heads of a row per wave
template <int M, typename T>
__global__ __launch_bounds__(256) void attn_win_delta(AttnWinArgs a) {
  constexpr int V = 16 / sizeof(T);
  const int lane = threadIdx.x & 63;
  if (M == MASK_SPANS && blockIdx.x == 0) {   // (a workgroup of its own)
    docs_plan<M>(a);
    return;
  }
  const long row = (long)(blockIdx.x - (M == MASK_SPANS)) * 4 + (threadIdx.x >> 6);
  if (row >= (long)a.b * a.s) return;
  const int bi = (int)(row / a.s), qi = (int)(row % a.s);
  if (qi >= len_of<M>(a, bi)) return;   // (nothing reads it)
  const T *G = (const T*)a.dctx + row * a.lddc, *O = (const T*)a.ctx + row * a.ldc;
  const float* O32 = a.ctx32 ? a.ctx32 + row * a.ldc : nullptr;
  for (int h = lane >> 4; h - (lane >> 4) < a.A; h += 4) {
    float t = 0.f;
    if (h < a.A)
      for (int c = (lane & 15) * V; c < a.d; c += 16 * V) {
        const int at = h * a.d + c;
        typedef T TV __attribute__((ext_vector_type(V)));
        const TV g = *(const TV*)(G + at);
        if (O32) {
          typedef float FV __attribute__((ext_vector_type(V)));
          const FV o = *(const FV*)(O32 + at);
#pragma unroll
          for (int e = 0; e < V; ++e) t = fmaf(to_f32((T)g[e]), o[e], t);
        } else {
          const TV o = *(const TV*)(O + at);
#pragma unroll
          for (int e = 0; e < V; ++e) t = fmaf(to_f32((T)g[e]), to_f32((T)o[e]), t);
        }
      }
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) t += __shfl_xor(t, x, 64);
    if (h < a.A && (lane & 15) == 0) a.delta[((long)bi * a.A + h) * a.s + qi] = -t;
  }
}

constexpr int join_threads(int elements) { return elements / 4 < 256 ? elements / 4 : 256; }
// dk (z = 0), dv of the tiles whose walk has parts: the parts' sums in ascending order.  RW: rows (keys) of a wave; an
// accumulator block is RW rows x 64 * 4 / RW columns.
template <int M, typename T, int D, int KT, int RW, int BLK>
__global__ __launch_bounds__(256) void attn_win_join(AttnWinArgs a, float scale) {
  constexpr int JT = join_threads(KT * D), UNITS = KT * D / 4 / JT;   // workgroups per tile, four elements to a lane
  const WinPlan& p = a.plan;
  const int head = blockIdx.y;
  const int u = (blockIdx.x % UNITS) * JT + threadIdx.x, lane = u & 63, blk = u >> 6;
  constexpr int CB = 256 / RW;              // columns of an accumulator register block
  const int row = blk / (D / CB) * RW + (lane & (RW - 1)), col = blk % (D / CB) * CB + 4 * (lane / RW);
  auto join = [&](int bi, int kv, int k0, int slot, int used) {
    const float* src = a.partial + ((long)slot * 2 + blockIdx.z) * KT * D + (long)u * 4;
    f32x4 t{0.f, 0.f, 0.f, 0.f};
    int i = 0;
    for (; i + 3 < used; i += 4) {
      f32x4 x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = *(const f32x4*)(src + (long)(i + q) * 2 * KT * D);
#pragma unroll
      for (int q = 0; q < 4; ++q) t += x[q];
    }
    for (; i < used; ++i) t += *(const f32x4*)(src + (long)i * 2 * KT * D);
    if (k0 + row >= a.s || col >= a.d) return;
    if (blockIdx.z == 0) t *= scale;
    T* const out = (T*)(blockIdx.z ? a.dv : a.dk) + ((long)bi * a.s + k0 + row) * (blockIdx.z ? a.lddv : a.lddk) + kv * a.d + col;
    if constexpr (sizeof(T) == 2) {
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (bf16)t[e];
      *(bf16x4*)out = o;
    } else {
      *(f32x4*)out = t;
    }
  };
  if constexpr (M == MASK_SPANS) {   // (how many there are is known on the device alone)
    const int32_t* const cuts = a.table + 4 + 4L * p.max_tasks;
    for (int c = blockIdx.x / UNITS; c < a.table[1]; c += gridDim.x / UNITS)
      join(0, head, cuts[4 * c] * KT, head * p.slots + cuts[4 * c + 1], cuts[4 * c + 2]);
  } else {
    const int nt = (p.sink_parts > 1 ? p.sink_tiles : 0);
    int tile = blockIdx.x / UNITS;
    if (nt == 0) tile += p.sink_tiles;   // (then the other tiles have parts)
    const bool sink = tile < p.sink_tiles;
    const int sinks = p.sink_tiles * p.sink_parts;
    // the tile's first task (KeyTask counts the same)
    KeyTask<M> w;
    w.init(a, head * (sinks + (p.key_tiles - p.sink_tiles) * p.parts) + (sink ? tile * p.sink_parts : sinks + (tile - p.sink_tiles) * p.parts), KT, BLK);
    const int all = w.nq * (a.A / a.Ak), steps = sink ? p.sink_steps : p.steps;
    join(w.bi, w.kv, w.k0, w.slot, (all + steps - 1) / steps);
  }
}

// ------------------------------------------------------------------ launchers
// Workgroups of four waves, or of two where four would leave a quarter of the 256 units without one (bf16; as in attention.hip), the
// gradient's where they give few units a second one.  Us with two / four waves, workgroups of four: forward, heads of 64, 128 of them 9.2 / 9.8,
// 168 12.4 / 11.6, 256 13.2 / 12.0, 512 32 / 26; forward and backward 128 30 / 31, 256 56 / 62 and 34 / 35, 320 67 / 57, 512 53 / 46
inline int fwd_waves(const AttnWinArgs& a) { return (long)((a.s + 127) / 128) * a.b * a.A < 160 ? 2 : 4; }
inline int bwd_waves(const AttnWinArgs& a) { return (long)((a.s + 127) / 128) * a.b * (a.A + a.Ak) < 288 ? 2 : 4; }
// fp32: waves of a group (16 rows each).  Four where their tiles make two workgroups for each unit, else two: us forward and
// backward with four / two waves: 4 x 512 rows, 16 heads of 64 211 / 227; 2 x 2048, window none 879 / 914; 2 x 777, 12 heads, window
// 200 110 / 101; 300 rows, 8 heads of 32 31 / 24
inline int f32_rows(const AttnWinArgs& a) { return (long)((a.s + 63) / 64) * a.b * a.A < 512 ? 2 : 4; }
// The forward of wide heads, whose blocks take two groups of two waves twice as long to bring: us 256 tiles of 64 rows, heads of 128, 31 / 27, 512
// 89 / 70, 1024 167 / 124, but 80 39 / 50 (heads of 64: 256 14 / 15 and 51 / 48, 312 25 / 29, 512 37 / 33)
inline int f32_fwd_rows(const AttnWinArgs& a) { return a.d > 64 && (long)((a.s + 63) / 64) * a.b * a.A >= 192 ? 4 : f32_rows(a); }
// keys of a workgroup of the backward
inline int key_tile(Dtype dt, const AttnWinArgs& a) { return dt != DT_BF16 ? 16 * f32_rows(a) : a.d > 64 ? 128 : 32 * bwd_waves(a); }

// queries of a block of their walks
inline int walk_block(Dtype dt, const AttnWinArgs& a) { return dt != DT_BF16 ? BR : a.d > 64 ? 32 : 64; }

// How the walks of dk and dv are cut.  Parts: as long as the walk of a tile without sinks where that walk is short or the tiles are
// many -- fewer than units, for dq's workgroups fill the others; but where the walks grow with the tile (causal, no window) the longest
// is twice the mean -- else as long as two workgroups to a unit leave, eight blocks at least.  Us forward and backward, cut / whole, key
// tiles: bf16 heads of 64, window 512, 248 tiles 73 / 60; no mask, 96 83 / 79; window 200, 72 39 / 43; causal, 84 90 / 119, 162 64 / 62, 172
// 120 / 124; of 128, window 256, 120 145 / 114; causal, 88 200 / 225.  fp32, window 300, 372 104 / 87; window 200, 92 59 / 56; causal, 352 209 /
// 162, 256 339 / 335, 152 170 / 189, 64 109 / 145.  (What lies on the other side of 192 by 3%, 162 causal tiles, is left there.)
// Tiles of sinks, whose walks are the longest, are cut likewise, but into no more than two parts for each unit in all: there
// fp32 sums of every part are written and read again, and with parts of the others' length their number grew with sinks times
// rows.  Gradient, us and workspace, parts of the others' length / these: 16384 rows, 32 heads of 128 on 8, window 64, 1024 sinks 1535, 623 MB /
// 1235, 69 MB; 32768 rows, 16 heads of 64, window 64, 1024 sinks 1063, 1076 MB / 720, 36 MB; 65536 rows, window 128, 4 sinks 663, 219 MB / 600,
// 38 MB.  (One part for each unit 716 to 1262 in the first two; four 737, 1263.)
inline void make_plan(Dtype dt, AttnWinArgs& a) {
  const int kt = key_tile(dt, a), blk = walk_block(dt, a);
  WinPlan& p = a.plan;
  const long G = a.A / a.Ak, nb = (a.s + blk - 1) / blk, heads = (long)a.b * a.Ak;
  p.key_tiles = (a.s + kt - 1) / kt;
  p.sink_tiles = a.W ? (int)std::min<long>(p.key_tiles, ((long)a.S + kt - 1) / kt) : 0;
  const long rest = p.key_tiles - p.sink_tiles;
  // the most blocks that a walk without sinks has, per head
  const long reach = !a.W ? nb : std::min(nb, ((a.causal ? 1L : 2L) * (a.W - 1) + kt + blk - 2) / blk + 1);
  const long total = heads * G * (rest * reach + p.sink_tiles * nb), fair = (total + 511) / 512;
  const bool whole = rest && (heads * rest * (a.causal && !a.W ? 1 : 2) >= 192 || G * reach <= 10);
  const long steps = whole ? G * reach : std::min(G * (rest ? reach : nb), std::max(8L, fair));
  const long sink_steps = std::min(G * nb, std::max(steps, (heads * G * p.sink_tiles * nb + 511) / 512));
  p.parts = (int)((G * reach + steps - 1) / steps);
  p.sink_parts = (int)((G * nb + sink_steps - 1) / sink_steps);
  if (!p.sink_tiles) p.sink_parts = 1;
  if (!rest) p.parts = 1;
  p.steps = (int)steps;
  p.sink_steps = (int)sink_steps;
  p.slots = (p.sink_parts > 1 ? p.sink_tiles * p.sink_parts : 0) + (p.parts > 1 ? (int)rest * p.parts : 0);
  p.key_tasks = (unsigned)(heads * (p.sink_tiles * p.sink_parts + rest * p.parts));
}

template <typename F>
auto pick_width(Dtype dt, int d, F&& f) {
  if (dt != DT_BF16 && d <= 16) return f(std::integral_constant<int, 16>{});
  if (d <= 32) return f(std::integral_constant<int, 32>{});
  if (d <= 64) return f(std::integral_constant<int, 64>{});
  return f(std::integral_constant<int, 128>{});
}

inline size_t delta_bytes(const AttnWinArgs& a) { return ((size_t)a.b * a.A * a.s * 4 + 255) / 256 * 256; }

// D = 128: whether dq's workgroups of 256 queries (a unit holds one) are in the launch of dk and dv
inline bool pair_has_dq(const AttnWinArgs& a) { return (long)((a.s + 255) / 256) * a.b * a.A >= 256; }

// what docs_plan may cut the walks into (b = 1)
inline void make_docs_plan(Dtype dt, AttnWinArgs& a) {
  WinPlan& p = a.plan;
  p.kt = key_tile(dt, a);
  p.blk = walk_block(dt, a);
  // Parts of up to one of `units` shares of all walks of dk and dv: the longest begin first, and dq's workgroups, in the same launch behind them,
  // fill what they leave; where those are alone, a share for each unit.  Us forward and gradient with 170 / 340 / 512 shares, of 3, 6 and 12 documents:
  // 8192 rows of 16 heads of 128 on 4 1003 / 1010 / 1026, 544 / 560 / 571, 345 / 360 / 378; 6001 rows of 16 heads of 64, of 6, 8 and 14
  // documents 265 / 281 / 278, 177 / 184 / 184, 145 / 146 / 151; fp32, 1554 rows, 3, 6 and 7 documents 152 / 163 / 167, 134 / 142 / 145, 125 /
  // 127 / 126.
  p.units = dt == DT_BF16 && a.d > 64 && !pair_has_dq(a) ? 256 : 170;
  p.min_steps = 16;
  p.key_tiles = (a.s + p.kt - 1) / p.kt;
  const long parts = ((long)(a.s + p.blk - 1) / p.blk * (a.A / a.Ak) + p.min_steps - 1) / p.min_steps;   // of the longest walk there can be
  const long share = p.units / a.Ak;   // walks longer than a unit's share, of a head
  p.max_cuts = parts > 1 ? (int)std::min<long>(share, p.key_tiles) : 0;
  p.slots = parts > 1 ? (int)std::min<long>(2L * p.units / a.Ak, p.key_tiles * parts) : 0;
  p.max_tasks = p.key_tiles + (int)std::min<long>(share, p.key_tiles * parts);
  p.key_tasks = heads_grid(a.Ak, p.max_tasks);
}
inline size_t table_bytes(const AttnWinArgs& a) { return (16 + 16 * ((size_t)a.plan.max_tasks + a.plan.max_cuts) + 255) / 256 * 256; }

template <typename K>
hipError_t allow_lds(K kern, int bytes) {
  return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

// workgroups of the query tiles of so many rows
template <int M>
unsigned query_grid(const AttnWinArgs& a, int rows) {
  const long tiles = (a.s + rows - 1) / rows;
  return M == MASK_SPANS ? heads_grid(a.A, tiles) : (unsigned)(tiles * a.b * a.A);
}

template <int M, int S>
hipError_t attn_win_fwd_launch_f32(const AttnWinArgs& a, hipStream_t st) {
  const float scale2 = LOG2E * a.scale;
  return pick_width(DT_F32, a.d, [&](auto D) {
    constexpr int d = decltype(D)::value;
    auto go = [&](auto RG) {
      constexpr int rg = decltype(RG)::value, lds = F32Lds<d, rg, 2>::FLOATS * 4;
      static const hipError_t rc = allow_lds(attn_win_fwd_f32<M, S, d, rg, 2>, lds);
      if (rc != hipSuccess) return rc;
      hipLaunchKernelGGL((attn_win_fwd_f32<M, S, d, rg, 2>), dim3(query_grid<M>(a, 16 * rg)), dim3(128 * rg), lds, st, a, scale2);
      return hipGetLastError();
    };
    return f32_fwd_rows(a) == 4 ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 2>{});
  });
}

template <int M, int S>
hipError_t attn_win_fwd_launch_bf16(const AttnWinArgs& a, hipStream_t st) {
  const float scale2 = LOG2E * a.scale;
  return pick_width(DT_BF16, a.d, [&](auto D) {
    constexpr int d = decltype(D)::value;
    if constexpr (d >= 32) {
      auto go = [&](auto NW) {
        constexpr int nw = decltype(NW)::value, lds = WinRing<d, nw, false>::BYTES;
        static const hipError_t rc = allow_lds(attn_win_fwd<M, S, d, nw>, lds);
        if (rc != hipSuccess) return rc;
        hipLaunchKernelGGL((attn_win_fwd<M, S, d, nw>), dim3(query_grid<M>(a, 32 * nw)), dim3(64 * nw), lds, st, a, scale2);
        return hipGetLastError();
      };
      return fwd_waves(a) == 4 ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 2>{});
    }
    return hipErrorInvalidValue;
  });
}

// the plan, the workspace's parts, -delta
template <int M, typename T>
hipError_t attn_win_bwd_begin(Dtype dt, AttnWinArgs& a, void* workspace, hipStream_t st) {
  if (M == MASK_SPANS) make_docs_plan(dt, a);
  else make_plan(dt, a);
  a.delta = (float*)workspace;
  a.partial = (float*)((char*)workspace + delta_bytes(a));
  if (M == MASK_SPANS) {
    a.table = (int32_t*)a.partial;
    a.partial = (float*)((char*)a.table + table_bytes(a));
  }
  hipLaunchKernelGGL((attn_win_delta<M, T>), dim3((unsigned)(((long)a.b * a.s + 3) / 4) + (M == MASK_SPANS)), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename K>
hipError_t attn_win_bwd_join(K kern, const AttnWinArgs& a, int kt, int d, hipStream_t st) {
  int joined = a.plan.slots ? (a.plan.sink_parts > 1 ? a.plan.sink_tiles : 0) + (a.plan.parts > 1 ? a.plan.key_tiles - a.plan.sink_tiles : 0) : 0;
  const int threads = join_threads(kt * d);
  if (a.spans) {   // (workgroups enough for the memory; what finds no cut tile costs time, too)
    const long per = (long)(kt * d / 4 / threads) * a.Ak * 2;
    joined = std::min<long>(a.plan.max_cuts, std::max<long>(1, 512 / per));
  }
  if (!joined) return hipSuccess;
  hipLaunchKernelGGL(kern, dim3(joined * (kt * d / 4 / threads), a.b * a.Ak, 2), dim3(threads), 0, st, a, a.scale);
  return hipGetLastError();
}

template <int M, int S>
hipError_t attn_win_bwd_launch_f32(AttnWinArgs a, void* workspace, hipStream_t st) {
  hipError_t e = attn_win_bwd_begin<M, float>(DT_F32, a, workspace, st);
  if (e != hipSuccess) return e;
  const float scale = a.scale, scale2 = LOG2E * scale;
  return pick_width(DT_F32, a.d, [&](auto D) {
    constexpr int d = decltype(D)::value;
    auto go = [&](auto RG) {
      constexpr int rg = decltype(RG)::value, lds = F32Lds<d, rg, 2>::FLOATS * 4;
      static const hipError_t rc = allow_lds(attn_win_bwd_f32<M, S, d, rg, 2>, lds);
      if (rc != hipSuccess) return rc;
      const unsigned grid = a.plan.key_tasks + query_grid<M>(a, 16 * rg);
      hipLaunchKernelGGL((attn_win_bwd_f32<M, S, d, rg, 2>), dim3(grid), dim3(128 * rg), lds, st, a, scale2, scale);
      e = hipGetLastError();
      return e != hipSuccess ? e : attn_win_bwd_join(attn_win_join<M, float, d, 16 * rg, 16, BR>, a, 16 * rg, d, st);
    };
    return f32_rows(a) == 4 ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 2>{});
  });
}

template <int M, int S>
hipError_t attn_win_bwd_launch_bf16(AttnWinArgs a, void* workspace, hipStream_t st) {
  hipError_t e = attn_win_bwd_begin<M, bf16>(DT_BF16, a, workspace, st);
  if (e != hipSuccess) return e;
  const float scale = a.scale, scale2 = LOG2E * scale;
  return pick_width(DT_BF16, a.d, [&](auto D) {
    constexpr int d = decltype(D)::value;
    if constexpr (d == 128) {
      static const hipError_t rc = allow_lds(attn_win_bwd_pair<M, S>, PAIR_BYTES);
      if (rc != hipSuccess) return rc;
      const bool both = pair_has_dq(a);
      hipLaunchKernelGGL((attn_win_bwd_pair<M, S>), dim3(a.plan.key_tasks + (both ? query_grid<M>(a, 256) : 0)), dim3(512), PAIR_BYTES, st, a, scale2, scale);
      e = hipGetLastError();
      if (e == hipSuccess) e = attn_win_bwd_join(attn_win_join<M, bf16, d, 128, 32, 32>, a, 128, d, st);
      if (e != hipSuccess || both) return e;
      auto dq = [&](auto NW) {
        constexpr int nw = decltype(NW)::value, lds = WinRing<d, nw, true>::BYTES;
        static const hipError_t rc = allow_lds(attn_win_dq<M, S, nw>, lds);
        if (rc != hipSuccess) return rc;
        hipLaunchKernelGGL((attn_win_dq<M, S, nw>), dim3(query_grid<M>(a, 32 * nw)), dim3(64 * nw), lds, st, a, scale2, scale);
        return hipGetLastError();
      };
      return fwd_waves(a) == 4 ? dq(std::integral_constant<int, 4>{}) : dq(std::integral_constant<int, 2>{});
    } else if constexpr (d >= 32) {
      auto go = [&](auto NW) {
        constexpr int nw = decltype(NW)::value, lds = WinRing<d, nw, true>::BYTES;
        static const hipError_t rc = allow_lds(attn_win_bwd<M, S, d, nw>, lds);
        if (rc != hipSuccess) return rc;
        const unsigned grid = a.plan.key_tasks + query_grid<M>(a, 32 * nw);
        hipLaunchKernelGGL((attn_win_bwd<M, S, d, nw>), dim3(grid), dim3(64 * nw), lds, st, a, scale2, scale);
        e = hipGetLastError();
        return e != hipSuccess ? e : attn_win_bwd_join(attn_win_join<M, bf16, d, 32 * nw, 32, 64>, a, 32 * nw, d, st);
      };
      return bwd_waves(a) == 4 ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 2>{});
    }
    return hipErrorInvalidValue;
  });
}

}  // namespace dapple
