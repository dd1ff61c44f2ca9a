// The division of a ragged batch's attention over a paged cache among workgroups, and what the kernels do at its ends (attn_paged_one.hip, attn_paged_rows.hip).
//
// Contexts of a batch differ by orders of magnitude, and their lengths are known on the GPU only.  All items (sequence, K head, block of BR rows) are laid out on one
// line, an item's stretch as long as the keys it sees, and every workgroup ("slot") takes an equal stretch of the line: a part of one item, or the
// end of one, some whole items, the start of another.  Every workgroup works its own stretch out from the lengths.  Pieces of a cut item leave (m, l, O) in
// the workspace, and a second kernel joins them in their order: sums do not depend on which workgroup ends first.
// Rows: the G heads that share a K head are rows of the same block, row = token * G + head, so that a tile of K serves all of them.
#pragma once
#include "attn_paged.h"
#include "attn_tiles.h"

namespace attn {

constexpr int kItemKeys = 64;   // what an item costs beside its keys, in keys: Q, the wait for its first tile, its end

// A sequence of the batch, every number taken from device memory forced into its range.
struct Sequence {
  int first;   // its first token's row of Q
  int m, L;
  int rows, blocks;   // m * G, and in blocks of BR
  // The line's unit is 1 / G key.  Block t is V(t) = a + step (t + 1) long (an upper bound of the keys its last row sees), the first t blocks are S(t).
  int64_t a;
  int step;
  __device__ __forceinline__ int64_t length(int t) const { return a + (int64_t)step * (t + 1); }
  __device__ __forceinline__ int64_t upto(int64_t t) const { return t * a + step * (t * (t + 1) / 2); }
};
template <int BR> __device__ __forceinline__ Sequence sequence_of(const PagedCall& c, int first, int m, int L) {
  Sequence s;
  s.first = first;
  s.m = m;
  s.L = L;
  s.rows = m * c.G;
  s.blocks = (s.rows + BR - 1) / BR;
  s.a = (int64_t)c.G * ((c.causal ? max(L - m, 0) : L) + kItemKeys);
  s.step = c.causal ? BR : 0;
  return s;
}
// Sequence b (one a lane)
template <int BR> __device__ __forceinline__ Sequence load_sequence(const PagedCall& c, int b) {
  const PagedBatch& p = c.b;
  const int L = min(max(p.lengths[b], 0), p.capacity);
  int first = b, end = b + 1;   // (the host checks T >= B)
  if (p.starts) {
    first = min(max(p.starts[b], 0), p.T);
    end = min(max(p.starts[b + 1], first), p.T);
  }
  return sequence_of<BR>(c, first, end - first, L);
}
// the same for one that all lanes share, in scalar registers
template <int BR> __device__ __forceinline__ Sequence load_sequence_uniform(const PagedCall& c, int b) {
  const Sequence s = load_sequence<BR>(c, b);
  return sequence_of<BR>(c, __builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.m), __builtin_amdgcn_readfirstlane(s.L));
}
template <int BR> __device__ __forceinline__ Sequence lane_sequence(const PagedCall& c, const Sequence& s, int lane) {
  return sequence_of<BR>(c, __builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.m, lane), __builtin_amdgcn_readlane(s.L, lane));
}

__device__ __forceinline__ int64_t lane64(int64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
// x / y for 0 <= x < 2^52, 0 < y < 2^52, rounded down (the 64-bit division of the compiler is five times as long)
__device__ __forceinline__ int64_t divided(int64_t x, int64_t y) {
  int64_t q = (int64_t)((double)x / (double)y);
  if (q * y > x) --q;
  return q;
}

// A point of the line: item (sequence b, K head h, block t), where on the line that starts, and the distance z from there.
struct Point {
  int b, h, t;
  int64_t at, z;
};

// 64 sequences of the line, one a lane: its stretch, and the sum up to its end.
struct Round {
  Sequence s;
  int64_t cost, incl;
  template <int BR> __device__ __forceinline__ void load(const PagedCall& c, int b0) {
    const int lane = threadIdx.x & 63, n = c.b.B - b0;
    s = load_sequence<BR>(c, b0 + min(lane, n - 1));
    cost = lane < n ? s.upto(s.blocks) * c.b.Hk : 0;
    incl = cost;
    for (int d = 1; d < min(n, 64); d <<= 1) {
      const int64_t other = __shfl_up(incl, d, 64);
      if (lane >= d) incl += other;
    }
  }
};

// The line, seen by one wavefront.
template <int BR> struct Line {
  int64_t total;
  Round first;            // all there is for up to 64 sequences
  int n;                  // slots that get a stretch
  int64_t each;           // stretches are `each` long, the first `longer` one more
  int longer;
  int64_t slack;          // a cut nearer than this to an item's end is made there

  // least: keys that a stretch has at least, with what an item costs
  __device__ __forceinline__ void init(const PagedCall& c, int least, int slack_share) {
    first.load<BR>(c, 0);
    total = lane64(first.incl, min(c.b.B, 64) - 1);
    for (int b0 = 64; b0 < c.b.B; b0 += 64) {
      Round r;
      r.load<BR>(c, b0);
      total += lane64(r.incl, min(c.b.B - b0, 64) - 1);
    }
    const int64_t worth = divided(total, (int64_t)(least + kItemKeys) * c.G);
    n = (int)(worth < 1 ? 1 : (worth > c.slots ? c.slots : worth));
    each = divided(total, n);
    longer = (int)(total - each * n);
    slack = slack_share > 0 ? each / slack_share : 0;
  }
  __device__ __forceinline__ int64_t start(int slot) const { return each * slot + min(slot, longer); }
  // The item at 0 <= x < total, and its sequence.
  __device__ __forceinline__ Point locate(const PagedCall& c, int64_t x, Sequence& s) const {
    Point p;
    int64_t before = 0;
    Round r = first;
    for (int b0 = 0;; b0 += 64) {
      if (b0 > 0) r.load<BR>(c, b0);
      const int in_round = min(c.b.B - b0, 64);
      const uint64_t beyond = __ballot((int)(threadIdx.x & 63) < in_round && before + r.incl > x);
      if (beyond != 0 || b0 + 64 >= c.b.B) {
        const int i = beyond != 0 ? __builtin_ctzll(beyond) : in_round - 1;
        p.b = b0 + i;
        p.at = before + lane64(r.incl, i) - lane64(r.cost, i);
        s = lane_sequence<BR>(c, r.s, i);
        break;
      }
      before += lane64(r.incl, 63);
    }
    const int64_t in = x - p.at;
    int64_t head = s.a + s.step;
    int h, t = 0;
    if (s.blocks == 1) {
      h = (int)divided(in, head);
    } else {
      head = s.upto(s.blocks);
      h = (int)divided(in, head);
      const int64_t y = in - h * head;   // t with S(t) <= y < S(t + 1)
      if (s.step == 0) {
        t = (int)divided(y, s.a);
      } else {
        const double q = (double)s.a + 0.5 * s.step;
        t = (int)((sqrt(q * q + 2.0 * s.step * (double)y) - q) / s.step);
        t = min(max(t, 0), s.blocks - 1);
        while (t > 0 && s.upto(t) > y) --t;
        while (t + 1 < s.blocks && s.upto(t + 1) <= y) ++t;
      }
    }
    p.t = __builtin_amdgcn_readfirstlane(t);
    p.h = __builtin_amdgcn_readfirstlane(h);
    p.at += p.h * head + s.upto(p.t);
    p.z = x - p.at;
    return p;
  }
};

// What the second kernel joins at a slot: pieces (0: nothing) of the slots from the one before on, rows `row0` to row0 + rows - 1 of K head h of the sequence
// whose first token is `first`.
struct Join { int pieces, row0, rows, first, h, unused[3]; };
static_assert(sizeof(Join) == kJoinBytes, "the workspace counts them");
__device__ __forceinline__ int* join_slots(const PagedCall& c) { return (int*)c.part; }
__device__ __forceinline__ Join* join_list(const PagedCall& c) { return (Join*)((char*)c.part + kJoinBytes); }

// How a kernel divides its line: rows of a block, keys of a stretch at least, and the share of a stretch (0: none) that a cut is moved by to an item's end.
template <int BR_, int LEAST, int SLACK> struct Division {
  static constexpr int BR = BR_;
  static __device__ __forceinline__ void init(Line<BR>& line, const PagedCall& c) { line.init(c, LEAST, SLACK); }
};
// The item behind `at`, whose stretch ends at x on the line: false if there is none.  s: its sequence, of at before.
template <int BR> __device__ __forceinline__ bool next_item(const PagedCall& c, int64_t x, Point& at, Sequence& s) {
  at.at = x;
  at.z = 0;
  if (++at.t < s.blocks) return true;
  at.t = 0;
  if (++at.h < c.b.Hk) return true;
  at.h = 0;
  do {
    if (++at.b >= c.b.B) return false;
    s = load_sequence_uniform<BR>(c, at.b);
  } while (s.rows == 0);
  return true;
}

// The stretch of a slot: from `at` (s: its sequence) to x_end.  False: there is none.  Leaves in the workspace how many slots there are, and for the first
// cut of an item what is to be joined there.
template <class DIV> __device__ __forceinline__ bool stretch(const PagedCall& c, int& slot, Point& at, Sequence& s, int64_t& x_end) {
  constexpr int BR = DIV::BR;
  Line<BR> line;
  DIV::init(line, c);
  if (blockIdx.x == 0 && threadIdx.x == 0) *join_slots(c) = line.total == 0 ? 0 : line.n;
  slot = xcd_item(line.n, (line.n + kXcds - 1) / kXcds);   // neighbours on the line share an XCD's L2
  if (slot < 0 || line.total == 0) return false;
  at = line.locate(c, line.start(slot), s);
  if (slot > 0) {
    const int64_t near_end = at.at + s.length(at.t) - line.slack;
    int pieces = 0;
    if (at.z > line.slack && line.start(slot) < near_end && line.start(slot - 1) - at.at <= line.slack) {
      // slots slot - 1 to the last that starts in the item: the smallest k with start(k) >= near_end
      int k = (int)min((int64_t)line.n, divided(max(near_end - line.longer, (int64_t)0), line.each));
      while (k < line.n && line.start(k) < near_end) ++k;
      while (line.start(k - 1) >= near_end) --k;
      pieces = k - (slot - 1);
    }
    if (threadIdx.x == 0) {
      const Join j = {pieces, at.t * BR, min(BR, s.rows - at.t * BR), s.first, at.h, {0, 0, 0}};
      join_list(c)[slot] = j;
    }
  }
  x_end = line.start(slot + 1);
  if (line.slack > 0) {
    if (slot + 1 < line.n) {
      Sequence last;
      const Point e = line.locate(c, x_end, last);
      const int64_t v = last.length(e.t);
      if (e.z <= line.slack) x_end = e.at;
      else if (v - e.z <= line.slack) x_end = e.at + v;
    }
    const int64_t v = s.length(at.t);
    if (at.z <= line.slack) at.z = 0;
    else if (v - at.z <= line.slack && !next_item<BR>(c, at.at + v, at, s)) return false;
  }
  return true;
}

// What the 32 rows of an item from row0 on are: lane r has row `row0 + r` = token * G + head of the item's sequence (a copy of the last one beyond the end).
struct Rows {
  int token, head, pos;      // head: of Q
  bool ok;
  int pos_first, pos_last;   // of the first and the last row, the same in all lanes
};
__device__ __forceinline__ Rows rows_of(const PagedCall& c, const Sequence& s, int h, int row0, int r) {
  Rows w;
  w.ok = row0 + r < s.rows;
  const int row = min(row0 + r, s.rows - 1);
  const int i = row / c.G;
  w.head = h * c.G + (row - i * c.G);
  w.token = s.first + i;
  const int base = s.L - s.m, all = s.L - 1;
  w.pos = c.causal ? base + i : all;
  w.pos_first = __builtin_amdgcn_readfirstlane(c.causal ? base + min(row0, s.rows - 1) / c.G : all);
  w.pos_last = __builtin_amdgcn_readfirstlane(c.causal ? base + min(row0 + 31, s.rows - 1) / c.G : all);
  return w;
}

// Tiles of `keys` keys that block t sees: those of its last row.
template <int BR> __device__ __forceinline__ int tiles_of(const PagedCall& c, const Sequence& s, int t, int keys) {
  const int last_row = min((t + 1) * BR, s.rows) - 1;
  const int last = c.causal ? s.L - s.m + last_row / c.G : s.L - 1;
  return last < 0 ? 0 : last / keys + 1;
}
// Where a cut at distance z of an item of length v falls among its tiles (the same for the pieces on both sides).
__device__ __forceinline__ int cut_at(int64_t z, int64_t v, int tiles) {
  return __builtin_amdgcn_readfirstlane(z >= v ? tiles : min(tiles, (int)((double)z / (double)v * tiles)));
}

// 16 zeros: what rows beyond a sequence's length, and pages whose number is not one, are copied from.  (What stands in the unwritten part of a page may be
// NaN, and 0 * NaN is not 0.)
__device__ const u32x4 zero_line[1] = {{0u, 0u, 0u, 0u}};

// O rows and row statistics of a finished item's 32 rows.  l_tot, lr_sum: the exact sum and that of the rounded probabilities.  stage: 32 D elements of LDS of
// this wavefront.  (Lane numbers that the compiler does not keep through the tile loop.)
template <typename T, int D>
__device__ __forceinline__ void write_rows(const PagedCall& c, const Sequence& s, int h, int row0, const f32x16 (&o)[D / 32], float m_run, float l_tot, float lr_sum,
                                           T* stage) {
  typedef typename Vec<T>::x4 T4;
  typedef typename Vec<T>::x8 T8;
  constexpr int CPR = D / 8, RPP = 64 / CPR;
  const int lane = lane_id_here(), r = lane & 31, g = lane >> 5;
  const Rows w = rows_of(c, s, h, row0, r);
  const float inv = (l_tot > 0.f && lr_sum > 0.f) ? 1.f / lr_sum : (l_tot == l_tot ? 0.f : l_tot);   // (a row of NaN stays one)
  if (g == 0 && w.ok)
    c.LSE[(int64_t)w.head * c.b.T + w.token] =
        l_tot > 0.f ? (m_run + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f : (l_tot == l_tot ? -INFINITY : l_tot);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      T4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (T)(o[db][4 * i4 + e] * inv);
      const int chunk = (4 * db + i4) ^ (r & (CPR - 1));
      *(T4*)(stage + r * D + 8 * chunk + 4 * g) = v;
    }
  __builtin_amdgcn_wave_barrier();   // same wavefront: LDS operations complete in program order
  const int64_t off = w.ok ? (int64_t)w.token * c.ot + (int64_t)w.head * c.oh : -1;
#pragma unroll
  for (int p = 0; p < 32 / RPP; ++p) {
    if (row0 + p * RPP >= s.rows) break;
    const int row = p * RPP + lane / CPR, ch = lane % CPR;
    const T8 v = *(const T8*)(stage + row * D + 8 * (ch ^ (row & (CPR - 1))));
    const int64_t dst = __shfl(off, row, 64);
    if (dst >= 0 && 8 * ch < c.d) *(T8*)((T*)c.O + dst + 8 * ch) = v;
  }
  __builtin_amdgcn_wave_barrier();
}

// A cut item's pieces in the workspace: O, not yet divided by the sum, and (m, l, sum of the rounded probabilities) of its rows, kFloats = BR (D + 4) floats.
template <int D, int BR> __device__ __forceinline__ float* piece_of(const PagedCall& c, int index) {
  return (float*)((char*)c.part + (int64_t)(c.slots + 1) * kJoinBytes) + (int64_t)index * (BR * (D + 4));
}
// Its index: a slot has at most one piece that starts inside an item and one that does not.
__device__ __forceinline__ int piece_index(int slot, bool from_start) { return 2 * slot + (from_start ? 1 : 0); }

}  // namespace attn
