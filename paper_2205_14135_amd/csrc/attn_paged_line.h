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

// How a kernel divides its line.  BR: rows of a block.  KEYS: of a tile.  ITEM: what an item costs beside its keys, in keys (Q, the wait for its first tile, its end); a piece costs
// as much, and a join.  SLACK: keys that a cut is moved by to an end of its item.  SPREAD: a stretch has at least the square root of SPREAD times the longest item's keys, so that joining the pieces takes no longer than making one:
// with k keys in each of n / k pieces the kernel takes c k for a piece, the join C n / k, and the sum is least at k^2 = n C / c.
// WINDOW: tokens see a window of keys and sinks only.
template <int BR_, int KEYS_, int ITEM_, int SLACK_, int SPREAD_, bool WINDOW_ = false> struct Division {
  static constexpr int BR = BR_, KEYS = KEYS_, ITEM = ITEM_, SLACK = SLACK_, SPREAD = SPREAD_;
  static constexpr bool WINDOW = WINDOW_;
};
// A sequence of the batch, every number taken from device memory forced into its range.
struct Sequence {
  int first;   // its first token's row of Q
  int base;    // the position of its first new token: may be negative
  int L;       // its keys: no more than a row of the table holds
  int rows, blocks;   // m * G, and in blocks of BR
  // The line's unit is 1 / G key; its points are whole numbers below 2^50 (the host checks that) in double: exact, and an instruction where a 64-bit integer takes four.
  // Block t is length(t) = a + step (t + 1) long (an upper bound of the keys its last row sees), the first t blocks are upto(t).
  double a, step;
  __device__ __forceinline__ double length(int t) const { return a + step * (t + 1); }
  __device__ __forceinline__ double upto(int t) const { return t * a + step * (0.5 * t * (t + 1)); }
};
template <class DIV> __device__ __forceinline__ Sequence sequence_of(const PagedCall& c, int first, int base, int L, int rows) {
  Sequence s;
  s.first = first;
  s.base = base;
  s.L = L;
  s.rows = rows;
  if constexpr (DIV::WINDOW) {
    if (c.only != 0 && (rows > 32) != (c.only == 1)) s.rows = 0;
  }
  s.blocks = (s.rows + DIV::BR - 1) / DIV::BR;
  s.a = (double)c.G * ((c.causal ? max(min(base, L), 0) : L) + DIV::ITEM);
  s.step = c.causal ? DIV::BR : 0;
  if constexpr (DIV::WINDOW) {
    // Blocks of a sequence that is longer than the window see about as many keys each: the window of the first row, the rows behind it, the sinks, and what tiles are rounded by.
    const int64_t reach = (int64_t)c.window + c.sinks + DIV::BR / c.G + 2 * DIV::KEYS;
    if (L > reach) {
      s.a = (double)c.G * (double)(reach + DIV::ITEM);
      s.step = 0;
    }
  }
  return s;
}
// The numbers of sequence b (one a lane) as they are in memory, and the sequence.
struct Numbers {
  int L, first, end;
  __device__ __forceinline__ Numbers(const PagedCall& c, int b) : L(c.b.lengths[b]), first(b), end(b + 1) {   // (the host checks T >= B)
    if (c.b.starts) {
      first = c.b.starts[b];
      end = c.b.starts[b + 1];
    }
  }
};
template <class DIV> __device__ __forceinline__ Sequence load_sequence(const PagedCall& c, const Numbers& n) {
  int first = n.first, end = n.end;
  force_rows(c.b, first, end);
  // (a length beyond what the table holds: the new tokens keep their positions, which are those that the append gives them, and see the keys that there are)
  const int length = max(n.L, 0), m = end - first;
  return sequence_of<DIV>(c, first, length - m, min(length, c.b.capacity), m * c.G);
}
// the same for one that all lanes share, in scalar registers
template <class DIV> __device__ __forceinline__ Sequence load_sequence_uniform(const PagedCall& c, int b) {
  const Sequence s = load_sequence<DIV>(c, Numbers(c, b));
  return sequence_of<DIV>(c, __builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.base), __builtin_amdgcn_readfirstlane(s.L),
                          __builtin_amdgcn_readfirstlane(s.rows));
}
template <class DIV> __device__ __forceinline__ Sequence lane_sequence(const PagedCall& c, const Sequence& s, int lane) {
  return sequence_of<DIV>(c, __builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.base, lane), __builtin_amdgcn_readlane(s.L, lane),
                          __builtin_amdgcn_readlane(s.rows, lane));
}

__device__ __forceinline__ double lane_double(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

// A double that all lanes share, in scalar registers: the arithmetic is the vector unit's, and the tile loops have no vector registers to keep it in.
__device__ __forceinline__ double uniform(double v) { return lane_double(v, 0); }
__device__ __forceinline__ void uniform(Sequence& s) {
  s.a = uniform(s.a);
  s.step = uniform(s.step);
}

// A point of the line: item (sequence b, K head h, block t), where on the line that starts, and the distance z from there.
struct Point {
  int b, h, t;
  double at, z;
};

// 64 sequences of the line, one a lane: its stretch, and the sum up to its end.
struct Round {
  Sequence s;
  double cost, incl, longest;   // longest: of the items of all 64
  static __device__ __forceinline__ Numbers numbers(const PagedCall& c, int b0) { return Numbers(c, min(b0 + (int)(threadIdx.x & 63), c.b.B - 1)); }
  template <class DIV> __device__ __forceinline__ void load(const PagedCall& c, int b0, const Numbers& numbers) {
    const int lane = threadIdx.x & 63, n = c.b.B - b0;
    s = load_sequence<DIV>(c, numbers);
    cost = lane < n ? s.upto(s.blocks) * c.b.Hk : 0.0;
    incl = cost;
    longest = s.blocks > 0 ? s.length(s.blocks - 1) : 0.0;
    for (int d = 1; d < min(n, 64); d <<= 1) {
      const double other = __shfl_up(incl, d, 64);
      longest = fmax(longest, __shfl_xor(longest, d, 64));
      if (lane >= d) incl += other;
    }
  }
};

// The line, seen by one wavefront.
template <class DIV> struct Line {
  double total;
  Round first;      // all there is for up to 64 sequences
  int n;            // slots that get a stretch
  double each;      // its length, not a whole number
  double slack;     // a cut no farther than this from an item's start, or else from its end, is made there

  __device__ __forceinline__ void init(const PagedCall& c, const Numbers& numbers) {
    first.load<DIV>(c, 0, numbers);
    total = lane_double(first.incl, min(c.b.B, 64) - 1);
    double longest = lane_double(first.longest, 0);
#pragma clang loop unroll(disable)
    for (int b0 = 64; b0 < c.b.B; b0 += 64) {
      Round r;
      r.load<DIV>(c, b0, Round::numbers(c, b0));
      total += lane_double(r.incl, min(c.b.B - b0, 64) - 1);
      longest = fmax(longest, lane_double(r.longest, 0));
    }
    // (with stretches no longer than an item without keys, every end of an item has a cut near it)
    const float item = (float)longest / (float)c.G;   // in keys
    const float least = fmaxf((float)DIV::ITEM, sqrtf((float)DIV::SPREAD * item));
    n = __builtin_amdgcn_readfirstlane((int)fmin(fmax(total / ((double)least * c.G), 1.0), (double)c.slots));
    each = total / n;
    slack = (double)DIV::SLACK * c.G;
  }
  __device__ __forceinline__ double start(int slot) const { return slot < n ? floor(each * slot) : total; }   // (each * slot < total: grows with the slot)
  // The item at 0 <= x < total, and its sequence.
  __device__ __forceinline__ Point locate(const PagedCall& c, double x, Sequence& s) const {
    Point p;
    double before = 0.0;
    Round r = first;
#pragma clang loop unroll(disable)
    for (int b0 = 0;; b0 += 64) {
      if (b0 > 0) r.load<DIV>(c, b0, Round::numbers(c, b0));
      const int in_round = min(c.b.B - b0, 64);
      const uint64_t beyond = __ballot((int)(threadIdx.x & 63) < in_round && before + r.incl > x);
      if (beyond != 0 || b0 + 64 >= c.b.B) {
        const int i = beyond != 0 ? __builtin_ctzll(beyond) : in_round - 1;
        p.b = b0 + i;
        p.at = before + lane_double(r.incl, i) - lane_double(r.cost, i);
        s = lane_sequence<DIV>(c, r.s, i);
        break;
      }
      before += lane_double(r.incl, 63);
    }
    // (quotients of whole numbers below 2^50, rounded down, are exact)
    const double head = s.upto(s.blocks);
    p.h = __builtin_amdgcn_readfirstlane((int)((x - p.at) / head));
    p.at += p.h * head;
    p.t = 0;
    if (s.blocks > 1) {   // t with upto(t) <= x - at < upto(t + 1)
      const double y = x - p.at, q = s.a + 0.5 * s.step;
      int t = (int)(s.step == 0.0 ? y / s.a : (sqrt(q * q + 2.0 * s.step * y) - q) / s.step);
      t = min(max(t, 0), s.blocks - 1);
      while (t > 0 && s.upto(t) > y) --t;
      while (t + 1 < s.blocks && s.upto(t + 1) <= y) ++t;
      p.t = __builtin_amdgcn_readfirstlane(t);
      p.at += s.upto(p.t);
    }
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

// The item behind `at`, whose stretch ends at x on the line: false if there is none.  s: its sequence, of at before.
template <class DIV> __device__ __forceinline__ bool next_item(const PagedCall& c, double x, Point& at, Sequence& s) {
  at.at = uniform(x);
  at.z = 0.0;
  if (++at.t < s.blocks) return true;
  at.t = 0;
  if (++at.h < c.b.Hk) return true;
  at.h = 0;
  do {
    if (++at.b >= c.b.B) return false;
    s = load_sequence_uniform<DIV>(c, at.b);
    uniform(s);
  } while (s.rows == 0);
  return true;
}

// What there is to join at the start of a slot's stretch, left in the workspace.
template <class DIV> __device__ __forceinline__ void leave_join(const PagedCall& c, const Line<DIV>& line, int slot, const Point& at, const Sequence& s) {
  if (slot == 0) return;
  const double near_end = at.at + s.length(at.t) - line.slack;
  int pieces = 0;
  if (at.z > line.slack && line.start(slot) < near_end && line.start(slot - 1) - at.at <= line.slack) {   // an item's first cut
    // slots slot - 1 to the last that starts in the item: the smallest k with start(k) >= near_end
    int k = max((int)(near_end / line.each), slot + 1);
    while (k < line.n && line.start(k) < near_end) ++k;
    while (line.start(k - 1) >= near_end) --k;
    pieces = __builtin_amdgcn_readfirstlane(k - (slot - 1));
  }
  if (threadIdx.x == 0) {
    const Join j = {pieces, at.t * DIV::BR, min(DIV::BR, s.rows - at.t * DIV::BR), s.first, at.h, {0, 0, 0}};
    join_list(c)[slot] = j;
  }
}
// What a workgroup does: the items of its stretch, one after the other.
template <class DIV> struct Work {
  Line<DIV> line;
  Point at;          // the item, from distance at.z from its start ...
  Sequence s;        // ... of this sequence
  int slot;
  double x_end;      // the stretch's end

  // numbers: of the first 64 sequences, loaded before the kernel does what else it can.  False: there is nothing to do.  Leaves in the workspace how many slots there are, and
  // what there is to join.
  __device__ __forceinline__ bool begin(const PagedCall& c, const Numbers& numbers) {
    line.init(c, numbers);
    // (starts that fall can give rows to several sequences, up to B T in all: what is longer than any line of rising starts is not begun, since its points need not be
    // exact, its items need not exist, and its end may be hours away)
    const bool some = line.total > 0.0 && line.total <= c.longest_line;
    if (blockIdx.x == 0 && threadIdx.x == 0) *join_slots(c) = some ? line.n : 0;
    if (!some) return false;
    slot = xcd_item(line.n, (line.n + kXcds - 1) / kXcds);   // neighbours on the line share an XCD's L2
    if (slot < 0) return false;
    at = line.locate(c, line.start(slot), s);
    x_end = line.start(slot + 1);
    leave_join<DIV>(c, line, slot, at, s);
    // a cut near an item's end is made there
    const double v = s.length(at.t);
    if (at.z <= line.slack) at.z = 0.0;
    else if (v - at.z <= line.slack && !next_item<DIV>(c, at.at + v, at, s)) return false;
    x_end = uniform(x_end);
    line.slack = uniform(line.slack);
    at.at = uniform(at.at);
    at.z = uniform(at.z);
    uniform(s);
    return true;
  }
  // Where the stretch ends in the item, v long: v at its end or behind, 0 in front of it.
  __device__ __forceinline__ double up_to(double v) const {
    const double z1 = x_end - at.at;
    if (slot + 1 < line.n && z1 <= line.slack) return 0.0;
    return uniform(v - z1 <= line.slack ? v : z1);
  }
  __device__ __forceinline__ bool next(const PagedCall& c, double v) {
    const double x = at.at + v;
    return x < x_end && next_item<DIV>(c, x, at, s);
  }
};

// row / G
__device__ __forceinline__ int token_of(const PagedCall& c, int row) { return (int)(((uint64_t)(uint32_t)row * c.g_factor) >> c.g_shift); }

// What the 32 rows of an item from row0 on are: lane r has row `row0 + r` = token * G + head of the item's sequence (a copy of the last one beyond the end).
struct Rows {
  int token, head, pos;      // head: of Q; pos: the last key that it sees
  bool ok;
  int pos_first, pos_last;   // of the first and the last row, the same in all lanes
};
// With a window, beside that: the first key of it (its position may lie beyond the keys that there are, and this with it).
struct FarEdge {
  int from;
  int from_first, from_last;
};
// (of the sequence's first new token; far below zero it hides nothing either way)
__device__ __forceinline__ int first_from(const PagedCall& c, const Sequence& s) { return (int)max((int64_t)s.base - c.window + 1, -((int64_t)1 << 30)); }
__device__ __forceinline__ FarEdge far_edge_of(const PagedCall& c, const Sequence& s, int row0, int r) {
  const int base = first_from(c, s);
  FarEdge f;
  f.from = base + token_of(c, min(row0 + r, s.rows - 1));
  f.from_first = __builtin_amdgcn_readfirstlane(base + token_of(c, min(row0, s.rows - 1)));
  f.from_last = __builtin_amdgcn_readfirstlane(base + token_of(c, min(row0 + 31, s.rows - 1)));
  return f;
}
// Keys of a tile of 32 NB from k0 on that lie in front of the row's window and are no sinks.
template <int NB> __device__ __forceinline__ void hide_far(const PagedCall& c, const FarEdge& f, f32x16 (&st)[NB], int k0, int g) {
  if (k0 < f.from_last && k0 + 32 * NB > c.sinks) {
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + 32 * kb + 8 * (i >> 2) + 4 * g + (i & 3);
        if (key < f.from && key >= c.sinks) st[kb][i] = -INFINITY;
      }
  }
}
__device__ __forceinline__ Rows rows_of(const PagedCall& c, const Sequence& s, int h, int row0, int r) {
  Rows w;
  w.ok = row0 + r < s.rows;
  const int row = min(row0 + r, s.rows - 1);
  const int i = token_of(c, row);
  w.head = h * c.G + (row - i * c.G);
  w.token = s.first + i;
  const int all = s.L - 1;
  w.pos = c.causal ? min(s.base + i, all) : all;
  w.pos_first = __builtin_amdgcn_readfirstlane(c.causal ? min(s.base + token_of(c, min(row0, s.rows - 1)), all) : all);
  w.pos_last = __builtin_amdgcn_readfirstlane(c.causal ? min(s.base + token_of(c, min(row0 + 31, s.rows - 1)), all) : all);
  return w;
}

// Tiles of `keys` keys that block t sees: those of its last row.
template <int BR> __device__ __forceinline__ int tiles_of(const PagedCall& c, const Sequence& s, int t, int keys) {
  const int last_row = min((t + 1) * BR, s.rows) - 1;
  const int last = c.causal ? min(s.base + token_of(c, last_row), s.L - 1) : s.L - 1;
  return last < 0 ? 0 : last / keys + 1;
}
// The tiles that block t sees, numbered from 0: those of the sinks, then those from the first that its first row's window reaches to that of its last row's position.
struct SeenTiles {
  int sink_tiles, first, count;
  int from;   // the first key of the first row's window
  // Sixteen rows of a page from `row` on that hold no key that any row of the block sees: their page may belong to another sequence by now, and zeros stand for them.
  __device__ __forceinline__ bool hidden(const PagedCall& c, int row) const { return row >= c.sinks && row + 16 <= from; }
  __device__ __forceinline__ int operator()(int i) const { return i < sink_tiles ? i : i - sink_tiles + first; }
};
template <int BR> __device__ __forceinline__ SeenTiles seen_tiles(const PagedCall& c, const Sequence& s, int t, int keys) {
  const int end = tiles_of<BR>(c, s, t, keys);
  const int from = max(first_from(c, s) + token_of(c, t * BR), 0);
  SeenTiles m;
  m.from = __builtin_amdgcn_readfirstlane(from);
  m.first = __builtin_amdgcn_readfirstlane(from / keys);
  m.sink_tiles = __builtin_amdgcn_readfirstlane(min((c.sinks + keys - 1) / keys, min(m.first, end)));
  m.count = __builtin_amdgcn_readfirstlane(m.sink_tiles + max(end - m.first, 0));
  return m;
}
// Without a window: all tiles up to that of the last row's position.
struct AllTiles {
  int count;
  __device__ __forceinline__ bool hidden(const PagedCall&, int) const { return false; }
  __device__ __forceinline__ int operator()(int i) const { return i; }
};
template <bool WINDOW, int BR> __device__ __forceinline__ auto item_tiles(const PagedCall& c, const Sequence& s, int t, int keys) {
  if constexpr (WINDOW) return seen_tiles<BR>(c, s, t, keys);
  else return AllTiles{tiles_of<BR>(c, s, t, keys)};
}
// Where a cut at distance z of an item of length v falls among its tiles (the same for the pieces on both sides).
__device__ __forceinline__ int cut_at(double z, double v, int tiles) { return __builtin_amdgcn_readfirstlane(z >= v ? tiles : min(tiles, (int)(z / v * tiles))); }

// 16 zeros: what rows beyond a sequence's length, and pages whose number is not one, are copied from.  (What stands in the unwritten part of a page may be
// NaN, and 0 * NaN is not 0.)
__device__ const u32x4 zero_line[1] = {{0u, 0u, 0u, 0u}};

// O rows and row statistics of a finished item's 32 rows.  l_tot, lr_sum: the exact sum and that of the rounded probabilities.  stage: 32 D elements of LDS of
// this wavefront.  (Lane numbers that the compiler does not keep through the tile loop.)
template <typename T, int D>
__device__ __forceinline__ void write_rows(const PagedCall& c, const Sequence& s, int h, int row0, const f32x16 (&o)[D / 32], float m_run, float l_tot, float lr_sum,
                                           T* stage, bool with_lse = true) {
  typedef typename Vec<T>::x4 T4;
  typedef typename Vec<T>::x8 T8;
  constexpr int CPR = D / 8, RPP = 64 / CPR;
  const int lane = lane_id_here(), r = lane & 31, g = lane >> 5;
  const Rows w = rows_of(c, s, h, row0, r);
  const float inv = (l_tot > 0.f && lr_sum > 0.f) ? 1.f / lr_sum : (l_tot == l_tot ? 0.f : l_tot);   // (a row of NaN stays one)
  if (with_lse && g == 0 && w.ok)
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
