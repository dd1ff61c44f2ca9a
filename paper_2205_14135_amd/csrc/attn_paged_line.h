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
// UNIFORM: b is the same in all lanes, and so is what comes back, in scalar registers.
template <int BR, bool UNIFORM = true> __device__ __forceinline__ Sequence sequence(const PagedCall& c, int b) {
  Sequence s;
  const PagedBatch& p = c.b;
  auto number = [](int v) { return UNIFORM ? __builtin_amdgcn_readfirstlane(v) : v; };
  s.L = min(max(number(p.lengths[b]), 0), p.capacity);
  int end;
  if (p.starts) {
    const int first = number(p.starts[b]);
    end = number(p.starts[b + 1]);
    s.first = min(max(first, 0), p.T);
    end = min(max(end, s.first), p.T);
  } else {
    s.first = b;
    end = b + 1;   // (the host checks T >= B)
  }
  s.m = end - s.first;
  s.rows = s.m * c.G;
  s.blocks = (s.rows + BR - 1) / BR;
  s.a = (int64_t)c.G * ((c.causal ? max(s.L - s.m, 0) : s.L) + kItemKeys);
  s.step = c.causal ? BR : 0;
  return s;
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

// The line, seen by one wavefront: lane i of a round over 64 sequences has the length of sequence (round + i), summed up to it.
template <int BR> struct Line {
  int64_t total;
  int64_t incl0, cost0;   // of the first round, which is all there is for up to 64 sequences
  int n;                  // slots that get a stretch
  int64_t each;           // stretches are `each` long, the first `longer` one more
  int longer;
  int64_t slack;          // a cut nearer than this to an item's end is made there

  __device__ __forceinline__ void round(const PagedCall& c, int b0, int64_t& cost, int64_t& incl) const {
    const int lane = threadIdx.x & 63;
    cost = 0;
    if (b0 + lane < c.b.B) {
      const Sequence s = sequence<BR, false>(c, b0 + lane);
      cost = s.upto(s.blocks) * c.b.Hk;
    }
    incl = cost;
    for (int d = 1; d < min(c.b.B - b0, 64); d <<= 1) {
      const int64_t other = __shfl_up(incl, d, 64);
      if (lane >= d) incl += other;
    }
  }
  // least: keys that a stretch has at least, with what an item costs
  __device__ __forceinline__ void init(const PagedCall& c, int least, int slack_share) {
    round(c, 0, cost0, incl0);
    total = lane64(incl0, min(c.b.B, 64) - 1);
    for (int b0 = 64; b0 < c.b.B; b0 += 64) {
      int64_t cost, incl;
      round(c, b0, cost, incl);
      total += lane64(incl, min(c.b.B - b0, 64) - 1);
    }
    const int64_t worth = divided(total, (int64_t)(least + kItemKeys) * c.G);
    n = (int)(worth < 1 ? 1 : (worth > c.slots ? c.slots : worth));
    each = divided(total, n);
    longer = (int)(total - each * n);
    slack = slack_share > 0 ? each / slack_share : 0;
  }
  __device__ __forceinline__ int64_t start(int slot) const { return each * slot + min(slot, longer); }
  __device__ __forceinline__ Point locate(const PagedCall& c, int64_t x) const {   // 0 <= x < total
    Point p;
    int64_t before = 0, cost = cost0, incl = incl0;
    for (int b0 = 0;; b0 += 64) {
      if (b0 > 0) round(c, b0, cost, incl);
      const int in_round = min(c.b.B - b0, 64);
      const uint64_t beyond = __ballot((int)(threadIdx.x & 63) < in_round && before + incl > x);
      if (beyond != 0 || b0 + 64 >= c.b.B) {
        const int i = beyond != 0 ? __builtin_ctzll(beyond) : in_round - 1;
        p.b = b0 + i;
        p.at = before + lane64(incl, i) - lane64(cost, i);
        break;
      }
      before += lane64(incl, 63);
    }
    const Sequence s = sequence<BR>(c, p.b);
    const int64_t head = s.upto(s.blocks), in = x - p.at;
    int h = (int)divided(in, head);
    const int64_t y = in - h * head;
    // t with S(t) <= y < S(t + 1)
    int t = 0;
    if (s.blocks > 1) {
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
    p.b = __builtin_amdgcn_readfirstlane(p.b);
    p.at = lane64(p.at + p.h * head + s.upto(p.t), 0);
    p.z = x - p.at;
    return p;
  }
};

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
    s = sequence<BR>(c, at.b);
  } while (s.rows == 0);
  return true;
}

// The stretch of a slot: from `at` (s: its sequence) to x_end.  False: there is none.
template <class DIV> __device__ __forceinline__ bool stretch(const PagedCall& c, int& slot, Point& at, Sequence& s, int64_t& x_end) {
  constexpr int BR = DIV::BR;
  Line<BR> line;
  DIV::init(line, c);
  slot = xcd_item(line.n, (line.n + kXcds - 1) / kXcds);   // neighbours on the line share an XCD's L2
  if (slot < 0 || line.total == 0) return false;
  at = line.locate(c, line.start(slot));
  s = sequence<BR>(c, at.b);
  x_end = line.start(slot + 1);
  if (line.slack > 0) {
    if (slot + 1 < line.n) {
      const Point e = line.locate(c, x_end);
      const int64_t v = sequence<BR>(c, e.b).length(e.t);
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

// A cut item's piece in the workspace: rows of O, not yet divided by the sum, and (m, l, sum of the rounded probabilities) of every row.
template <int D, int BR> struct Piece {
  static constexpr int kFloats = BR * (D + 4);
  float* o;
  float* s;
  __device__ __forceinline__ Piece(const PagedCall& c, int index) {
    o = c.part + (int64_t)index * kFloats;
    s = o + BR * D;
  }
};
// Its index: a slot has at most one piece that starts inside an item and one that does not.
__device__ __forceinline__ int piece_index(int slot, bool from_start) { return 2 * slot + (from_start ? 1 : 0); }

// 32 rows of a piece, from row0 of the block on (row0 + 32 t of the item's rows exist up to s.rows).
template <int D, int BR>
__device__ __forceinline__ void write_piece(const PagedCall& c, const Sequence& s, int t, int row0, int index, const f32x16 (&o)[D / 32], float m_run, float l_tot,
                                            float lr_sum) {
  const int lane = lane_id_here(), r = lane & 31, g = lane >> 5;
  if (t * BR + row0 + r >= s.rows) return;
  const Piece<D, BR> piece(c, index);
  float* const row = piece.o + (row0 + r) * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4 v = {o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]};
      *(f32x4*)(row + 32 * db + 8 * i4 + 4 * g) = v;
    }
  if (g == 0) {
    const f32x4 v = {m_run, l_tot, lr_sum, 0.f};
    *(f32x4*)(piece.s + 4 * (row0 + r)) = v;
  }
}

// Joins the pieces of the items that were cut.  The workgroup of slot i (from 1 on) looks at the cut at the start of that slot's stretch, and does the item if the
// cut is its first one.  A wavefront does a row: lane k weighs piece k, then the lanes are columns.  One piece after the other, rows in the accumulators' layout, took
// 98.6 us for the 16 items of two contexts of 10^5 tokens (16 pieces each), mostly waiting.
template <typename T, int D, class DIV>
__global__ __launch_bounds__(512) void paged_join_kernel(const PagedCall c) {
  constexpr int BR = DIV::BR;
  Line<BR> line;
  DIV::init(line, c);
  const int slot = (int)blockIdx.x + 1;
  if (slot >= line.n) return;
  const Point at = line.locate(c, line.start(slot));
  const Sequence s = sequence<BR>(c, at.b);
  const int64_t length = s.length(at.t), near_end = at.at + length - line.slack;   // (stretch() above makes the same cuts)
  if (at.z <= line.slack || line.start(slot) >= near_end || line.start(slot - 1) - at.at > line.slack) return;   // no cut, or not the first one
  int pieces = 2;   // of the slots from slot - 1 on
  while (slot - 1 + pieces < line.n && line.start(slot - 1 + pieces) < near_end) ++pieces;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = min(BR, s.rows - at.t * BR);
  constexpr int C = D / 64 > 0 ? D / 64 : 1;   // columns of a lane
  const int col = C * lane;
  for (int row = wave; row < rows; row += 8) {
    // the item's statistic: rounds of 64 pieces
    float m = -INFINITY;
    for (int k0 = 0; k0 < pieces; k0 += 64) {
      const int k = k0 + lane;
      float mk = -INFINITY;
      if (k < pieces) mk = Piece<D, BR>(c, piece_index(slot - 1 + k, k == 0)).s[4 * row];
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) mk = fmaxf(mk, __shfl_xor(mk, d, 64));
      m = fmaxf(m, mk);
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f, lr = 0.f, acc[C];
#pragma unroll
    for (int e = 0; e < C; ++e) acc[e] = 0.f;
    for (int k0 = 0; k0 < pieces; k0 += 64) {
      const int k = k0 + lane, n = min(64, pieces - k0);
      float wk = 0.f, lk = 0.f, rk = 0.f;
      if (k < pieces) {
        const f32x4 st = *(const f32x4*)(Piece<D, BR>(c, piece_index(slot - 1 + k, k == 0)).s + 4 * row);
        wk = __builtin_amdgcn_exp2f(st[0] - ref);
        lk = st[1] * wk;
        rk = st[2] * wk;
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        lk += __shfl_xor(lk, d, 64);
        rk += __shfl_xor(rk, d, 64);
      }
      l += lk;
      lr += rk;
      for (int i0 = 0; i0 < n; i0 += 8) {   // eight loads in flight
        float v[8][C];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int piece = min(k0 + i0 + i, pieces - 1);
          const float* const o = Piece<D, BR>(c, piece_index(slot - 1 + piece, piece == 0)).o + row * D + min(col, D - C);
#pragma unroll
          for (int e = 0; e < C; ++e) v[i][e] = o[e];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float w = i0 + i < n ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wk), (i0 + i) & 63)) : 0.f;
#pragma unroll
          for (int e = 0; e < C; ++e) acc[e] += i0 + i < n ? v[i][e] * w : 0.f;
        }
      }
    }
    const float inv = (l > 0.f && lr > 0.f) ? 1.f / lr : (l == l ? 0.f : l);   // (a row of NaN stays one)
    const int i = (at.t * BR + row) / c.G, head = at.h * c.G + (at.t * BR + row) % c.G, token = s.first + i;
    if (lane == 0) c.LSE[(int64_t)head * c.b.T + token] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
    if (col < c.d) {
      T* const dst = (T*)c.O + (int64_t)token * c.ot + (int64_t)head * c.oh + col;
#pragma unroll
      for (int e = 0; e < C; ++e) dst[e] = (T)(acc[e] * inv);
    }
  }
}

}  // namespace attn
