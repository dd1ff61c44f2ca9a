// Attention of the new tokens of a ragged batch over a paged key/value cache, gfx950.
//
// For sequence b with m new tokens and L tokens in its pages (the new ones among them), token i = 0 .. m - 1 at position L - m + i, Q head h and
// its K head h / G:   O_i = sum_j softmax_j(tau q_i k_j) v_j,   LSE_i = ln sum_j exp(tau q_i k_j),   j <= L - m + i (causal) or j < L.
//
// One token a sequence reads 4 d bytes of cache for 4 d G operations: the memory bounds it.  A chunk of hundreds of tokens does the same products for all
// of them: the matrix and vector units bound it.  Both run on the tile step of the dense forward (attn_fwd.hip): S^T = K Q^T with 32x32x16 MFMA, a lane holds
// the logits of one row, online softmax, O^T += V^T P^T, 64 keys at a time through LDS, the next tile in flight.
//   Rows: the G heads that share a K head are rows of the same tile, row = token * G + head, so that a K tile is read once for all of them: one token of
// 8 heads a group fills 8 of the 32 columns of an MFMA.
//   Division: contexts of a batch differ by orders of magnitude, and their lengths are known on the GPU only.  The work of all (sequence, K head, block of rows)
// items is laid out on one line, an item's stretch as long as the keys it sees, and every workgroup ("slot") takes an equal stretch of the line: of one item,
// or the end of one, some whole items, the start of another.  Pieces of a cut item leave (m, l, O) in the workspace, which the second kernel joins in their order:
// sums do not depend on which workgroup ends first.
//   Pages: a tile copy instruction covers at most 16 rows, and a page holds 16 or more, so each copy reads one page.  The page numbers of a tile sit in one
// register, one lane a copy, loaded a tile ahead; a copy's address is then scalar work.  Rows beyond the length, and pages whose number is not one, read zeros from a line of
// their own: what stands in the unwritten part of a page (it may be NaN) never meets a probability of zero.
#include "attn_paged.h"
#include "attn_tiles.h"

namespace attn {
namespace {

constexpr int BC = 64;   // keys per tile
constexpr int kItemKeys = 64;   // what an item costs beside its keys, in keys: Q, the first tile's wait, the epilogue

__device__ const u32x4 zero_line[1] = {{0u, 0u, 0u, 0u}};

// A sequence of the batch, every number taken from device memory forced into its range.
struct Sequence {
  int first;   // its first token's row of Q
  int m, L;
  int rows, blocks;   // m * G, and in blocks of BR
  // The line's unit is 1 / G key.  Block t is V(t) = a + step (t + 1) long (an upper bound of the keys its last row sees), t blocks are S(t).
  int64_t a;
  int step;
  __device__ __forceinline__ int64_t upto(int64_t t) const { return t * a + step * (t * (t + 1) / 2); }
};
template <int BR> __device__ __forceinline__ Sequence sequence(const PagedCall& c, int b) {
  Sequence s;
  const PagedBatch& p = c.b;
  int end;
  if (p.starts) {
    s.first = min(max(p.starts[b], 0), p.T);
    end = min(max(p.starts[b + 1], s.first), p.T);
  } else {
    s.first = b;
    end = b + 1;   // (the host checks T >= B)
  }
  s.m = end - s.first;
  s.L = min(max(p.lengths[b], 0), p.capacity);
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

// A point of the line: item (sequence b, K head h, block t) and the distance z from the item's start.
struct Point {
  int b, h, t;
  int64_t z, at;   // at: the item's start on the line
};

// The line, seen by one wavefront: lane i of a round over 64 sequences holds the length of sequence (round + i).
template <int BR> struct Line {
  int64_t total;
  int64_t incl0, cost0;   // of the first round, which is all there is for up to 64 sequences
  int n;                  // slots that get a stretch

  __device__ __forceinline__ void round(const PagedCall& c, int b0, int64_t& cost, int64_t& incl) const {
    const int lane = threadIdx.x & 63;
    cost = 0;
    if (b0 + lane < c.b.B) {
      const Sequence s = sequence<BR>(c, b0 + lane);
      cost = s.upto(s.blocks) * c.b.Hk;
    }
    incl = cost;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t other = __shfl_up(incl, d, 64);
      if (lane >= d) incl += other;
    }
  }
  __device__ __forceinline__ void init(const PagedCall& c) {
    round(c, 0, cost0, incl0);
    total = lane64(incl0, 63);
    for (int b0 = 64; b0 < c.b.B; b0 += 64) {
      int64_t cost, incl;
      round(c, b0, cost, incl);
      total += lane64(incl, 63);
    }
    // (a stretch of less than kSlotKeys keys is not worth a workgroup and a join)
    constexpr int64_t kSlotKeys = 4 * BC + kItemKeys;
    const int64_t worth = total / (kSlotKeys * c.G);
    n = (int)(worth < 1 ? 1 : (worth > c.slots ? c.slots : worth));
  }
  __device__ __forceinline__ int64_t start(int slot) const { return total * slot / n; }   // (total < 2^50: the host checks the sizes)
  __device__ __forceinline__ Point locate(const PagedCall& c, int64_t x) const {   // 0 <= x < total
    Point p;
    int64_t before = 0, cost = cost0, incl = incl0;
    for (int b0 = 0;; b0 += 64) {
      if (b0 > 0) round(c, b0, cost, incl);
      const uint64_t beyond = __ballot(before + incl > x);
      if (beyond != 0 || b0 + 64 >= c.b.B) {
        const int i = beyond != 0 ? __builtin_ctzll(beyond) : 63;
        p.b = b0 + i;
        p.at = before + lane64(incl, i) - lane64(cost, i);
        break;
      }
      before += lane64(incl, 63);
    }
    p.b = min(p.b, c.b.B - 1);
    const Sequence s = sequence<BR>(c, p.b);
    const int64_t head = s.upto(s.blocks), in = x - p.at;
    p.h = (int)(in / head);
    const int64_t y = in - p.h * head;
    // t with S(t) <= y < S(t + 1)
    int t;
    if (s.step == 0) {
      t = (int)(y / s.a);
    } else {
      const double q = (double)s.a + 0.5 * s.step;
      t = (int)((sqrt(q * q + 2.0 * s.step * (double)y) - q) / s.step);
      t = min(max(t, 0), s.blocks - 1);
      while (t > 0 && s.upto(t) > y) --t;
      while (t + 1 < s.blocks && s.upto(t + 1) <= y) ++t;
    }
    p.t = __builtin_amdgcn_readfirstlane(t);
    p.h = __builtin_amdgcn_readfirstlane(p.h);
    p.b = __builtin_amdgcn_readfirstlane(p.b);
    p.at += p.h * head + s.upto(p.t);
    p.z = x - p.at;
    return p;
  }
};

// What the rows of an item's wavefront are: lane r has row `row` = token * G + head of the item's sequence.
struct Rows {
  int token, head, pos;   // of this lane's row (a copy of the last one beyond the end); head: of Q
  bool ok;
  int pos_first, pos_last;   // of the wavefront's first and last row, the same in all lanes
};
__device__ __forceinline__ Rows rows_of(const PagedCall& c, const Sequence& s, int h, int row0) {
  Rows w;
  const int r = threadIdx.x & 31;
  w.ok = row0 + r < s.rows;
  const int row = min(row0 + r, s.rows - 1);
  const int i = row / c.G;
  w.head = h * c.G + (row - i * c.G);
  w.token = s.first + i;
  const int base = s.L - s.m, all = s.L - 1;
  w.pos = c.causal ? base + i : all;
  w.pos_first = c.causal ? base + min(row0, s.rows - 1) / c.G : all;
  w.pos_last = c.causal ? base + min(row0 + 31, s.rows - 1) / c.G : all;
  w.pos_first = __builtin_amdgcn_readfirstlane(w.pos_first);
  w.pos_last = __builtin_amdgcn_readfirstlane(w.pos_last);
  return w;
}

// Key tiles of block t: those its last row sees.
template <int BR> __device__ __forceinline__ int tiles_of(const PagedCall& c, const Sequence& s, int t) {
  const int last_row = min((t + 1) * BR, s.rows) - 1;
  const int last = c.causal ? s.L - s.m + last_row / c.G : s.L - 1;
  return last < 0 ? 0 : last / BC + 1;
}
// Where a cut at distance z of an item of length v falls among its `tiles` tiles.
__device__ __forceinline__ int cut_at(int64_t z, int64_t v, int tiles) {
  return z >= v ? tiles : min(tiles, (int)((double)z / (double)v * tiles));   // (the same for the pieces on both sides)
}

// O rows and row statistics of a finished item.  stage: 32 D elements of LDS of this wavefront.
template <typename T, int D>
__device__ __forceinline__ void write_rows(const PagedCall& c, const Rows& w, const f32x16 (&o)[D / 32], float m_run, float l_tot, float lr_sum, T* stage) {
  typedef typename Vec<T>::x4 T4;
  typedef typename Vec<T>::x8 T8;
  constexpr int CPR = D / 8, RPP = 64 / CPR;
  const int lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5;
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
    const int row = p * RPP + lane / CPR, ch = lane % CPR;
    const T8 v = *(const T8*)(stage + row * D + 8 * (ch ^ (row & (CPR - 1))));
    const int64_t dst = __shfl(off, row, 64);
    if (dst >= 0 && 8 * ch < c.d) *(T8*)((T*)c.O + dst + 8 * ch) = v;
  }
  __builtin_amdgcn_wave_barrier();
}

// A piece in the workspace: O as the accumulators lie (16 bytes a lane at a time), then the reference and the two sums.
template <int D, int RW> struct Piece {
  static constexpr int kLanes = 64 * RW, kFloats = kLanes * (D / 2 + 3);
  f32x4* o;
  float* s;
  __device__ __forceinline__ Piece(const PagedCall& c, int index, int wave) {
    float* const base = c.part + (int64_t)index * kFloats;
    o = (f32x4*)base + wave * 64 + (threadIdx.x & 63);
    s = base + kLanes * (D / 2) + wave * 64 + (threadIdx.x & 63);
  }
};

template <typename T, int D, int RW, int KG>
__global__ __launch_bounds__(64 * RW * KG, KG == 1 && D <= 64 ? 3 : 2) void paged_kernel(const PagedCall c) {
  typedef typename Vec<T>::x8 T8;
  constexpr int KK = D / 16, DB = D / 32, BR = 32 * RW;
  constexpr int CPR = D / 8, RPC = 64 / CPR, COPIES = BC / RPC / RW;   // copies of a tile that a wavefront issues
  typedef T Tile[BC * D];
  __shared__ __attribute__((aligned(16))) Tile bufs[4 * KG];   // K and V, twice, for every group
  __shared__ float sums[KG > 1 ? (KG - 1) * 3 * 64 * RW : 1];
  Tile* const Ks = bufs;
  Tile* const Vs = bufs + 2 * KG;

  Line<BR> line;
  line.init(c);
  const int slot = xcd_item(line.n, (line.n + kXcds - 1) / kXcds);   // neighbours on the line share an XCD's L2
  if (slot < 0 || line.total == 0) return;
  int64_t x = line.start(slot);
  const int64_t x_end = line.start(slot + 1);
  if (x >= x_end) return;

  const int lane = threadIdx.x & 63;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = KG == 1 ? 0 : wave_all / RW;
  const int wave = wave_all - RW * group;
  const int r = lane & 31, g = lane >> 5;
  const T8 ones = row_sum_ones<T>();
  const float cs = c.scale_log2;
  const int page_mask = (1 << c.b.page_log2) - 1;

  if (D == 32 && c.d < D) {   // head dimension 16: the copies leave columns >= 16 untouched
    zero_tiles(&bufs[0][0], 4 * KG * BC * D);
    __syncthreads();
  }
  TrOffsets<D> tro;
  tro.init();
  // byte offsets of this lane's K fragments in a tile, and of its chunk in a copy relative to the copy's first row
  uint32_t k_off[KK], goff[COPIES];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) k_off[kk] = lds_addr(&Ks[2 * group][0]) + (uint32_t)(lds_off<D>(r, 2 * kk + g) * sizeof(T));
  uint32_t beyond = 0;   // D = 32: copies whose chunk of this lane lies beyond the tensors' columns
#pragma unroll
  for (int p = 0; p < COPIES; ++p) {
    const int row = (wave * COPIES + p) * RPC + lane / CPR, chunk = (lane % CPR) ^ swz_bits<D>(row);
    goff[p] = (uint32_t)(((int64_t)(lane / CPR) * c.b.sn + 8 * chunk) * (int64_t)sizeof(T));
    if (D == 32 && 8 * chunk >= c.d) beyond |= 1u << p;
  }

  Point at = line.locate(c, x);
  Sequence s = sequence<BR>(c, at.b);
  while (true) {
    const int64_t length = s.a + (int64_t)s.step * (at.t + 1);
    const int64_t z1 = min(x_end - at.at, length);
    const int tiles = tiles_of<BR>(c, s, at.t);
    const int j0 = __builtin_amdgcn_readfirstlane(cut_at(at.z, length, tiles)), j1 = __builtin_amdgcn_readfirstlane(cut_at(z1, length, tiles));
    const bool whole = at.z == 0 && z1 == length;
    const int L = s.L;
    const int* const table = c.b.table + (int64_t)at.b * c.b.table_stride;
    const T* const Kg = (const T*)c.K + (int64_t)at.h * c.b.sh;
    const T* const Vg = (const T*)c.V + (int64_t)at.h * c.b.sh;
    const Rows w = rows_of(c, s, at.h, at.t * BR + wave * 32);

    // page numbers of a tile's copies of this wavefront, one lane each
    auto page_numbers = [&](int j) {
      const int row = min(j * BC + (wave * COPIES + min(lane, COPIES - 1)) * RPC, L - 1);
      return table[row >> c.b.page_log2];
    };
    auto copy_tile = [&](int j, int ids, int buf) {
      const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_addr(&Ks[2 * group + buf][0]) + wave * COPIES * 1024);
      const uint32_t v_lds = __builtin_amdgcn_readfirstlane(lds_addr(&Vs[2 * group + buf][0]) + wave * COPIES * 1024);
      if ((j + 1) * BC <= L && __ballot((uint32_t)ids >= (uint32_t)c.b.pages) == 0) {
#pragma unroll
        for (int p = 0; p < COPIES; ++p) {
          const int row = j * BC + (wave * COPIES + p) * RPC;
          const int64_t off = (int64_t)__builtin_amdgcn_readlane(ids, p) * c.b.sp + (int64_t)(row & page_mask) * c.b.sn;
          if (D != 32 || !((beyond >> p) & 1u)) {
            async_copy_b128(Kg + off, goff[p], k_lds + p * 1024);
            async_copy_b128(Vg + off, goff[p], v_lds + p * 1024);
          }
        }
      } else {
        const int lane_row = lane_id_here() / CPR;
#pragma unroll
        for (int p = 0; p < COPIES; ++p) {
          const int row = j * BC + (wave * COPIES + p) * RPC;
          const int id = __builtin_amdgcn_readlane(ids, p);
          const int64_t off = (int64_t)id * c.b.sp + (int64_t)(row & page_mask) * c.b.sn;
          const bool there = (uint32_t)id < (uint32_t)c.b.pages && row + lane_row < L;
          const void* const kp = there ? (const void*)((const char*)(Kg + off) + goff[p]) : (const void*)zero_line;
          const void* const vp = there ? (const void*)((const char*)(Vg + off) + goff[p]) : (const void*)zero_line;
          if (D != 32 || !((beyond >> p) & 1u)) {
            async_copy_b128(kp, k_lds + p * 1024);
            async_copy_b128(vp, v_lds + p * 1024);
          }
        }
      }
    };

    // ---- the first tile, then Q
    int jt = j0 + group;
    int ids = 0;
    if (jt < j1) {
      ids = page_numbers(jt);
      copy_tile(jt, ids, 0);
      if (jt + KG < j1) ids = page_numbers(jt + KG);
    }
    T8 qf[KK];
    {
      const T* const q_row = (const T*)c.Q + (int64_t)w.token * c.qt + (int64_t)w.head * c.qh;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (D == 32 && 16 * kk + 8 * g >= c.d) {
#pragma unroll
          for (int e = 0; e < 8; ++e) qf[kk][e] = (T)0.f;
        } else {
          qf[kk] = *(const T8*)(q_row + 16 * kk + 8 * g);
        }
      }
    }
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    f32x4 lr_run = {0.f, 0.f, 0.f, 0.f};
    int calm = kFirstTile;
    wait_async_copies();
    __syncthreads();

    int buf = 0;
    for (int j = j0; j < j1; j += KG) {
      const int jn = jt + KG;
      if (jn < j1) {   // the next tile streams into the other buffer while this one is used
        copy_tile(jn, ids, buf ^ 1);
        if (jn + KG < j1) ids = page_numbers(jn + KG);
      }
      const T* const Vt = Vs[2 * group + buf];
      const int k0 = jt * BC;
      if (jt < j1 && k0 <= w.pos_last) {
        constexpr int PF = 4;
        f32x16 st[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) st[kb][i] = 0.f;
        {
          auto k_frag = [&](int f) {   // f = 2 kk + kb
            const auto* p = (const __attribute__((address_space(3))) T8*)(k_off[f >> 1] + (uint32_t)(buf * BC * D * sizeof(T)));
            return p[32 * (f & 1) * D / 8];
          };
          T8 ring[PF];
#pragma unroll
          for (int f = 0; f < PF; ++f) ring[f] = k_frag(f);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int f = 0; f < 2 * KK; ++f) {
            const T8 cur = ring[f % PF];
            st[f & 1] = mfma32(cur, qf[f >> 1], st[f & 1]);
            if (f + PF < 2 * KK) ring[f % PF] = k_frag(f + PF);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        T8 pf[4];
        const KArgs no_dropout = {};
        softmax_tile_lane_query<T, DB, true, false, D == 128>(no_dropout, st, o, pf, m_run, l_run, lr_run, calm, ones, cs, k0, w.pos_first, w.pos, L, g, 0);
        {
          auto v_frag = [&](int f) {   // f = DB cc + db: consecutive MFMAs hit different accumulators
            const T* base = Vt + 16 * (f / DB) * D;
            return tr_frag<T8>(base + tro.off[f % DB][0], base + tro.off[f % DB][1]);
          };
          T8 ring[PF];
#pragma unroll
          for (int f = 0; f < PF; ++f) ring[f] = v_frag(f);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int f = 0; f < 4 * DB; ++f) {
            const T8 cur = ring[f % PF];
            o[f % DB] = mfma32(cur, pf[f / DB], o[f % DB]);
            if (f + PF < 4 * DB) ring[f % PF] = v_frag(f + PF);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      wait_async_copies();
      __syncthreads();   // the next tile has landed, and everyone is done with this buffer
      jt = jn;
      buf ^= 1;
    }

    if constexpr (KG > 1) {   // groups of wavefronts took every KG-th tile: join them in the tile buffers, as the dense forward does
      constexpr int kLanes = 64 * RW;
      static_assert((KG - 1) * RW + 2 <= 4 * KG && RW <= 2 && sizeof(Tile) == 4 * D * 32, "LDS holds the groups' O and the output rows");
      f32x4* const o_part = (f32x4*)&bufs[0][0] + (group - 1) * (4 * DB * kLanes) + wave * 64 + lane;
      float* const s_part = sums + (group - 1) * 3 * kLanes + wave * 64 + lane;
      if (group > 0) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const f32x4 v = {o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]};
            o_part[(4 * db + i4) * kLanes] = v;
          }
        s_part[0] = m_run;
        s_part[kLanes] = l_run;
        s_part[2 * kLanes] = lr_run[0];
      }
      __syncthreads();
      if (group == 0) {
#pragma unroll
        for (int k = 1; k < KG; ++k) {
          const float* const sp = s_part + k * 3 * kLanes;
          const f32x4* const op = o_part + k * (4 * DB * kLanes);
          const float mk = sp[0], m = fmaxf(m_run, mk), ref = m == -INFINITY ? 0.f : m;
          const float w0 = __builtin_amdgcn_exp2f(m_run - ref), w1 = __builtin_amdgcn_exp2f(mk - ref);
          m_run = m;
          l_run = l_run * w0 + sp[kLanes] * w1;
          lr_run[0] = lr_run[0] * w0 + sp[2 * kLanes] * w1;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
              const f32x4 v = op[(4 * db + i4) * kLanes];
#pragma unroll
              for (int e = 0; e < 4; ++e) o[db][4 * i4 + e] = o[db][4 * i4 + e] * w0 + v[e] * w1;
            }
        }
      }
    }
    if (group == 0) {
      const float l_tot = l_run + xchg32(l_run);
      if (whole) {
        // (two buffers that hold nothing of the join above)
        T* const stage = KG > 1 ? &bufs[4 * KG - 1][0] + wave * 32 * D : &bufs[0][0] + wave * 32 * D;
        write_rows<T, D>(c, w, o, m_run, l_tot, lr_run[0], stage);
      } else {
        const Piece<D, RW> piece(c, 2 * slot + (at.z == 0 ? 1 : 0), wave);
        if (w.ok) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
              const f32x4 v = {o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]};
              piece.o[(4 * db + i4) * piece.kLanes] = v;
            }
          piece.s[0] = m_run;
          piece.s[piece.kLanes] = l_tot;
          piece.s[2 * piece.kLanes] = lr_run[0];
        }
      }
    }
    // ---- the next item of the stretch
    x = at.at + length;
    if (x >= x_end) break;
    at.at = x;
    at.z = 0;
    if (++at.t == s.blocks) {
      at.t = 0;
      if (++at.h == c.b.Hk) {
        at.h = 0;
        do {
          if (++at.b >= c.b.B) return;   // (not reached: x < total, so there is one with rows)
          s = sequence<BR>(c, at.b);
        } while (s.rows == 0);
      }
    }
    __syncthreads();   // the buffers are free again
    if (D == 32 && c.d < D) {   // (O has stood in them)
      zero_tiles(&bufs[0][0], 4 * KG * BC * D);
      __syncthreads();
    }
  }
}

// Joins the pieces of the items that were cut: the workgroup of slot i looks at the cut at the start of that slot's stretch, and does the item if the cut
// is its first one.
template <typename T, int D, int RW>
__global__ __launch_bounds__(64 * RW) void paged_join_kernel(const PagedCall c) {
  constexpr int DB = D / 32, BR = 32 * RW;
  __shared__ __attribute__((aligned(16))) T stage[RW * 32 * D];
  Line<BR> line;
  line.init(c);
  const int slot = (int)blockIdx.x + 1;
  if (slot >= line.n) return;
  const int64_t x = line.start(slot), x_before = line.start(slot - 1);
  if (x >= line.total) return;
  const Point at = line.locate(c, x);
  if (at.z == 0 || x_before > at.at) return;   // no cut, or not the first one
  const Sequence s = sequence<BR>(c, at.b);
  const int64_t end = at.at + s.a + (int64_t)s.step * (at.t + 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rows w = rows_of(c, s, at.h, at.t * BR + wave * 32);
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m_run = -INFINITY, l_tot = 0.f, lr = 0.f;
  for (int k = slot - 1; k < line.n && line.start(k) < end; ++k) {
    const Piece<D, RW> piece(c, 2 * k + (k < slot ? 1 : 0), wave);
    if (!w.ok) continue;
    const float mk = piece.s[0], m = fmaxf(m_run, mk), ref = m == -INFINITY ? 0.f : m;
    const float w0 = __builtin_amdgcn_exp2f(m_run - ref), w1 = __builtin_amdgcn_exp2f(mk - ref);
    m_run = m;
    l_tot = l_tot * w0 + piece.s[piece.kLanes] * w1;
    lr = lr * w0 + piece.s[2 * piece.kLanes] * w1;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const f32x4 v = piece.o[(4 * db + i4) * piece.kLanes];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[db][4 * i4 + e] = o[db][4 * i4 + e] * w0 + v[e] * w1;
      }
  }
  write_rows<T, D>(c, w, o, m_run, l_tot, lr, stage + wave * 32 * D);
}

template <typename T, int D, int RW, int KG> int launch(const PagedCall& c, hipStream_t s) {
  hipLaunchKernelGGL((paged_kernel<T, D, RW, KG>), dim3(c.slots), dim3(64 * RW * KG), 0, s, c);
  int e = (int)hipGetLastError();
  if (e != 0) return e;
  hipLaunchKernelGGL((paged_join_kernel<T, D, RW>), dim3(c.slots - 1), dim3(64 * RW), 0, s, c);
  return (int)hipGetLastError();
}

constexpr int one_wave_groups(int D) { return D == 128 ? 2 : 4; }   // 128 KB of tiles

template <typename T, int D> int launch_d(const PagedCall& c, const PagedShape& shape, hipStream_t s) {
  if (shape.waves == 1) return launch<T, D, 1, one_wave_groups(D)>(c, s);
  return launch<T, D, 4, 1>(c, s);
}
template <typename T> int launch_t(const PagedCall& c, const PagedShape& shape, hipStream_t s) {
  if (c.d <= 32) return launch_d<T, 32>(c, shape, s);
  if (c.d == 64) return launch_d<T, 64>(c, shape, s);
  return launch_d<T, 128>(c, shape, s);
}

}  // namespace

// Few rows a sequence (single tokens): 32-row blocks, groups of wavefronts over the keys; else blocks of 128 rows.  Slots: the workgroups that the chip holds at a time.
PagedShape paged_shape(int64_t rows, int B, int d) {
  if (rows <= (int64_t)32 * B) return {1, one_wave_groups(d <= 32 ? 32 : d), d == 128 ? kComputeUnits : (d == 64 ? kComputeUnits : 2 * kComputeUnits)};
  return {4, 1, d == 128 ? 2 * kComputeUnits : 3 * kComputeUnits};
}
size_t paged_part_bytes(const PagedShape& s, int d) {
  const int D = d <= 32 ? 32 : d;
  return (size_t)2 * s.slots * 64 * s.waves * (D / 2 + 3) * sizeof(float);
}

int launch_paged_fwd(const PagedCall& c, const PagedShape& shape, int dtype, hipStream_t s) {
  return dtype == ATTN_FP16 ? launch_t<_Float16>(c, shape, s) : launch_t<__bf16>(c, shape, s);
}

}  // namespace attn
