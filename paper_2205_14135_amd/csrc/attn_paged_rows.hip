// Attention over a paged cache for many rows a sequence (chunks of a prompt), gfx950.
//
// Hundreds of rows use every tile of K and V: the matrix and the vector units bound it.  Arithmetic and register layout are those of the dense forward, in two schedules:
//   d = 128: two wavefront groups in ping-pong (attn_fwd_pp.hip), 8 wavefronts of 32 rows, one group a block behind the other, so that one issues MFMA while the other
// does its softmax; K and V tiles of 64 keys in rings of three, group A copies K and group B V.
//   d <= 64: four wavefronts of 32 rows, three workgroups to a compute unit (attn_fwd.hip).
// us, blocks of 128 rows | 256, the main kernel, causal, 16 heads: d = 32, 4 x 4096 tokens 152 | 204; d = 64, a chunk of 1000 tokens among 32 single ones, contexts up to 4000, 22.5 | 28.5;
// d = 128, 2 x 8192 tokens 620 | 560, not causal 1036 | 967.
//   Pages: a wavefront copies 16 rows of a tile, which lie in one page.  Its page number is a lane of a register that holds those of sixteen tiles, loaded sixteen tiles
// ahead: the address of a copy is scalar work alone.  (One load a tile, used in the next, makes the compiler wait for the copies issued since: its count
// of loads in flight does not know them.)
//   The stretches of the line (attn_paged_line.h) make up for blocks of unequal length, short batches and single tokens in between.  Rates, 16 heads, against the dense
// forward without pages, pages of 16 in any order | of 256: d = 128, 2 x 8192 not causal 1160 TFLOP/s, 97 % of it | 97 %, causal 980, 87 % | 92 %; d = 64, 820, 95 % | 103 %, and 810, 87 % | 88 %.  What the
// causal batches lose is the start and the end of stretches.
#include "attn_paged_line.h"

namespace attn {
namespace {

// us, ITEM and SLACK of 256 and 160 | 320 and 320, 128 and 96 | 256 and 256, 16 heads: d = 128, 8 x 256 tokens 25 | 18, 8 x 1024 67 | 67; d = 64, 8 x 256 22 | 14, 32 x 64 on 100 20 | 13, 4 x 4096
// 195 | 195.  Over 76 batches, 32 of them ragged, the same within 1 per cent at d = 128, 6 to 8 less at d = 64; 25 per cent more or less of either changes nothing.
// SPREAD, us with the join, 4 | 18 | 72 | 288: d = 64, 4 heads, 128 tokens on 60000 65 | 65 | 62 | 76; d = 128, 8 heads, 8 x 16 on 2000 22 | 22 | 22 | 29, 256 on 60000 237 | 240 | 238 | 241, 2048 on 14336 and
// 8 x 256 the same with all four: anything between 4 and 72 will do.
typedef Division<256, 64, 320, 320, 18> PairDiv;    // two groups of four wavefronts
typedef Division<128, 64, 256, 256, 18> BlockDiv;   // four wavefronts
constexpr int BC = 64;

// The copies of a tile that a wavefront makes: 16 rows, which lie in one page.  Page numbers come sixteen tiles at a time, those of their 16-row groups one a lane.
// An address is scalar work: two 32-bit products (the host checks that a page, and the step from one to the next, are less than 4 GiB).
template <typename T, int D> struct RowCopies {
  static constexpr int CPR = D / 8, RPC = 64 / CPR, COPIES = 16 / RPC;
  const int* table;
  int L, part;             // rows 16 part .. + 15 of a tile
  int window, ids, ids_next;
  uint32_t goff[COPIES];   // byte offset of this lane's chunk of a copy from the first of the 16 rows
  bool beyond;             // D = 32: that chunk lies beyond the tensors' 16 columns
  __device__ __forceinline__ int numbers(const PagedCall& c, int tile) const {
    return table[min(tile * BC + 16 * (int)(threadIdx.x & 63), L - 1) >> c.b.page_log2];
  }
  __device__ __forceinline__ void init(const PagedCall& c, int b, int length, int part_, int first_tile, int lane) {
    table = c.b.table + (int64_t)b * c.b.table_stride;
    L = length;
    part = part_;
    window = first_tile & ~15;
    ids = ids_next = numbers(c, window);
    beyond = false;
#pragma unroll
    for (int p = 0; p < COPIES; ++p) {
      const int row = p * RPC + lane / CPR, chunk = (lane % CPR) ^ swz_bits<D>(16 * part + row);
      goff[p] = (uint32_t)(((int64_t)row * c.b.sn + 8 * chunk) * (int64_t)sizeof(T));
      if (D == 32) beyond = 8 * chunk >= c.d;
    }
  }
  // Copies tile j's 16 rows of N tensors; lds: of the wavefront's part of the tile.  Tiles are asked for in order, and each one once; ids_next has to be loaded once the first
  // has arrived.
  template <int N> __device__ __forceinline__ void copy(const PagedCall& c, int j, const T* const (&tensor)[N], const uint32_t (&lds_part)[N]) {
    if ((j & ~15) != window) {
      window = j & ~15;
      ids = ids_next;
#if defined(__HIP_DEVICE_COMPILE__)
      asm volatile("" : "+v"(ids));   // (arrived from here on: else every tile waits for what might be its load, and for the copies behind that)
#endif
      ids_next = numbers(c, window + 16);
    }
    const uint32_t id = (uint32_t)__builtin_amdgcn_readlane(ids, 4 * (j & 15) + part);
    const int row = j * BC + 16 * part;
    const uint64_t offset = (uint64_t)id * c.b.page_bytes + (uint32_t)(row & c.b.page_mask) * c.b.row_bytes;
    if (D == 32 && beyond) return;
    if (__builtin_expect(row + 16 <= L && id < (uint32_t)c.b.pages, 1)) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_part[n]);
#pragma unroll
        for (int p = 0; p < COPIES; ++p) async_copy_b128((const char*)tensor[n] + offset, goff[p], lds + p * 1024);
      }
    } else {
      const int lane_row = lane_id_here() / CPR;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_part[n]);
#pragma unroll
        for (int p = 0; p < COPIES; ++p)
          async_copy_b128(id < (uint32_t)c.b.pages && row + p * RPC + lane_row < L ? (const void*)((const char*)tensor[n] + offset + goff[p]) : (const void*)zero_line,
                          lds + p * 1024);
      }
    }
  }
};

// Q^T fragments (B operand) of this lane's row
template <typename T, int D> __device__ __forceinline__ void load_q(const PagedCall& c, const Rows& w, int g, typename Vec<T>::x8 (&qf)[D / 16]) {
  typedef typename Vec<T>::x8 T8;
  const T* const q_row = (const T*)c.Q + (int64_t)w.token * c.qt + (int64_t)w.head * c.qh;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    if (D == 32 && 16 * kk + 8 * g >= c.d) {   // head dimension 16: the upper columns are zeros
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[kk][e] = (T)0.f;
    } else {
      qf[kk] = *(const T8*)(q_row + 16 * kk + 8 * g);
    }
  }
}

// A piece in the layout of the accumulators: 16 bytes a lane at a time, whole lines; then the statistics of every wavefront's 32 rows.
template <int D> __device__ __forceinline__ f32x4* piece_o(float* piece, int wave, int lane) { return (f32x4*)piece + wave * (8 * D) + lane; }
template <int D, int BR> __device__ __forceinline__ f32x4* piece_s(float* piece, int wave, int lane) { return (f32x4*)(piece + BR * D) + 32 * wave + (lane & 31); }
template <int D, int BR> __device__ __forceinline__ void write_piece(const PagedCall& c, int wave, int index, const f32x16 (&o)[D / 32], float m_run, float l_tot, float lr_sum) {
  const int lane = lane_id_here();
  float* const piece = piece_of<D, BR>(c, index);
  f32x4* const po = piece_o<D>(piece, wave, lane);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4 v = {o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]};
      po[64 * (4 * db + i4)] = v;
    }
  if (lane < 32) {
    const f32x4 v = {m_run, l_tot, lr_sum, 0.f};
    *piece_s<D, BR>(piece, wave, lane) = v;
  }
}

// Joins the pieces of the items that were cut: blockIdx.x + 1 is the slot of an item's first cut, blockIdx.y 32 columns; a wavefront does 32 rows, four pieces at a time.
// (Rows one after the other, and lanes as columns, as for single tokens: chunk of 2048 tokens on 14336, two or three pieces of most of 256 items, 32 us; all columns by one
// wavefront, a piece at a time, 14.6.)
template <typename T, int D, int BR>
__global__ __launch_bounds__(2 * BR) void paged_rows_join_kernel(const PagedCall c) {
  constexpr int NP = 4;
  __shared__ __attribute__((aligned(16))) T stage[BR / 32][32 * 32];
  const int slot = (int)blockIdx.x + 1, db = (int)blockIdx.y;
  const Join j = join_list(c)[slot];
  if (slot >= *join_slots(c) || j.pieces == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (32 * wave >= j.rows) return;
  f32x16 o[1];
#pragma unroll
  for (int i = 0; i < 16; ++i) o[0][i] = 0.f;
  float m = -INFINITY, l = 0.f, lr = 0.f;
  for (int k0 = 0; k0 < j.pieces; k0 += NP) {
    f32x4 st[NP], v[NP][4];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int k = min(k0 + i, j.pieces - 1);
      float* const piece = piece_of<D, BR>(c, piece_index(slot - 1 + k, k == 0));
      const f32x4* const po = piece_o<D>(piece, wave, lane) + 256 * db;
      st[i] = *piece_s<D, BR>(piece, wave, lane);
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) v[i][i4] = po[64 * i4];
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < NP; ++i) top = fmaxf(top, st[i][0]);   // (the last piece more than once: no harm)
    const float ref = top == -INFINITY ? 0.f : top, w0 = __builtin_amdgcn_exp2f(m - ref);
    m = top;
    l *= w0;
    lr *= w0;
#pragma unroll
    for (int e = 0; e < 16; ++e) o[0][e] *= w0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (k0 + i >= j.pieces) break;
      const float w = __builtin_amdgcn_exp2f(st[i][0] - ref);
      l += st[i][1] * w;
      lr += st[i][2] * w;
#pragma unroll
      for (int e = 0; e < 16; ++e) o[0][e] += v[i][e / 4][e % 4] * w;
    }
  }
  Sequence s = {};
  s.first = j.first;
  s.rows = j.row0 + j.rows;   // (of the item's sequence, as far as this block goes)
  PagedCall slice = c;
  slice.O = (T*)c.O + 32 * db;
  write_rows<T, 32>(slice, s, j.h, j.row0 + 32 * wave, o, m, l, lr, stage[wave], db == 0);
}

template <typename T, int D>
__global__ __launch_bounds__(512) void paged_pair_kernel(const PagedCall c) {
  typedef typename Vec<T>::x8 T8;
  typedef RowCopies<T, D> Copies;
  constexpr int BR = PairDiv::BR, KK = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) T Ks[3][BC * D];
  __shared__ __attribute__((aligned(16))) T Vs[3][BC * D];

  Work<PairDiv> work;
  if (!work.begin(c, Round::numbers(c, 0))) return;
  const Point& at = work.at;
  const Sequence& s = work.s;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool group_b = wave >= 4;
  const float cs = c.scale_log2;

  while (true) {
    const double length = uniform(s.length(at.t));
    const double z1 = work.up_to(length);
    if (z1 == 0.0) break;
    const bool whole = at.z == 0.0 && z1 == length;
    const int tiles = tiles_of<BR>(c, s, at.t, BC);
    const int j0 = cut_at(at.z, length, tiles), J = cut_at(z1, length, tiles) - j0;   // tiles j0 .. j0 + J - 1
    const int L = s.L, row0 = at.t * BR + 32 * wave;
    const bool valid = row0 < s.rows;   // wavefronts past the end only keep the barriers company
    // (a lane number that the compiler does not derive things from ahead of the loop over items)
    const int lane = lane_id_here(), r = lane & 31, g = lane >> 5;
    const Rows w = rows_of(c, s, at.h, row0, r);

    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    f32x4 lr_run = {0.f, 0.f, 0.f, 0.f};

    if (J > 0) {
      const T* const Tg = (const T*)(group_b ? c.V : c.K) + (int64_t)at.h * c.b.sh;   // what this group copies
      Copies dma;
      dma.init(c, at.b, L, wave & 3, j0, lane);
      const uint32_t ring0 = __builtin_amdgcn_readfirstlane(lds_addr(group_b ? &Vs[0][0] : &Ks[0][0]) + dma.part * Copies::COPIES * 1024);
      auto copy_tile = [&](int j, int k) { dma.template copy<1>(c, j, {Tg}, {ring0 + k * (BC * D * (uint32_t)sizeof(T))}); };
      T8 qf[KK];
      load_q<T, D>(c, w, g, qf);
      const int pos = w.pos;
      int calm = kFirstTile;
      const T8 ones = row_sum_ones<T>();
      TrOffsets<D> tro;
      tro.init();
      f32x16 st[2];
      T8 pf[4];
      auto active = [&](int i) { return valid && (j0 + i) * BC <= w.pos_last; };

      constexpr int PF = 4;
      auto k_frag = [&](const T* kbuf, int f) {  // f = 2 * kk + kb
        return *(const T8*)(kbuf + lds_off<D>(32 * (f & 1) + r, 2 * (f >> 1) + g));
      };
      auto v_frag = [&](const T* vbuf, int f) {  // f = DB * cc + db: consecutive MFMAs hit different accumulators
        const T* base = vbuf + 16 * (f / DB) * D;
        return tr_frag<T8>(base + tro.off[f % DB][0], base + tro.off[f % DB][1]);
      };
      // M block: O^T += V^T P^T (if do_pv) followed by S^T = K Q^T (if do_s), as one software-pipelined stream
      auto do_M = [&](bool do_pv, const T* vbuf, bool do_s, const T* kbuf) {
        constexpr int NV = 4 * DB, NK = 2 * KK;
        T8 ring[PF];
        if (do_pv) {
#pragma unroll
          for (int f = 0; f < PF; ++f) ring[f] = v_frag(vbuf, f);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int f = 0; f < NV; ++f) {
            const T8 cur = ring[f % PF];
            o[f % DB] = mfma32(cur, pf[f / DB], o[f % DB]);
            if (f + PF < NV) ring[f % PF] = v_frag(vbuf, f + PF);
            else if (do_s) ring[f % PF] = k_frag(kbuf, f + PF - NV);
            __builtin_amdgcn_sched_barrier(0);   // keep the prefetch distance the source states
          }
        } else if (do_s) {
#pragma unroll
          for (int f = 0; f < PF; ++f) ring[f] = k_frag(kbuf, f);
        }
        if (do_s) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) st[kb][i] = 0.f;
#pragma unroll
          for (int f = 0; f < NK; ++f) {
            const int ring_slot = do_pv ? (NV + f) % PF : f % PF;
            const T8 cur = ring[ring_slot];
            st[f & 1] = mfma32(cur, qf[f >> 1], st[f & 1]);
            if (f + PF < NK) ring[ring_slot] = k_frag(kbuf, f + PF);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      };
      copy_tile(j0, 0);
      wait_async_copies();   // (and Q)
      dma.ids_next = dma.numbers(c, dma.window + 16);
      if (J > 1) copy_tile(j0 + 1, 1);
      __syncthreads();
      if (group_b) {
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();   // B runs one block behind A
      }
      int cur = 0;   // ring slot of tile i
      for (int i = 0; i < J; ++i) {
        const int nxt = cur == 2 ? 0 : cur + 1, prv = cur == 0 ? 2 : cur - 1;
        do_M(i > 0 && active(i - 1), Vs[prv], active(i), Ks[cur]);
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        const bool more = i + 2 < J;
        if (more) copy_tile(j0 + i + 2, prv);
        if (active(i)) {
          const KArgs no_dropout = {};
          softmax_tile_lane_query<T, DB, true, false, false>(no_dropout, st, o, pf, m_run, l_run, lr_run, calm, ones, cs, (j0 + i) * BC, w.pos_first, pos, L, g, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) wait_async_copies_but<Copies::COPIES>(); else wait_async_copies();
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        cur = nxt;
      }
      do_M(active(J - 1), Vs[cur == 0 ? 2 : cur - 1], false, Ks[0]);
      if (!group_b) { __builtin_amdgcn_sched_barrier(0); __syncthreads(); }  // equal barrier counts
      __builtin_amdgcn_sched_barrier(0);
      __syncthreads();   // every wavefront is done with the tiles: the buffers become output staging
    }

    if (valid) {
      const float l_tot = l_run + xchg32(l_run), lr_sum = lr_run[0];
      if (whole) {
        T* const stage = wave < 4 ? &Ks[0][0] + wave * 32 * D : &Vs[0][0] + (wave - 4) * 32 * D;
        write_rows<T, D>(c, s, at.h, row0, o, m_run, l_tot, lr_sum, stage);
      } else {
        write_piece<D, BR>(c, wave, piece_index(work.slot, at.z == 0.0), o, m_run, l_tot, lr_sum);
      }
    }
    if (!work.next(c, length)) break;
    __syncthreads();   // the buffers are free again
  }
}

// The same with four wavefronts of 32 rows to a workgroup, which share tiles of K and V in two buffers: three workgroups to a compute unit, so that one's first tiles, ends and
// diagonal tiles fall into another's full ones.
template <typename T, int D>
__global__ __launch_bounds__(256, 3) void paged_block_kernel(const PagedCall c) {
  typedef typename Vec<T>::x8 T8;
  typedef RowCopies<T, D> Copies;
  constexpr int BR = BlockDiv::BR, KK = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) T Ks[2][BC * D];
  __shared__ __attribute__((aligned(16))) T Vs[2][BC * D];

  Work<BlockDiv> work;
  if (!work.begin(c, Round::numbers(c, 0))) return;
  const Point& at = work.at;
  const Sequence& s = work.s;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float cs = c.scale_log2;

  while (true) {
    const double length = uniform(s.length(at.t));
    const double z1 = work.up_to(length);
    if (z1 == 0.0) break;
    const bool whole = at.z == 0.0 && z1 == length;
    const int tiles = tiles_of<BR>(c, s, at.t, BC);
    const int j0 = cut_at(at.z, length, tiles), j1 = cut_at(z1, length, tiles);
    const int L = s.L, row0 = at.t * BR + 32 * wave;
    const bool valid = row0 < s.rows;   // wavefronts past the end copy their part of the tiles
    // (a lane number that the compiler does not derive things from ahead of the loop over items)
    const int lane = lane_id_here(), r = lane & 31, g = lane >> 5;
    const Rows w = rows_of(c, s, at.h, row0, r);

    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    f32x4 lr_run = {0.f, 0.f, 0.f, 0.f};

    if (j0 < j1) {
      const T* const Kg = (const T*)c.K + (int64_t)at.h * c.b.sh;
      const T* const Vg = (const T*)c.V + (int64_t)at.h * c.b.sh;
      if (D == 32 && c.d < D) {   // head dimension 16: the copies leave columns >= 16 untouched
        zero_tiles(&Ks[0][0], 2 * BC * D);
        zero_tiles(&Vs[0][0], 2 * BC * D);
        __syncthreads();
      }
      Copies dma;
      dma.init(c, at.b, L, wave, j0, lane);
      const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_addr(&Ks[0][0]) + wave * Copies::COPIES * 1024);
      const uint32_t v_lds = __builtin_amdgcn_readfirstlane(lds_addr(&Vs[0][0]) + wave * Copies::COPIES * 1024);
      auto copy_tile = [&](int j, int buf) {
        const uint32_t at_buf = buf * (BC * D * (uint32_t)sizeof(T));
        dma.template copy<2>(c, j, {Kg, Vg}, {k_lds + at_buf, v_lds + at_buf});
      };
      copy_tile(j0, 0);
      T8 qf[KK];
      load_q<T, D>(c, w, g, qf);
      const int pos = w.pos;
      int calm = kFirstTile;
      const T8 ones = row_sum_ones<T>();
      TrOffsets<D> tro;
      tro.init();
      uint32_t k_off[KK];   // byte offsets of this lane's K fragments in a tile
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        k_off[kk] = lds_addr(&Ks[0][0]) + (uint32_t)(lds_off<D>(r, 2 * kk + g) * sizeof(T));
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(k_off[kk]));   // (kept whole: derived again on every tile otherwise)
#endif
      }
      wait_async_copies();   // (and Q)
      dma.ids_next = dma.numbers(c, dma.window + 16);
      __syncthreads();
      int buf = 0;
      for (int j = j0; j < j1; ++j) {
        const int k0 = j * BC;
        const bool active = valid && k0 <= w.pos_last;
        constexpr int PF = 4;   // operand reads run ahead of their MFMA
        f32x16 st[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) st[kb][i] = 0.f;
        if (active) {
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
        // The next tile streams into the other buffer while this one is used.  (Its addresses are made while the products above are under way: d = 64, 2 x 8192 tokens not causal,
        // with one address for K and V and a branch for both, 736 -> 632 us.)
        if (j + 1 < j1) copy_tile(j + 1, buf ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        if (active) {
          T8 pf[4];
          const KArgs no_dropout = {};
          softmax_tile_lane_query<T, DB, true, false, false>(no_dropout, st, o, pf, m_run, l_run, lr_run, calm, ones, cs, k0, w.pos_first, pos, L, g, 0);
          {
            const T* const Vt = Vs[buf];
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
        buf ^= 1;
      }
    }

    if (valid) {
      const float l_tot = l_run + xchg32(l_run), lr_sum = lr_run[0];
      if (whole) write_rows<T, D>(c, s, at.h, row0, o, m_run, l_tot, lr_sum, &Ks[0][0] + wave * 32 * D);
      else write_piece<D, BR>(c, wave, piece_index(work.slot, at.z == 0.0), o, m_run, l_tot, lr_sum);
    }
    if (!work.next(c, length)) break;
    __syncthreads();   // the buffers are free again
  }
}

template <typename T, int D> int launch(const PagedCall& c, hipStream_t s) {
  constexpr int BR = paged_block_rows(D);
  if constexpr (BR == PairDiv::BR) hipLaunchKernelGGL((paged_pair_kernel<T, D>), dim3(c.slots), dim3(2 * BR), 0, s, c);
  else hipLaunchKernelGGL((paged_block_kernel<T, D>), dim3(c.slots), dim3(2 * BR), 0, s, c);
  const int e = (int)hipGetLastError();
  if (e != 0) return e;
  hipLaunchKernelGGL((paged_rows_join_kernel<T, D, BR>), dim3(c.slots - 1, D / 32), dim3(2 * BR), 0, s, c);
  return (int)hipGetLastError();
}
template <typename T> int launch_t(const PagedCall& c, hipStream_t s) {
  if (c.d <= 32) return launch<T, 32>(c, s);
  if (c.d == 64) return launch<T, 64>(c, s);
  return launch<T, 128>(c, s);
}

}  // namespace

// Workgroups that the chip holds, by the kernels' registers and LDS.
int paged_rows_slots(int d) { return kComputeUnits * (d == 128 ? 1 : 3); }
int launch_paged_rows(const PagedCall& c, int dtype, hipStream_t s) { return dtype == ATTN_FP16 ? launch_t<_Float16>(c, s) : launch_t<__bf16>(c, s); }

}  // namespace attn
