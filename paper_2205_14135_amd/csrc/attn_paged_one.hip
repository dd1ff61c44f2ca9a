// Attention over a paged cache for few rows a sequence (single tokens), gfx950.
//
// A token of G heads a group reads 4 d bytes of cache for 4 d G operations: the memory bounds it, and what counts is how much of K and V is on its way at any time.
// A workgroup is one wavefront with tiles of its own (d = 128: 48 KB of LDS, three to a compute unit, 96 KB in flight): no barriers, and while one of them
// ends an item and waits for the page numbers and the first tile of the next, the others stream on.
//   A tile is 32 keys of K and V.  S^T = K Q^T with 32x32x16 MFMA: a lane holds the logits of one row (G of the 32 are real), online softmax,
// O^T += V^T P^T; the matrix and vector work is a fifth of what the memory takes.
//   A page holds 16 rows or more, so a tile has two page numbers at most, which scalar loads bring a tile ahead.
#include "attn_paged_line.h"

#include <algorithm>

namespace attn {
namespace {

// (cuts moved by up to 48 keys or 64 instead of 32: single tokens of mixed lengths 1 and 3 per cent slower.  SPREAD, us with the join, 0 | 1 | 4 | 16: one token on 30000, 4 heads of 64, 30.0 | 20.5 |
// 19.8 | 26.1, on 4000 10.6 | 10.6 | 11.0 | 14.1, 8 heads of 128 15.7 | 15.4 | 17.0 | 20.2; two on 10^5 and 64 of 128 to 8192 the same with all four.)
typedef Division<32, 32, 64, 32, 1> Div;
constexpr int BR = Div::BR;

// (us, the main kernel.  d = 64, tiles of 64 keys | 32: one token over 777 keys 9.5 | 7.6, 32 sequences of up to 2000 35.9 | 35.1 with the join.  d = 128, 64 sequences and two contexts of
// 10^5 tokens: two tiles of 32 keys and five wavefronts to a compute unit 108, 163; three and three 97, 143; four and two 103, 151; two tiles of 64 and two wavefronts 110, 148.)
template <int D> struct OneShape {
  static constexpr int kKeys = 32;     // of a tile
  static constexpr int kStages = 3;    // tiles: one in use, two on their way
  static constexpr int kLds = kStages * 2 * kKeys * D * 2;
  static constexpr int kPerUnit = 160 * 1024 / kLds < 8 ? 160 * 1024 / kLds : 8;   // wavefronts that a compute unit holds
};

// Online softmax of a tile of 32 NB keys, lane = row (two lanes a row): as softmax_tile_lane_query in attn_common.h, but the reference follows the maximum of every tile,
// and the sum of the rounded probabilities is taken on the vector unit, which is idle here.
// Probabilities are rounded to 16 bits, half a step each, because the matrix unit takes the product with V in 16 bits, as in the dense forward; O is divided by the sum of the rounded
// ones, so that weights still sum to 1, and maxima, sums, pieces and joins are in 32 bits.  O is off by 0.0020 to 0.0023 of its norm in bf16, 0.0017 with 32-bit weights rounded once at the end.
template <typename T, int DB, int NB>
__device__ __forceinline__ void softmax_tile(f32x16 (&st)[NB], f32x16 (&o)[DB], typename Vec<T>::x8 (&pf)[2 * NB], float& m_run, float& l_run, float& lr_run, float cs, int k0,
                                             const Rows& w, int L, int g) {
  if (k0 + 32 * NB - 1 > w.pos_first || k0 + 32 * NB > L) {
    const int last = min(w.pos, L - 1);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (k0 + 32 * kb + 8 * (i >> 2) + 4 * g + (i & 3) > last) st[kb][i] = -INFINITY;
  }
  float mx = st[0][0];
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[kb][i]);
  mx = fmaxf(mx, xchg32(mx)) * cs;
  if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
    const float m_new = fmaxf(m_run, mx);
    const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
    m_run = m_new;
    l_run *= alpha;
    lr_run *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
  }
  const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][i], cs, neg_m));
      const T rounded = (T)p;
      l_run += p;
      lr_run += (float)rounded;
      pf[2 * kb + (i >> 3)][i & 7] = rounded;
    }
}

// A piece: rows of O one after the other (few of the 32 are real), then their statistics.
template <int D>
__device__ __forceinline__ void write_piece(const PagedCall& c, const Sequence& s, int t, int index, const f32x16 (&o)[D / 32], float m_run, float l_tot, float lr_sum) {
  const int lane = lane_id_here(), r = lane & 31, g = lane >> 5;
  if (t * BR + r >= s.rows) return;
  float* const piece = piece_of<D, BR>(c, index);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4 v = {o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]};
      *(f32x4*)(piece + r * D + 32 * db + 8 * i4 + 4 * g) = v;
    }
  if (g == 0) {
    const f32x4 v = {m_run, l_tot, lr_sum, 0.f};
    *(f32x4*)(piece + BR * D + 4 * r) = v;
  }
}

// Joins the pieces of the items that were cut: blockIdx.x + 1 is the slot of an item's first cut, blockIdx.y four of its rows (eight at d <= 32).  The four wavefronts take
// pieces by eights in turn, 16 bytes of a row a lane, all loads in flight together, and meet in LDS.
// us, the join alone, two contexts of 10^5 tokens and 64 sequences (16 items of 48 pieces, about 400 of 2 or 3, 4 rows): this 7.6, 5.4; eight rows, pieces by fours 12.6, 6.7, with eight
// wavefronts 9.5, 9.8.  (One piece after the other took 98.6 for 16 pieces; most of the grid has nothing to join, and large workgroups are slow to find that out.)
template <int D> struct JoinShape {
  static constexpr int kWaves = 4, kPieces = 8;                              // of a workgroup; pieces at a time
  static constexpr int kLanes = D / 4, kRowsOfLoad = 64 / kLanes;            // lanes of a row
  static constexpr int kLoads = kRowsOfLoad < 4 ? 4 / kRowsOfLoad : 1, kRows = kLoads * kRowsOfLoad;
};
template <typename T, int D>
__global__ __launch_bounds__(64 * JoinShape<D>::kWaves) void paged_one_join_kernel(const PagedCall c) {
  typedef JoinShape<D> Shape;
  constexpr int WAVES = Shape::kWaves, LPR = Shape::kLanes, RPI = Shape::kRowsOfLoad, NR = Shape::kLoads, NP = Shape::kPieces;
  __shared__ f32x4 part_o[WAVES][NR][64];
  __shared__ f32x4 part_s[WAVES][NR][RPI];
  const int slot = (int)blockIdx.x + 1, row0 = Shape::kRows * (int)blockIdx.y;
  const Join j = join_list(c)[slot];
  if (slot >= *join_slots(c) || j.pieces == 0 || row0 >= j.rows) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = lane / LPR, col = 4 * (lane % LPR);
  f32x4 acc[NR], st[NR];   // st: m, l, sum of the rounded ones
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    st[n] = f32x4{-INFINITY, 0.f, 0.f, 0.f};
  }
  for (int k0 = NP * wave; k0 < j.pieces; k0 += NP * WAVES) {
    f32x4 v[NP][NR], t[NP][NR];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int k = min(k0 + i, j.pieces - 1);
      const float* const piece = piece_of<D, BR>(c, piece_index(slot - 1 + k, k == 0));
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const int row = min(row0 + n * RPI + sub, j.rows - 1);
        t[i][n] = *(const f32x4*)(piece + BR * D + 4 * row);
        v[i][n] = *(const f32x4*)(piece + row * D + col);
      }
    }
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float top = st[n][0];
#pragma unroll
      for (int i = 0; i < NP; ++i) top = fmaxf(top, t[i][n][0]);   // (the last piece more than once: no harm)
      const float ref = top == -INFINITY ? 0.f : top, w0 = __builtin_amdgcn_exp2f(st[n][0] - ref);
      st[n][0] = top;
      st[n][1] *= w0;
      st[n][2] *= w0;
      acc[n] *= w0;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const bool there = k0 + i < j.pieces;
        const float w = __builtin_amdgcn_exp2f(t[i][n][0] - ref);
        if (there) {
          st[n][1] += t[i][n][1] * w;
          st[n][2] += t[i][n][2] * w;
          acc[n] += v[i][n] * w;
        }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    part_o[wave][n][lane] = acc[n];
    if (col == 0) part_s[wave][n][sub] = st[n];
  }
  __syncthreads();
  // wavefront w ends rows of load n = w, w + 4, ...
#pragma unroll
  for (int n0 = 0; n0 < NR; n0 += WAVES) {
    const int n = n0 + wave, row = row0 + n * RPI + sub;
    if (n >= NR || row >= j.rows) continue;
    float m = -INFINITY, l = 0.f, lr = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < WAVES; ++k) m = fmaxf(m, part_s[k][n][sub][0]);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      const f32x4 s = part_s[k][n][sub];
      const float w = __builtin_amdgcn_exp2f(s[0] - ref);
      l += s[1] * w;
      lr += s[2] * w;
      o += part_o[k][n][lane] * w;
    }
    const float inv = (l > 0.f && lr > 0.f) ? 1.f / lr : (l == l ? 0.f : l);   // (a row of NaN stays one)
    const int i = token_of(c, j.row0 + row), head = j.h * c.G + (j.row0 + row) - i * c.G, token = j.first + i;
    if (col == 0) c.LSE[(int64_t)head * c.b.T + token] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
    if (col < c.d) {
      typename Vec<T>::x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (T)(o[e] * inv);
      *(typename Vec<T>::x4*)((T*)c.O + (int64_t)token * c.ot + (int64_t)head * c.oh + col) = v;
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(64, 2) void paged_one_kernel(const PagedCall c) {
  typedef typename Vec<T>::x8 T8;
  typedef OneShape<D> Shape;
  constexpr int KEYS = Shape::kKeys, STAGES = Shape::kStages, NB = KEYS / 32, KK = D / 16, DB = D / 32;
  constexpr int CPR = D / 8, RPC = 64 / CPR, COPIES = KEYS / RPC, PER_PAGE = 16 / RPC, NP = KEYS / 16;
  __shared__ __attribute__((aligned(16))) T Ks[Shape::kStages][KEYS * D];
  __shared__ __attribute__((aligned(16))) T Vs[Shape::kStages][KEYS * D];

  const Numbers numbers = Round::numbers(c, 0);   // (on their way while the lane's constants are made)
  const int lane = threadIdx.x, r = lane & 31, g = lane >> 5;
  const float cs = c.scale_log2;
  TrOffsets<D> tro;
  tro.init();
  uint32_t goff[COPIES];   // byte offset of this lane's chunk of a copy from the copy's first row
#pragma unroll
  for (int p = 0; p < COPIES; ++p) {
    const int chunk = (lane % CPR) ^ swz_bits<D>(p * RPC + lane / CPR);
    goff[p] = (uint32_t)(((int64_t)(lane / CPR) * c.b.sn + 8 * chunk) * (int64_t)sizeof(T));
  }
  uint32_t beyond = 0;   // D = 32: copies whose chunk of this lane lies beyond the tensors' 16 columns
  if constexpr (D == 32) {
#pragma unroll
    for (int p = 0; p < COPIES; ++p)
      if (8 * ((lane % CPR) ^ swz_bits<D>(p * RPC + lane / CPR)) >= c.d) beyond |= 1u << p;
  }
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" ::"v"(tro.off[0][0]), "v"(goff[0]), "v"(goff[COPIES - 1]));
#endif

  Work<Div> work;
  if (!work.begin(c, numbers)) return;
  const Point& at = work.at;
  const Sequence& s = work.s;

  while (true) {
    const double length = uniform(s.length(at.t));
    const double z1 = work.up_to(length);
    if (z1 == 0.0) break;
    const int tiles = tiles_of<BR>(c, s, at.t, KEYS);
    const int j0 = cut_at(at.z, length, tiles), j1 = cut_at(z1, length, tiles);
    const int L = s.L;
    const Rows w = rows_of(c, s, at.h, at.t * BR, r);
    typedef const __attribute__((address_space(4))) int* ScalarInts;   // (scalar loads)
    const ScalarInts table = (ScalarInts)(uintptr_t)(c.b.table + (int64_t)at.b * c.b.table_stride);
    const T* const Kg = (const T*)c.K + (int64_t)at.h * c.b.sh;
    const T* const Vg = (const T*)c.V + (int64_t)at.h * c.b.sh;

    if (D == 32 && c.d < D) {   // (the copies leave columns >= 16 untouched, and O rows have stood there)
      zero_tiles(&Ks[0][0], Shape::kStages * KEYS * D);
      zero_tiles(&Vs[0][0], Shape::kStages * KEYS * D);
      __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    }

    int ids[NP];
    auto page_numbers = [&](int j) {
#pragma unroll
      for (int i = 0; i < NP; ++i) ids[i] = table[min(j * KEYS + 16 * i, L - 1) >> c.b.page_log2];
    };
    auto copy_tile = [&](int j, int buf) {
      const uint32_t k_lds = lds_addr(&Ks[buf][0]), v_lds = lds_addr(&Vs[buf][0]);
      bool all = (j + 1) * KEYS <= L;
#pragma unroll
      for (int i = 0; i < NP; ++i) all = all && (uint32_t)ids[i] < (uint32_t)c.b.pages;
      if (all) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const uint64_t off = (uint64_t)(uint32_t)ids[i] * c.b.page_bytes + (uint32_t)((j * KEYS + 16 * i) & c.b.page_mask) * c.b.row_bytes;
#pragma unroll
          for (int p = i * PER_PAGE; p < (i + 1) * PER_PAGE; ++p) {
            const uint64_t at_row = off + (p - i * PER_PAGE) * RPC * c.b.row_bytes;
            if (D != 32 || !((beyond >> p) & 1u)) {
              async_copy_b128((const char*)Kg + at_row, goff[p], k_lds + p * 1024);
              async_copy_b128((const char*)Vg + at_row, goff[p], v_lds + p * 1024);
            }
          }
        }
      } else {
        const int lane_row = lane_id_here() / CPR;
#pragma unroll
        for (int p = 0; p < COPIES; ++p) {
          const int id = ids[p / PER_PAGE], row = j * KEYS + p * RPC;
          const uint64_t off = (uint64_t)(uint32_t)id * c.b.page_bytes + (uint32_t)(row & c.b.page_mask) * c.b.row_bytes;
          const bool there = (uint32_t)id < (uint32_t)c.b.pages && row + lane_row < L;
          const void* const kp = there ? (const void*)((const char*)Kg + off + goff[p]) : (const void*)zero_line;
          const void* const vp = there ? (const void*)((const char*)Vg + off + goff[p]) : (const void*)zero_line;
          if (D != 32 || !((beyond >> p) & 1u)) {
            async_copy_b128(kp, k_lds + p * 1024);
            async_copy_b128(vp, v_lds + p * 1024);
          }
        }
      }
    };

    T8 qf[KK];
    const T* const q_row = (const T*)c.Q + (int64_t)w.token * c.qt + (int64_t)w.head * c.qh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (D == 32 && 16 * kk + 8 * g >= c.d) {   // head dimension 16: the upper columns are zeros
#pragma unroll
        for (int e = 0; e < 8; ++e) qf[kk][e] = (T)0.f;
      } else {
        qf[kk] = *(const T8*)(q_row + 16 * kk + 8 * g);
      }
    }
    if (j0 < j1) page_numbers(j0);
    wait_async_copies();   // Q (the compiler would wait for its loads, and all copies with them, in the loop)
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f, lr_run = 0.f;

    // Tile j is used while those behind it, up to j + STAGES - 1, are on their way.  (One place for the copies, also the first ones: short calls wait for instructions
    // more than for anything else.)
    int buf = 0, to = 0;
#pragma clang loop unroll(disable)
    for (int j = j0 - (STAGES - 1); j < j1; ++j) {
      const int ahead = j + STAGES - 1;
      if (ahead < j1) {   // into the buffer of tile j - 1, which this wavefront is done with
        copy_tile(ahead, to);
        to = to + 1 == STAGES ? 0 : to + 1;
        if (ahead + 1 < j1) page_numbers(ahead + 1);
      }
      if (j < j0) continue;
      static_assert(STAGES == 3, "the waits below");
      if (j + 2 < j1) wait_async_copies_but<2 * 2 * COPIES>();
      else if (j + 1 < j1) wait_async_copies_but<2 * COPIES>();
      else wait_async_copies();
      const T* const Kt = Ks[buf];
      const T* const Vt = Vs[buf];
      f32x16 st[NB];
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[kb][i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
          st[kb] = mfma32(*(const T8*)(Kt + lds_off<D>(32 * kb + r, 2 * kk + g)), qf[kk], st[kb]);
      T8 pf[2 * NB];
      softmax_tile<T, DB, NB>(st, o, pf, m_run, l_run, lr_run, cs, j * KEYS, w, L, g);
#pragma unroll
      for (int cc = 0; cc < 2 * NB; ++cc)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const T* const base = Vt + 16 * cc * D;
          o[db] = mfma32(tr_frag<T8>(base + tro.off[db][0], base + tro.off[db][1]), pf[cc], o[db]);
        }
      buf = buf + 1 == STAGES ? 0 : buf + 1;
    }

    const float l_tot = l_run + xchg32(l_run), lr_sum = lr_run + xchg32(lr_run);
    if (at.z == 0.0 && z1 == length) write_rows<T, D>(c, s, at.h, at.t * BR, o, m_run, l_tot, lr_sum, &Ks[0][0]);
    else write_piece<D>(c, s, at.t, piece_index(work.slot, at.z == 0.0), o, m_run, l_tot, lr_sum);
    if (!work.next(c, length)) break;
  }
}

template <typename T, int D> int launch(const PagedCall& c, hipStream_t s) {
  hipLaunchKernelGGL((paged_one_kernel<T, D>), dim3((c.slots + kXcds - 1) / kXcds * kXcds), dim3(64), 0, s, c);
  const int e = (int)hipGetLastError();
  if (e != 0) return e;
  const int rows = c.b.starts ? BR : std::min(c.G, BR);   // of a block, at most
  hipLaunchKernelGGL((paged_one_join_kernel<T, D>), dim3(c.slots - 1, (rows + JoinShape<D>::kRows - 1) / JoinShape<D>::kRows), dim3(64 * JoinShape<D>::kWaves), 0, s, c);
  return (int)hipGetLastError();
}
template <typename T> int launch_t(const PagedCall& c, hipStream_t s) {
  if (c.d <= 32) return launch<T, 32>(c, s);
  if (c.d == 64) return launch<T, 64>(c, s);
  return launch<T, 128>(c, s);
}

}  // namespace

int paged_one_slots(int d) {
  return kComputeUnits * (d <= 32 ? OneShape<32>::kPerUnit : (d == 64 ? OneShape<64>::kPerUnit : OneShape<128>::kPerUnit));
}
int launch_paged_one(const PagedCall& c, int dtype, hipStream_t s) { return dtype == ATTN_FP16 ? launch_t<_Float16>(c, s) : launch_t<__bf16>(c, s); }

}  // namespace attn
