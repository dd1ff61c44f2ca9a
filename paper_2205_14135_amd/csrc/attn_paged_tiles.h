// What a wavefront does with the tiles of an item of at most 32 rows: single tokens, and few of them (attn_paged_one.hip, attn_paged_few.hip).
#pragma once
#include "attn_paged_line.h"

namespace attn {
namespace {

constexpr int kFewRows = 32;   // of an item

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

// What a lane keeps for all tiles: where its chunks of a copy lie, and its offsets of the transposing reads.
template <typename T, int D> struct OneLane {
  static constexpr int CPR = D / 8, RPC = 64 / CPR, COPIES = OneShape<D>::kKeys / RPC;
  TrOffsets<D> tro;
  uint32_t goff[COPIES];   // byte offset of this lane's chunk of a copy from the copy's first row
  uint32_t beyond;         // D = 32: copies whose chunk of this lane lies beyond the tensors' 16 columns
  __device__ __forceinline__ void init(const PagedCall& c, int lane) {
    tro.init();
#pragma unroll
    for (int p = 0; p < COPIES; ++p) {
      const int chunk = (lane % CPR) ^ swz_bits<D>(p * RPC + lane / CPR);
      goff[p] = (uint32_t)(((int64_t)(lane / CPR) * c.b.sn + 8 * chunk) * (int64_t)sizeof(T));
    }
    beyond = 0;
    if constexpr (D == 32) {
#pragma unroll
      for (int p = 0; p < COPIES; ++p)
        if (8 * ((lane % CPR) ^ swz_bits<D>(p * RPC + lane / CPR)) >= c.d) beyond |= 1u << p;
    }
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" ::"v"(tro.off[0][0]), "v"(goff[0]), "v"(goff[COPIES - 1]));
#endif
  }
};

// Tiles j0 .. j1 - 1 (as `tile` counts them) of K head h of sequence b, whose rows w and L keys these are: O^T, not divided, and this lane's share of the sums.  Ks, Vs: kStages tiles each, the
// wavefront's own.
template <typename T, int D, bool WINDOW, class TILES>
__device__ __forceinline__ void stream_tiles(const PagedCall& c, const OneLane<T, D>& my, T (*Ks)[OneShape<D>::kKeys * D], T (*Vs)[OneShape<D>::kKeys * D], const TILES& tile, int j0, int j1,
                                             int b, int h, int L, const Rows& w, const FarEdge& far, f32x16 (&o)[D / 32], float& m_run, float& l_run, float& lr_run) {
  typedef typename Vec<T>::x8 T8;
  typedef OneShape<D> Shape;
  constexpr int KEYS = Shape::kKeys, STAGES = Shape::kStages, NB = KEYS / 32, KK = D / 16, DB = D / 32;
  constexpr int CPR = D / 8, RPC = 64 / CPR, COPIES = KEYS / RPC, PER_PAGE = 16 / RPC, NP = KEYS / 16;
  const int lane = threadIdx.x & 63, g = lane >> 5, r = lane & 31;
  const float cs = c.scale_log2;
  typedef const __attribute__((address_space(4))) int* ScalarInts;   // (scalar loads)
  const ScalarInts table = (ScalarInts)(uintptr_t)(c.b.table + (int64_t)b * c.b.table_stride);
  const T* const Kg = (const T*)c.K + (int64_t)h * c.b.sh;
  const T* const Vg = (const T*)c.V + (int64_t)h * c.b.sh;

  if (D == 32 && c.d < D) {   // (the copies leave columns >= 16 untouched, and O rows have stood there)
    T8 zeros;
#pragma unroll
    for (int e = 0; e < 8; ++e) zeros[e] = (T)0.f;
    for (int i = 8 * lane; i < Shape::kStages * KEYS * D; i += 8 * 64) {
      *(T8*)(&Ks[0][0] + i) = zeros;
      *(T8*)(&Vs[0][0] + i) = zeros;
    }
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
    for (int i = 0; i < NP; ++i) all = all && (uint32_t)ids[i] < (uint32_t)c.b.pages && !tile.hidden(c, j * KEYS + 16 * i);
    if (all) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const uint64_t off = (uint64_t)(uint32_t)ids[i] * c.b.page_bytes + (uint32_t)((j * KEYS + 16 * i) & c.b.page_mask) * c.b.row_bytes;
#pragma unroll
        for (int p = i * PER_PAGE; p < (i + 1) * PER_PAGE; ++p) {
          const uint64_t at_row = off + (p - i * PER_PAGE) * RPC * c.b.row_bytes;
          if (D != 32 || !((my.beyond >> p) & 1u)) {
            async_copy_b128((const char*)Kg + at_row, my.goff[p], k_lds + p * 1024);
            async_copy_b128((const char*)Vg + at_row, my.goff[p], v_lds + p * 1024);
          }
        }
      }
    } else {
      const int lane_row = lane_id_here() / CPR;
#pragma unroll
      for (int p = 0; p < COPIES; ++p) {
        const int id = ids[p / PER_PAGE], row = j * KEYS + p * RPC;
        const uint64_t off = (uint64_t)(uint32_t)id * c.b.page_bytes + (uint32_t)(row & c.b.page_mask) * c.b.row_bytes;
        const bool there = (uint32_t)id < (uint32_t)c.b.pages && row + lane_row < L && !tile.hidden(c, j * KEYS + 16 * (p / PER_PAGE));
        const void* const kp = there ? (const void*)((const char*)Kg + off + my.goff[p]) : (const void*)zero_line;
        const void* const vp = there ? (const void*)((const char*)Vg + off + my.goff[p]) : (const void*)zero_line;
        if (D != 32 || !((my.beyond >> p) & 1u)) {
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
  if (j0 < j1) page_numbers(tile(j0));
  wait_async_copies();   // Q (the compiler would wait for its loads, and all copies with them, in the loop)
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  m_run = -INFINITY;
  l_run = lr_run = 0.f;

  // Tile j is used while those behind it, up to j + STAGES - 1, are on their way.  (One place for the copies, also the first ones: short calls wait for instructions
  // more than for anything else.)
  int buf = 0, to = 0;
#pragma clang loop unroll(disable)
  for (int j = j0 - (STAGES - 1); j < j1; ++j) {
    const int ahead = j + STAGES - 1;
    if (ahead < j1) {   // into the buffer of tile j - 1, which this wavefront is done with
      copy_tile(tile(ahead), to);
      to = to + 1 == STAGES ? 0 : to + 1;
      if (ahead + 1 < j1) page_numbers(tile(ahead + 1));
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
    if constexpr (WINDOW) hide_far<NB>(c, far, st, tile(j) * KEYS, g);
    softmax_tile<T, DB, NB>(st, o, pf, m_run, l_run, lr_run, cs, tile(j) * KEYS, w, L, g);
#pragma unroll
    for (int cc = 0; cc < 2 * NB; ++cc)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const T* const base = Vt + 16 * cc * D;
        o[db] = mfma32(tr_frag<T8>(base + my.tro.off[db][0], base + my.tro.off[db][1]), pf[cc], o[db]);
      }
    buf = buf + 1 == STAGES ? 0 : buf + 1;
  }
}

}  // namespace
}  // namespace attn
