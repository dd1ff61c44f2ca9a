// Attention over a paged cache for few rows a sequence (single tokens), gfx950.
//
// A token of G heads a group reads 4 d bytes of cache for 4 d G operations: the memory bounds it, and what counts is how much of K and V is on its way at any time.
// A workgroup is one wavefront with tiles of its own, 32 KB of LDS: five to a compute unit, no barriers, 80 KB in flight, and while one of them
// ends an item and waits for the lengths, page numbers and first tile of the next, the others stream on.
//   A tile is kKeys keys of K and V.  S^T = K Q^T with 32x32x16 MFMA: a lane holds the logits of one row (G of the 32 are real), online softmax,
// O^T += V^T P^T; the matrix and vector work is a fifth of what the memory takes.
//   A page holds 16 rows or more, so a tile is kKeys / 16 page numbers at most, which scalar loads bring two tiles ahead.
#include "attn_paged_line.h"

namespace attn {
namespace {

typedef Division<32, 64, 0> Div;
constexpr int BR = Div::BR;

template <int D> struct OneShape {
  static constexpr int kKeys = D == 128 ? 32 : 64;
#ifdef V_STAGES
  static constexpr int kStages = V_STAGES;
#else
  static constexpr int kStages = 3;
#endif
  static constexpr int kLds = kStages * 2 * kKeys * D * 2;
  static constexpr int kPerUnit = 160 * 1024 / kLds;   // wavefronts that a compute unit holds
};

// Online softmax of a tile of 32 NB keys, lane = row (two lanes a row): as softmax_tile_lane_query in attn_common.h, but the reference follows the maximum of every tile,
// and the sum of the rounded probabilities is taken on the vector unit, which is idle here.
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

// Joins the pieces of the items that were cut: blockIdx.x + 1 is the slot of an item's first cut.  16 wavefronts; with few rows several of them share a row and take
// its pieces by eights in turn.  A lane is C columns.
// (One piece after the other, in the layout of the accumulators: 98.6 us for the 16 items of two contexts of 10^5 tokens, 16 pieces each.)
template <typename T, int D>
__global__ __launch_bounds__(1024) void paged_one_join_kernel(const PagedCall c) {
  constexpr int WAVES = 16, C = D / 64 > 0 ? D / 64 : 1;
  __shared__ float sums[WAVES][64 * C + 4];
  const int slot = (int)blockIdx.x + 1;
  const Join j = join_list(c)[slot];
  if (slot >= *join_slots(c) || j.pieces == 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = j.rows;
  int share = 1;   // wavefronts of a row
  while (2 * share * rows <= WAVES && 8 * share < j.pieces) share *= 2;
  const int col = min(C * lane, D - C), turn = wave % share;
  for (int r0 = 0; r0 < rows; r0 += WAVES / share) {
    const bool active = r0 + wave / share < rows;
    const int row = min(r0 + wave / share, rows - 1);
    float m = -INFINITY, l = 0.f, lr = 0.f, acc[C];
#pragma unroll
    for (int e = 0; e < C; ++e) acc[e] = 0.f;
    for (int k0 = 8 * turn; k0 < j.pieces; k0 += 8 * share) {
      f32x4 st[8];
      float v[8][C];
#pragma unroll
      for (int i = 0; i < 8; ++i) {   // sixteen loads in flight
        const int k = min(k0 + i, j.pieces - 1);
        const float* const piece = piece_of<D, BR>(c, piece_index(slot - 1 + k, k == 0));
        st[i] = *(const f32x4*)(piece + BR * D + 4 * row);
#pragma unroll
        for (int e = 0; e < C; ++e) v[i][e] = piece[row * D + col + e];
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, st[i][0]);   // (a piece twice: no harm)
      const float ref = top == -INFINITY ? 0.f : top, w0 = __builtin_amdgcn_exp2f(m - ref);
      m = top;
      l *= w0;
      lr *= w0;
#pragma unroll
      for (int e = 0; e < C; ++e) acc[e] *= w0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (k0 + i >= j.pieces) break;
        const float w = __builtin_amdgcn_exp2f(st[i][0] - ref);
        l += st[i][1] * w;
        lr += st[i][2] * w;
#pragma unroll
        for (int e = 0; e < C; ++e) acc[e] += v[i][e] * w;
      }
    }
    if (share > 1) {   // (the same for the whole workgroup)
      if (r0 > 0) __syncthreads();
#pragma unroll
      for (int e = 0; e < C; ++e) sums[wave][C * lane + e] = acc[e];
      if (lane == 0) {
        sums[wave][64 * C] = m;
        sums[wave][64 * C + 1] = l;
        sums[wave][64 * C + 2] = lr;
      }
      __syncthreads();
      if (turn == 0)
        for (int k = 1; k < share; ++k) {
          const float* const other = sums[wave + k];
          const float mk = other[64 * C], top = fmaxf(m, mk), ref = top == -INFINITY ? 0.f : top;
          const float w0 = __builtin_amdgcn_exp2f(m - ref), w1 = __builtin_amdgcn_exp2f(mk - ref);
          m = top;
          l = l * w0 + other[64 * C + 1] * w1;
          lr = lr * w0 + other[64 * C + 2] * w1;
#pragma unroll
          for (int e = 0; e < C; ++e) acc[e] = acc[e] * w0 + other[C * lane + e] * w1;
        }
    }
    if (turn != 0 || !active) continue;
    const float inv = (l > 0.f && lr > 0.f) ? 1.f / lr : (l == l ? 0.f : l);   // (a row of NaN stays one)
    const int i = (j.row0 + row) / c.G, head = j.h * c.G + (j.row0 + row) - i * c.G, token = j.first + i;
    if (lane == 0) c.LSE[(int64_t)head * c.b.T + token] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
    if (C * lane < c.d) {
      T* const dst = (T*)c.O + (int64_t)token * c.ot + (int64_t)head * c.oh + C * lane;
#pragma unroll
      for (int e = 0; e < C; ++e) dst[e] = (T)(acc[e] * inv);
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

  int slot;
  Point at;
  Sequence s;
  int64_t x_end;
  if (!stretch<Div>(c, slot, at, s, x_end)) return;

  const int lane = threadIdx.x, r = lane & 31, g = lane >> 5;
  const float cs = c.scale_log2;
  const int page_mask = (1 << c.b.page_log2) - 1;
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

  while (true) {
    const int64_t length = s.length(at.t);
    const int64_t z1 = min(x_end - at.at, length);
    const int tiles = tiles_of<BR>(c, s, at.t, KEYS);
    const int j0 = cut_at(at.z, length, tiles), j1 = cut_at(z1, length, tiles);
    const int L = s.L;
    const Rows w = rows_of(c, s, at.h, at.t * BR, r);
    typedef const __attribute__((address_space(4))) int* ScalarInts;   // (scalar loads)
    const ScalarInts table = (ScalarInts)(uintptr_t)(c.b.table + (int64_t)at.b * c.b.table_stride);
    const T* const Kg = (const T*)c.K + (int64_t)at.h * c.b.sh;
    const T* const Vg = (const T*)c.V + (int64_t)at.h * c.b.sh;

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
          const int64_t off = (int64_t)ids[i] * c.b.sp + (int64_t)((j * KEYS + 16 * i) & page_mask) * c.b.sn;
#pragma unroll
          for (int p = i * PER_PAGE; p < (i + 1) * PER_PAGE; ++p) {
            const int64_t row = (p - i * PER_PAGE) * RPC * c.b.sn;
            if (D != 32 || !((beyond >> p) & 1u)) {
              async_copy_b128(Kg + off + row, goff[p], k_lds + p * 1024);
              async_copy_b128(Vg + off + row, goff[p], v_lds + p * 1024);
            }
          }
        }
      } else {
        const int lane_row = lane_id_here() / CPR;
#pragma unroll
        for (int p = 0; p < COPIES; ++p) {
          const int id = ids[p / PER_PAGE], row = j * KEYS + p * RPC;
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

    if (j0 < j1) page_numbers(j0);
    wait_async_copies();   // Q
#pragma unroll
    for (int i = 0; i + 1 < STAGES; ++i)
      if (j0 + i < j1) {
        copy_tile(j0 + i, i);
        if (j0 + i + 1 < j1) page_numbers(j0 + i + 1);
      }
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f, lr_run = 0.f;

    int buf = 0;
    for (int j = j0; j < j1; ++j) {
      // tile j has landed, those behind it are on their way
      if (STAGES > 2 && j + STAGES - 2 < j1) wait_async_copies_but<(STAGES - 2) * 2 * COPIES>();
      else if (STAGES > 3 && j + 1 < j1) wait_async_copies_but<2 * COPIES>();
      else wait_async_copies();
      if (j + STAGES - 1 < j1) {   // into the buffer of tile j - 1, which this wavefront is done with
        copy_tile(j + STAGES - 1, buf == 0 ? STAGES - 1 : buf - 1);
        if (j + STAGES < j1) page_numbers(j + STAGES);
      }
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
    if (at.z == 0 && z1 == length) write_rows<T, D>(c, s, at.h, at.t * BR, o, m_run, l_tot, lr_sum, &Ks[0][0]);
    else write_piece<D>(c, s, at.t, piece_index(slot, at.z == 0), o, m_run, l_tot, lr_sum);
    const int64_t x = at.at + length;
    if (x >= x_end || !next_item<BR>(c, x, at, s)) break;
  }
}

template <typename T, int D> int launch(const PagedCall& c, hipStream_t s) {
  hipLaunchKernelGGL((paged_one_kernel<T, D>), dim3((c.slots + kXcds - 1) / kXcds * kXcds), dim3(64), 0, s, c);
  const int e = (int)hipGetLastError();
  if (e != 0) return e;
  hipLaunchKernelGGL((paged_one_join_kernel<T, D>), dim3(c.slots - 1), dim3(1024), 0, s, c);
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
