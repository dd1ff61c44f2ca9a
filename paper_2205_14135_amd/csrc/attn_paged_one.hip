// Attention over a paged cache for few rows a sequence (single tokens), gfx950.
//
// A token of G heads a group reads 4 d bytes of cache for 4 d G operations: the memory bounds it, and what counts is how much of K and V is on its way at any time.
// A workgroup is one wavefront with tiles of its own (d = 128: 48 KB of LDS, three to a compute unit, 96 KB in flight): no barriers, and while one of them
// ends an item and waits for the page numbers and the first tile of the next, the others stream on.
//   A tile is 32 keys of K and V.  S^T = K Q^T with 32x32x16 MFMA: a lane holds the logits of one row (G of the 32 are real), online softmax,
// O^T += V^T P^T; the matrix and vector work is a fifth of what the memory takes.
//   With a window (WINDOW) the tiles of an item are those that its rows see, the sinks' and the window's: 64 sequences of 500 to 30000 tokens, 32 / 8 heads of 128, window 2048 and four sinks, 443 MB
// in 90 us (4.9 TB/s) and the join 5.
//   A page holds 16 rows or more, so a tile has two page numbers at most, which scalar loads bring a tile ahead.
#include "attn_paged_tiles.h"

#include <algorithm>

namespace attn {
namespace {

// (cuts moved by up to 48 keys or 64 instead of 32: single tokens of mixed lengths 1 and 3 per cent slower.  SPREAD, us with the join, 0 | 1 | 4 | 16: one token on 30000, 4 heads of 64, 30.0 | 20.5 |
// 19.8 | 26.1, on 4000 10.6 | 10.6 | 11.0 | 14.1, 8 heads of 128 15.7 | 15.4 | 17.0 | 20.2; two on 10^5 and 64 of 128 to 8192 the same with all four.)
template <bool WINDOW> using DivOf = Division<kFewRows, 32, 64, 32, 1, WINDOW>;
constexpr int BR = DivOf<false>::BR;

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

template <typename T, int D, bool WINDOW>
__global__ __launch_bounds__(64, 2) void paged_one_kernel(const PagedCall c) {
  typedef OneShape<D> Shape;
  constexpr int KEYS = Shape::kKeys, DB = D / 32;
  __shared__ __attribute__((aligned(16))) T Ks[Shape::kStages][KEYS * D];
  __shared__ __attribute__((aligned(16))) T Vs[Shape::kStages][KEYS * D];

  const Numbers numbers = Round::numbers(c, 0);   // (on their way while the lane's constants are made)
  const int lane = threadIdx.x, r = lane & 31;
  OneLane<T, D> my;
  my.init(c, lane);

  Work<DivOf<WINDOW>> work;
  if (!work.begin(c, numbers)) return;
  const Point& at = work.at;
  const Sequence& s = work.s;

  while (true) {
    const double length = uniform(s.length(at.t));
    const double z1 = work.up_to(length);
    if (z1 == 0.0) break;
    const auto tile = item_tiles<WINDOW, BR>(c, s, at.t, KEYS);   // (tiles are counted among those that are seen)
    const int tiles = tile.count;
    const int j0 = cut_at(at.z, length, tiles), j1 = cut_at(z1, length, tiles);
    const Rows w = rows_of(c, s, at.h, at.t * BR, r);
    FarEdge far;
    if constexpr (WINDOW) far = far_edge_of(c, s, at.t * BR, r);
    f32x16 o[DB];
    float m_run, l_run, lr_run;
    stream_tiles<T, D, WINDOW>(c, my, Ks, Vs, tile, j0, j1, at.b, at.h, s.L, w, far, o, m_run, l_run, lr_run);

    const float l_tot = l_run + xchg32(l_run), lr_sum = lr_run + xchg32(lr_run);
    if (at.z == 0.0 && z1 == length) write_rows<T, D>(c, s, at.h, at.t * BR, o, m_run, l_tot, lr_sum, &Ks[0][0]);
    else write_piece<D>(c, s, at.t, piece_index(work.slot, at.z == 0.0), o, m_run, l_tot, lr_sum);
    if (!work.next(c, length)) break;
  }
}

template <typename T, int D> int launch(const PagedCall& c, hipStream_t s) {
  if (c.window > 0) hipLaunchKernelGGL((paged_one_kernel<T, D, true>), dim3((c.slots + kXcds - 1) / kXcds * kXcds), dim3(64), 0, s, c);
  else hipLaunchKernelGGL((paged_one_kernel<T, D, false>), dim3((c.slots + kXcds - 1) / kXcds * kXcds), dim3(64), 0, s, c);
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
