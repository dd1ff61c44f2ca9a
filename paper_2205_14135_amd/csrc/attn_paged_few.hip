// Attention over a paged cache for one new token a sequence that sees a short window, gfx950.
//
// Where a token's window and sinks are a few tiles, dividing them over the device (attn_paged_one.hip) costs more than it gives: every workgroup works out the line, pieces go through
// memory, and a second launch joins them.  Here a workgroup has an item (32 rows of one K head's group) to itself: its wavefronts take contiguous shares of the item's tiles, each with copies in
// LDS of its own, and meet in LDS: with maxima m_i, sums l_i and rows O_i of the shares,
//   m = max m_i, w_i = 2^(m_i - m), l = sum w_i l_i, O = sum w_i O_i / sum w_i lr_i (lr: the sums of the rounded probabilities).
// What bounds it is latency, of lengths, page numbers, K and V, and of the joining: one token of 16 heads of 64 with 2 K heads, a window of 512 and 4 sinks (264 KB of cache) 6.7 us, 64 such sequences
// 7.9 us; divided 9.8 (6.0 and the join 3.8) and 14.0.
#include "attn_paged_tiles.h"

namespace attn {
namespace {

using Item = Division<kFewRows, 32, 64, 32, 1, true>;

template <typename T, int D>
__global__ __launch_bounds__(64 * paged_few_waves(D), 1) void paged_few_kernel(const PagedCall c) {
  typedef typename Vec<T>::x4 T4;
  typedef OneShape<D> Shape;
  constexpr int KEYS = Shape::kKeys, WAVES = paged_few_waves(D), DB = D / 32, QUADS = D / 4;
  // (a wavefront's O^T, kFewRows D floats, takes the place of its tiles)
  static_assert(kFewRows * D * 4 <= Shape::kLds, "O in place of the tiles");
  __shared__ __attribute__((aligned(16))) T tiles_lds[WAVES][2 * Shape::kStages][KEYS * D];
  __shared__ f32x4 sums[WAVES][kFewRows];   // m, l, sum of the rounded ones
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5;
  const int blocks = (c.G + kFewRows - 1) / kFewRows, pair = (int)blockIdx.x / blocks, t = (int)blockIdx.x - pair * blocks, b = pair / c.b.Hk, h = pair - b * c.b.Hk;
  const Sequence s = load_sequence_uniform<Item>(c, b);
  OneLane<T, D> my;
  my.init(c, lane);
  const SeenTiles tile = seen_tiles<kFewRows>(c, s, t, KEYS);
  const Rows w = rows_of(c, s, h, t * kFewRows, r);
  const FarEdge far = far_edge_of(c, s, t * kFewRows, r);
  f32x16 o[DB];
  float m_run, l_run, lr_run;
  stream_tiles<T, D, true>(c, my, &tiles_lds[wave][0], &tiles_lds[wave][Shape::kStages], tile, tile.count * wave / WAVES, tile.count * (wave + 1) / WAVES, b, h, s.L, w, far, o, m_run, l_run,
                           lr_run);

  const float l_tot = l_run + xchg32(l_run), lr_sum = lr_run + xchg32(lr_run);
  float* const part = (float*)&tiles_lds[wave][0][0];   // (same wavefront: LDS operations complete in program order)
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const int quad = 8 * db + 2 * i4 + g;
      *(f32x4*)(part + r * D + 4 * (quad ^ (r & 7))) = f32x4{o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]};
    }
  if (g == 0) sums[wave][r] = f32x4{m_run, l_tot, lr_sum, 0.f};
  __syncthreads();

  const int rows = min(s.rows - t * kFewRows, kFewRows);
  for (int i = threadIdx.x; i < rows * QUADS; i += 64 * WAVES) {
    const int row = i / QUADS, quad = i % QUADS;
    float m = -INFINITY, l = 0.f, lr = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < WAVES; ++k) m = fmaxf(m, sums[k][row][0]);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      const f32x4 v = sums[k][row];
      const float weight = __builtin_amdgcn_exp2f(v[0] - ref);
      l += v[1] * weight;
      lr += v[2] * weight;
      sum += *(const f32x4*)((const float*)&tiles_lds[k][0][0] + row * D + 4 * (quad ^ (row & 7))) * weight;
    }
    const float inv = (l > 0.f && lr > 0.f) ? 1.f / lr : (l == l ? 0.f : l);   // (a row of NaN stays one)
    const int head = h * c.G + t * kFewRows + row;
    if (quad == 0) c.LSE[(int64_t)head * c.b.T + s.first] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
    if (4 * quad < c.d) {
      T4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (T)(sum[e] * inv);
      *(T4*)((T*)c.O + (int64_t)s.first * c.ot + (int64_t)head * c.oh + 4 * quad) = v;
    }
  }
}

template <typename T, int D> int launch(const PagedCall& c, hipStream_t s) {
  hipLaunchKernelGGL((paged_few_kernel<T, D>), dim3((uint32_t)paged_few_items(c)), dim3(64 * paged_few_waves(D)), 0, s, c);
  return (int)hipGetLastError();
}
template <typename T> int launch_t(const PagedCall& c, hipStream_t s) {
  if (c.d <= 32) return launch<T, 32>(c, s);
  if (c.d == 64) return launch<T, 64>(c, s);
  return launch<T, 128>(c, s);
}

}  // namespace

int launch_paged_few(const PagedCall& c, int dtype, hipStream_t s) { return dtype == ATTN_FP16 ? launch_t<_Float16>(c, s) : launch_t<__bf16>(c, s); }

}  // namespace attn
