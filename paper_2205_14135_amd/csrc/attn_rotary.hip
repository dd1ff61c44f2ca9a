// Rotary positions, and the append of new tokens to a paged key/value cache, gfx950.
//
// Pair i of the first r columns of a row at position p turns by the angle p f_i, and its length is multiplied by a factor m:
//   y_a = m (x_a cos - x_b sin),   y_b = m (x_b cos + x_a sin),   (a, b) = (2 i, 2 i + 1) or (i, i + r / 2).
// The rotation is linear with the transpose R(-p f), so the gradient is the same kernel with the sine negated.
//
// Memory bounds it: 4 bytes a column, read and written once.  A thread has 16 columns of one token (a "unit": the two 16-byte pieces that pair up) and walks
// over heads, so that its eight sines and cosines serve all of them.  There is no table: the angle in turns, p (f / 2 pi), is a product in 64 bits whose
// whole part is dropped before it is rounded to 32: exact to 2^-22 radians at any position that 31 bits hold, where a table in 32 bits of angles in 32 bits
// is off by 2^-7 at position 10^5.
#include "attn_turn.h"

#include <algorithm>

namespace attn {
namespace {

// blockIdx.x: NT / (d / 16) tokens of B N; blockIdx.y: `per` of the heads of both tensors.
template <typename T, Pairing P>
__global__ __launch_bounds__(NT) void rotary_kernel(const RotaryCall c, const int units_log2, const int per) {
  const int u = (int)threadIdx.x & ((1 << units_log2) - 1);
  const int64_t token = (int64_t)blockIdx.x * (NT >> units_log2) + ((int)threadIdx.x >> units_log2);
  if (token >= (int64_t)c.B * c.N) return;
  const int b = (int)(token / c.N), n = (int)(token - (int64_t)b * c.N);
  const int position = c.positions ? c.positions[b * c.position_sb + n] : n;
  Turn<T, P> turn;
  turn.columns(c.rot, u);
  turn.angles(c.rot, u, position);
  const int heads = c.t[0].H + (c.n_tensors > 1 ? c.t[1].H : 0);
  const int h0 = (int)blockIdx.y * per, h1 = min(heads, h0 + per);
  for (int i = 0; i < c.n_tensors; ++i) {
    const RotaryTensor& t = c.t[i];
    const int first = i == 0 ? 0 : c.t[0].H;
    const T* const x = (const T*)t.x + b * t.xb + n * t.xn;
    T* const y = (T*)t.y + b * t.yb + n * t.yn;
    turn.template rows<true, false>(x, t.xh, y, t.yh, max(h0 - first, 0), min(h1 - first, t.H));
  }
}

// blockIdx.x: NT / (d / 16) tokens; blockIdx.y: `per` of the heads of Q (if there is one), K and V, in this order.
template <typename T, Pairing P>
__global__ __launch_bounds__(NT) void append_kernel(const AppendCall c, const int units_log2, const int per) {
  const PagedBatch& p = c.b;
  const int u = (int)threadIdx.x & ((1 << units_log2) - 1);
  const int token = (int)blockIdx.x * (NT >> units_log2) + ((int)threadIdx.x >> units_log2);
  int b = token, first = token, m = 1;
  if (p.starts) {
    b = sequence_of(p, token, 6 - units_log2);
    if (b >= p.B || token >= p.T) return;
    first = p.starts[b];
    int end = p.starts[b + 1];
    force_rows(p, first, end);
    if (token < first || token >= end) return;
    m = end - first;
  } else if (b >= p.B) {
    return;   // (the host checks T >= B)
  }
  const int64_t position = (int64_t)p.lengths[b] - m + (token - first);
  const int hq = c.Q ? p.Hq : 0, heads = hq + 2 * p.Hk;
  const int h0 = (int)blockIdx.y * per, h1 = min(heads, h0 + per);
  Turn<T, P> turn;
  turn.columns(c.rot, u);
  if (h0 < hq + p.Hk) turn.angles(c.rot, u, (int)position);
  {
    const T* const x = (const T*)c.Q + (int64_t)token * c.qt;
    T* const y = (T*)c.Qo + (int64_t)token * c.ot;
    turn.template rows<true, false>(x, c.qh, y, c.oh, h0, min(h1, hq));
  }
  if (position < 0 || position >= p.capacity) return;
  const int id = p.table[b * p.table_stride + (position >> p.page_log2)];
  if ((uint32_t)id >= (uint32_t)p.pages) return;
  const int64_t slot = id * p.sp + (position & ((1 << p.page_log2) - 1)) * p.sn;
  {
    const T* const x = (const T*)c.K + (int64_t)token * c.kt;
    T* const y = (T*)c.Kc + slot;
    turn.template rows<true, true>(x, c.kh, y, p.sh, max(h0 - hq, 0), min(h1 - hq, p.Hk));
  }
  {
    const T* const x = (const T*)c.V + (int64_t)token * c.vt;
    T* const y = (T*)c.Vc + slot;
    turn.template rows<false, true>(x, c.vh, y, p.sh, max(h0 - hq - p.Hk, 0), min(h1 - hq - p.Hk, p.Hk));
  }
}

template <typename T, Pairing P> int launch_rotary_p(const RotaryCall& c, hipStream_t s) {
  const int units_log2 = log2_units(c.d), tokens = NT >> units_log2;
  const int64_t n = (int64_t)c.B * c.N;
  const int heads = c.t[0].H + (c.n_tensors > 1 ? c.t[1].H : 0), per = heads_per_thread(n << units_log2, heads);
  hipLaunchKernelGGL((rotary_kernel<T, P>), dim3((unsigned)((n + tokens - 1) / tokens), (unsigned)((heads + per - 1) / per)), dim3(NT), 0, s, c, units_log2, per);
  return (int)hipGetLastError();
}
template <typename T> int launch_rotary_t(const RotaryCall& c, hipStream_t s) {
  switch (pairing_of(c.rot)) {
    case kHalves: return launch_rotary_p<T, kHalves>(c, s);
    case kNeighbours: return launch_rotary_p<T, kNeighbours>(c, s);
    default: return launch_rotary_p<T, kHalvesAny>(c, s);
  }
}
template <typename T, Pairing P> int launch_append_p(const AppendCall& c, hipStream_t s) {
  const int units_log2 = log2_units(c.d), tokens = NT >> units_log2;
  const int heads = (c.Q ? c.b.Hq : 0) + 2 * c.b.Hk, per = heads_per_thread((int64_t)c.b.T << units_log2, heads);
  hipLaunchKernelGGL((append_kernel<T, P>), dim3((unsigned)((c.b.T + tokens - 1) / tokens), (unsigned)((heads + per - 1) / per)), dim3(NT), 0, s, c, units_log2, per);
  return (int)hipGetLastError();
}
template <typename T> int launch_append_t(const AppendCall& c, hipStream_t s) {
  switch (pairing_of(c.rot)) {
    case kHalves: return launch_append_p<T, kHalves>(c, s);
    case kNeighbours: return launch_append_p<T, kNeighbours>(c, s);
    default: return launch_append_p<T, kHalvesAny>(c, s);
  }
}

}  // namespace

int launch_rotary(const RotaryCall& c, int dtype, hipStream_t s) {
  return dtype == ATTN_FP16 ? launch_rotary_t<_Float16>(c, s) : launch_rotary_t<__bf16>(c, s);
}
int launch_append(const AppendCall& c, int dtype, hipStream_t s) {
  return dtype == ATTN_FP16 ? launch_append_t<_Float16>(c, s) : launch_append_t<__bf16>(c, s);
}

}  // namespace attn
