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
#include "attn_paged.h"

#include <algorithm>

namespace attn {
namespace {

constexpr int NT = 256;

// How the columns of a unit u (of d / 16) pair up.
//   kHalves (r a multiple of 16): 8 columns from 8 u on and the 8 that lie r / 2 behind; behind the turning columns, 16 in a row
//   kNeighbours: columns 16 u .. 16 u + 15, pairs inside
//   kHalvesAny: the same columns, each partner read by itself: sixteen loads of two bytes a thread and head bound it.  128 MiB of Q and K in and out, d = 64, r = 20: 72 us
//   (1.9 TB/s), r = 6 at d = 16 69, where kHalves takes 23 to 25 and kNeighbours 24 to 25 (5.3 to 5.8 TB/s)
enum Pairing { kHalves, kNeighbours, kHalvesAny };

// cosine and sine, times the factor, of the angle at `position` of pair i (of no use behind the last)
__device__ __forceinline__ void turn_of(const RotaryArgs& a, int position, int i, float& cs, float& sn) {
  cs = 1.f;
  sn = 0.f;
  if (2 * i >= a.r) return;
  const double turns = (double)position * (a.freq[i] * 0.15915494309189533577);
  float s, c;
  sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
  cs = c * a.magnitude;
  sn = (a.inverse ? -s : s) * a.magnitude;
}

// The turn of one unit of one token, kept for all heads.  What does not turn is copied, bit by bit: a product with cosine 1 and sine 0 would make NaN of an infinity in the
// other column, and lose the sign of zeros.
template <typename T, Pairing P> struct Turn {
  typedef typename Vec<T>::x8 T8;
  static constexpr int kAngles = P == kHalvesAny ? 16 : 8;
  int lo, hi;                     // first columns of the two pieces
  float cs[kAngles], sn[kAngles];
  int partner[P == kHalvesAny ? 16 : 1];   // kHalvesAny: the other column of a column's pair
  int turning;                    // how many of the unit's eight pairs of neighbouring columns turn: the first ones (r is even)

  __device__ __forceinline__ void columns(const RotaryArgs& a, int u) {
    if (P == kHalves) {
      const int units = a.r / 16;   // that turn
      lo = u < units ? 8 * u : a.r + 16 * (u - units);
      hi = u < units ? lo + a.r / 2 : lo + 8;
      turning = u < units ? 8 : 0;
    } else {
      lo = 16 * u;
      hi = lo + 8;
      turning = a.r / 2 - 8 * u;
    }
  }
  __device__ __forceinline__ void angles(const RotaryArgs& a, int u, int position) {
#pragma unroll
    for (int e = 0; e < kAngles; ++e) {
      if (P == kHalves) {
        turn_of(a, position, u < a.r / 16 ? 8 * u + e : a.r, cs[e], sn[e]);
      } else if (P == kNeighbours) {
        turn_of(a, position, 8 * u + e, cs[e], sn[e]);
      } else {
        const int col = 16 * u + e, half = a.r / 2;
        partner[e] = col;
        cs[e] = 1.f;
        sn[e] = 0.f;
        if (col < a.r) {
          turn_of(a, position, col < half ? col : col - half, cs[e], sn[e]);
          partner[e] = col < half ? col + half : col - half;
          if (col < half) sn[e] = -sn[e];
        }
      }
    }
  }
  // the two pieces of a row x of one head
  __device__ __forceinline__ void turn_pieces(T8& a, T8& b, const T* x) const {
    T8 ya, yb;
    if constexpr (P == kHalves) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float fa = (float)a[e], fb = (float)b[e];
        ya[e] = (T)(fa * cs[e] - fb * sn[e]);
        yb[e] = (T)(fb * cs[e] + fa * sn[e]);
      }
    } else if constexpr (P == kNeighbours) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const T8& v = e < 4 ? a : b;
        const float fa = (float)v[(2 * e) & 7], fb = (float)v[(2 * e + 1) & 7];
        T8& w = e < 4 ? ya : yb;
        w[(2 * e) & 7] = (T)(fa * cs[e] - fb * sn[e]);
        w[(2 * e + 1) & 7] = (T)(fb * cs[e] + fa * sn[e]);
      }
    } else {
      float other[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) other[e] = (float)x[partner[e]];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float own = (float)(e < 8 ? a[e & 7] : b[e & 7]);
        const T v = (T)(own * cs[e] + other[e] * sn[e]);
        if (e < 8) ya[e & 7] = v; else yb[e & 7] = v;
      }
    }
    // (Two columns at a time.  us, a column at a time | a branch around what is copied | this: 12 prompts of up to 2048 tokens appended, half of each row turning, 17.7 | 17.5 | 17.0;
    // 8192 tokens appended without a rotation, 16 heads of 64 columns, 17.3 | 17.2 | 13.1; rotations within 2 per cent.)
    const u32x4 ua = __builtin_bit_cast(u32x4, a), ub = __builtin_bit_cast(u32x4, b);
    u32x4 va = __builtin_bit_cast(u32x4, ya), vb = __builtin_bit_cast(u32x4, yb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      va[i] = i < turning ? va[i] : ua[i];
      vb[i] = i + 4 < turning ? vb[i] : ub[i];
    }
    a = __builtin_bit_cast(T8, va);
    b = __builtin_bit_cast(T8, vb);
  }
  // Heads h0 .. h1 - 1 of one token, x and y at head 0; TURN: they turn, else they are copied; STREAM: past the caches (rows of pages: 12 prompts of up to 2048 tokens, 16 heads of 64
  // columns, 22.4 -> 17.4 us; not Q, which the next call reads, 17.8, nor a rotation's outputs, 33.6 -> 39.1 for 16384 tokens of 20 heads of 128).  Four rows are read before the first is written, so that their
  // loads are in flight together.  All threads of a row are in one wavefront, whose loads are complete before its stores: y may be x.
  template <bool TURN, bool STREAM> __device__ __forceinline__ void rows(const T* x, int64_t xh, T* y, int64_t yh, int h0, int h1) const {
    constexpr int N = 4;
    for (int h = h0; h < h1; h += N) {
      T8 a[N], b[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const T* const row = x + min(h + k, h1 - 1) * xh;
        a[k] = *(const T8*)(row + lo);
        b[k] = *(const T8*)(row + hi);
      }
      if (TURN) {
#pragma unroll
        for (int k = 0; k < N; ++k) turn_pieces(a[k], b[k], x + min(h + k, h1 - 1) * xh);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (h + k >= h1) break;
        T8* const y_lo = (T8*)(y + (h + k) * yh + lo);
        T8* const y_hi = (T8*)(y + (h + k) * yh + hi);
        if (STREAM) {
          __builtin_nontemporal_store(a[k], y_lo);
          __builtin_nontemporal_store(b[k], y_hi);
        } else {
          *y_lo = a[k];
          *y_hi = b[k];
        }
      }
    }
  }
};

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

// Which sequence a token belongs to: the number of sequences that end at it or before.  A wavefront's tokens are consecutive: the ends up to its first
// token are counted 64 at a time, those that fall among its tokens one by one.  (c.B where there is none.)
__device__ __forceinline__ int sequence_of(const PagedBatch& p, int token, int tokens_log2) {
  const int lane = threadIdx.x & 63;
  const int first = __builtin_amdgcn_readfirstlane(token), last = first + (1 << tokens_log2) - 1;
  int seq = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int end = b0 + lane < p.B ? p.starts[b0 + lane + 1] : INT32_MAX;
    seq += __popcll(__ballot(end <= first));
    uint64_t among = __ballot(end > first && end <= last);
    while (among != 0) {
      seq += token >= __builtin_amdgcn_readlane(end, __builtin_ctzll(among));
      among &= among - 1;
    }
  }
  return seq;
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

// Heads a thread walks over: as many as leave 8 wavefronts to a compute unit (its angles are then computed once for all of them), at most 8; and at least so many
// that a grid's second axis holds the rest.  us, 8 wavefronts | 32: 8 x 1024 tokens of 16 + 16 heads of 64 13.0 | 15.1, 4 x 2048 of 8 + 8 heads of 32 6.2 | 7.6, 197 of 12 + 12 of 64 4.4 | 4.4,
// 16384 of 16 + 4 of 128 29.8 | 29.7.
int heads_per_thread(int64_t token_units, int heads) {
  const int64_t enough = (int64_t)kComputeUnits * 8 * 64;
  int per = 8;
  while (per > 1 && token_units * ((heads + per - 1) / per) < enough && (heads + per / 2 - 1) / (per / 2) < 65536) per /= 2;
  return per;
}
int log2_units(int d) { return d == 128 ? 3 : (d == 64 ? 2 : (d == 32 ? 1 : 0)); }

Pairing pairing_of(const RotaryArgs& a) { return a.interleaved ? kNeighbours : (a.r % 16 == 0 ? kHalves : kHalvesAny); }

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
