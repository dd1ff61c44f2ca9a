// What the kernels that turn rows of Q and K by their positions share (attn_rotary.hip, attn_norm.hip): the columns and angles of a thread, the
// sequence that a new token belongs to, and how tokens and heads are divided.
#pragma once
#include "attn_paged.h"

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

}  // namespace
}  // namespace attn
