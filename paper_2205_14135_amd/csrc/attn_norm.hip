// Norm of every row of Q and K with the rotation by its position in the same pass, its gradients, and the append of new tokens with both, gfx950.
//
//   y = R(p) (w o x r),   r = (mean(x^2) + eps)^(-1/2),   R(p) as in attn_rotary.hip.
// With g = R(p)^T dy, h = g o w:
//   dx = r (h - x r^2 mean(h o x)),   dw = sum over all rows of g o x r.
//
// Memory bounds all of it: 4 bytes a column forward, 6 backward, each row read and written once.  A thread has 16 columns of one token and walks over heads, as in
// attn_rotary.hip, so that its angles and its 16 weights serve all of them; the d / 16 threads of a row are neighbours in a wavefront and add their
// shares of a row's sums by cross-lane moves.  All arithmetic between the load and the one rounding at the end is in 32 bits.
// One MI355X: 16384 tokens of 16 + 4 heads of 128 in fp16, half of each row turning, forward 33 us (168 MB, 5.1 TB/s), backward 54 + 4 us (252 MB, 4.7 TB/s in the first launch); 12 prompts of up to 2048
// tokens appended, 16 heads of 64, 16.9 us (91 MB, 5.4 TB/s); 64 single tokens of 32 + 8 heads of 128 5.4 us, a launch and the chain length, angles, row, store.  (Rows loaded ahead of the angles: 5.4 -> 6.4 us for 197
// tokens of 12 + 12 heads of 64, 33 -> 35 us for the 16384.)  (Times of a trace; among others in a replayed graph the single tokens take 5.2.)
// Halves with r no multiple of 16 read every partner by itself, two bytes at a time, and keep 246 to 256 registers: 16384 tokens of 16 + 4 heads of 64 in bf16, 20 columns turning, forward 53 us (84 MB, 1.6 TB/s), backward 65
// (126 MB, 1.9 TB/s), where neighbours take 17 and 30.
//   dw: a thread adds up its own rows, a workgroup its threads', and a second launch the workgroups' sums, each in a fixed order: the same inputs give the same bits.
#include "attn_turn.h"

#include <algorithm>

namespace attn {
namespace {

// Sum over the d / 16 neighbouring lanes that share a row.
__device__ __forceinline__ float row_sum(float v, int units_log2) {
  auto moved = [](float x, auto ctrl) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true)); };
  if (units_log2 > 0) v += moved(v, std::integral_constant<int, 0xB1>());    // lane ^ 1
  if (units_log2 > 1) v += moved(v, std::integral_constant<int, 0x4E>());    // lane ^ 2
  if (units_log2 > 2) v += moved(v, std::integral_constant<int, 0x141>());   // mirrored in eight: the other four
  return v;
}

// Eight weights from column `col` (a multiple of 8) on.
template <typename T> __device__ __forceinline__ void weights_at(const void* w, bool fp32, int col, float* out) {
  typedef typename Vec<T>::x8 T8;
  if (fp32) {
    const float* const p = (const float*)w + col;
    if (((uintptr_t)w & 15u) == 0) {
      const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) { out[e] = a[e]; out[4 + e] = b[e]; }
    } else {   // (a part of a longer vector)
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = p[e];
    }
  } else {
    const T* const p = (const T*)w + col;
    if (((uintptr_t)w & 15u) == 0) {
      const T8 a = *(const T8*)p;
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = (float)a[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = (float)p[e];
    }
  }
}

// One unit of one token, as a row of it passes through: 16 values in 32 bits, 8 from column lo on and 8 from hi on.
template <typename T, Pairing P> struct NormUnit {
  typedef typename Vec<T>::x8 T8;
  Turn<T, P> turn;
  float w[16], wp[P == kHalvesAny ? 16 : 1];   // wp: of the partner columns

  __device__ __forceinline__ void weights(const void* p, bool fp32) {
    weights_at<T>(p, fp32, turn.lo, w);
    weights_at<T>(p, fp32, turn.hi, w + 8);
    if constexpr (P == kHalvesAny) {
#pragma unroll
      for (int e = 0; e < 16; ++e) wp[e] = fp32 ? ((const float*)p)[turn.partner[e]] : (float)((const T*)p)[turn.partner[e]];
    }
  }
  static __device__ __forceinline__ void widen(const T8& a, const T8& b, float (&v)[16]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = (float)a[e];
      v[8 + e] = (float)b[e];
    }
  }
  // v with all of its pairs turned; other: the partners (kHalvesAny)
  __device__ __forceinline__ void turn_all(float (&v)[16], const float (&other)[P == kHalvesAny ? 16 : 1]) const {
    if constexpr (P == kHalvesAny) {
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = v[e] * turn.cs[e] + other[e] * turn.sn[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float &a = P == kHalves ? v[e] : v[2 * e], &b = P == kHalves ? v[8 + e] : v[2 * e + 1];
        const float fa = a, fb = b;
        a = fa * turn.cs[e] - fb * turn.sn[e];
        b = fb * turn.cs[e] + fa * turn.sn[e];
      }
    }
  }
  // The same, but what does not turn stays as it is, as in attn_turn.h: cosine 1 and sine 0 would make NaN of it where an infinity stands in the other column, and lose the sign of zeros.
  __device__ __forceinline__ void apply(float (&v)[16], const float (&other)[P == kHalvesAny ? 16 : 1]) const {
    float was[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) was[e] = v[e];
    turn_all(v, other);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = (P == kHalves ? e & 7 : e / 2) < turn.turning ? v[e] : was[e];
  }
  static __device__ __forceinline__ void narrow(const float (&v)[16], T8& a, T8& b) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[e] = (T)v[e];
      b[e] = (T)v[8 + e];
    }
  }
  // apply and narrow, the selection two rounded columns at a time.  us, all columns by products alone | a column at a time, in 32 bits | this: 197 tokens of 12 + 12 heads of 64 5.1 | 5.3 | 5.1, 64 tokens appended 5.1 | 5.3 | 5.2,
  // 8 x 1024 of 16 + 16 heads of 64 14.0 | 14.1 | 14.2, 16384 of 16 + 4 of 128, halves of them turning, 28.9 | 29.1 | 29.1, neighbours 29.8 | 30.4 | 30.4.
  __device__ __forceinline__ void apply_and_narrow(float (&v)[16], const float (&other)[P == kHalvesAny ? 16 : 1], T8& a, T8& b) const {
    narrow(v, a, b);
    turn_all(v, other);
    T8 ta, tb;
    narrow(v, ta, tb);
    const u32x4 ua = __builtin_bit_cast(u32x4, a), ub = __builtin_bit_cast(u32x4, b);
    u32x4 va = __builtin_bit_cast(u32x4, ta), vb = __builtin_bit_cast(u32x4, tb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      va[i] = i < turn.turning ? va[i] : ua[i];
      vb[i] = i + 4 < turn.turning ? vb[i] : ub[i];
    }
    a = __builtin_bit_cast(T8, va);
    b = __builtin_bit_cast(T8, vb);
  }
  // Heads h0 .. h1 - 1 of one token, x and y at head 0; STREAM: past the caches, as in attn_turn.h.  y may be x: all threads of a row are in one wavefront, whose loads are
  // complete before its stores.
  template <bool STREAM> __device__ __forceinline__ void rows(const T* x, int64_t xh, T* y, int64_t yh, int h0, int h1, float eps, float inv_d, int units_log2) const {
    constexpr int N = 4;
    for (int h = h0; h < h1; h += N) {
      T8 a[N], b[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const T* const row = x + min(h + k, h1 - 1) * xh;
        a[k] = *(const T8*)(row + turn.lo);
        b[k] = *(const T8*)(row + turn.hi);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float v[16], other[P == kHalvesAny ? 16 : 1] = {}, ss = 0.f;
        widen(a[k], b[k], v);
#pragma unroll
        for (int e = 0; e < 16; ++e) ss += v[e] * v[e];
        const float r = 1.f / sqrtf(row_sum(ss, units_log2) * inv_d + eps);
        if constexpr (P == kHalvesAny) {
          const T* const row = x + min(h + k, h1 - 1) * xh;
#pragma unroll
          for (int e = 0; e < 16; ++e) other[e] = (float)row[turn.partner[e]] * r * wp[e];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = v[e] * r * w[e];
        apply_and_narrow(v, other, a[k], b[k]);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (h + k >= h1) break;
        T8* const y_lo = (T8*)(y + (h + k) * yh + turn.lo);
        T8* const y_hi = (T8*)(y + (h + k) * yh + turn.hi);
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
__global__ __launch_bounds__(NT) void norm_rotary_kernel(const NormCall c, const int units_log2, const int per) {
  const RotaryCall& rc = c.rotary;
  const int u = (int)threadIdx.x & ((1 << units_log2) - 1);
  const int64_t token = (int64_t)blockIdx.x * (NT >> units_log2) + ((int)threadIdx.x >> units_log2);
  if (token >= (int64_t)rc.B * rc.N) return;
  const int b = (int)(token / rc.N), n = (int)(token - (int64_t)b * rc.N);
  const int position = rc.positions ? rc.positions[b * rc.position_sb + n] : n;
  NormUnit<T, P> unit;
  unit.turn.columns(rc.rot, u);
  unit.turn.angles(rc.rot, u, position);
  const int heads = rc.t[0].H + (rc.n_tensors > 1 ? rc.t[1].H : 0);
  const int h0 = (int)blockIdx.y * per, h1 = min(heads, h0 + per);
  const float inv_d = 1.f / (float)rc.d;
  for (int i = 0; i < rc.n_tensors; ++i) {
    const RotaryTensor& t = rc.t[i];
    const int first = i == 0 ? 0 : rc.t[0].H;
    const int lo = max(h0 - first, 0), hi = min(h1 - first, t.H);
    if (lo >= hi) continue;
    unit.weights(c.norm.w[i], c.norm.w_fp32);
    unit.template rows<false>((const T*)t.x + b * t.xb + n * t.xn, t.xh, (T*)t.y + b * t.yb + n * t.yn, t.yh, lo, hi, c.norm.eps, inv_d, units_log2);
  }
}

// blockIdx.x: NT / (d / 16) tokens; blockIdx.y: `per` of the heads of Q (if there is one), K and V, in this order; see append_kernel in attn_rotary.hip.
template <typename T, Pairing P>
__global__ __launch_bounds__(NT) void norm_append_kernel(const AppendCall c, const NormArgs norm, const int units_log2, const int per) {
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
  const float inv_d = 1.f / (float)c.d;
  NormUnit<T, P> unit;
  unit.turn.columns(c.rot, u);
  // (the weights are on their way while the angles are made: 64 single tokens 5.8 -> 5.5 us; kHalvesAny learns its partners' columns with the angles)
  if (P != kHalvesAny && h0 < hq) unit.weights(norm.w[0], norm.w_fp32);
  if (h0 < hq + p.Hk) unit.turn.angles(c.rot, u, (int)position);
  if (h0 < hq) {
    if (P == kHalvesAny) unit.weights(norm.w[0], norm.w_fp32);
    unit.template rows<false>((const T*)c.Q + (int64_t)token * c.qt, c.qh, (T*)c.Qo + (int64_t)token * c.ot, c.oh, h0, min(h1, hq), norm.eps, inv_d, units_log2);
  }
  if (position < 0 || position >= p.capacity) return;
  const int id = p.table[b * p.table_stride + (position >> p.page_log2)];
  if ((uint32_t)id >= (uint32_t)p.pages) return;
  const int64_t slot = id * p.sp + (position & ((1 << p.page_log2) - 1)) * p.sn;
  if (h0 < hq + p.Hk && h1 > hq) {
    unit.weights(norm.w[1], norm.w_fp32);
    unit.template rows<true>((const T*)c.K + (int64_t)token * c.kt, c.kh, (T*)c.Kc + slot, p.sh, max(h0 - hq, 0), min(h1 - hq, p.Hk), norm.eps, inv_d, units_log2);
  }
  unit.turn.template rows<false, true>((const T*)c.V + (int64_t)token * c.vt, c.vh, (T*)c.Vc + slot, p.sh, max(h0 - hq - p.Hk, 0), min(h1 - hq - p.Hk, p.Hk));
}

// The gradients.  Workgroups 0 .. blocks[0] - 1 have Q's items, the others K's; an item is NT / (d / 16) tokens and `per` heads.
struct NormItems { int blocks[2]; int64_t items[2]; int groups[2], per[2]; };   // groups: of heads

template <typename T, Pairing P>
__global__ __launch_bounds__(NT, P == kHalvesAny ? 2 : 3) void norm_rotary_bwd_kernel(const NormBwdCall c, const NormItems w, const int units_log2) {
  typedef typename Vec<T>::x8 T8;
  const int i = (int)blockIdx.x < w.blocks[0] ? 0 : 1;
  const int block = (int)blockIdx.x - (i == 0 ? 0 : w.blocks[0]);
  const NormGrad& t = c.t[i];
  const int units = 1 << units_log2, tokens = NT >> units_log2;
  const int u = (int)threadIdx.x & (units - 1);
  const float inv_d = 1.f / (float)c.d;
  NormUnit<T, P> unit;
  unit.turn.columns(c.rot, u);
  if constexpr (P == kHalvesAny) unit.turn.angles(c.rot, u, 0);   // (the partners)
  unit.weights(c.norm.w[i], c.norm.w_fp32);
  float dw[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) dw[e] = 0.f;
  for (int64_t item = block; item < w.items[i]; item += w.blocks[i]) {
    const int64_t tb = item / w.groups[i];
    const int h0 = (int)(item - tb * w.groups[i]) * w.per[i], h1 = min(t.H, h0 + w.per[i]);
    const int64_t token = tb * tokens + ((int)threadIdx.x >> units_log2);
    if (token >= (int64_t)c.B * c.N) continue;
    const int b = (int)(token / c.N), n = (int)(token - (int64_t)b * c.N);
    unit.turn.angles(c.rot, u, c.positions ? c.positions[b * c.position_sb + n] : n);
    const T* const x = (const T*)t.x + b * t.xb + n * t.xn;
    const T* const g = (const T*)t.dy + b * t.gb + n * t.gn;
    T* const y = (T*)t.dx + b * t.yb + n * t.yn;
    // one row is worked on while the next one is on its way
    auto load = [&](int h, T8 (&v)[4]) {
      v[0] = *(const T8*)(x + h * t.xh + unit.turn.lo);
      v[1] = *(const T8*)(x + h * t.xh + unit.turn.hi);
      v[2] = *(const T8*)(g + h * t.gh + unit.turn.lo);
      v[3] = *(const T8*)(g + h * t.gh + unit.turn.hi);
    };
    T8 next[4];
    load(h0, next);
    for (int h = h0; h < h1; ++h) {
      T8 now[4] = {next[0], next[1], next[2], next[3]};
      if (h + 1 < h1) load(h + 1, next);
      float v[16], gv[16], other[P == kHalvesAny ? 16 : 1] = {}, ss = 0.f, hx = 0.f;
      unit.widen(now[0], now[1], v);
      unit.widen(now[2], now[3], gv);
      if constexpr (P == kHalvesAny) {
#pragma unroll
        for (int e = 0; e < 16; ++e) other[e] = (float)g[h * t.gh + unit.turn.partner[e]];
      }
      unit.apply(gv, other);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ss += v[e] * v[e];
        hx += gv[e] * unit.w[e] * v[e];
      }
      const float r = 1.f / sqrtf(row_sum(ss, units_log2) * inv_d + c.norm.eps);
      if (__builtin_expect(r == 0.f, 0)) {
        // Squares beyond 32 bits: the forward pass made zeros of a finite row, and it has no gradient.  (Its products with h may be infinities, 0 times which would be in dx and in all rows' dw.)  What
        // is infinite in x itself becomes NaN here, and all of dx with it.
        hx = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          v[e] *= r;
          hx += gv[e] * unit.w[e] * v[e];
        }
      }
      const float back = row_sum(hx, units_log2) * inv_d * r * r;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        dw[e] += gv[e] * v[e] * r;
        gv[e] = r * (gv[e] * unit.w[e] - v[e] * back);
      }
      unit.narrow(gv, now[0], now[1]);
      *(T8*)(y + h * t.yh + unit.turn.lo) = now[0];
      *(T8*)(y + h * t.yh + unit.turn.hi) = now[1];
    }
  }
  if (t.dw == nullptr) return;
  // the workgroup's sum: thread rows of 16 columns in LDS, then NT / d (or so) threads a column
  __shared__ __attribute__((aligned(16))) float sums[NT * 16];
#pragma unroll
  for (int e4 = 0; e4 < 4; ++e4) {
    const f32x4 v = {dw[4 * e4], dw[4 * e4 + 1], dw[4 * e4 + 2], dw[4 * e4 + 3]};
    *(f32x4*)(sums + 16 * (int)threadIdx.x + 4 * e4) = v;
  }
  __syncthreads();
  // column `col` of the d = 16 units that a token's threads have, and every `parts`-th token of the workgroup from `part` on
  const int d = 16 << units_log2, col = (int)threadIdx.x & (d - 1), part = (int)threadIdx.x >> (4 + units_log2), parts = NT >> (4 + units_log2);
  float s = 0.f;
  for (int k = part; k < tokens; k += parts) s += sums[k * d + col];
  __syncthreads();
  sums[(int)threadIdx.x] = s;
  __syncthreads();
  if ((int)threadIdx.x < d) {
    for (int k = 1; k < parts; ++k) s += sums[k * d + col];
    Turn<T, P> owner;
    owner.columns(c.rot, col >> 4);
    const int e = col & 15;
    c.partial[(int64_t)blockIdx.x * c.d + (e < 8 ? owner.lo + e : owner.hi + e - 8)] = s;
  }
}

// The weights' gradient: blockIdx.x is 16 columns, blockIdx.y the tensor.  64 rows of 16 threads take the workgroups' sums in turn and meet in LDS.
template <typename T>
__global__ __launch_bounds__(1024) void norm_weights_kernel(const NormBwdCall c, const NormItems w) {
  __shared__ float sums[64][17];
  const int i = blockIdx.y;
  if (c.t[i].dw == nullptr) return;
  const int row = (int)threadIdx.x >> 4, lane = threadIdx.x & 15, col = 16 * (int)blockIdx.x + lane;
  const float* const part = c.partial + (i == 0 ? 0 : (int64_t)w.blocks[0] * c.d) + col;
  float s = 0.f;
#pragma unroll 8
  for (int k = row; k < w.blocks[i]; k += 64) s += part[(int64_t)k * c.d];
  sums[row][lane] = s;
  __syncthreads();
  for (int n = 32; n > 0; n >>= 1) {
    if (row < n) sums[row][lane] += sums[row + n][lane];
    __syncthreads();
  }
  if (row == 0) {
    if (c.norm.w_fp32) ((float*)c.t[i].dw)[col] = sums[0][lane];
    else ((T*)c.t[i].dw)[col] = (T)sums[0][lane];
  }
}

template <typename T, Pairing P> int launch_norm_p(const NormCall& c, hipStream_t s) {
  const RotaryCall& r = c.rotary;
  const int units_log2 = log2_units(r.d), tokens = NT >> units_log2;
  const int64_t n = (int64_t)r.B * r.N;
  const int heads = r.t[0].H + (r.n_tensors > 1 ? r.t[1].H : 0), per = heads_per_thread(n << units_log2, heads);
  hipLaunchKernelGGL((norm_rotary_kernel<T, P>), dim3((unsigned)((n + tokens - 1) / tokens), (unsigned)((heads + per - 1) / per)), dim3(NT), 0, s, c, units_log2, per);
  return (int)hipGetLastError();
}
template <typename T, Pairing P> int launch_norm_append_p(const AppendCall& c, const NormArgs& norm, hipStream_t s) {
  const int units_log2 = log2_units(c.d), tokens = NT >> units_log2;
  const int heads = (c.Q ? c.b.Hq : 0) + 2 * c.b.Hk, per = heads_per_thread((int64_t)c.b.T << units_log2, heads);
  hipLaunchKernelGGL((norm_append_kernel<T, P>), dim3((unsigned)((c.b.T + tokens - 1) / tokens), (unsigned)((heads + per - 1) / per)), dim3(NT), 0, s, c, norm, units_log2, per);
  return (int)hipGetLastError();
}
template <typename T, Pairing P> int launch_norm_bwd_p(const NormBwdCall& c, hipStream_t s) {
  const int units_log2 = log2_units(c.d), tokens = NT >> units_log2;
  const int64_t n = (int64_t)c.B * c.N, token_blocks = (n + tokens - 1) / tokens;
  NormItems w = {};
  for (int i = 0; i < c.n_tensors; ++i) {
    w.per[i] = std::min(c.t[i].H, heads_per_thread(n << units_log2, c.t[i].H));
    w.groups[i] = (c.t[i].H + w.per[i] - 1) / w.per[i];
    w.items[i] = token_blocks * w.groups[i];
  }
  const int64_t all = w.items[0] + w.items[1];
  if (all <= kNormBlocks) {
    w.blocks[0] = (int)w.items[0];
    w.blocks[1] = (int)w.items[1];
  } else if (c.n_tensors == 1) {
    w.blocks[0] = kNormBlocks;
  } else {
    w.blocks[0] = (int)std::min<int64_t>(std::max<int64_t>((int64_t)((double)w.items[0] / (double)all * kNormBlocks + 0.5), 1), kNormBlocks - 1);
    w.blocks[1] = kNormBlocks - w.blocks[0];
  }
  hipLaunchKernelGGL((norm_rotary_bwd_kernel<T, P>), dim3((unsigned)(w.blocks[0] + w.blocks[1])), dim3(NT), 0, s, c, w, units_log2);
  const int e = (int)hipGetLastError();
  if (e != 0 || (c.t[0].dw == nullptr && c.t[1].dw == nullptr)) return e;
  hipLaunchKernelGGL((norm_weights_kernel<T>), dim3((unsigned)(c.d / 16), (unsigned)c.n_tensors), dim3(1024), 0, s, c, w);
  return (int)hipGetLastError();
}

// the launcher for a type and a way to pair columns
#define ATTN_BY_PAIRING(ROT, CALL)                                    \
  (pairing_of(ROT) == kHalves ? CALL(kHalves) : pairing_of(ROT) == kNeighbours ? CALL(kNeighbours) : CALL(kHalvesAny))

}  // namespace

int launch_norm_rotary(const NormCall& c, int dtype, hipStream_t s) {
#define ATTN_CALL(P) (dtype == ATTN_FP16 ? launch_norm_p<_Float16, P>(c, s) : launch_norm_p<__bf16, P>(c, s))
  return ATTN_BY_PAIRING(c.rotary.rot, ATTN_CALL);
#undef ATTN_CALL
}
int launch_norm_append(const AppendCall& c, const NormArgs& norm, int dtype, hipStream_t s) {
#define ATTN_CALL(P) (dtype == ATTN_FP16 ? launch_norm_append_p<_Float16, P>(c, norm, s) : launch_norm_append_p<__bf16, P>(c, norm, s))
  return ATTN_BY_PAIRING(c.rot, ATTN_CALL);
#undef ATTN_CALL
}
int launch_norm_rotary_bwd(const NormBwdCall& c, int dtype, hipStream_t s) {
#define ATTN_CALL(P) (dtype == ATTN_FP16 ? launch_norm_bwd_p<_Float16, P>(c, s) : launch_norm_bwd_p<__bf16, P>(c, s))
  return ATTN_BY_PAIRING(c.rot, ATTN_CALL);
#undef ATTN_CALL
}

}  // namespace attn
