// Forward pass and dQ of attention with a sliding window and first tokens that stay visible, gfx950.
//
// Key j is visible to query i iff j <= i and (i - j < window or j < sinks).  The arithmetic is that of the causal kernels (attn_fwd.hip, attn_bwd.hip); a block of 128 rows sweeps the
// tiles of 64 keys that hold sinks and those from the first one that its first row's window reaches to the diagonal: (window + 128) / 64 + 1 of them and the sinks', whatever the length.  Blocks cost
// the same but for the first of a head, which come last (16 x 16384, window 8192, d = 128: forward 847 -> 790 us, backward pass 2440 -> 2368; narrower windows the same); neighbours go to the same XCD, whose L2 has loaded
// most of their keys already.
// Masks are looked at in the tiles that the edges cross only, the diagonal, the window's far edge and the last sink; wavefronts whose 32 rows see nothing of a tile skip it.
//   One MI355X, bf16, operations of the visible pairs: 16 heads x 16384, d = 128, window 1024 and four sinks forward 175 us (765 TFLOP/s; 19 tiles are swept for 16 of pairs: 930 of what is executed), dQ 235 (855); the
// matrix and vector units bound it, matrix units busy in 41 and 47 per cent of the cycles.  128 heads x 1024, d = 64, window 256: 26 and 40 us: a block has 7 tiles, and what it waits for at its start and its end, and 16
// exponentials a lane to an MFMA, are most of it; HBM bytes (67 and 102 MB) take 12 and 19.
//   With dropout (of probability 0.1) forward and backward pass take 206 and 612 us instead of 174 and 520, and 34 and 93 instead of 26 and 76; 5 x 12 x 1000, d = 32, window 300, padded, 15.3 and 41 instead of 13.0 and 30.
#include "attn_window.h"

#include "attn_tiles.h"

namespace attn {
namespace {

constexpr int TILE = 64;   // keys

// The tiles of a block of rows r0 .. r0 + BR - 1, in order: those of the sinks, then those of the window.  len: keys that there are.
struct WindowTiles {
  int at, sink_end, first, limit;
  template <int BR> __device__ __forceinline__ void init(const WindowArgs& a, int r0, int len) {
    const int lo = max(r0 - a.window + 1, 0);   // the first key in reach
    first = lo / TILE;
    limit = r0 >= len ? 0 : (min(r0 + BR, len) + TILE - 1) / TILE;
    sink_end = min((a.sinks + TILE - 1) / TILE, first);
    at = sink_end > 0 ? 0 : first;
    if (limit == 0) at = 0;
  }
  __device__ __forceinline__ int next() {   // -1: no more
    if (at >= limit) return -1;
    const int t = at++;
    if (at == sink_end) at = first;
    return t;
  }
  // The next GROUPS tiles, one for each group of wavefronts; own: that of `group`, -1 past the end.  False once there is none for any.
  template <int GROUPS> __device__ __forceinline__ bool next_of(int group, int& own) {
    own = next();
    const bool any = own >= 0;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) {
      const int t = next();
      if (group == k) own = t;
    }
    return any;
  }
};
// Whether rows q0 .. q0 + 31 see any of the tile's keys from k0 on.
__device__ __forceinline__ bool wave_sees(const WindowArgs& a, int k0, int q0) { return k0 <= q0 + 31 && (q0 - k0 < a.window + TILE - 1 || k0 < a.sinks); }
// The far edge: keys that lie a window or more before the row and are no sinks.  (The near one and the length are the caller's.)
__device__ __forceinline__ void hide_far(const WindowArgs& a, f32x16 (&s)[2], int k0, int q0, int qi, int g) {
  if (q0 + 31 - k0 >= a.window && k0 + TILE > a.sinks) {
    const int first = qi - a.window + 1;   // of the row's window
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + 32 * kb + 8 * (i >> 2) + 4 * g + (i & 3);
        if (key < first && key >= a.sinks) s[kb][i] = -INFINITY;
      }
  }
}

// Probabilities are rounded to 16 bits for their product with V and O is divided by the sum of the rounded ones, as in the dense forward; maxima, sums and O are in 32 bits until the one rounding at the end.
// RW wavefronts of 32 rows share the tiles of a workgroup, and KG groups of them work on the same rows, group k on every KG-th tile, in buffers of its own; their (m, l, O) are merged
// through LDS at the end, as in attn_fwd.hip.
// PER_UNIT: workgroups, of four wavefronts, that a compute unit is to hold.
template <typename T, int D, bool DROPOUT, int RW, int KG, int PER_UNIT>
__global__ __launch_bounds__(64 * RW * KG, PER_UNIT) void window_fwd_kernel(const WindowArgs w) {
  typedef typename Vec<T>::x8 T8;
  constexpr int KK = D / 16, DB = D / 32, BR = 32 * RW, PF = 4;
  typedef T Tile[TILE * D];
  __shared__ __attribute__((aligned(16))) Tile bufs[4 * KG];
  Tile* const Ks = bufs;            // buffers 2 k and 2 k + 1: group k's
  Tile* const Vs = bufs + 2 * KG;
  const KArgs& a = w.k;
  args_at_once(a);
  const int item = xcd_item(a.n_items, a.chunk);
  if (item < 0) return;
  const int n_qt = (a.N + BR - 1) / BR;
  const int bh = dealt_head(a, item / n_qt), qt = n_qt - 1 - item % n_qt;
  const int b = bh / a.H, h = bh % a.H;
  const int64_t head_off = (int64_t)b * a.sb + (int64_t)h * a.sh;
  const T* __restrict__ Qg = (const T*)a.Q + head_off;
  const T* __restrict__ Kg = (const T*)a.K + head_off;
  const T* __restrict__ Vg = (const T*)a.V + head_off;
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / RW;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - RW * group;
  const int r = lane & 31, g = lane >> 5;
  const int q0 = qt * BR + wave * 32;
  const bool row_ok = q0 + r < a.N;   // (lanes beyond a ragged end work on a copy of the last row and store nothing)
  const int qi = min(q0 + r, a.N - 1);
  // What stands at padded positions is not read: the last row that is none stands for it, so that nothing but finite numbers meets the weights 0.
  const int len = a.klen ? min(max(a.klen[b], 0), a.N) : a.N;
  const int q_row = min(qi, max(len - 1, 0));

  T8 qf[KK];   // Q^T fragments (B operand): query qi, d = 16 kk + 8 g .. +7
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    if (D == 32 && 16 * kk + 8 * g >= a.dvalid) {   // head dimension 16: the upper columns are zeros
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[kk][e] = (T)0.f;
    } else {
      qf[kk] = *(const T8*)(Qg + (int64_t)q_row * a.sn + 16 * kk + 8 * g);
    }
  }
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  f32x4 lr_run = {0.f, 0.f, 0.f, 0.f};
  int calm = kFirstTile;
  const T8 ones = row_sum_ones<T>();

  WindowTiles it;
  it.init<BR>(w, qt * BR, len);
  TrOffsets<D> tro;
  tro.init();
  TileAsync<T, D, RW> dma;
  dma.init(a.sn, wave, D == 32 ? a.dvalid : D);
  if (D == 32 && a.dvalid < D) {   // the copies leave columns >= 16 of the tile buffers untouched
    zero_tiles(&bufs[0][0], 4 * KG * TILE * D);
    __syncthreads();
  }
  const float c = a.scale_log2;
  int jt, buf = 0;   // this group's tile, -1 if there is none; more: some group (then the first) has one
  bool more = it.next_of<KG>(group, jt);
  if (jt >= 0) {
    dma.copy_rows(Kg, a.sn, jt * TILE, len, Ks[2 * group]);
    dma.copy_rows(Vg, a.sn, jt * TILE, len, Vs[2 * group]);
  }
  wait_async_copies();
  __syncthreads();   // the first tile has landed, and so have the Q fragments
  asm volatile("" ::"s"(c));
  uint32_t k_off[KK];   // byte offsets of this lane's K fragments in a tile, kept whole
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    k_off[kk] = lds_addr(&Ks[2 * group][0]) + (uint32_t)(lds_off<D>(r, 2 * kk + g) * sizeof(T));
    asm volatile("" : "+v"(k_off[kk]));
  }
  while (KG == 1 ? jt >= 0 : more) {
    int jn;
    const bool more_next = it.next_of<KG>(group, jn);
    if (jn >= 0) {   // the next tile streams into the other buffer while this one is used
      dma.copy_rows(Kg, a.sn, jn * TILE, len, Ks[2 * group + (buf ^ 1)]);
      dma.copy_rows(Vg, a.sn, jn * TILE, len, Vs[2 * group + (buf ^ 1)]);
    }
    const T* Vt = Vs[2 * group + buf];
    const int k0 = jt * TILE;
    if ((KG == 1 || jt >= 0) && wave_sees(w, k0, q0)) {
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
      {   // S^T = K Q^T; operand reads run PF fragments ahead of their MFMA
        auto k_frag = [&](int f) {   // f = 2 kk + kb
          const auto* p = (const __attribute__((address_space(3))) T8*)(k_off[f >> 1] + (uint32_t)(buf * TILE * D * sizeof(T)));
          return p[32 * (f & 1) * D / 8];
        };
        T8 ring[PF];
#pragma unroll
        for (int f = 0; f < PF; ++f) ring[f] = k_frag(f);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < 2 * KK; ++f) {
          const T8 cur = ring[f % PF];
          s[f & 1] = mfma32(cur, qf[f >> 1], s[f & 1]);
          if (f + PF < 2 * KK) ring[f % PF] = k_frag(f + PF);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      hide_far(w, s, k0, q0, qi, g);
      T8 pf[4];
      softmax_tile_lane_query<T, DB, true, DROPOUT, D == 128>(a, s, o, pf, m_run, l_run, lr_run, calm, ones, c, k0, q0, qi, len, g, bh);
      {   // O^T += V^T P^T
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
    jt = jn;
    more = more_next;
    buf ^= 1;
  }
  if constexpr (KG > 1) {
    // (the loop ended on a barrier) the groups but the first leave O in the tile buffers from the first one on; the last two take the output rows
    constexpr int kLanes = 64 * RW;
    static_assert((KG - 1) * RW + 2 <= 4 * KG && RW <= 4 && sizeof(Tile) == 4 * D * 32, "LDS holds the groups' O and the output rows");
    __shared__ float sums[(KG - 1) * 3 * kLanes];   // references and row sums
    f32x4* const o_part = (f32x4*)Ks + (group - 1) * (4 * DB * kLanes) + wave * 64 + lane;
    float* const s_part = sums + (group - 1) * 3 * kLanes + wave * 64 + lane;
    if (group > 0) {
#pragma unroll
      for (int f = 0; f < 4 * DB; ++f) {
        const int i = 4 * (f % 4);
        const f32x4 v = {o[f / 4][i], o[f / 4][i + 1], o[f / 4][i + 2], o[f / 4][i + 3]};
        o_part[f * kLanes] = v;
      }
      s_part[0] = m_run;
      s_part[kLanes] = l_run;
      s_part[2 * kLanes] = lr_run[0];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 1; k < KG; ++k) {
      const float* const sp = s_part + k * 3 * kLanes;
      const f32x4* const op = o_part + k * (4 * DB * kLanes);
      const float mk = sp[0], m = fmaxf(m_run, mk), ref = m == -INFINITY ? 0.f : m;
      const float w0 = __builtin_amdgcn_exp2f(m_run - ref), w1 = __builtin_amdgcn_exp2f(mk - ref);
      m_run = m;
      l_run = l_run * w0 + sp[kLanes] * w1;
      lr_run[0] = lr_run[0] * w0 + sp[2 * kLanes] * w1;
#pragma unroll
      for (int f = 0; f < 4 * DB; ++f) {
        const f32x4 v = op[f * kLanes];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[f / 4][4 * (f % 4) + e] = o[f / 4][4 * (f % 4) + e] * w0 + v[e] * w1;
      }
    }
  }

  const float l_sum = l_run + xchg32(l_run);
  const float lr_sum = lr_run[0];
  const float l_tot = qi < len ? l_sum : 0.f;   // padding rows: O = 0, LSE = -inf
  const float inv = (l_tot > 0.f && lr_sum > 0.f) ? (DROPOUT ? a.keep_scale : 1.f) / lr_sum : (l_tot == l_tot ? 0.f : l_tot);   // (a row of NaN stays one)
  if (g == 0 && row_ok)
    a.LSE[(int64_t)bh * a.N + qi] = l_tot > 0.f ? (m_run + __builtin_amdgcn_logf(l_tot)) * 0.6931471805599453f : -INFINITY;
  if (a.o_fp32) {
    float* Og = (float*)a.O + head_off + (int64_t)qi * a.sn;
    if (row_ok) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = o[db][4 * i4 + e] * inv;
          if (D != 32 || 8 * i4 + 4 * g < a.dvalid) *(f32x4*)(Og + 32 * db + 8 * i4 + 4 * g) = v;
        }
    }
  } else {   // through the (now idle) tile buffers
    T* stage = KG > 1 ? &Vs[2 * KG - 2][0] + wave * 32 * D : &bufs[0][0] + wave * 32 * D;
    store_rows_coalesced<T, D>(stage, (T*)a.O + head_off + (int64_t)q0 * a.sn, a.sn, o, inv, a.N - q0, D == 32 ? a.dvalid : D);
  }
}

// dQ, and -D and the row statistic in base 2 for the dK/dV kernels, as in attn_bwd.hip.
// S, dP, P and the sums are in 32 bits; dS is rounded to 16, half a step each, for its product with K, because the matrix unit takes 16-bit operands: dQ, itself rounded once, is off by 0.0025 of its norm in bf16 and 0.0003 in fp16,
// where 32-bit arithmetic rounded once is off by 0.0017 and 0.0002.  (What the rounding drops as a second operand: a third more matrix products here for that factor of 1.5; the dense kernels round as this one does.)
template <typename T, int D, bool DROPOUT, int RW, int KG>
__global__ __launch_bounds__(64 * RW * KG, 2) void window_dq_kernel(const WindowArgs w) {
  typedef typename Vec<T>::x8 T8;
  constexpr int KK = D / 16, DB = D / 32, BR = 32 * RW, PF = 4;
  __shared__ __attribute__((aligned(16))) T all[KG * 4 * TILE * D];
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / RW;
  T* const Ks = all + group * 4 * TILE * D;   // K tile of buffer b at b TILE D, V tile at (2 + b) TILE D
  T* const Vs = Ks + 2 * TILE * D;
  const KArgs& a = w.k;
  args_at_once(a);
  const int item = xcd_item(a.n_items, a.chunk);
  if (item < 0) return;
  const int n_qt = a.T * (4 / RW);   // blocks of BR rows, to the end of the last 128-row block: the scratch vectors are written whole
  const int bh = dealt_head(a, item / n_qt), qt = n_qt - 1 - item % n_qt;
  const int b = bh / a.H, h = bh % a.H;
  const int64_t head_off = (int64_t)b * a.sb + (int64_t)h * a.sh;
  const T* __restrict__ Kg = (const T*)a.K + head_off;
  const T* __restrict__ Vg = (const T*)a.V + head_off;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - RW * group;
  const int r = lane & 31, g = lane >> 5;
  const int q0 = qt * BR + wave * 32;
  const bool row_ok = q0 + r < a.N;
  const int qi = min(q0 + r, a.N - 1);
  const int len = a.klen ? min(max(a.klen[b], 0), a.N) : a.N;
  const int q_row = min(qi, max(len - 1, 0));   // (as in the forward pass)

  T8 qf[KK], gf[KK];   // Q^T and dO^T fragments of this lane's query
  float d_part = 0.f;
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    const int64_t off = head_off + (int64_t)q_row * a.sn + 16 * kk + 8 * g;
    if (D == 32 && 16 * kk + 8 * g >= a.dvalid) {
#pragma unroll
      for (int e = 0; e < 8; ++e) { qf[kk][e] = (T)0.f; gf[kk][e] = (T)0.f; }
      continue;
    }
    qf[kk] = *(const T8*)((const T*)a.Q + off);
    gf[kk] = *(const T8*)((const T*)a.dO + off);
    if (a.o_fp32) {
      const f32x4 o0 = *(const f32x4*)((const float*)a.O + off);
      const f32x4 o1 = *(const f32x4*)((const float*)a.O + off + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) d_part += (float)gf[kk][e] * o0[e] + (float)gf[kk][4 + e] * o1[e];
    } else {
      const T8 o = *(const T8*)((const T*)a.O + off);
#pragma unroll
      for (int e = 0; e < 8; ++e) d_part += (float)gf[kk][e] * (float)o[e];
    }
  }
  const float lse = a.LSE[(int64_t)bh * a.N + qi];
  const float l2 = (lse == -INFINITY || !row_ok) ? INFINITY : lse * 1.4426950408889634f;
  const float neg_d = row_ok ? -(d_part + xchg32(d_part)) : 0.f;   // -D_i
  if (g == 0 && group == 0) {   // (the scratch is padded to whole blocks: this workgroup writes all of its block)
    a.Dvec[(int64_t)bh * a.Nr + q0 + r] = neg_d;
    a.L2vec[(int64_t)bh * a.Nr + q0 + r] = l2;
  }
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) dq[db][i] = 0.f;

  WindowTiles it;
  it.init<BR>(w, qt * BR, len);
  TrOffsets<D> tro;
  tro.init();
  TileAsync<T, D, RW> dma;
  dma.init(a.sn, wave, D == 32 ? a.dvalid : D);
  if (D == 32 && a.dvalid < D) {
    zero_tiles(all, KG * 4 * TILE * D);
    __syncthreads();
  }
  const float c = a.scale_log2;
  int jt, buf = 0;
  bool more = it.next_of<KG>(group, jt);
  if (jt >= 0) {
    dma.copy_rows(Kg, a.sn, jt * TILE, len, Ks);
    dma.copy_rows(Vg, a.sn, jt * TILE, len, Vs);
  }
  wait_async_copies();
  __syncthreads();
  while (KG == 1 ? jt >= 0 : more) {
    int jn;
    const bool more_next = it.next_of<KG>(group, jn);
    if (jn >= 0) {
      dma.copy_rows(Kg, a.sn, jn * TILE, len, Ks + (buf ^ 1) * TILE * D);
      dma.copy_rows(Vg, a.sn, jn * TILE, len, Vs + (buf ^ 1) * TILE * D);
    }
    const T* Kt = Ks + buf * TILE * D;
    const T* Vt = Vs + buf * TILE * D;
    const int k0 = jt * TILE;
    if ((KG == 1 || jt >= 0) && wave_sees(w, k0, q0)) {
      f32x16 s[2], dp[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kb][i] = 0.f;
          dp[kb][i] = DROPOUT ? 0.f : neg_d;   // without dropout the product starts from -D and ends as dP - D
        }
      // S^T = K Q^T and dP^T = V dO^T as one stream
      auto kv_frag = [&](int f) {   // f = 4 kk + 2 kb + (0: K, 1: V)
        const int off = lds_off<D>(32 * ((f >> 1) & 1) + r, 2 * (f >> 2) + g);
        return *(const T8*)(((f & 1) ? Vt : Kt) + off);
      };
      {
        T8 ring[PF];
#pragma unroll
        for (int f = 0; f < PF; ++f) ring[f] = kv_frag(f);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < 4 * KK; ++f) {
          const T8 cur = ring[f % PF];
          const int kk = f >> 2, kb = (f >> 1) & 1;
          if (f & 1) dp[kb] = mfma32(cur, gf[kk], dp[kb]);
          else s[kb] = mfma32(cur, qf[kk], s[kb]);
          if (f + PF < 4 * KK) ring[f % PF] = kv_frag(f + PF);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      hide_far(w, s, k0, q0, qi, g);
      if (k0 + TILE - 1 > q0 || k0 + TILE > len) {
        const int last = min(qi, len - 1);   // last visible key of this row
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (k0 + 32 * kb + 8 * (i >> 2) + 4 * g + (i & 3) > last) s[kb][i] = -INFINITY;
      }
      KeepLQ kq = {};
      if constexpr (DROPOUT) kq = keep_tile_lane_query(k0, qi, bh, g, a.offset_lo, a.seed_lo, a.seed_hi);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * i4 + e;
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], c, -l2));
            float dpv = dp[kb][i];
            if constexpr (DROPOUT) dpv = dropped(kq.w[kb][i4], e, a.drop_thr) ? neg_d : __builtin_fmaf(dpv, a.keep_scale, neg_d);
            s[kb][i] = p * dpv;
          }
      T8 dsf[4];
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
#pragma unroll
        for (int t = 0; t < 8; ++t) dsf[cc][t] = (T)s[cc >> 1][8 * (cc & 1) + t];
      auto kt_frag = [&](int f) {   // f = DB cc + db
        const T* base = Kt + 16 * (f / DB) * D;
        return tr_frag<T8>(base + tro.off[f % DB][0], base + tro.off[f % DB][1]);
      };
      {   // dQ^T += K^T dS^T
        T8 ring[PF];
#pragma unroll
        for (int f = 0; f < PF; ++f) ring[f] = kt_frag(f);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < 4 * DB; ++f) {
          const T8 cur = ring[f % PF];
          dq[f % DB] = mfma32(cur, dsf[f / DB], dq[f % DB]);
          if (f + PF < 4 * DB) ring[f % PF] = kt_frag(f + PF);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    wait_async_copies();
    __syncthreads();
    jt = jn;
    more = more_next;
    buf ^= 1;
  }
  if constexpr (KG > 1) {
    // (the loop ended on a barrier) the groups but the first leave their dQ in the tile buffers
    constexpr int kLanes = 64 * RW;
    static_assert((KG - 1) * DB * 16 * kLanes * 4 <= KG * 4 * TILE * D * (int)sizeof(T), "LDS holds the groups' dQ");
    f32x4* const part = (f32x4*)all + wave * 64 + lane;
    if (group > 0) {
#pragma unroll
      for (int f = 0; f < 4 * DB; ++f) {
        const int i = 4 * (f % 4);
        const f32x4 v = {dq[f / 4][i], dq[f / 4][i + 1], dq[f / 4][i + 2], dq[f / 4][i + 3]};
        part[((group - 1) * 4 * DB + f) * kLanes] = v;
      }
    }
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int k = 0; k < KG - 1; ++k)
#pragma unroll
        for (int f = 0; f < 4 * DB; ++f) {
          const f32x4 v = part[(k * 4 * DB + f) * kLanes];
#pragma unroll
          for (int e = 0; e < 4; ++e) dq[f / 4][4 * (f % 4) + e] += v[e];
        }
    }
    __syncthreads();   // the buffers stage the output rows
    if (group > 0) return;
  }
  T* stage = all + wave * 32 * D;
  store_rows_coalesced<T, D>(stage, (T*)a.dQ + head_off + (int64_t)q0 * a.sn, a.sn, dq, a.tau, a.N - q0, D == 32 ? a.dvalid : D);
}

// The division of the forward and of dQ among wavefronts: with few blocks of rows, half as many rows to a block and two groups of wavefronts that take every other tile.
// us of calls in a replayed graph, without sinks, {4, 1} | {2, 2} (wavefronts of rows, groups), heads x N, window: forward d = 64 12 x 197, 64 7.2 | 5.1, 16 x 1024, 256 11.1 | 8.0, 8 x 4096, 512 15.8 | 12.9, 32 x 1024, 256 11.5 | 10.1,
// 48 x 1024, 256 15.1 | 15.7, 16 x 4096, 512 21.1 | 23.4; d = 128 1 x 16384, 1024 28.7 | 22.6, 16 x 1024, 256 13.9 | 11.7, 32 x 1024, 256 14.8 | 22.0; d = 32 60 x 1000, 300 14.4 | 11.8.
// Backward (dQ alone so): d = 64 8 x 4096, 512 35.2 | 33.3, 32 x 1024, 256 27.4 | 26.8, 48 x 1024, 256 35.9 | 38.9; d = 128 1 x 16384, 1024 142 | 134, 4 x 8192, 1024 112 | 122; d = 32 30 x 1000, 300
// 23.5 | 20.9, 60 x 1000, 300 30.2 | 31.7.
bool window_divided(const WindowArgs& a, int64_t compute_units_blocks) {
  const int64_t blocks64 = (int64_t)a.k.B * a.k.H * ((a.k.N + 63) / 64);
  return blocks64 <= compute_units_blocks * kComputeUnits;
}
// (d = 64 in 128 registers, four workgroups to a compute unit instead of three, where there are more blocks than three to each: two of them go through scratch memory, 12 bytes a lane, and it is faster all the same; with dropout, which needs more, it stays at three.  us, heads x N, window, blocks, three | four:
// 97 x 1024, 256, 776 25.8 | 22.7, 128 x 1024, 1024 28.5 | 26.4, 32 x 4096, 512, 1024 40.0 | 35.5, 128 x 2048, 1024, 2048 87.3 | 86.8, 300 x 1024, 128, 2400 42.8 | 40.8; 96 x 512, 100, 384 12.6 | 13.4, 64 x
// 1024, 256, 512 16.4 | 16.9.)
template <typename T, int D, int RW, int KG> int launch_fwd(WindowArgs a, bool dropout, hipStream_t s) {
  constexpr int PER = KG == 1 && D <= 64 ? 3 : 2;
  a.k.n_items = a.k.B * a.k.H * ((a.k.N + 32 * RW - 1) / (32 * RW));
  a.k.chunk = (a.k.n_items + kXcds - 1) / kXcds;
  const dim3 grid(kXcds * a.k.chunk), block(64 * RW * KG);
  if constexpr (D == 64 && KG == 1) {
    if (!dropout && a.k.n_items > PER * kComputeUnits) {
      hipLaunchKernelGGL((window_fwd_kernel<T, D, false, RW, KG, PER + 1>), grid, block, 0, s, a);
      return (int)hipGetLastError();
    }
  }
  if (dropout) hipLaunchKernelGGL((window_fwd_kernel<T, D, true, RW, KG, PER>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((window_fwd_kernel<T, D, false, RW, KG, PER>), grid, block, 0, s, a);
  return (int)hipGetLastError();
}
template <typename T, int D, int RW, int KG> int launch_dq(WindowArgs a, bool dropout, hipStream_t s) {
  a.k.n_items = a.k.B * a.k.H * a.k.T * (4 / RW);
  a.k.chunk = (a.k.n_items + kXcds - 1) / kXcds;
  const dim3 grid(kXcds * a.k.chunk), block(64 * RW * KG);
  if (dropout) hipLaunchKernelGGL((window_dq_kernel<T, D, true, RW, KG>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((window_dq_kernel<T, D, false, RW, KG>), grid, block, 0, s, a);
  return (int)hipGetLastError();
}
template <typename T, int D> int launch_fwd(const WindowArgs& a, bool dropout, hipStream_t s) {
  return window_divided(a, D == 128 ? 1 : (D == 64 ? 2 : 4)) ? launch_fwd<T, D, 2, 2>(a, dropout, s) : launch_fwd<T, D, 4, 1>(a, dropout, s);
}
template <typename T, int D> int launch_dq(const WindowArgs& a, bool dropout, hipStream_t s) {
  return window_divided(a, D == 128 ? 1 : 2) ? launch_dq<T, D, 2, 2>(a, dropout, s) : launch_dq<T, D, 4, 1>(a, dropout, s);
}

}  // namespace

int launch_window_fwd(const WindowArgs& a, int dtype, int d, bool dropout, hipStream_t s) {
  if (d == 32) return dtype == 0 ? launch_fwd<_Float16, 32>(a, dropout, s) : launch_fwd<__bf16, 32>(a, dropout, s);
  if (d == 64) return dtype == 0 ? launch_fwd<_Float16, 64>(a, dropout, s) : launch_fwd<__bf16, 64>(a, dropout, s);
  return dtype == 0 ? launch_fwd<_Float16, 128>(a, dropout, s) : launch_fwd<__bf16, 128>(a, dropout, s);
}
int launch_window_bwd(const WindowArgs& a, int dtype, int d, bool dropout, hipStream_t s) {
  int e;
  if (d == 32) e = dtype == 0 ? launch_dq<_Float16, 32>(a, dropout, s) : launch_dq<__bf16, 32>(a, dropout, s);
  else if (d == 64) e = dtype == 0 ? launch_dq<_Float16, 64>(a, dropout, s) : launch_dq<__bf16, 64>(a, dropout, s);
  else e = dtype == 0 ? launch_dq<_Float16, 128>(a, dropout, s) : launch_dq<__bf16, 128>(a, dropout, s);
  return e != 0 ? e : launch_window_dkv(a, dtype, d, dropout, s);
}

}  // namespace attn
