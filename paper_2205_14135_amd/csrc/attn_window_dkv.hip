// dK and dV of attention with a sliding window and first tokens that stay visible, gfx950.
//
// Arithmetic and register layout are those of attn_bwd_dkv_fr128.hip (lane = key; one wavefront does all four tile products of its 32 keys).
// A block of 128 keys is swept by the (window + 128) / QT tiles of queries from the diagonal on, whatever the length.  What is left are the pairs of a sink and a query a window or more
// behind it: few keys and many queries.  Either the blocks that hold sinks are swept by all queries (WindowArgs::swept_through), or workgroups in front of the others take 32 keys and a
// stretch of the queries each, their four wavefronts every fourth tile of it, in buffers of their own (window_plan says which).
// Then wavefronts whose 32 keys hold sinks leave dV^T and dK^T of either part in the workspace, in 32 bits, and window_join_kernel adds the pieces up in their order and rounds once: no
// atomics, the same bits every time.
// (The stretches in a launch of their own: us of the backward pass with four sinks 16 x 1024, window 256, d = 64 35.4 -> 25.6, 16 x 4096, 1024, d = 128 147 -> 131, 16 x 2048, 512 75 -> 58;
// 16 x 16384, 1024, whose other blocks fill the chip four times exactly, the same.)
// One MI355X, bf16: 16 heads x 16384, d = 128, window 1024, four sinks 290 us and the join 7.5 (920 TFLOP/s of the visible pairs' four products, matrix units busy in 50 per cent of the cycles);
// 128 heads x 1024, d = 64, window 256, swept through, 40 us.
// P and dS are rounded to 16 bits, half a step each, for their products with dO and Q, as in the dense kernels: dK and dV are no further off than dQ (attn_window.hip).
// Vector registers: d = 128 keeps the V rows in LDS (as there) and 32 queries to a tile, d <= 64 both operands in registers and 64 queries.
// (At d = 128 four registers go through scratch memory, 20 bytes a lane.)
#include "attn_window.h"

#include <type_traits>

#include "attn_tiles.h"

namespace attn {
namespace {

// A piece: dV^T, then dK^T, 16 bytes a lane at a time.
template <int D> __device__ __forceinline__ f32x4* window_piece(const WindowArgs& w, int bh, int block, int index) {
  return (f32x4*)(w.part + (((int64_t)bh * w.sink_blocks + block) * (1 + w.segments) + index) * (2 * 32 * D));
}

// What a workgroup of either kind has in LDS, one block, so that every address is a per-lane register plus an immediate: for each group of wavefronts row statistics and tiles of Q and dO, in
// BUFS buffers, and at d = 128 the V rows of the keys.
template <typename T, int D, bool SINKS> struct DkvShape {
  static constexpr int QT = window_query_tile(D), RW = SINKS ? 1 : 4, KG = SINKS ? 4 : 1, BUFS = SINKS ? 1 : 2, BR = 32 * RW;
  static constexpr int kVecBytes = 2 * BUFS * 64 * 4, kGroupBytes = kVecBytes + 2 * BUFS * QT * D * (int)sizeof(T);
  static constexpr int kBytes = KG * kGroupBytes + (D == 128 ? BR * D * (int)sizeof(T) : 0);
};

// SINKS: a block of 32 keys and a stretch of queries, else a block of 128 keys.  number: of the workgroup among those of its kind.
template <typename T, int D, bool DROPOUT, bool SINKS>
__device__ __forceinline__ void window_dkv_block(const WindowArgs& w, unsigned char* const all, uint32_t* const keep_table, const int number) {
  typedef typename Vec<T>::x8 T8;
  typedef DkvShape<T, D, SINKS> Shape;
  constexpr int KK = D / 16, DB = D / 32, QT = Shape::QT, QB = QT / 32, RW = Shape::RW, KG = Shape::KG, BUFS = Shape::BUFS, BR = Shape::BR;
  constexpr bool V_IN_LDS = D == 128;
  const KArgs& a = w.k;
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = KG == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  unsigned char* const smem = all + group * Shape::kGroupBytes;
  float* const Ls0 = (float*)smem;                 // base-2 row statistic, 64 a buffer
  float* const Ds0 = Ls0 + BUFS * 64;              // -D_i
  T* const Qs0 = (T*)(smem + Shape::kVecBytes);
  T* const Gs0 = Qs0 + BUFS * QT * D;
  T* const Vb = (T*)(all + KG * Shape::kGroupBytes);
  KeepLK keep;
  if constexpr (DROPOUT) keep.init(keep_table, a.drop_thr);

  // The heads are dealt round the XCDs.  The blocks of an XCD's heads come in their order, the first of all of them first: they may be swept through, and neighbours read the same queries.
  const int place = number / kXcds, heads = a.chunk;   // heads of an XCD, rounded up
  const int bh = place % heads * kXcds + number % kXcds;
  if (bh >= a.B * a.H) return;
  const int kt = SINKS ? place / heads / w.segments : place / heads, segment = SINKS ? place / heads % w.segments : 0;
  const int b = bh / a.H, h = bh % a.H;
  const int64_t head_off = (int64_t)b * a.sb + (int64_t)h * a.sh;
  const T* __restrict__ Qg = (const T*)a.Q + head_off;
  const T* __restrict__ Gg = (const T*)a.dO + head_off;
  const T* __restrict__ Vg = (const T*)a.V + head_off;
  const float* __restrict__ Lg = a.L2vec + (int64_t)bh * a.Nr;
  const float* __restrict__ Dg = a.Dvec + (int64_t)bh * a.Nr;
  const int lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5;
  const int kb0 = kt * BR, kw0 = kb0 + wave * 32, kj = kw0 + r;

  // (what stands at padded positions is not read, as in the forward pass: the last row that is none stands for it)
  const int len = a.klen ? min(max(a.klen[b], 0), a.N) : a.N;
  T8 kf[KK], vf[V_IN_LDS ? 1 : KK];
  {
    const int64_t row_off = head_off + (int64_t)min(kj, max(len - 1, 0)) * a.sn;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (D == 32 && 16 * kk + 8 * g >= a.dvalid) {   // head dimension 16: the upper columns are zeros
#pragma unroll
        for (int e = 0; e < 8; ++e) { kf[kk][e] = (T)0.f; if constexpr (!V_IN_LDS) vf[kk][e] = (T)0.f; }
        continue;
      }
      kf[kk] = *(const T8*)((const T*)a.K + row_off + 16 * kk + 8 * g);
      if constexpr (!V_IN_LDS) vf[kk] = *(const T8*)((const T*)a.V + row_off + 16 * kk + 8 * g);
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): before any asynchronous copy is in flight
  f32x16 dv[DB], dk[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) { dv[db][i] = 0.f; dk[db][i] = 0.f; }

  // Tiles of queries first .. limit - 1
  int first, limit = (len + QT - 1) / QT;
  if constexpr (SINKS) {
    first = max(segment * w.segment_tiles, (kb0 + w.window) / QT);
    limit = min(limit, (segment + 1) * w.segment_tiles);
  } else {
    first = kb0 / QT;
    if (!(w.swept_through && kb0 < w.sinks)) limit = min((int64_t)limit, ((int64_t)kb0 + BR - 1 + w.window - 1) / QT + 1);
  }
  const bool to_the_end = !SINKS && w.swept_through && kw0 < w.sinks;   // of this wavefront's keys
  if (kb0 >= len) limit = 0;

  TrOffsets<D> tro;
  tro.init();
  TileAsync<T, D, RW, QT> dma;
  dma.init(a.sn, wave, D == 32 ? a.dvalid : D);
  if (D == 32 && a.dvalid < D) {   // the copies leave columns >= 16 of the tile buffers untouched
    zero_tiles((T*)all, KG * Shape::kGroupBytes / (int)sizeof(T));
    __syncthreads();
  }
  auto fetch_tile = [&](int t, int buf) {
    dma.copy_rows(Qg, a.sn, t * QT, len, Qs0 + buf * QT * D);
    dma.copy_rows(Gg, a.sn, t * QT, len, Gs0 + buf * QT * D);
    const int row = min(t * QT + lane, a.Nr - 1);   // whole-wavefront copies: 64 floats, clamped to the head
    if (wave == (RW - 1) / 2) async_copy_b32(Lg + row, __builtin_amdgcn_readfirstlane(lds_addr(Ls0 + 64 * buf)));
    if (wave == RW / 2) async_copy_b32(Dg + row, __builtin_amdgcn_readfirstlane(lds_addr(Ds0 + 64 * buf)));
  };
  const float c = a.scale_log2;
  if constexpr (V_IN_LDS) {   // (rows >= len repeat the last one; their keys are masked)
    constexpr int VR = BR < 64 ? BR : 64;
    TileAsync<T, D, RW, VR> dma_v;
    dma_v.init(a.sn, wave);
    if (group == 0) {
      if (kb0 < len) dma_v.copy_rows(Vg, a.sn, kb0, len, Vb);
      if constexpr (BR > 64) {
        if (kb0 + 64 < len) dma_v.copy_rows(Vg, a.sn, kb0 + 64, len, Vb + 64 * D);
        else if (kb0 < len) dma_v.copy_rows(Vg, a.sn, kb0, len, Vb + 64 * D);   // all of these keys are masked
      }
    }
  }
  if (!SINKS && first < limit) fetch_tile(first, 0);
  wait_async_copies();
  __syncthreads();

  // the first and the last query of the pairs of this lane's key
  int first_query = kj < len ? kj : 0x7fffffff, last_query = kj + w.window - 1;
  if constexpr (SINKS) {
    first_query = kj < len && kj < w.sinks ? kj + w.window : 0x7fffffff;
    last_query = 0x7fffffff;
  }
  if (to_the_end && kj < w.sinks) last_query = 0x7fffffff;
  const bool short_of_keys = kw0 + 32 > len || (SINKS && kw0 + 32 > w.sinks);
  auto products = [&](int t, auto buf_c) __attribute__((always_inline)) {
    constexpr int buf = decltype(buf_c)::value;
    const int i0 = t * QT;
    // (rows of the workgroup's tiles that this wavefront's keys have no pair with)
    if ((SINKS || (i0 + QT > kw0 && (to_the_end || i0 <= kw0 + 31 + w.window - 1)))) {
      const T* Qt = Qs0 + buf * QT * D;
      const T* Gt = Gs0 + buf * QT * D;
      f32x16 s[QB], dp[QB];
      {   // S = Q K^T and dP = dO V^T, alternating; dP starts from -D
        auto qfrag = [&](int f) { return *(const T8*)(Qt + lds_off<D>(32 * (f % QB) + r, 2 * (f / QB) + g)); };   // f = QB kk + qb
        auto gfrag = [&](int f) { return *(const T8*)(Gt + lds_off<D>(32 * (f % QB) + r, 2 * (f / QB) + g)); };
        auto vfrag = [&](int kk) {
          if constexpr (V_IN_LDS) return *(const T8*)(Vb + lds_off<D>(wave * 32 + r, 2 * kk + g));
          else return vf[kk];
        };
        constexpr int PF2 = 2;
        T8 rq[PF2], rg[PF2], rv[PF2];
#pragma unroll
        for (int f = 0; f < PF2; ++f) { rq[f] = qfrag(f); rg[f] = gfrag(f); if constexpr (V_IN_LDS) rv[f] = vfrag(f); }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            f32x4 c4 = {0.f, 0.f, 0.f, 0.f};   // (with dropout -D joins after the mask)
            if constexpr (!DROPOUT) c4 = *(const f32x4*)(Ds0 + 64 * buf + 32 * qb + 8 * i4 + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) { dp[qb][4 * i4 + e] = c4[e]; s[qb][4 * i4 + e] = 0.f; }
          }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < QB * KK; ++f) {
          const T8 cq = rq[f % PF2], cg = rg[f % PF2];
          T8 cv;
          if constexpr (V_IN_LDS) cv = rv[f % PF2]; else cv = vf[f / QB];
          s[f % QB] = mfma32(cq, kf[f / QB], s[f % QB]);
          dp[f % QB] = mfma32(cg, cv, dp[f % QB]);
          if (f + PF2 < QB * KK) { rq[f % PF2] = qfrag(f + PF2); rg[f % PF2] = gfrag(f + PF2); if constexpr (V_IN_LDS) rv[f % PF2] = vfrag(f + PF2); }
          __builtin_amdgcn_sched_barrier(0);
        }
        static_assert(!V_IN_LDS || QB == 1, "the V fragments are read one an MFMA");
      }
      // hidden pairs get the logit -inf, hence P = 0: tiles that an edge crosses, and keys that are none
      if (short_of_keys || (SINKS ? i0 < kw0 + 31 + w.window : i0 < kw0 + 31 || i0 + QT > kw0 + w.window)) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int q = i0 + 32 * qb + 8 * (i >> 2) + 4 * g + (i & 3);
            if (q < first_query || q > last_query) s[qb][i] = -INFINITY;
          }
      }
      uint32_t kept = 0;   // dropout: the keep flags of this lane's key for the tile's queries it holds
      if constexpr (DROPOUT) kept = keep.draw<QB>(i0, kw0, bh, a.offset_lo, a.seed_lo, a.seed_hi);
      T8 pf[2 * QB], dsf[2 * QB];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const f32x4 l4 = *(const f32x4*)(Ls0 + 64 * buf + 32 * qb + 8 * i4 + 4 * g);
          f32x4 d4 = {0.f, 0.f, 0.f, 0.f};
          if constexpr (DROPOUT) d4 = *(const f32x4*)(Ds0 + 64 * buf + 32 * qb + 8 * i4 + 4 * g);   // -D_i
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * i4 + e, cc = 2 * qb + (i4 >> 1), at = 4 * (i4 & 1) + e;
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qb][i], c, -l4[e]));
            if constexpr (DROPOUT) {
              const uint32_t mask = KeepLK::mask(kept, QB == 1 ? 1 : qb, i4, e);
              pf[cc][at] = (T)keep_or_zero(p, mask);
              dsf[cc][at] = (T)(p * dropped_dp_minus_d(dp[qb][i], a.keep_scale, mask, d4[e]));
            } else {
              pf[cc][at] = (T)p;
              dsf[cc][at] = (T)(p * dp[qb][i]);
            }
          }
        }
      {   // dV^T += dO^T P and dK^T += Q^T dS, alternating
        auto tr = [&](const T* tile, int f) {   // f = DB cc + db
          const T* base = tile + 16 * (f / DB) * D;
          return tr_frag<T8>(base + tro.off[f % DB][0], base + tro.off[f % DB][1]);
        };
        constexpr int PF2 = 2, NF = 2 * QB * DB;
        T8 rg[PF2], rq[PF2];
#pragma unroll
        for (int f = 0; f < PF2; ++f) { rg[f] = tr(Gt, f); rq[f] = tr(Qt, f); }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const T8 cg = rg[f % PF2], cq = rq[f % PF2];
          dv[f % DB] = mfma32(cg, pf[f / DB], dv[f % DB]);
          dk[f % DB] = mfma32(cq, dsf[f / DB], dk[f % DB]);
          if (f + PF2 < NF) { rg[f % PF2] = tr(Gt, f + PF2); rq[f % PF2] = tr(Qt, f + PF2); }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  const std::integral_constant<int, 0> buf0;
  const std::integral_constant<int, 1> buf1;
  if constexpr (SINKS) {   // (buffers of the wavefront's own: no barriers; other workgroups fill its waits)
    for (int t = first + group; t < limit; t += KG) {
      fetch_tile(t, 0);
      wait_async_copies();
      products(t, buf0);
    }
  } else {
    auto step = [&](int t, auto buf_c) __attribute__((always_inline)) {
      if (t + 1 < limit) fetch_tile(t + 1, decltype(buf_c)::value ^ 1);
      products(t, buf_c);
      wait_async_copies();
      __syncthreads();
    };
    for (int t = first; t < limit; t += 2) {
      step(t, buf0);
      if (t + 1 < limit) step(t + 1, buf1);
    }
  }

  if constexpr (SINKS) {
    // the groups but the first leave dV, then dK in the buffers, and the first one adds them up
    f32x4* const part = (f32x4*)all + lane;
    static_assert(3 * 4 * DB * 64 * 16 <= Shape::kBytes, "LDS holds one gradient of the groups");
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      f32x16 (&x)[DB] = which == 0 ? dv : dk;
      __syncthreads();
      if (group > 0) {
#pragma unroll
        for (int f = 0; f < 4 * DB; ++f) {
          const int i = 4 * (f % 4);
          const f32x4 v = {x[f / 4][i], x[f / 4][i + 1], x[f / 4][i + 2], x[f / 4][i + 3]};
          part[((group - 1) * 4 * DB + f) * 64] = v;
        }
      }
      __syncthreads();
      if (group == 0) {
#pragma unroll
        for (int k = 0; k < KG - 1; ++k)
#pragma unroll
          for (int f = 0; f < 4 * DB; ++f) {
            const f32x4 v = part[(k * 4 * DB + f) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[f / 4][4 * (f % 4) + e] += v[e];
          }
      }
    }
    if (group > 0) return;
  }
  if (SINKS || (w.sink_blocks > 0 && kw0 < w.sinks)) {   // a piece (the same for all lanes: a sink among the 32 keys)
    f32x4* const piece = window_piece<D>(w, bh, SINKS ? kt : kw0 / 32, SINKS ? 1 + segment : 0) + lane;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const f32x16 (&x)[DB] = which == 0 ? dv : dk;
#pragma unroll
      for (int f = 0; f < 4 * DB; ++f) {
        const int i = 4 * (f % 4);
        const f32x4 v = {x[f / 4][i], x[f / 4][i + 1], x[f / 4][i + 2], x[f / 4][i + 3]};
        piece[(which * 4 * DB + f) * 64] = v;
      }
    }
    return;
  }
  if constexpr (!SINKS) {
    // (the loop ended on a barrier: the tile buffers stage the output rows)
    static_assert(4 * 32 * D <= 2 * BUFS * QT * D, "room for a gradient's rows");
    T* const stage = Qs0 + wave * 32 * D;
    store_rows_coalesced<T, D>(stage, (T*)a.dV + head_off + (int64_t)kw0 * a.sn, a.sn, dv, DROPOUT ? a.keep_scale : 1.f, a.N - kw0, D == 32 ? a.dvalid : D);
    __builtin_amdgcn_wave_barrier();
    store_rows_coalesced<T, D>(stage, (T*)a.dK + head_off + (int64_t)kw0 * a.sn, a.sn, dk, a.tau, a.N - kw0, D == 32 ? a.dvalid : D);
  }
}

// The first `sink_groups` workgroups (a multiple of the XCDs) take the sinks' stretches, so that their waits for memory fall into the others' products.
template <typename T, int D, bool DROPOUT>
__global__ __launch_bounds__(256, 2) void window_dkv_kernel(const WindowArgs w, const int sink_groups) {
  constexpr int kBytes = DkvShape<T, D, true>::kBytes > DkvShape<T, D, false>::kBytes ? DkvShape<T, D, true>::kBytes : DkvShape<T, D, false>::kBytes;
  __shared__ __attribute__((aligned(16))) unsigned char all[kBytes];
  __shared__ __attribute__((aligned(16))) uint32_t keep_table[DROPOUT ? KeepLK::kTable : 4];
  if ((int)blockIdx.x < sink_groups) window_dkv_block<T, D, DROPOUT, true>(w, all, keep_table, (int)blockIdx.x);
  else window_dkv_block<T, D, DROPOUT, false>(w, all, keep_table, (int)blockIdx.x - sink_groups);
}

// blockIdx.x: a head's block of 32 keys with sinks; blockIdx.y: 32 columns of dV (the first D / 32) or of dK, a wavefront each.  Four pieces are on their way at a time.  (All columns of
// a gradient by one wavefront, a piece at a time: 16 heads of 16384 tokens, d = 128, eight pieces 41 us.)
template <typename T, int D>
__global__ __launch_bounds__(64) void window_join_kernel(const WindowArgs w, const float v_scale) {
  constexpr int DB = D / 32, NP = 4;
  __shared__ __attribute__((aligned(16))) T stage[32 * 32];
  const KArgs& a = w.k;
  const int lane = threadIdx.x;
  const int bh = (int)blockIdx.x / w.sink_blocks, block = (int)blockIdx.x % w.sink_blocks, which = (int)blockIdx.y / DB, db = (int)blockIdx.y % DB;
  const f32x4* const piece = window_piece<D>(w, bh, block, 0) + (which * DB + db) * 256 + lane;
  f32x4 sum[4] = {};
  for (int k0 = 0; k0 <= w.segments; k0 += NP) {
    f32x4 v[NP][4];
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) v[k][i4] = piece[(int64_t)min(k0 + k, w.segments) * (2 * 4 * DB * 64) + i4 * 64];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      if (k0 + k > w.segments) break;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) sum[i4] += v[k][i4];
    }
  }
  f32x16 x[1];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[0][i] = sum[i / 4][i % 4];
  const int b = bh / a.H, h = bh % a.H;
  const int64_t row0 = (int64_t)b * a.sb + (int64_t)h * a.sh + (int64_t)32 * block * a.sn + 32 * db;
  store_rows_coalesced<T, 32>(stage, (T*)(which == 0 ? a.dV : a.dK) + row0, a.sn, x, which == 0 ? v_scale : a.tau, a.N - 32 * block, D == 32 ? a.dvalid : 32);
}

template <typename T, int D, bool DROPOUT> int launch(WindowArgs a, hipStream_t s) {
  KArgs& k = a.k;
  const int heads = k.B * k.H;
  k.chunk = (heads + kXcds - 1) / kXcds;
  const int sink_groups = kXcds * k.chunk * a.sink_blocks * a.segments;
  hipLaunchKernelGGL((window_dkv_kernel<T, D, DROPOUT>), dim3(sink_groups + kXcds * k.chunk * k.T), dim3(256), 0, s, a, sink_groups);
  const int e = (int)hipGetLastError();
  if (e != 0 || a.sink_blocks == 0) return e;
  hipLaunchKernelGGL((window_join_kernel<T, D>), dim3(heads * a.sink_blocks, 2 * (D / 32)), dim3(64), 0, s, a, DROPOUT ? k.keep_scale : 1.f);
  return (int)hipGetLastError();
}
template <typename T, int D> int launch_d(const WindowArgs& a, bool dropout, hipStream_t s) { return dropout ? launch<T, D, true>(a, s) : launch<T, D, false>(a, s); }
template <typename T> int launch_t(const WindowArgs& a, int d, bool dropout, hipStream_t s) {
  if (d == 32) return launch_d<T, 32>(a, dropout, s);
  if (d == 64) return launch_d<T, 64>(a, dropout, s);
  return launch_d<T, 128>(a, dropout, s);
}

}  // namespace

int launch_window_dkv(const WindowArgs& a, int dtype, int d, bool dropout, hipStream_t s) {
  return dtype == 0 ? launch_t<_Float16>(a, d, dropout, s) : launch_t<__bf16>(a, d, dropout, s);
}

}  // namespace attn
