// Internal declarations of attention with a sliding window and first tokens that stay visible ("sinks"): key j is visible to query i iff j <= i and (i - j < window or j < sinks).
#pragma once
#include "attn_common.h"

namespace attn {

struct WindowArgs {
  KArgs k;
  int window, sinks;   // 1 .. N and 0 .. N - 1
  // Gradients of the sinks: pieces of 32 keys, a head's `sink_blocks` times (1 + segments), each dV^T and dK^T in 32 bits in the layout of the accumulators
  // (window_piece).  The first is of the queries less than a window behind, the others divide those behind them.
  float* part;
  int sink_blocks, segments, segment_tiles;
  int swept_through;   // != 0: instead, blocks of 128 keys that hold sinks are swept by all queries from the diagonal on, in the one launch (sink_blocks is 0 then)
};

// Whether the window hides anything at all: if not, the dense causal kernels take the call.
inline bool window_hides(int N, int window, int sinks) { return (int64_t)window + sinks < N; }

// Rows of a tile of queries in the dK/dV kernels.
constexpr int window_query_tile(int d) { return d == 128 ? 32 : 64; }
constexpr size_t window_piece_floats(int d) { return (size_t)2 * 32 * (d <= 32 ? 32 : d); }
// How the gradients of the sinks are made.  Blocks of keys that hold sinks are swept by the queries behind the window too where that takes no longer than the launch: they come first, two
// workgroups to a compute unit.  Else those queries are divided in stretches, which four wavefronts each take the tiles of in turn: about 128 in all where heads and sinks are few, of at least 16 tiles, and of no more than
// the other blocks of keys leave time for (a stretch's tile takes a quarter of twice as long as theirs).  There is one at least for every head and 32 sinks, so that with many sinks
// time and workspace grow with them: stretches, us of the backward pass and MB, 16 x 16384, d = 128, window 1024, 4 | 256 | 1024 sinks 128, 520, 6.8 | 256, 620, 14.7 | 1024, 930, 52; window 128, 8000 sinks 4000, 2840, 264.
// us of the backward pass with four sinks, stretches of 32 tiles | swept through, heads x N, window, tiles behind it, tiles of the launch's longest unit: d = 64 16 x 1024, 256, 12 of 2 25.6 | 38.3;
// 128 x 1024, 256, 12 of 12 82.0 | 80.2; 64 x 2048, 256, 28 of 12 78.2 | 97.3; 300 x 300, 150, 3 of 7 56.5 | 50.9; d = 128 16 x 4096, 1024, 96 of 36 135 | 223; 210 x 333, 200, 5 of 12 85.8 | 70.6;
// 64 x 16384, 1024, 480 of 576 2053 | 2040; 1 x 16384, 1024, 480 of 9 154 | 600.  Stretches of 16 | 32 | 64: d = 64 4 x 2048, 128 22.4 | 28.1 | 27.9; d = 32 8 x 8192, 100 28.1 | 30.1 | 39.8,
// 60 x 3000, 300, 40 sinks 77.1 | 78.8 | 75.8; d = 128 16 x 16384, 1024 553 | 534 | 527.
inline void window_plan(WindowArgs& a, int d) {
  const int qt = window_query_tile(d);
  a.sink_blocks = a.segments = a.segment_tiles = a.swept_through = 0;
  if (a.sinks == 0) return;
  const int64_t tiles = ((int64_t)a.k.N + qt - 1) / qt, heads = (int64_t)a.k.B * a.k.H, behind = tiles - a.window / qt, own = (a.window + 128) / qt;
  const int64_t unit = heads * a.k.T * own / (2 * kComputeUnits);   // tiles that a compute unit's two workgroups take one after the other
  if (behind * 2 * kComputeUnits <= heads * a.k.T * own) {
    a.swept_through = 1;
    return;
  }
  a.sink_blocks = (a.sinks + 31) / 32;
  int64_t stretch = tiles * heads * a.sink_blocks / 128;
  if (stretch > 2 * unit && stretch > 64) stretch = 2 * unit > 64 ? 2 * unit : 64;
  if (stretch < 16) stretch = 16;
  // (no more pieces than two workgroups a compute unit and one a block: the workspace stays linear in the sinks and the heads)
  int64_t n = (tiles + stretch / 2) / stretch;
  const int64_t most = 2 * kComputeUnits / (heads * a.sink_blocks) + 1;
  if (n > most) n = most;
  if (n < 1) n = 1;
  a.segment_tiles = (int)((tiles + n - 1) / n);
  a.segments = (int)((tiles + a.segment_tiles - 1) / a.segment_tiles);
}
inline size_t window_part_bytes(const WindowArgs& a, int d) {
  return (size_t)a.k.B * a.k.H * a.sink_blocks * (1 + a.segments) * window_piece_floats(d) * sizeof(float);
}

int launch_window_fwd(const WindowArgs& a, int dtype, int d, bool dropout, hipStream_t s);
int launch_window_dkv(const WindowArgs& a, int dtype, int d, bool dropout, hipStream_t s);   // attn_window_dkv.hip
int launch_window_bwd(const WindowArgs& a, int dtype, int d, bool dropout, hipStream_t s);

}  // namespace attn
