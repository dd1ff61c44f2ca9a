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
};

// Whether the window hides anything at all: if not, the dense causal kernels take the call.
inline bool window_hides(int N, int window, int sinks) { return (int64_t)window + sinks < N; }

// Rows of a tile of queries in the dK/dV kernels.
constexpr int window_query_tile(int d) { return d == 128 ? 32 : 64; }
constexpr size_t window_piece_floats(int d) { return (size_t)2 * 32 * (d <= 32 ? 32 : d); }
// Blocks of 32 keys that hold sinks, and how the queries at a window's distance and more behind them are divided: stretches of four wavefronts that take as many tiles each as half
// of those that an ordinary block of keys is swept by, at least 4; fewer stretches where there are many sinks.
inline void window_plan(WindowArgs& a, int d) {
  const int qt = window_query_tile(d);
  a.sink_blocks = (a.sinks + 31) / 32;
  a.segments = 0;
  a.segment_tiles = 0;
  if (a.sink_blocks == 0) return;
  const int64_t tiles = ((int64_t)a.k.N + qt - 1) / qt, heads = (int64_t)a.k.B * a.k.H;
  const int64_t least = 32;
  int64_t n = (tiles + least - 1) / least;
  const int64_t most = 8 * kComputeUnits / (heads * a.sink_blocks) + 1;
  if (n > most) n = most;
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
