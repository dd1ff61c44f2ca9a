// Internal declarations of the operators over a paged key/value cache and of the rotary positions: the kernels' arguments and the launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/attn.h"
#include "attn_common.h"

namespace attn {

// The frequencies and how they pair the columns (attn_rotary_spec, checked).
struct RotaryArgs {
  const double* freq;   // [r / 2] radians a position, nullptr: nothing turns (r = 0)
  int r;                // columns that turn
  int interleaved;
  int inverse;
  float magnitude;
};

// One [B,H,N,d] tensor of a rotary call.
struct RotaryTensor {
  const void* x;
  void* y;
  int H;
  int64_t xb, xh, xn, yb, yh, yn;
};

struct RotaryCall {
  RotaryTensor t[2];
  int n_tensors;
  int B, N, d;
  RotaryArgs rot;
  const int* positions;   // nullptr: 0 .. N - 1
  int64_t position_sb;
};

// The norm of rows of Q and K (attn_norm_spec, checked).
struct NormArgs {
  const void* w[2];     // weights [d] of Q and of K
  int w_fp32;           // in 32 bits, else in the tensors' type
  float eps;
};
struct NormCall {
  RotaryCall rotary;    // rotary.rot.r = 0: nothing turns
  NormArgs norm;
};
// One tensor of its backward pass.
struct NormGrad {
  const void* x; const void* dy;
  void* dx;
  void* dw;             // nullptr: not asked for
  int H;
  int64_t xb, xh, xn, gb, gh, gn, yb, yh, yn;
};
struct NormBwdCall {
  NormGrad t[2];
  int n_tensors;
  int B, N, d;
  RotaryArgs rot;       // by the negative angle
  NormArgs norm;
  const int* positions;
  int64_t position_sb;
  float* partial;       // [workgroups][d]: their shares of the weights' gradients
};
// Workgroups of the backward pass at most: what the chip holds at three wavefronts a SIMD, so that each adds up the weights' gradient of many rows before it leaves a share.
// us, two wavefronts | three | four, with registers for as many: 8 x 1024 tokens of 16 + 16 heads of 64 24.7 | 22.3 | 31.0, 16384 of 16 + 4 of 128 60.7 | 54.5 | 84.6 (one row on its way).
constexpr int kNormBlocks = 768;
inline size_t norm_workspace_bytes(int d) { return (size_t)kNormBlocks * d * sizeof(float); }

// The sequences of a batch and their pages; see attn_paged_params.
struct PagedBatch {
  const int* table;
  const int* lengths;
  const int* starts;      // nullptr: token b is the one new token of sequence b
  int64_t table_stride;
  int B, T;
  int Hq, Hk;
  int pages, page_log2, width;
  int capacity;           // width << page_log2: tokens that a row of the table holds
  int64_t sp, sh, sn;     // strides of the caches: page, head, row
  uint32_t page_bytes, row_bytes, page_mask;   // sp and sn in bytes; rows of a page - 1
};

// The rows first .. end - 1 of a sequence, out of its starts as they are in memory: forced into 0 .. T, for the append and for the attention alike.
__device__ __forceinline__ void force_rows(const PagedBatch& b, int& first, int& end) {
  first = min(max(first, 0), b.T);
  end = min(max(end, first), b.T);
}

struct AppendCall {
  PagedBatch b;
  RotaryArgs rot;
  int d;
  const void* K; const void* V; const void* Q;
  void* Kc; void* Vc; void* Qo;
  int64_t kt, kh, vt, vh, qt, qh, ot, oh;
};

struct PagedCall {
  PagedBatch b;
  const void* Q; const void* K; const void* V;
  void* O;
  float* LSE;
  float* part;            // pieces of divided items
  int64_t qt, qh, ot, oh;
  int G;                  // Q heads to a K head
  uint32_t g_factor;      // n / G = n g_factor >> g_shift for 0 <= n < 2^31: g_factor = ceil(2^g_shift / G), g_shift = 31 + ceil(log2 G)
  int g_shift;
  int d;                  // of the tensors: 16 runs on the D = 32 kernels
  int causal;
  int slots;              // workgroups that share the work
  float scale_log2;       // tau * log2(e)
  double longest_line;    // no rising starts make more of the line (attn_paged_line.h) than this
  int window, sinks;      // a token sees the last `window` keys up to its own, and the first `sinks` (window 0: all up to its own)
  int only;               // with a window: 0 all sequences, 1 those of more than 32 rows, 2 the others
};

// How attn_paged_fwd runs: blocks of 32 rows, a wavefront each (attn_paged_one.hip), or of 128 or 256 (attn_paged_rows.hip), and the workgroups that share the work.
struct PagedShape { int rows, slots; };
int paged_one_slots(int d);
int paged_rows_slots(int d);
// rows of the larger blocks (attn_paged_rows.hip)
constexpr int paged_block_rows(int d) { return d == 128 ? 256 : 128; }
// Blocks of 32 rows where a sequence has no more on average (single tokens), or where all blocks together are few, so that their keys are divided over many workgroups:
// pieces of 32 rows are joined sooner than larger ones.  Else larger blocks use a tile of K and V four or eight times as often.  us, 32 rows | larger, with the join, sequences x new
// tokens on tokens before.  d = 128, 32 / 8 heads: 1 x 1 on 4000 17 | 22, on 30000 33 | 39, 256 x 1 on 100 40 | 56, 64 x 1 on 4000 195 | 188, 120 x 1 and 1 x 256 on 2000 211 | 245;
// 1 x 16 on 16000 (16 blocks of 32 rows) 35 | 33, 1 x 32 (32) 48 | 36, 1 x 128 (128) 138 | 59, 8 x 16 on 2000 (120) 36 | 24.  d = 64, 16 / 4 heads: 1 x 1 on 4000 11 | 17, on 30000 20 | 35;
// 1 x 32 on 16000 (16) 25 | 31, 1 x 64 on 2000 (32) 18 | 18, on 16000 28 | 33, 1 x 128 (64) 39 | 38, 8 x 16 on 2000 (92) 21 | 19, 32 x 32 on 2000 39 | 27.
inline PagedShape paged_shape(int64_t rows, int B, int Hk, int d) {
  if (rows <= (int64_t)32 * B || Hk * ((rows + 31) / 32 + B - 1) < 32) return {32, paged_one_slots(d)};
  return {paged_block_rows(d), paged_rows_slots(d)};
}
// With a window: whether sequences of at most 32 rows are worked on in launches of their own, by the kernel for single tokens, behind those of more.  In blocks of 256 rows (d = 128) a tile of one
// takes nearly as long as of a whole block, and the window, the heads and the batch say how many tiles there may be at most; two launches more are 8 to 12 us.  us, together | apart, 32 / 8 heads
// of 128, window: 8 single tokens and a chunk of 2048, 4096 214 | 192, 1024 76 | 72; 32 and 2048, 4096 289 | 262; 60 and 4 x 500, 512 83 | 72; two and 2 x 512, 8 / 8 heads, 4096 54 | 62; no single ones, 4 x 512 on 8000,
// 4096 162 | 167.  d = 64: 32 and a chunk of 1000, 16 / 4 heads, 1024 29 | 44.
inline bool paged_window_apart(const attn_paged_params& p, const PagedShape& shape, int window, int sinks) {
  const int64_t reach = (int64_t)window + sinks, capacity = (int64_t)p.table_width * p.page_size;
  return shape.rows == 256 && (int64_t)p.Hk * (p.B - 1) * (reach < capacity ? reach : capacity) >= 3000 * 64;
}
// With a window and one new token a sequence: a workgroup for each block of 32 rows, of wavefronts with three tiles of 32 keys of K and of V each, in one launch
// (attn_paged_few.hip): as many as LDS has room for at d >= 64, eight (of thirteen) at d <= 32.  Where a wavefront has up to 6 tiles, one more where the window's edges and the last sink cut some, or up to 12 and the workgroups are not so few that most of the device would idle, and up to 512 workgroups: more of them take turns on a
// compute unit, and a division by keys is evener.  us, divided with the join | this, sequences x K heads (workgroups), window.  d = 64: 1 x 2, 512 (3 tiles) 9.9 | 7.0, 1024 10.1 | 9.9, 2048 (11) 10.8 | 15.2;
// 64 x 2, 512 14.0 | 7.9, 2048 23.1 | 17.3; 256 x 2, 512 27.6 | 19.3, 2048 59 | 50; 1024 x 2, 512 80 | 67.  d = 128: 1 x 8, 256 (3) 13.7 | 9.9, 512 (6) 13.8 | 13.2, 1024 (11) 14.5 | 21.0; 16 x 8, 256 14.3 |
// 10.6, 1024 22.4 | 22.3; 33 x 8, 512 26.5 | 27.5; 64 x 8, 256 27.4 | 24.7, 512 35.6 | 33.0; 128 x 8, 512 58 | 62; 256 x 8, 256 71 | 83.  d = 32: 1 x 12, 2048 (8) 11.6 | 12.1; 20 x 12, 512 15.0 | 7.3, 2048 24.4 |
// 15.3; 200 x 12, 512 48 | 55.
constexpr int paged_few_waves(int d) { return d <= 32 ? 8 : (d == 64 ? 6 : 3); }
inline int64_t paged_few_items(const PagedCall& c) { return (int64_t)c.b.B * c.b.Hk * ((c.G + 31) / 32); }
inline bool paged_few(const PagedCall& c) {
  if (c.window == 0 || c.b.starts != nullptr) return false;
  const int64_t items = paged_few_items(c), reach = (int64_t)c.window + c.sinks, keys = reach < c.b.capacity ? reach : c.b.capacity;
  return items <= 512 && keys <= (int64_t)(items < 64 ? 6 : 12) * 32 * paged_few_waves(c.d);
}
// The number of slots and what to join at each of them (Join in attn_paged_line.h), then two pieces a slot: 32-bit rows of O and three statistics.  Room for either
// kernel, so that a workspace serves every call at its head dimension.
constexpr int kJoinBytes = 32;
inline size_t paged_part_bytes(const PagedShape& s, int d) {
  return (size_t)(s.slots + 1) * kJoinBytes + (size_t)2 * s.slots * s.rows * ((d <= 32 ? 32 : d) + 4) * sizeof(float);
}
inline size_t paged_workspace_bytes(int d) {
  const size_t one = paged_part_bytes({32, paged_one_slots(d)}, d), rows = paged_part_bytes({paged_block_rows(d), paged_rows_slots(d)}, d);
  return one > rows ? one : rows;
}

int launch_rotary(const RotaryCall& c, int dtype, hipStream_t s);
int launch_append(const AppendCall& c, int dtype, hipStream_t s);
int launch_norm_rotary(const NormCall& c, int dtype, hipStream_t s);
int launch_norm_append(const AppendCall& c, const NormArgs& norm, int dtype, hipStream_t s);
int launch_norm_rotary_bwd(const NormBwdCall& c, int dtype, hipStream_t s);
int launch_paged_one(const PagedCall& c, int dtype, hipStream_t s);
int launch_paged_few(const PagedCall& c, int dtype, hipStream_t s);
int launch_paged_rows(const PagedCall& c, int dtype, hipStream_t s);
// pairs: host memory, (source, destination) page numbers, checked by the caller; bytes of a row: d * 2.
struct CopyCall {
  void* Kc; void* Vc;
  int layers, Hk, page_size, d;
  int64_t sl, sp, sh, sn;
};
int launch_page_copy(const CopyCall& c, const int* pairs, int64_t n_pairs, hipStream_t s);

}  // namespace attn
