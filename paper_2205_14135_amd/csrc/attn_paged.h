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
int launch_paged_one(const PagedCall& c, int dtype, hipStream_t s);
int launch_paged_rows(const PagedCall& c, int dtype, hipStream_t s);
// pairs: host memory, (source, destination) page numbers, checked by the caller; bytes of a row: d * 2.
struct CopyCall {
  void* Kc; void* Vc;
  int layers, Hk, page_size, d;
  int64_t sl, sp, sh, sn;
};
int launch_page_copy(const CopyCall& c, const int* pairs, int64_t n_pairs, hipStream_t s);

}  // namespace attn
