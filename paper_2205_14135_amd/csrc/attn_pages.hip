// Copies of pages of a key/value cache, in all its layers and in K and V, gfx950: what a fork of a sequence (its last, partly filled page) and a compaction ask
// for.  Memory bounds it: 8 bytes a cached column.  The page numbers travel in the kernel's arguments: the list is the caller's host memory,
// nothing is uploaded, and a captured graph holds its own copy.
#include "attn_paged.h"

#include <algorithm>
#include <cstring>

namespace attn {
namespace {

constexpr int NT = 256;
constexpr int kPairs = 480;   // of a launch: 3840 bytes of the 4096 that a kernel's arguments may take

struct Pairs { int src[kPairs], dst[kPairs]; };

// blockIdx.x: a run of 16-byte pieces of one page of one tensor; .y: pair; .z: layer, K or V.  A page is rows of head h, row n; `pieces` of a row
template <bool PACKED>
__global__ __launch_bounds__(NT) void copy_kernel(const CopyCall c, const Pairs pairs, const int row_log2, const int page_log2, const int total) {
  const int z = (int)blockIdx.z;
  char* const base = (char*)(z & 1 ? c.Vc : c.Kc) + 2 * (z >> 1) * c.sl;
  const char* const src = base + 2 * pairs.src[blockIdx.y] * c.sp;
  char* const dst = base + 2 * pairs.dst[blockIdx.y] * c.sp;
  const int i0 = (int)blockIdx.x * (4 * NT) + (int)threadIdx.x;
  u32x4 v[4];
  int64_t off[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = i0 + k * NT;
    if (PACKED) {
      off[k] = 16 * (int64_t)i;
    } else {
      const int row = i >> row_log2, head = row >> page_log2;
      off[k] = 2 * (head * c.sh + (row & ((1 << page_log2) - 1)) * c.sn) + 16 * (i & ((1 << row_log2) - 1));
    }
    if (i < total) v[k] = *(const u32x4*)(src + off[k]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (i0 + k * NT < total) *(u32x4*)(dst + off[k]) = v[k];
}

int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

}  // namespace

int launch_page_copy(const CopyCall& c, const int* pairs, int64_t n_pairs, hipStream_t s) {
  const int row_log2 = log2_of(c.d / 8), page_log2 = log2_of(c.page_size);
  const int total = c.Hk << (page_log2 + row_log2);
  const bool packed = c.sn == c.d && c.sh == (int64_t)c.page_size * c.d;
  for (int64_t at = 0; at < n_pairs; at += kPairs) {
    const int n = (int)std::min<int64_t>(kPairs, n_pairs - at);
    Pairs list;
    for (int i = 0; i < n; ++i) {
      list.src[i] = pairs[2 * (at + i)];
      list.dst[i] = pairs[2 * (at + i) + 1];
    }
    for (int i = n; i < kPairs; ++i) list.src[i] = list.dst[i] = 0;
    const dim3 grid((unsigned)((total + 4 * NT - 1) / (4 * NT)), (unsigned)n, (unsigned)(2 * c.layers));
    if (packed) hipLaunchKernelGGL((copy_kernel<true>), grid, dim3(NT), 0, s, c, list, row_log2, page_log2, total);
    else hipLaunchKernelGGL((copy_kernel<false>), grid, dim3(NT), 0, s, c, list, row_log2, page_log2, total);
    const int e = (int)hipGetLastError();
    if (e != 0) return e;
  }
  return 0;
}

}  // namespace attn
