// Device code of the paged key-value cache (gfx950): page copies, entries of its table, rows between a context and pages.
#pragma once
#include "river_pages.h"

namespace river {
namespace pg {

constexpr int kPairs = 448;               // of a launch: they travel as kernel arguments (below 4 KiB)
struct Pairs { int src[kPairs], dst[kPairs]; };

// One workgroup per 16 KiB of a page, four 16-byte pieces a thread in flight; grid (pieces, pairs, layers x {k, v}).  Bound: memory
// (200 pages of 2 MiB over 32 layers, 839 MB read and written, 148 .. 157 us, 5.3 .. 5.7 TB/s; a large copy reaches 5.0).
constexpr int kCopyPiece = 16384;
__global__ __launch_bounds__(256) void k_copy_pages(char *k, char *v, long long page_bytes, long long layer_bytes, long long used, Pairs w) {
  char *base = (blockIdx.z & 1 ? v : k) + (blockIdx.z >> 1) * layer_bytes;
  const char *src = base + w.src[blockIdx.y] * page_bytes;
  char *dst = base + w.dst[blockIdx.y] * page_bytes;
  const long long at = (long long)blockIdx.x * kCopyPiece + threadIdx.x * 16;
#pragma unroll
  for (int i = 0; i < kCopyPiece / 4096; ++i)
    if (at + i * 4096 < used) *(u32x4 *)(dst + at + i * 4096) = *(const u32x4 *)(src + at + i * 4096);
}

__global__ void k_set_entries(int *state, int n, Pairs w) {        // state[src[i]] = dst[i]
  for (int i = threadIdx.x; i < n; i += blockDim.x) state[w.src[i]] = w.dst[i];
}
__global__ void k_clear_state(int *state, int max_seqs, long long n) {     // no positions, no pages
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x)
    state[i] = i < max_seqs ? 0 : -1;
}

// A context's cache rows [position][head][HD] <-> pages [head][slot][HD], 16 bytes a thread; grid (rows' pieces, layers).
__global__ __launch_bounds__(256) void k_move_rows(Cache c, const int *row, int max_pages, long long layer_stride_bytes, char *kc, char *vc,
                                                   long long ctx_layer_bytes, int head_bytes, int first, int n, int to_pages) {
  const int per_head = head_bytes / 16, per_row = c.n_kv_heads * per_head;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)n * per_row) return;
  const int p = first + (int)(i / per_row), r = (int)(i % per_row), h = r / per_head, e = r % per_head;
  const int at = c.by_page.quot(p);
  if (at >= max_pages) return;
  const int page = row[at], slot = p - at * c.page_size;
  if ((unsigned)page >= (unsigned)c.n_pages) return;
  const long long in_page = (long long)blockIdx.y * layer_stride_bytes + page * c.page_stride +
                            ((long long)h * c.page_size + slot) * head_bytes + e * 16;
  const long long in_ctx = (long long)blockIdx.y * ctx_layer_bytes + (long long)p * per_row * 16 + r * 16;
  u32x4 *pk = (u32x4 *)((char *)c.k + in_page), *pv = (u32x4 *)((char *)c.v + in_page);
  u32x4 *xk = (u32x4 *)(kc + in_ctx), *xv = (u32x4 *)(vc + in_ctx);
  if (to_pages) { *pk = *xk; *pv = *xv; }
  else { *xk = *pk; *xv = *pv; }
}

}  // namespace pg
}  // namespace river
