// What the paged cache's translation units share on the host side: errors, launches, checks of arguments.
#pragma once
#include <algorithm>
#include <atomic>
#include <cstdint>
#include <string>

#include "river_host.h"
#include "river_pages.h"

namespace river {
namespace pg {

inline int refuse(const char *why, int code = RIVER_EINVAL) {
  call_error() = why;
  return code;
}
inline int hip_failed(const char *what, hipError_t e) {
  call_error() = std::string(what) + ": " + hipGetErrorString(e);
  return RIVER_EHIP;
}
// Every entry point: no exception leaves the library (what is left to throw is memory that runs out).
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (...) {
    try { call_error() = "out of host memory"; } catch (...) {}
    return RIVER_ENOSPC;
  }
}
// The launch's own result (an error of the caller's that is pending stays his).
template <class T> struct As { typedef T type; };
template <class... A>
hipError_t launch(void (*k)(A...), dim3 grid, dim3 block, size_t lds, hipStream_t s, typename As<A>::type... a) {
  void *args[] = {(void *)&a...};
  return hipLaunchKernel((const void *)k, grid, block, args, lds, s);
}

// The same with more than 64 KiB of dynamic LDS, which each kernel asks for once per device.
template <auto K, class... A>
hipError_t launch_lds(dim3 grid, dim3 block, size_t lds, hipStream_t s, A... a) {
  static std::atomic<uint64_t> asked{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(asked.load(std::memory_order_relaxed) & bit)) {
    if ((e = hipFuncSetAttribute((const void *)K, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) != hipSuccess) return e;
    asked.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch(K, grid, block, lds, s, a...);
}

inline Div div_by(int d) {
  uint32_t s = 0;
  while ((1ll << s) < d) ++s;
  return Div{(uint32_t)d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
}
inline int elem_bytes(const river_pages *p) { return p->dtype == RIVER_F32 ? 4 : 2; }
inline long long page_elems(const river_pages *p) { return (long long)p->n_kv_heads * p->page_size * p->head_dim; }

// (a launch holds fewer than 2^32 threads in a dimension; a larger one would be cut off without an error)
constexpr int kMostTokens = 1 << 22;
constexpr int kMostPositions = 1 << 30;                          // of a sequence: indices of keys are 32-bit numbers

inline Cache layer_cache(const river_pages *p, int layer) {
  const size_t at = (size_t)layer * p->layer_stride * elem_bytes(p);
  return Cache{(char *)p->k + at, (char *)p->v + at, p->page_stride, (uint32_t)(p->page_stride * elem_bytes(p) / 16), p->n_pages, p->page_size, p->n_kv_heads, div_by(p->page_size)};
}

inline const char *bad_batch(const river_batch *b) {
  if (!b) return "null batch";
  if (b->n_seq < 0 || b->n_tokens < 0 || b->max_pages < 1 || b->table_stride < b->max_pages || b->max_new < 0 || b->max_len < 0)
    return "bad batch: n_seq, n_tokens, max_new, max_len >= 0, 1 <= max_pages <= table_stride";
  if (b->n_tokens > kMostTokens || b->n_seq > kMostTokens) return "more than 2^22 tokens or sequences in a call";
  if (b->n_seq == 0 || b->n_tokens == 0) return nullptr;         // (nothing to do: null pointers will do)
  if (!b->table || !b->lens) return "null table or lengths";
  if (((uintptr_t)b->table | (uintptr_t)b->lens | (uintptr_t)b->q_start) % 4) return "misaligned table, lengths or q_start";
  if (!b->q_start && b->n_tokens != b->n_seq) return "without q_start every sequence has one token: n_tokens must be n_seq";
  return nullptr;
}
inline Batch device_batch(const river_batch *b, int page_size) {
  return Batch{b->table, b->lens, b->q_start, b->n_seq, b->n_tokens, b->max_pages, b->table_stride,
               (int)std::min<long long>((long long)b->max_pages * page_size, kMostPositions)};
}

// The kernels of a configuration: f(T{}, C{}, HD) with the activations' type, the pages' and the head size.
template <int N> struct Int { static constexpr int v = N; };
template <class F>
auto by_types(const river_pages *p, F f) {
  const bool big = p->head_dim == 128;
  if (p->dtype == RIVER_F32) return big ? f(float{}, float{}, Int<128>{}) : f(float{}, float{}, Int<64>{});
  if (p->kv_dtype == RIVER_KV_F16) return big ? f(__bf16{}, _Float16{}, Int<128>{}) : f(__bf16{}, _Float16{}, Int<64>{});
  return big ? f(__bf16{}, __bf16{}, Int<128>{}) : f(__bf16{}, __bf16{}, Int<64>{});
}

const char *bad_attention(const river_pages *pages, const river_batch *batch, int n_q_heads, int window, int sinks, std::string *why);

// How a call is divided: which kernel, tiles of rows, splits of the keys.
struct AttnPlan {
  bool many;                                                     // k_attn_many, else k_attn_split
  bool fused;                                                    // its last workgroups join the splits, where they have tickets
  int max_new, tiles, tile_rows, n_splits, split_len;
  size_t o_bytes, bytes;                                         // of the partial results
};
constexpr int kSplitRows = 16;            // of a tile of k_attn_split
// Up to 16 splits are joined by a row's last workgroup, where there are tickets (8B shape, one sequence of 512: 8.1 us, with a
// second launch 6.4 + 3.8; 16 sequences of up to 1201 15.8, 14.3 + 3.9; 64 splits of 131072 105, 96 + 6)
constexpr int kFewSplits = 16;
AttnPlan plan_attention(const river_pages *p, const river_batch *b, int nq, int window, int sinks);

}  // namespace pg
}  // namespace river
