// Host side of a step that is laid out on the device (include/river.h): checks of arguments, launches.
#include "river.h"

#include <algorithm>
#include <climits>
#include <cstdint>
#include <string>

#include "river_pages_host.h"
#include "river_step.h"

using namespace river;
using namespace river::pg;

// More tokens than these have a launch of their own
constexpr int kTokensInOne = 4096;

extern "C" int river_build_batch(const river_tables *t, const int32_t *n_new, int32_t n_tokens, int32_t *q_start, int64_t *slots,
                                 int32_t *positions, int32_t *refused, void *hip_stream) {
  return guarded([&]() -> int {
    if (!t) return refuse("null tables");
    if (t->n_seq < 0 || t->n_seq > kBuildSeqs) return refuse("build: n_seq in [0, 4096]");
    if (t->n_pages < 1 || t->n_pages > (1 << 28) || t->page_size < 1 || t->page_size > 65536 || t->max_pages < 1 || t->table_stride < t->max_pages)
      return refuse("build: n_pages in [1, 2^28], page_size in [1, 65536], 1 <= max_pages <= table_stride");
    if ((long long)t->n_seq * t->max_pages > (long long)kMuch) return refuse("build: more than 2^30 entries");      // (sums of pages given back end there)
    if (n_tokens < 0 || n_tokens > kMostTokens) return refuse("build: n_tokens in [0, 2^22]");
    if (!t->n_free || !t->n_free_out || !t->free_pages || !q_start) return refuse("build: null free list or q_start");
    if (t->n_seq && (!t->table || !t->lens || !t->lens_out || !n_new)) return refuse("build: null table, lengths or n_new");
    if (((uintptr_t)t->table | (uintptr_t)t->lens | (uintptr_t)t->lens_out | (uintptr_t)t->free_pages | (uintptr_t)t->n_free | (uintptr_t)t->n_free_out |
         (uintptr_t)t->n_shared | (uintptr_t)n_new | (uintptr_t)q_start | (uintptr_t)positions | (uintptr_t)refused) % 4 || (uintptr_t)slots % 8)
      return refuse("build: misaligned arrays");
    const BuildArgs a{t->table, t->lens, n_new, t->n_free, t->n_shared, t->lens_out, t->free_pages, t->n_free_out, t->n_seq, t->max_pages,
                      t->table_stride, t->n_pages, t->page_size, n_tokens, (int)std::min<long long>((long long)t->max_pages * t->page_size, kMostPositions),
                      div_by(t->page_size), q_start, (long long *)slots, positions, refused};
    const bool tokens = slots || positions, apart = tokens && n_tokens > kTokensInOne;
    // Threads: one a token or a sixteenth of the table's entries, as far as one workgroup reaches, and four a sequence.  Any entry may come or go, and most do not:
    // a wavefront more takes longer to meet.  (us, taken and given back, without entries / a sixteenth / all: a sequence of 8192 pages 85 / 19.0 / 17.7, of 131072
    // 1286 / 165 / 165, 64 of 188 60.6 / 27.2 / 27.2; drafts of 64 sequences that have 252 entries each
    // 11.5 / 11.6 / 11.6, the kernel that gives them back 3.9 / 5.0 / 5.0; a token of four that have 77 the same)
    const long long some = (long long)t->n_seq * t->max_pages / 16;
    const int threads = (int)std::min<long long>(kBuildThreads, (std::max<long long>({64, 4 * t->n_seq, tokens ? n_tokens : 0, some}) + 63) / 64 * 64);
    const size_t lds = (3 * (size_t)t->n_seq + 1) * 4;
    const hipStream_t st = (hipStream_t)hip_stream;
    auto go = [&](auto k) { return launch(k, dim3(1), dim3(threads), lds, st, a); };
    auto by_seqs = [&](auto with_tokens) {
      constexpr bool TOKENS = decltype(with_tokens)::value;
      return t->n_seq <= 64 ? go(k_build<TOKENS, true, 1>) : t->n_seq <= kBuildThreads ? go(k_build<TOKENS, false, 1>) : go(k_build<TOKENS, false, kBuildEach>);
    };
    hipError_t e = tokens && !apart ? by_seqs(True{}) : by_seqs(False{});
    if (e == hipSuccess && apart)
      e = launch(k_slots, dim3((n_tokens + 256 * kSlotsEach - 1) / (256 * kSlotsEach)), dim3(256), 0, st, a);
    return e == hipSuccess ? RIVER_OK : hip_failed("river_build_batch", e);
  });
}

extern "C" int river_store_slots(const river_pages *pages, int32_t layer, const int64_t *slots, int32_t n_tokens, const void *k,
                                 int64_t k_stride, const void *v, int64_t v_stride, void *hip_stream) {
  return guarded([&]() -> int {
    std::string why;
    if (check_pages(pages, &why)) return refuse(why.c_str());
    if (layer < 0 || layer >= pages->n_layers) return refuse("layer out of range");
    if (n_tokens < 0 || n_tokens > kMostTokens) return refuse("more than 2^22 tokens in a call, or a negative number");
    const long long kw = (long long)pages->n_kv_heads * pages->head_dim;
    if (kw > (1 << 18)) return refuse("too many key heads");    // (2^17 pieces a token at most)
    if (k_stride < kw || v_stride < kw) return refuse("a stride is smaller than its row");
    const int es = elem_bytes(pages);
    if (((uintptr_t)k | (uintptr_t)v) % es || (uintptr_t)slots % 8) return refuse("misaligned keys, values or slots");
    if (n_tokens == 0) return RIVER_OK;
    if (!slots || !k || !v) return refuse("null slots, keys or values");
    const Cache c = layer_cache(pages, layer);
    const int per = 16 / es, row = (int)(2 * kw / per);
    StoreArgs a{(const long long *)slots, k, v, k_stride, v_stride, 1.0 / pages->page_size, (long long)pages->n_pages * pages->page_size,
                n_tokens, std::max(1, kStoreThreads * kStoreEach / row), div_by(row)};
    const bool wide = (((uintptr_t)k | (uintptr_t)v) & 15) == 0 && (k_stride | v_stride) % per == 0;
    const hipError_t e = by_types(pages, [&](auto t, auto ct, auto hd) {
      typedef decltype(t) T;
      typedef decltype(ct) C;
      constexpr int HD = decltype(hd)::v;
      const dim3 grid((n_tokens + a.tokens - 1) / a.tokens), block(kStoreThreads);
      return wide ? launch(k_store_slots<T, C, HD, true>, grid, block, 0, (hipStream_t)hip_stream, c, a)
                  : launch(k_store_slots<T, C, HD, false>, grid, block, 0, (hipStream_t)hip_stream, c, a);
    });
    return e == hipSuccess ? RIVER_OK : hip_failed("river_store_slots", e);
  });
}
