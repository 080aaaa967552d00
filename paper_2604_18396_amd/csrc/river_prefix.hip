// Host side of attention with common prefixes (include/river.h): checks of arguments, how a call is divided, launches.
#include "river.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <string>

#include "river_pages_host.h"
#include "river_prefix.h"

using namespace river;
using namespace river::pg;

namespace {

const char *bad_prefixes(const river_prefixes *x) {
  if (!x) return "null prefixes";
  if (x->n_groups < 0 || x->n_groups > kMostTokens || x->max_len < 0 || x->max_seqs < 0) return "bad prefixes: n_groups in [0, 2^22], max_len, max_seqs >= 0";
  if (x->n_groups == 0) return nullptr;
  if (x->max_pages < 1 || x->table_stride < x->max_pages) return "bad prefixes: 1 <= max_pages <= table_stride";
  if (!x->table || !x->lens || !x->seq_start) return "null table, lengths or seq_start of the prefixes";
  if (((uintptr_t)x->table | (uintptr_t)x->lens | (uintptr_t)x->seq_start) % 4) return "misaligned table, lengths or seq_start of the prefixes";
  return nullptr;
}

// How a call is divided: units of a group's rows and its prefix, units of a sequence's rows and its own keys.
struct SharePlan {
  bool many, p_many;                                             // tiles of 128 rows: of the sequences, of the prefixes
  bool two;                                                      // of the prefixes: bf16 probabilities as two numbers
  int max_new, tiles, n_splits, least;                           // of the sequences
  int p_tiles, p_splits, p_least;                                // of the prefixes, of all groups
  long long units;                                               // workgroups of the prefixes
  bool fused;                                                    // last workgroups join the splits, where they have tickets
  size_t o_bytes, bytes;                                         // of the partial results
};

// Prefixes have units of their own where that saves enough of reading them for each sequence: 24 MB, or 8 MB of a long one.  (A call then
// takes two launches, and its parts are written and read.  us, apart / each sequence through its prefix, 8B shape, 64 positions of their own:
// 2 sequences behind 1024 11.7 / 9.9, behind 4096 12.8 / 15.5; 8 behind 1024 12.1 / 11.9; 16 behind 256 11.8 / 9.8, behind 1024 12.9 / 19.7;
// 64 behind 16384 48 / 471; 1B shape: 2 behind 4096 11.8 / 11.6, 16 behind 1024 11.8 / 11.6, 32 behind 1024 12.0 / 14.6.)
constexpr double kSaves = 24e6, kSavesLong = 8e6;
constexpr int kLong = 4096;
// Several new tokens of 16-bit types: sequences whose rows nearly fill tiles of 128 read their prefixes hardly more often than a group's tiles do.
// An estimate of both in us: all tiles' work on the whole card (a tile of 128 rows, or of 16, per key and key head), or the keys of the longest
// workgroup (20 ns each) where that is more, and what it takes to begin, to end and to write and read parts (4 TB/s).
// (us, apart / through, 8B shape, 300 own positions: 24 sequences of up to 8 new tokens behind 1024 31 / 35, behind 8192 45 / 128; of 24 46 / 42,
// 91 / 136; of 48 73 / 46, 165 / 228; of 100 134 / 52, 318 / 415; 6 of 8 17.5 / 20.4, 27 / 39, of 48 36 / 32, 58 / 64; 1B shape: 24 of 24 27.9 / 29.8,
// 66 / 97, of 48 47 / 33, 102 / 166)
// Rows of sequences without a prefix count for their own keys alone: `members` sequences have one, with at most `grouped` rows in all.
// (us, apart / through, 8 .. 30 sequences without one: 8B shape, one of 100 tokens behind 20000 109 / 467, two of 8 behind 30000 67 / 390, one of 8
// behind 5000 35 / 47; 1B shape, one of 24 behind 8000 72 / 145)
bool pays(const river_pages *p, const river_batch *b, int nq, const AttnPlan &o, double groups, double members, double grouped, double common, double own) {
  const bool big = p->head_dim == 128;
  const double heads = p->n_kv_heads, all = (double)b->n_tokens * (nq / p->n_kv_heads), n = b->n_seq, keys = common + own;
  const double large = heads * (big ? 65e-6 : 50e-6), small = heads * (big ? 80e-6 : 50e-6);
  const double lone = ((all - grouped) / 128 + (n - members) / 2) * own * large;
  const double through = std::max((grouped / 128 + members / 2) * keys * large * 1.15 + lone, keys / o.n_splits * 0.02) + (o.n_splits > 1 ? 13 : 10);
  const double tiles = grouped / 128 + groups, splits = std::max(1., std::min(256 / (tiles * heads), common / 128));
  const double apart = std::max(tiles * common * large + (all / 16 + n / 2) * own * 0.6 * small, common / splits * 0.02) +
                       (double)b->n_tokens * nq * 2 * (p->head_dim * 4 + 8) * 2 / 4e6 + 14;
  return apart < through;
}
// Splits of a prefix: more than a CU each under one key head have no place (us, at most 64 / 256, one key head of 128: 14 sequences behind 131071 67 / 37,
// two key heads, 16 behind 100000 59 / 44; head size 64, 14 behind 62852 31.0 / 21.8)
constexpr int kMostSplits = 256;
// Splits of the prefixes, as workgroups: one a CU, or seven on four CUs (the eighth place is for the sequences) where that leaves them 1024
// keys of head size 128, 512 of 64, and where the sequences have no more keys of their own than the prefixes; six on four where three have place on a CU.
// (us, 256 / 448, 1B shape, up to 100 own positions: 24 sequences behind 30000 33.4 / 32.2, behind 40000 38.1 / 35.5, 32 behind 48000 43.9 / 41.0, 48 behind
// 20000 37.7 / 35.1, 18 of 64 heads behind 20937 39.7 / 34.7; 64 of up to 900 behind 16384 39.6 / 44.2; 8B shape, 64 of up to 900 behind 30000 84.6 / 86.3,
// 32 of up to 2047 behind 60000 100.9 / 101.3)
long long prefix_places(int head_dim, bool three, double common, double tiles, double groups, double own_keys) {
  
#ifdef FIT
  return FIT;
#endif
  return three ? 384 : common * tiles >= 3584 * head_dim && own_keys <= groups * common ? 448 : 256;
}
// Single tokens, a few long prefixes beside sequences without one: keys are split by the number of all sequences, and the long ones' workgroups
// go on alone.  Units of their own have more splits; 12 us less of the longest workgroup pay for the second launch.
// (us, apart / through, 30 sequences without one: 8B shape, one behind 30000 34.6 / 62, of four tokens 49 / 64, behind 5000 20.9 / 17.9, four behind 30000
// 47 / 63, one behind 100000 beside 60 104 / 353; 1B shape, one behind 30000 22.7 / 33.5, behind 6000 16.9 / 13.6)
bool unequal(const river_pages *p, const AttnPlan &o, double tiles, double groups, double common, double own_keys) {
  const double splits = std::max(1., std::min({(double)prefix_places(p->head_dim, false, common, tiles, groups, own_keys) / tiles, common / 128, (double)kMostSplits}));
  return common * (1. / o.n_splits - 1. / splits) * (p->head_dim == 128 ? 0.014 : 0.0063) > 12;
}
// By tiles of 128 rows (many_unit) where rows x keys x elements of a key head are more than these: they read a key once for 128 rows, those of 16 take
// less time to begin and end (us, 128 / 16, single tokens, 8B shape: 32 rows behind 4096 19.1 / 15.8, behind 16384 28.6 / 26.7, behind 60000 51 / 86; 128
// behind 1024 18.1 / 16.2, behind 4096 25.2 / 26.0; 256 behind 1024 19.6 / 22.0; 1B shape: 64 behind 16384 22.4 / 29.2, 128 behind 4096 18.7 / 20.5, 256
// behind 4096 18.6 / 29.1)
#ifndef KMANY
#define KMANY 3e8
#endif
constexpr double kManyWork = KMANY;

SharePlan plan_share(const river_pages *p, const river_batch *b, const river_prefixes *x, int nq) {
  SharePlan y{};
  const int rep = nq / p->n_kv_heads;
  y.max_new = b->q_start ? std::min(b->max_new, b->n_tokens) : 1;
  const long long rows = (long long)y.max_new * rep, group_rows = std::min<long long>(b->n_tokens, (long long)x->max_seqs * y.max_new) * rep;
  const long long common = x->n_groups ? std::min<long long>({x->max_len, (long long)x->max_pages * p->page_size, kMostPositions}) : 0;
  const long long keys = std::min<long long>({b->max_len, std::max<long long>((long long)b->max_pages * p->page_size, common), kMostPositions});
  const double key_bytes = 2. * p->n_kv_heads * p->head_dim * (p->dtype == RIVER_F32 ? 4 : 2);
  const long long in_group = std::min<long long>(x->max_seqs, b->n_seq), groups = std::min<long long>(x->n_groups, b->n_seq);
  const double saves = std::min<double>(groups * (in_group - 1.), b->n_seq) * common * key_bytes;
  const long long own = std::max(1ll, keys - common);
  bool apart = saves >= (common >= kLong ? kSavesLong : kSaves);
  const AttnPlan o = plan_attention(p, b, nq, 0, 0);
  // (several tokens beside sequences without a prefix: the long ones may be too few to fill the card by themselves)
  const double members = std::min<double>((double)groups * in_group, b->n_seq), grouped = std::min<double>((double)groups * group_rows, (double)b->n_tokens * rep);
  if (p->dtype == RIVER_BF16 && rows > kAttnRows)
    apart = (saves >= kSavesLong || (common >= kLong && members < b->n_seq)) && pays(p, b, nq, o, (double)groups, members, grouped, (double)common, (double)own);
  else if (p->dtype == RIVER_BF16 && !apart && common >= kLong && members < b->n_seq)
    apart = unequal(p, o, (double)groups * ((group_rows + kAttnRows - 1) / kAttnRows) * p->n_kv_heads, (double)groups, (double)common,
                    (double)b->n_seq * own);
  // (fp32 products take longer than their keys' way from the caches: what counts are tiles, which have to become fewer)
  if (p->dtype == RIVER_F32) apart = apart && 2 * b->n_seq * ((rows + 15) / 16) >= 3 * ((long long)b->n_tokens * rep / 16 + groups);
  constexpr int kManyRows = Many<__bf16, 128>::ROWS;
  if (!apart) {
    y.many = y.p_many = o.many;
    y.tiles = o.tiles;
    y.n_splits = o.n_splits;
    y.least = o.split_len;
    y.fused = o.fused;
  } else {
    y.p_many = p->dtype == RIVER_BF16 && group_rows > kAttnRows && (double)groups * group_rows * common * p->n_kv_heads * p->head_dim >= kManyWork;
    // river_paged_attention's roundings of the same batch: a sequence of few rows has two numbers for a probability, also where its group has many
    y.two = y.p_many && !o.many && p->kv_dtype != RIVER_KV_F16;
    y.least = y.p_least = 128;
    const int tile = y.p_many ? kManyRows : kAttnRows;
    const long long full = (group_rows + tile - 1) / tile;
    // (each group that has sequences may have a tile that is not full)
    y.p_tiles = (int)std::min<long long>(((long long)b->n_tokens * rep + tile - 1) / tile + std::max(0ll, groups - 1), INT_MAX);
    const long long p_groups = std::max(1ll, std::min<long long>(y.p_tiles, groups * full) * p->n_kv_heads);
    // Splits of the prefixes: see prefix_places.  But no more than it takes to be done (20 ns a key) in two fifths of the time that
    // all keys take to stream: every split is one more part of each row.
    // (us by splits: 24 sequences behind 131071 positions, 8 tiles and heads, 32 142, 48 140, 56 132, 64 130; 32 behind 65536 32 80, 48 82, 56 82,
    // 64 80; 32 behind 32768 32 47, 48 53, 56 51; 64 of 225 .. 900 own positions behind 8191, 16 tiles and heads, 6 64, 8 56.5, 12 60.2, 16 61;
    // head size 64: 24 behind 131071 32 93, 48 89, 56 80, 64 75; 48 behind 16384, 16 tiles and heads, 16 33, 24 35, 28 32, 32 34)
    const double stream = (groups * (double)common + (double)b->n_seq * own) * key_bytes / 5e6;
    const bool three = p->head_dim == 64 && !y.p_many;           // (workgroups that have place on a CU: see k_share)
    const long long places = three ? 768 : 512, fit = prefix_places(p->head_dim, three, (double)common, (double)p_groups, (double)groups, (double)b->n_seq * own);
    const long long hide = (long long)(common * 0.02 / (0.4 * stream)) + 1;
    y.p_splits = (int)std::max(1ll, std::min({fit / p_groups, (common + 127) / 128, hide, (long long)kMostSplits}));
    y.units = (long long)y.p_tiles * p->n_kv_heads * y.p_splits;
    y.tiles = (int)((rows + kAttnRows - 1) / kAttnRows);
    // of the sequences' own keys: see plan_attention; the places that are left.  Several tiles of a sequence's rows are that many workgroups
    // already: twice the keys in a split (us, 512 / 1024: 1B shape, half pages, four groups of up to 12 sequences behind 3000, drafts of five behind up to
    // 700 own positions 32.8 / 29.9; bf16 pages, behind up to 1400 37.4 / 36.4, 2047 43.4 / 42.0; 8B shape, 12 tokens behind up to 700 69.9 / 65.3)
    const long long o_groups = std::max(1ll, (long long)b->n_seq * p->n_kv_heads * y.tiles);
    auto by = [&](long long goal, long long least) { return std::min({goal / o_groups, (own + least - 1) / least, 64ll}); };
    y.n_splits = (int)std::max(1ll, std::max(by(std::max(256ll, places - p_groups * y.p_splits), 128), by(2048, y.tiles > 1 ? 1024 : 512)));
  }
  if (y.units || y.n_splits > 1) {
    const size_t parts = (size_t)b->n_tokens * nq * ((y.units ? y.p_splits : 0) + y.n_splits);
    y.o_bytes = parts * p->head_dim * 4;
    y.bytes = y.o_bytes + parts * 8;
  }
  return y;
}

}  // namespace

extern "C" int river_prefix_attention_workspace(const river_pages *pages, const river_batch *batch, const river_prefixes *prefixes,
                                                int32_t n_q_heads, size_t *bytes) {
  return guarded([&]() -> int {
    std::string why;
    if (!bytes) return refuse("null bytes");
    if (const char *m = bad_attention(pages, batch, n_q_heads, 0, 0, &why)) return refuse(m);
    if (const char *m = bad_prefixes(prefixes)) return refuse(m);
    *bytes = plan_share(pages, batch, prefixes, n_q_heads).bytes;
    return RIVER_OK;
  });
}

extern "C" int river_prefix_attention(const river_pages *pages, int32_t layer, const river_batch *batch, const river_prefixes *prefixes,
                                      int32_t n_q_heads, const void *q, int64_t q_stride, float scale, void *out, int64_t out_stride,
                                      void *workspace, size_t workspace_bytes, int32_t *tickets, void *hip_stream) {
  return guarded([&]() -> int {
    std::string why;
    if (const char *m = bad_attention(pages, batch, n_q_heads, 0, 0, &why)) return refuse(m);
    if (const char *m = bad_prefixes(prefixes)) return refuse(m);
    if (layer < 0 || layer >= pages->n_layers) return refuse("layer out of range");
    if (!(scale >= 0.f) || !std::isfinite(scale)) return refuse("scale must be positive (0: 1 / sqrt(head_dim))");
    const int es = elem_bytes(pages);
    const long long qw = (long long)n_q_heads * pages->head_dim;
    if (q_stride < qw || out_stride < qw) return refuse("a stride is smaller than its row");
    if ((((uintptr_t)q | (uintptr_t)out) & 15) || q_stride * es % 16 || out_stride * es % 16)
      return refuse("queries, output and their strides must be multiples of 16 bytes");
    if (batch->n_tokens == 0 || batch->n_seq == 0) return RIVER_OK;
    if (!q || !out) return refuse("null queries or output");
    if (q == out) return refuse("the output must not overlap the queries");
    if (scale == 0.f) scale = 1.f / std::sqrt((float)pages->head_dim);
    const float scale2 = scale * 1.44269504088896340736f;        // (powers of two are what the hardware has)
    if (!std::isfinite(scale2)) return refuse("scale is too large");
    if ((long long)batch->n_tokens * n_q_heads >= (1ll << 28)) return refuse("too many tokens and heads");
    const SharePlan y = plan_share(pages, batch, prefixes, n_q_heads);
    if (y.bytes && (!workspace || (uintptr_t)workspace % 16)) return refuse("null or misaligned (16 B) workspace");
    if (workspace_bytes < y.bytes) return refuse("workspace too small", RIVER_ENOSPC);
    if (tickets && (uintptr_t)tickets % 4) return refuse("misaligned tickets");
    if (y.tiles == 0) return RIVER_OK;
    const Cache c = layer_cache(pages, layer);
    const Batch b = device_batch(batch, pages->page_size);
    const int rep = n_q_heads / pages->n_kv_heads;
    auto turn = [](long long round) { int k = 0; while ((round << k) % 32) ++k; return k; };
    const int turn_z = turn((long long)y.n_splits * c.n_kv_heads), turn_s = turn((long long)b.n_seq * y.n_splits * c.n_kv_heads);
    const AttnArgs a{q, out, q_stride, out_stride, n_q_heads, rep, div_by(rep), scale2, 0, 0, y.n_splits, y.least, y.tiles, y.many ? Many<__bf16, 128>::ROWS : kAttnRows, turn_s, turn_z,
                     y.max_new, (float *)workspace, (float2 *)((char *)workspace + y.o_bytes), y.fused && tickets ? (unsigned int *)tickets : nullptr};
    const Prefixes x{prefixes->table, prefixes->lens, prefixes->seq_start, prefixes->n_groups, prefixes->max_pages, prefixes->table_stride,
                     (int)std::min<long long>((long long)prefixes->max_pages * pages->page_size, kMostPositions), std::max(1, y.p_splits), y.p_least,
                     (unsigned)y.units,
                     y.p_many && !y.many && pages->kv_dtype == RIVER_KV_F16 ? Mat<_Float16>::kBias - Mat<_Float16>::kLazyBias : 0.f};
    const long long workgroups = y.units + (long long)b.n_seq * c.n_kv_heads * y.n_splits * y.tiles;
    // (rows of a workgroup of the join: eight parts a thread, where there are more the lanes of several rows have one)
    const int parts = (y.units ? y.p_splits : 0) + y.n_splits, fit = 1024 / pages->head_dim;
    const int each = std::max(1, std::min(fit, fit * 8 / std::max(8, parts))), heads = each >= fit ? fit : each >= 4 ? 4 : each >= 2 ? 2 : 1;
    const int chunks = (n_q_heads + heads - 1) / heads;
    if (workgroups * kAttnThreads >= (1ll << 32) || (long long)b.n_tokens * chunks * 256 >= (1ll << 32))
      return refuse("too many sequences, groups, tokens and heads");
    const hipStream_t st = (hipStream_t)hip_stream;
    hipError_t e = by_types(pages, [&](auto t, auto ct, auto hd) {
      typedef decltype(t) T;
      typedef decltype(ct) C;
      constexpr int HD = decltype(hd)::v;
      auto go = [&](auto pm, auto om, auto two) {
        constexpr bool PM = decltype(pm)::value, OM = decltype(om)::value;
        return launch_lds<k_share<T, C, HD, PM, OM, decltype(two)::value>>(dim3((unsigned)workgroups), dim3(kAttnThreads), ShareLds<T, C, HD, PM, OM>::BYTES, st, c, b, a, x);
      };
      if constexpr (sizeof(T) == 2) {
        if (y.many) return go(True{}, True{}, False{});
        if constexpr (Mat<C>::kSplitP)
          if (y.two) return go(True{}, False{}, True{});
        if (y.p_many) return go(True{}, False{}, False{});
      }
      return go(False{}, False{}, False{});
    });
    if (e == hipSuccess && y.bytes && !a.tickets)
      e = by_types(pages, [&](auto t, auto, auto hd) {
        constexpr int HD = decltype(hd)::v;
        typedef decltype(t) T;
        if (!y.units && y.n_splits <= kFewSplits)
          return launch(k_share_join_few<T, HD>, dim3((unsigned)(((long long)b.n_tokens * n_q_heads + 15) / 16)), dim3(256), 0, st, b, a, x);
        const dim3 grid((unsigned)(b.n_tokens * chunks)), block(256);
        return heads == 1   ? launch(k_share_join<T, HD, 1>, grid, block, 0, st, b, a, x, chunks)
               : heads == 2 ? launch(k_share_join<T, HD, 2>, grid, block, 0, st, b, a, x, chunks)
               : heads == 4 ? launch(k_share_join<T, HD, 4>, grid, block, 0, st, b, a, x, chunks)
                            : launch(k_share_join<T, HD, 1024 / HD>, grid, block, 0, st, b, a, x, chunks);
      });
    return e == hipSuccess ? RIVER_OK : hip_failed("river_prefix_attention", e);
  });
}
