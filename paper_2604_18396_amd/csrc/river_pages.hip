// Host side of the paged key-value cache (include/river.h): checks of arguments, launches, the pool of pages.
#include "river.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <climits>
#include <cstdint>
#include <cstring>
#include <memory>
#include <new>
#include <string>

#include "river_host.h"
#include "river_pages.h"
#include "river_pool.h"

using namespace river;
using namespace river::pg;

namespace {

int refuse(const char *why, int code = RIVER_EINVAL) {
  call_error() = why;
  return code;
}
int hip_failed(const char *what, hipError_t e) {
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

Div div_by(int d) {
  uint32_t s = 0;
  while ((1ll << s) < d) ++s;
  return Div{(uint32_t)d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
}
int elem_bytes(const river_pages *p) { return p->dtype == RIVER_F32 ? 4 : 2; }
long long page_elems(const river_pages *p) { return (long long)p->n_kv_heads * p->page_size * p->head_dim; }

// (a launch holds fewer than 2^32 threads in a dimension; a larger one would be cut off without an error)
constexpr int kMostTokens = 1 << 22;
constexpr int kMostPositions = 1 << 30;                          // of a sequence: indices of keys are 32-bit numbers

Cache layer_cache(const river_pages *p, int layer) {
  const size_t at = (size_t)layer * p->layer_stride * elem_bytes(p);
  return Cache{(char *)p->k + at, (char *)p->v + at, p->page_stride, (uint32_t)(p->page_stride * elem_bytes(p) / 16), p->n_pages, p->page_size, p->n_kv_heads, div_by(p->page_size)};
}

const char *bad_batch(const river_batch *b) {
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
Batch device_batch(const river_batch *b, int page_size) {
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

}  // namespace

std::string &river::call_error() {
  static thread_local std::string text;
  return text;
}

int river::check_pages(const river_pages *p, std::string *why) {
  auto bad = [&](const char *m) { if (why) *why = m; return RIVER_EINVAL; };
  if (!p || !p->k || !p->v) return bad("null pages");
  if (p->n_layers < 1 || p->n_pages < 1 || p->n_kv_heads < 1 || p->page_size < 1 || p->page_size > 65536)
    return bad("bad pages: n_layers, n_pages, n_kv_heads >= 1, page_size in [1, 65536]");
  if (p->head_dim != 64 && p->head_dim != 128) return bad("head_dim must be 64 or 128");
  if (p->dtype != RIVER_F32 && p->dtype != RIVER_BF16) return bad("dtype must be RIVER_F32 or RIVER_BF16");
  if (p->kv_dtype != RIVER_KV_SAME && p->kv_dtype != RIVER_KV_F16) return bad("bad kv_dtype");
  if (p->kv_dtype == RIVER_KV_F16 && p->dtype != RIVER_BF16) return bad("RIVER_KV_F16 needs RIVER_BF16");
  const int es = elem_bytes(p);
  if ((((uintptr_t)p->k | (uintptr_t)p->v) & 15) || p->page_stride * es % 16 || p->layer_stride * es % 16)
    return bad("pages and their strides must be multiples of 16 bytes");
  if ((__int128)p->page_stride * es >= ((__int128)1 << 36)) return bad("page_stride must be below 64 GiB");
  // no two pages may overlap: the nearer stride holds a page, the further one all that the nearer one strides over
  const __int128 x = page_elems(p), ps = p->page_stride, ls = p->layer_stride;
  if (x > (1ll << 40) || ps < 0 || ls < 0) return bad("bad page size or strides");
  const bool apart = (p->n_pages == 1 || ps >= x) && (p->n_layers == 1 || ls >= x) &&
                     (p->n_pages == 1 || p->n_layers == 1 || ls >= (p->n_pages - 1) * ps + x || ps >= (p->n_layers - 1) * ls + x);
  if (!apart) return bad("pages overlap: page_stride or layer_stride is too small");
  if ((p->n_pages * ps + p->n_layers * ls + x) * es > ((__int128)1 << 60)) return bad("bad page size or strides");
  return RIVER_OK;
}

extern "C" int river_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len,
                                      double low, double high, double *inv_freq, float *mscale) {
  return guarded([&] {
    if (!inv_freq || rot_dim < 2 || rot_dim % 2 || rot_dim > 65536 || !(base > 1.0) || !std::isfinite(base))
      return refuse("rotary frequencies: an even rot_dim >= 2, a base > 1 and a place for the result");
    if (scaling < RIVER_ROPE_PLAIN || scaling > RIVER_ROPE_RAMP) return refuse("rotary frequencies: unknown scaling");
    if (scaling != RIVER_ROPE_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return refuse("rotary frequencies: factor must be >= 1");
    if (scaling == RIVER_ROPE_BASE && rot_dim < 4) return refuse("rotary frequencies: RIVER_ROPE_BASE needs rot_dim > 2");
    if (scaling >= RIVER_ROPE_BANDS &&
        !(original_len > 0 && std::isfinite(original_len) && low > 0 && low < high && std::isfinite(high)))
      return refuse("rotary frequencies: original_len > 0 and 0 < low < high are needed");
    const double pi = 3.14159265358979323846;
    const int n = rot_dim / 2;
    if (scaling == RIVER_ROPE_BASE) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
    double a = 0, b = 0;
    if (scaling == RIVER_ROPE_RAMP) {
      auto index = [&](double turns) { return rot_dim * std::log(original_len / (turns * 2 * pi)) / (2 * std::log(base)); };
      a = std::max(0.0, std::floor(index(high)));
      b = std::min(rot_dim - 1.0, std::ceil(index(low)));
    }
    for (int i = 0; i < n; ++i) {
      const double f = std::pow(base, -2.0 * i / rot_dim);
      double part = 0;                                           // of f / factor in the result
      if (scaling == RIVER_ROPE_LINEAR) part = 1;
      if (scaling == RIVER_ROPE_BANDS) part = 1 - std::min(1.0, std::max(0.0, (original_len * f / (2 * pi) - low) / (high - low)));
      if (scaling == RIVER_ROPE_RAMP) part = std::min(1.0, std::max(0.0, (i - a) / std::max(b - a, 0.001)));
      inv_freq[i] = part == 0 ? f : f * (1 - part) + f / factor * part;
    }
    if (mscale) *mscale = scaling == RIVER_ROPE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return (int)RIVER_OK;
  });
}

extern "C" int river_rope_store(const river_pages *pages, int32_t layer, const river_batch *batch, const river_rope *rope,
                                int32_t n_q_heads, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride, void *hip_stream) {
  return guarded([&]() -> int {
    std::string why;
    if (check_pages(pages, &why)) return refuse(why.c_str());
    if (layer < 0 || layer >= pages->n_layers) return refuse("layer out of range");
    if (const char *m = bad_batch(batch)) return refuse(m);
    if (!rope || !rope->inv_freq || (uintptr_t)rope->inv_freq % 8) return refuse("null or misaligned rotary frequencies");
    if (rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > pages->head_dim) return refuse("rot_dim must be even, in [2, head_dim]");
    if (rope->layout != RIVER_ROPE_HALF && rope->layout != RIVER_ROPE_INTERLEAVED) return refuse("bad rotary layout");
    if (n_q_heads < 1 || n_q_heads > 65536) return refuse("n_q_heads out of range");
    const long long qw = (long long)n_q_heads * pages->head_dim, kw = (long long)pages->n_kv_heads * pages->head_dim;
    if (kw > (1 << 24)) return refuse("too many key heads");
    if (q_stride < qw || q_out_stride < qw || k_stride < kw || v_stride < kw) return refuse("a stride is smaller than its row");
    if (q == q_out && q_stride != q_out_stride) return refuse("rotation in place needs the same stride");
    const int es = elem_bytes(pages);
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out) % es) return refuse("misaligned queries, keys or values");
    if (batch->n_tokens == 0 || batch->n_seq == 0) return RIVER_OK;
    if (!q || !k || !v || !q_out) return refuse("null queries, keys or values");
    const Cache c = layer_cache(pages, layer);
    const Batch b = device_batch(batch, pages->page_size);
    const RopeArgs a{rope->inv_freq, rope->rot_dim, rope->layout, rope->mscale, n_q_heads, q, k, v, q_out, q_stride, k_stride, v_stride, q_out_stride};
    // by pieces of 16 bytes where everything allows it: 4096 tokens of the 8B shape 17 us, element by element 29
    const int per = 16 / es;
    const bool wide = (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out) & 15) == 0 &&
                      (q_stride | k_stride | v_stride | q_out_stride) % per == 0 &&
                      rope->rot_dim % (rope->layout == RIVER_ROPE_HALF ? 2 * per : per) == 0;
    const int units = pages->head_dim / per - (rope->layout == RIVER_ROPE_HALF ? rope->rot_dim / (2 * per) : 0);   // of a head
    const hipError_t e = by_types(pages, [&](auto t, auto ct, auto hd) {
      typedef decltype(t) T;
      typedef decltype(ct) C;
      constexpr int HD = decltype(hd)::v;
      const dim3 grid(b.n_tokens), block(kRopeThreads);
      return wide ? launch(k_rope_store_wide<T, C, HD>, grid, block, 0, (hipStream_t)hip_stream, c, b, a, div_by(units))
                  : launch(k_rope_store<T, C, HD>, grid, block, 0, (hipStream_t)hip_stream, c, b, a);
    });
    return e == hipSuccess ? RIVER_OK : hip_failed("river_rope_store", e);
  });
}

// ------------------------------------------------------------------ attention

static const char *bad_attention(const river_pages *pages, const river_batch *batch, int n_q_heads, int window, int sinks, std::string *why) {
  if (check_pages(pages, why)) return why->c_str();
  if (const char *m = bad_batch(batch)) return m;
  if (n_q_heads < 1 || n_q_heads > 65536 || n_q_heads % pages->n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
  if (window < 0 || sinks < 0) return "window and sinks must not be negative";
  return nullptr;
}

// How a call is divided: which kernel, tiles of rows, splits of the keys.
struct AttnPlan {
  bool many;                                                     // k_attn_many, else k_attn_split
  bool fused;                                                    // its last workgroups join the splits, where they have tickets
  int max_new, tiles, tile_rows, n_splits, split_len;
  size_t o_bytes, bytes;                                         // of the partial results
};
// k_attn_many where the rows of a sequence and key head are more than a tile of k_attn_split and all of them see enough: rows x keys
// (of a row in the middle) x elements, 1.3e8 at head size 128 and 3e8 at 64.  It reads keys once for 128 rows, k_attn_split for 16, but
// takes longer to begin and end (us, k_attn_many / k_attn_split; 8B shape: 256 new tokens behind none 12.2 / 11.3, 32 behind 1024
// 18.4 / 21.5, 16 behind 4096 18.9 / 22.8, 8 behind 65536 56 / 104; eight sequences, 8 behind 2048 31.9 / 29.0; sixteen, 16 behind 512
// 22.2 / 24.2; 1B shape: 512 behind none 15.6 / 15.8, 32 behind 4096 17.0 / 17.3, 64 behind 4096 22.8 / 29.9, 8 behind 65536 39.5 / 47.4;
// sixteen, 16 behind 512 16.3 / 14.8, 32 behind 512 19.3 / 21.0.  One product does not part all of these: 256 behind none and eight sequences
// of 8 behind 2048 lie above the limit and are 8 .. 10 % slower there)
constexpr int kSplitRows = 16;
static double many_work(int head_dim) { return head_dim == 128 ? 1.3e8 : 3e8; }
// Up to 16 splits are joined by a row's last workgroup, where there are tickets (8B shape, one sequence of 512: 8.1 us, with a
// second launch 6.4 + 3.8; 16 sequences of up to 1201 15.8, 14.3 + 3.9; 64 splits of 131072 105, 96 + 6)
constexpr int kFewSplits = 16;

static AttnPlan plan_attention(const river_pages *p, const river_batch *b, int nq, int window, int sinks) {
  AttnPlan y{};
  const int rep = nq / p->n_kv_heads;
  y.max_new = b->q_start ? std::min(b->max_new, b->n_tokens) : 1;
  const long long rows = (long long)y.max_new * rep;
  long long keys = std::min<long long>({b->max_len, (long long)b->max_pages * p->page_size, kMostPositions});
  if (window) keys = std::min<long long>(keys, (long long)window + sinks + 15 / rep);
  const double seen = (double)std::min<long long>(keys, std::max(0, b->max_len - y.max_new / 2));
  y.many = p->dtype == RIVER_BF16 && rows > kSplitRows && b->n_seq * seen * rows * p->n_kv_heads * p->head_dim >= many_work(p->head_dim);
  y.tile_rows = y.many ? Many<__bf16, 128>::ROWS : kSplitRows;
  y.tiles = (int)((rows + y.tile_rows - 1) / y.tile_rows);
  // Workgroups without a split: sequences x key heads x tiles; splits so that every CU has two of k_attn_many of at least 256
  // keys.
  // k_attn_split (two at a time on a CU at head size 128, three at 64): three a CU of at least 128 keys (a step for each of the
  // four wavefronts), eight where that leaves them 512: more of them are more even where lengths differ.  us by workgroups a CU, 8B
  // shape: 64 sequences of 128 .. 512 keys 2 / 3 / 4: 21.4 / 21.1 / 27.0, 16 of 300 .. 1200 18.1 / 16.2 / 20.3, 16 of 2048 .. 8192
  // 4 / 8 / 16: 82 / 74 / 75; 1B shape, 32 windows of 1028 16.9 / 16.7 / 21.8; fp32, 8 of 1024 .. 4096 42.7 / 39.0 / 44.0.  At most 64
  // splits: their join
  const long long groups = std::max(1ll, (long long)b->n_seq * p->n_kv_heads * y.tiles);
  auto splits = [&](long long goal, long long least) { return std::min({goal / groups, (keys + least - 1) / least, 64ll}); };
  long long want = std::max(1ll, y.many ? splits(512, 256) : std::max(splits(768, 128), splits(2048, 512)));
  // k_attn_many: only where it saves more (48 keys take 1 us) than joining takes, 4 us and the partial results written and read (8B shape,
  // us, split / not: 384 tokens 19.9 / 15.2, 768 29.6 / 23.1, 1024 38.9 / 29.0; sixteen sequences, 32 behind 512 27.4 / 18.5)
  if (y.many && keys / 48. * (want - 1) / want < 4 + (double)b->n_seq * y.max_new * nq * p->head_dim * want * 8 / 5e6) want = 1;
  y.split_len = (int)std::max(128ll, std::min<long long>(((keys + want - 1) / want + 127) / 128 * 128, 1 << 30));
  y.n_splits = (int)std::max(1ll, (keys + y.split_len - 1) / y.split_len);
  y.fused = !y.many && groups <= RIVER_TICKETS && y.n_splits <= kFewSplits;
  if (y.n_splits > 1) {
    const size_t parts = (size_t)b->n_seq * y.max_new * nq * y.n_splits;
    y.o_bytes = parts * p->head_dim * 4;
    y.bytes = y.o_bytes + parts * 8;
  }
  return y;
}

extern "C" int river_paged_attention_workspace(const river_pages *pages, const river_batch *batch, int32_t n_q_heads,
                                               int32_t window, int32_t sinks, size_t *bytes) {
  return guarded([&]() -> int {
    std::string why;
    if (!bytes) return refuse("null bytes");
    if (const char *m = bad_attention(pages, batch, n_q_heads, window, sinks, &why)) return refuse(m);
    *bytes = plan_attention(pages, batch, n_q_heads, window, sinks).bytes;
    return RIVER_OK;
  });
}

extern "C" int river_paged_attention(const river_pages *pages, int32_t layer, const river_batch *batch, int32_t n_q_heads,
                                     const void *q, int64_t q_stride, float scale, int32_t window, int32_t sinks, void *out,
                                     int64_t out_stride, void *workspace, size_t workspace_bytes, int32_t *tickets, void *hip_stream) {
  return guarded([&]() -> int {
    std::string why;
    if (const char *m = bad_attention(pages, batch, n_q_heads, window, sinks, &why)) return refuse(m);
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
    const AttnPlan y = plan_attention(pages, batch, n_q_heads, window, sinks);
    if (y.bytes && (!workspace || (uintptr_t)workspace % 16)) return refuse("null or misaligned (16 B) workspace");
    if (workspace_bytes < y.bytes) return refuse("workspace too small", RIVER_ENOSPC);
    if (tickets && (uintptr_t)tickets % 4) return refuse("misaligned tickets");
    if (y.tiles == 0) return RIVER_OK;
    const Cache c = layer_cache(pages, layer);
    const Batch b = device_batch(batch, pages->page_size);
    const int rep = n_q_heads / pages->n_kv_heads;
    // Workgroups come back to the same shader engines after 32; a round of them is sequences x key heads (see work_of)
    auto turn = [](long long round) { int k = 0; while ((round << k) % 32) ++k; return k; };
    const int turn_z = turn((long long)y.n_splits * c.n_kv_heads), turn_s = turn((long long)b.n_seq * y.n_splits * c.n_kv_heads);
    AttnArgs a{q, out, q_stride, out_stride, n_q_heads, rep, div_by(rep), scale2, window, window ? sinks : 0,
               y.n_splits, y.split_len, y.tiles, y.tile_rows, turn_s, turn_z, y.max_new, (float *)workspace, (float2 *)((char *)workspace + y.o_bytes), y.fused && tickets ? (unsigned int *)tickets : nullptr};
    const long long groups = (long long)b.n_seq * c.n_kv_heads * y.n_splits * y.tiles;
    if (groups * kAttnThreads >= (1ll << 32) || (long long)b.n_tokens * n_q_heads >= (1ll << 28)) return refuse("too many sequences, tokens and heads");
    const hipStream_t st = (hipStream_t)hip_stream;
    hipError_t e = by_types(pages, [&](auto t, auto ct, auto hd) {
      if constexpr (sizeof(t) == 2)
        if (y.many)
          return launch_lds<k_attn_many<decltype(t), decltype(ct), decltype(hd)::v>>(dim3((unsigned)groups), dim3(256),
                                                                                    Many<decltype(ct), decltype(hd)::v>::LDS, st, c, b, a);
      return launch(k_attn_split<decltype(t), decltype(ct), decltype(hd)::v>, dim3((unsigned)groups), dim3(kAttnThreads), 0, st, c, b, a);
    });
    if (e == hipSuccess && y.n_splits > 1 && !a.tickets)
      e = by_types(pages, [&](auto t, auto, auto hd) {
        constexpr int HD = decltype(hd)::v;
        const unsigned rows = (unsigned)b.n_seq * y.max_new * n_q_heads, each = 16;            // (of 16 lanes)
        return y.n_splits <= kFewSplits ? launch(k_attn_join_few<decltype(t), HD>, dim3((rows + each - 1) / each), dim3(256), 0, st, b, a)
                                        : launch(k_attn_join_many<decltype(t), HD>, dim3(rows), dim3(256), 0, st, b, a);
      });
    return e == hipSuccess ? RIVER_OK : hip_failed("river_paged_attention", e);
  });
}

// ------------------------------------------------------------------ copies

// Pairs in launches of at most kPairs.  Within one, no page that is written is named twice: what depends on an
// earlier pair waits for the next launch.
static int copy_pairs(const river_pages *p, const int32_t *src, const int32_t *dst, int n, hipStream_t s) {
  const int es = elem_bytes(p);
  const long long used = page_elems(p) * es;
  constexpr int kSlots = 2048;
  int key[kSlots];
  char written[kSlots];
  Pairs w;
  int i = 0;
  while (i < n) {
    std::fill(key, key + kSlots, -1);
    auto slot = [&](int page) {
      unsigned h = (unsigned)page * 2654435761u >> 21;
      while (key[h] != -1 && key[h] != page) h = (h + 1) % kSlots;
      return h;
    };
    int m = 0;
    for (; i < n && m < kPairs; ++i) {
      if (src[i] == dst[i]) continue;
      const unsigned a = slot(src[i]), b = slot(dst[i]);
      if (key[b] != -1 || (key[a] != -1 && written[a])) break;
      key[a] = src[i];
      written[a] = 0;
      const unsigned b2 = slot(dst[i]);                          // (src may have taken the slot)
      key[b2] = dst[i];
      written[b2] = 1;
      w.src[m] = src[i];
      w.dst[m++] = dst[i];
    }
    if (!m) continue;
    const dim3 grid((unsigned)((used + kCopyPiece - 1) / kCopyPiece), m, 2);
    for (int l = 0; l < p->n_layers; l += 32767) {
      dim3 g = grid;
      g.z = 2 * std::min(32767, p->n_layers - l);
      const size_t at = (size_t)l * p->layer_stride * es;
      const hipError_t e = launch(k_copy_pages, g, dim3(256), 0, s, (char *)p->k + at, (char *)p->v + at, (long long)p->page_stride * es,
                                  (long long)p->layer_stride * es, used, w);
      if (e != hipSuccess) return hip_failed("river_copy_pages", e);
    }
  }
  return RIVER_OK;
}

extern "C" int river_copy_pages(const river_pages *pages, const int32_t *src, const int32_t *dst, int32_t n, void *hip_stream) {
  return guarded([&]() -> int {
    std::string why;
    if (check_pages(pages, &why)) return refuse(why.c_str());
    if (n < 0 || (n > 0 && (!src || !dst))) return refuse("null or negative list of pages");
    for (int i = 0; i < n; ++i)
      if (src[i] < 0 || src[i] >= pages->n_pages || dst[i] < 0 || dst[i] >= pages->n_pages) return refuse("page number out of range");
    return copy_pairs(pages, src, dst, n, (hipStream_t)hip_stream);
  });
}

hipError_t river::move_rows(const river_pages &p, const int32_t *row, int max_pages, void *kc, void *vc, int max_seq, int first, int n,
                            bool to_pages, hipStream_t stream) {
  const int es = elem_bytes(&p);
  Cache c = layer_cache(&p, 0);
  c.page_stride *= es;                                           // (this kernel counts bytes)
  const long long row_bytes = (long long)p.n_kv_heads * p.head_dim * es;
  const int most = (int)std::max(1ll, (1ll << 30) / (row_bytes / 16));       // rows of a launch
  hipError_t e = hipSuccess;
  for (int at = 0; at < n && e == hipSuccess; at += most) {
    const int m = std::min(most, n - at);
    e = launch(k_move_rows, dim3((unsigned)((m * (row_bytes / 16) + 255) / 256), p.n_layers), dim3(256), 0, stream, c, row, max_pages,
               (long long)p.layer_stride * es, (char *)kc, (char *)vc, max_seq * row_bytes, p.head_dim * es, first + at, m, (int)to_pages);
  }
  return e;
}

hipError_t river::set_word(int *at, int value, hipStream_t stream) {
  Pairs w;
  w.src[0] = 0;
  w.dst[0] = value;
  return launch(k_set_entries, dim3(1), dim3(64), 0, stream, at, 1, w);
}

// ------------------------------------------------------------------ the pool

extern "C" int river_pool_create(int32_t n_pages, int32_t page_size, int32_t max_seqs, int32_t max_pages, river_pool **out) {
  return guarded([&]() -> int {
    if (!out) return refuse("null out");
    *out = nullptr;
    if (n_pages < 1 || n_pages > (1 << 28) || page_size < 1 || page_size > 65536 || max_seqs < 1 || max_pages < 1)
      return refuse("bad pool: n_pages in [1, 2^28], max_seqs, max_pages >= 1, page_size in [1, 65536]");
    if ((long long)max_pages * page_size > INT_MAX || ((long long)max_pages + 1) * max_seqs > (1ll << 28))
      return refuse("bad pool: more than 2^31 positions of a sequence, or more than 2^28 table entries");
    *out = new river_pool(n_pages, page_size, max_seqs, max_pages);
    return RIVER_OK;
  });
}
extern "C" int river_pool_destroy(river_pool *p) {
  delete p;
  return RIVER_OK;
}
extern "C" int river_pool_extend(river_pool *p, int32_t seq, int32_t n_new) {
  return guarded([&]() -> int {
    if (!p || !p->has(seq) || n_new < 0) return refuse("bad sequence or number of positions");
    const char *why = nullptr;
    const int rc = p->extend(seq, n_new, &why);
    return rc ? refuse(why, rc) : RIVER_OK;
  });
}
extern "C" int river_pool_fork(river_pool *p, int32_t src, int32_t dst) {
  return guarded([&]() -> int {
    if (!p || !p->has(src) || !p->has(dst) || src == dst) return refuse("bad sequence");
    if (p->len[dst]) return refuse("the destination of a fork must have no positions", RIVER_ESTATE);
    p->fork(src, dst);
    return RIVER_OK;
  });
}
extern "C" int river_pool_rewind(river_pool *p, int32_t seq, int32_t new_len) {
  return guarded([&]() -> int {
    if (!p || !p->has(seq) || new_len < 0 || new_len > p->len[seq]) return refuse("bad rewind length");
    if (new_len % p->page_size && p->row(seq)[new_len / p->page_size] < 0)
      return refuse("the page that the sequence would go on in has been given back", RIVER_ESTATE);
    p->rewind(seq, new_len);
    return RIVER_OK;
  });
}
extern "C" int river_pool_trim(river_pool *p, int32_t seq, int32_t window, int32_t sinks) {
  return guarded([&]() -> int {
    if (!p || !p->has(seq) || window < 1 || sinks < 0) return refuse("bad sequence, window or sinks");
    p->trim(seq, window, sinks);
    return RIVER_OK;
  });
}
extern "C" int river_pool_compact(river_pool *p) {
  return guarded([&]() -> int { return p ? p->compact() : refuse("null pool"); });
}
extern "C" int river_pool_flush(river_pool *p, const river_pages *pages, int32_t *state, void *hip_stream) {
  return guarded([&]() -> int {
    if (!p || !state || (uintptr_t)state % 4) return refuse("null pool, or null or misaligned state");
    hipStream_t s = (hipStream_t)hip_stream;
    if (pages || !p->copies.empty()) {
      std::string why;
      if (check_pages(pages, &why)) return refuse(why.c_str());
      if (pages->n_pages != p->n_pages || pages->page_size != p->page_size) return refuse("these pages are not the pool's");
    }
    if (!p->copies.empty()) {
      std::vector<int32_t> src, dst;
      for (const auto &c : p->copies) { src.push_back(c.first); dst.push_back(c.second); }
      if (const int rc = copy_pairs(pages, src.data(), dst.data(), (int)src.size(), s)) return rc;
      p->copies.clear();
    }
    if (!p->on_device) {
      const long long n = (long long)p->max_seqs * (p->max_pages + 1);
      const hipError_t e = launch(k_clear_state, dim3((unsigned)std::min(1024ll, (n + 255) / 256)), dim3(256), 0, s, (int *)state, p->max_seqs, n);
      if (e != hipSuccess) return hip_failed("river_pool_flush", e);
      p->on_device = true;
    }
    Pairs w;
    while (!p->dirty.empty()) {
      const int n = std::min<int>(kPairs, (int)p->dirty.size());
      for (int i = 0; i < n; ++i) {
        const int word = p->dirty[p->dirty.size() - 1 - i];
        w.src[i] = word;
        w.dst[i] = word < p->max_seqs ? p->len[word] : p->table[word - p->max_seqs];
      }
      const hipError_t e = launch(k_set_entries, dim3(1), dim3(256), 0, s, (int *)state, n, w);
      if (e != hipSuccess) return hip_failed("river_pool_flush", e);
      for (int i = 0; i < n; ++i) { p->is_dirty[p->dirty.back()] = 0; p->dirty.pop_back(); }
    }
    return RIVER_OK;
  });
}
extern "C" int river_pool_length(const river_pool *p, int32_t seq) { return p && p->has(seq) ? p->len[seq] : RIVER_EINVAL; }
extern "C" int river_pool_free_pages(const river_pool *p) { return p ? (int)p->free_heap.size() : RIVER_EINVAL; }
extern "C" int river_pool_row(const river_pool *p, int32_t seq, int32_t *row) {
  return guarded([&]() -> int {
    if (!p || !p->has(seq) || !row) return refuse("bad sequence or null row");
    std::memcpy(row, p->row(seq), (size_t)p->max_pages * 4);
    return RIVER_OK;
  });
}
