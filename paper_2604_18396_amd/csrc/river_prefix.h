// Device code of attention over pages where groups of sequences go on from common prefixes (gfx950).
#pragma once
#include "river_pages.h"

namespace river {
namespace pg {

// Group g is the sequences seq_start[g] .. seq_start[g + 1] - 1, whose positions below lens[g] are the group's prefix, with a row of
// pages of its own.  A row's softmax over j <= p is the softmax over its parts, each with its own maximum m and sum l:
//   o = sum_i 2^(m_i - m) l_i o_i / sum_i 2^(m_i - m) l_i
// so the rows of all of a group's new tokens that share a key head are the rows of one product with the prefix's keys, which are
// read once for a tile of them, and each sequence's rows have a product with its own keys.  One launch has the units of both kinds, the
// prefixes' first; another joins a row's parts.
struct Prefixes {
  const int *table, *lens, *seq_start;
  int n_groups, max_pages, table_stride;
  int cap;                                // positions that a row has entries for
  int n_splits, least;                    // splits of a prefix at most, keys of a split at least
  unsigned units;                         // workgroups of the prefixes; 0: a sequence's rows go through its prefix too
  float shift;                            // added to the prefixes' maxima: both kernels scale fp16 probabilities, by different powers of two
};

// The group of sequence s (-1: none) and its prefix's positions.
__device__ __forceinline__ int cut_len(const Prefixes &x, int len) { return min(max(len, 0), x.cap); }
__device__ __forceinline__ void find_group(const Prefixes &x, int s, int &g, int &n) {
  g = -1;
  n = 0;
  if (x.n_groups == 0) return;
  if (x.n_groups < 64) {                  // (a lane a group: both are read at once)
    const int lane = threadIdx.x % 64, start = x.seq_start[min(lane, x.n_groups)], len = x.lens[min(lane, x.n_groups - 1)];
    const int c = __popcll(__ballot(lane <= x.n_groups && start <= s)) - 1;
    if (c < 0 || c >= x.n_groups) return;
    g = c;
    n = cut_len(x, __builtin_amdgcn_readlane(len, c));
  } else {
    const int c = __builtin_amdgcn_readfirstlane(count_up_to(x.seq_start, x.n_groups + 1, s)) - 1;
    if (c < 0 || c >= x.n_groups) return;
    g = c;
    n = cut_len(x, x.lens[c]);
  }
}

// Splits of n keys: whole steps of 128 keys, `least` at least and no more splits than `most`; one if there are none.
__device__ __forceinline__ int split_len(int n, int most, int least) { return max(least, ((n + most - 1) / most + 127) / 128 * 128); }
__device__ __forceinline__ int split_count(int n, int most, int least) {
  const int len = split_len(n, most, least);
  return max(1, (n + len - 1) / len);
}

// Keys that lie in the group's pages below position n, in the sequence's own from there on.
struct TwoRows {
  const int *common, *own;
  int n;
  __device__ __forceinline__ const int *place(int p, int i) const { return (p < n ? common : own) + i; }
  __device__ __forceinline__ int entry(int p, int i) const { return *place(p, i); }
};
// Rows whose positions were found before: this lane's, and the lowest and highest of its wavefront's.
struct Found {
  int mine, first, last;
  bool none;                              // no position: see prefix_unit
  __device__ __forceinline__ int position(int) const { return mine; }
  __device__ __forceinline__ void reach(int, int, int &lo, int &hi) const { lo = first; hi = last; }
  __device__ __forceinline__ bool nobody() const { return none; }
};
typedef Unit<TwoRows, Found> Share;

constexpr int kAttnRows = 16;              // of a tile of split_unit
// Steps of a prefix's keys in flight in many_unit: here they come from memory, where the prompts of k_attn_many read them again and again
// (us with two / four: 64 sequences behind 8191 59.2 / 56.5, 24 behind 131071 133 / 133, at head size 64 84 / 81; with one product a probability 58.1 / 53.8,
// 133 / 125, 92 / 87; five there 92, and no place at 128)
constexpr int kAhead = 4;
constexpr int kEverything = 1 << 30;       // a position that sees every key
template <int TR>
__device__ __forceinline__ int my_row(int r0, int r1) {           // this lane's row of a tile of TR
  return min(r0 + (TR == kAttnRows ? (int)threadIdx.x % 16 : (int)threadIdx.x / 64 * 32 + (int)threadIdx.x % 32), r1);
}

// The table's entries of a unit's first keys: those of the first two steps of a lane (split_unit), or CHUNK steps, a thread each (many_unit).
template <class C, int HD, int TR>
struct FirstOf {
  static constexpr int N = TR == kAttnRows ? 2 * Tile<C, HD>::KB : Many<C, HD, kAhead>::CHUNK * 32 / 256;
};
template <class C, int HD, int TR>
__device__ __forceinline__ void first_entries(const Cache &c, const Share &w, First<FirstOf<C, HD, TR>::N> &first) {
#pragma unroll
  for (int j = 0; j < FirstOf<C, HD, TR>::N; ++j) {
    constexpr int KB = Tile<C, HD>::KB;
    const int i = TR == kAttnRows ? (j / KB * kAttnWaves + (int)threadIdx.x / 64) * Mat<C>::kKeys + j % KB * 16 + (int)threadIdx.x % 16 : j * 256 + (int)threadIdx.x;
    const int p = max(w.sp.pos(min(w.i0 + i, w.i1 - 1)), 0);     // (a unit of no keys: any entry)
    first.e[j] = w.keys.entry(p, c.by_page.quot(p));
  }
}

// Tile `tile` of all groups' rows, one group after the other, with split z of its group's prefix.  A token without a position (it
// has no result) counts as one that sees all, with a query of zeros, so that it costs the others nothing, whatever its bits: a NaN there made the
// tile one of careful passes (64 single tokens behind 8191, one of them such a place, 36 us / 675).
template <class C, int HD, int TR>
__device__ __forceinline__ bool prefix_unit(const Cache &c, const Prefixes &x, const Batch &b, const AttnArgs &a, int tile, int z, int head, Share &w,
                                            First<FirstOf<C, HD, TR>::N> &first) {
  // a lane a group: where its tiles begin
  const int lane = threadIdx.x % 64;
  int g, s0, s1, t0, rows, n;
  for (int g0 = 0;; g0 += 64) {
    if (g0 >= x.n_groups) return false;
    g = min(g0 + lane, x.n_groups - 1);
    s0 = min(max(x.seq_start[g], 0), b.n_seq);
    s1 = min(max(x.seq_start[g + 1], s0), b.n_seq);
    n = cut_len(x, x.lens[g]);
    t0 = b.q_start ? min(max(b.q_start[s0], 0), b.n_tokens) : s0;
    rows = ((b.q_start ? min(max(b.q_start[s1], t0), b.n_tokens) : s1) - t0) * a.rep;
    const int tiles = g0 + lane < x.n_groups && n ? (rows + TR - 1) / TR : 0;
    int upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    const unsigned long long behind = __ballot(tile < upto);
    if (behind) {
      const int it = __ffsll(behind) - 1;
      tile -= __builtin_amdgcn_readlane(upto - tiles, it);
      g = __builtin_amdgcn_readlane(g, it);
      s0 = __builtin_amdgcn_readlane(s0, it);
      s1 = __builtin_amdgcn_readlane(s1, it);
      n = __builtin_amdgcn_readlane(n, it);
      t0 = __builtin_amdgcn_readlane(t0, it);
      rows = __builtin_amdgcn_readlane(rows, it);
      break;
    }
    tile -= __builtin_amdgcn_readlane(upto, 63);
  }
  const int parts = split_count(n, x.n_splits, x.least), len = split_len(n, x.n_splits, x.least), r0 = tile * TR;
  if (z >= parts || (unsigned)tile >= (unsigned)((rows + TR - 1) / TR)) return false;
  w.r0 = r0;
  w.r1 = min(r0 + TR - 1, rows - 1);
  const int *row = x.table + (long long)g * x.table_stride;
  w.keys = {row, row, n};
  w.sp = {0, 0, 0, 0, n};
  w.i0 = z * len;
  w.i1 = z == parts - 1 ? n : w.i0 + len;
  first_entries<C, HD, TR>(c, w, first);
  const int t = t0 + a.by_rep.quot(my_row<TR>(r0, w.r1));
  int p;
  if (!b.q_start) p = max(b.lens[t], 0) - 1;
  else if (s1 - s0 <= 64) {               // (a lane a sequence: where it ends, and its length; the token's is the first that ends behind it)
    const int ends = min(b.q_start[min(s0 + lane + 1, s1)], b.n_tokens), lens = b.lens[min(s0 + lane, s1 - 1)];
    int k = 0;
#pragma unroll
    for (int d = 32; d; d >>= 1)
      if (__shfl(ends, k + d - 1) <= t) k += d;
    p = max(__shfl(lens, k), 0) - (__shfl(ends, k) - t);
  } else {
    int s = s0, hi = s1;
    while (s + 1 < hi) {
      const int mid = (s + hi) >> 1;
      if (b.q_start[mid] <= t) s = mid; else hi = mid;
    }
    p = position_of(b, s, t);
  }
  const bool none = p < 0;
  if (none) p = kEverything;
  int lo = p, hi = p;
#pragma unroll
  for (int d = 1; d < (TR == kAttnRows ? 16 : 32); d <<= 1) {
    lo = min(lo, __shfl_xor(lo, d));
    hi = max(hi, __shfl_xor(hi, d));
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  w.rows = {p, lo, hi, none};
  w.sp = {lo, hi, 0, 0, n};
  w.first_token = t0;
  w.row0 = t0;
  w.head = head;
  w.part = z;
  w.whole = false;
  return true;
}

// Tile `tile` of sequence s's rows with split z of its own keys (of all that it sees, where the prefixes have no units).
template <class C, int HD, int TR, class F>
__device__ __forceinline__ bool own_unit(const Cache &c, const Prefixes &x, const Batch &b, const AttnArgs &a, int s, int tile, int z, int head, Share &w,
                                         F &first, int &parts) {
  int g, n;
  find_group(x, s, g, n);
  int first_token, count;
  seq_tokens(b, s, first_token, count);
  const int rows = min(count, a.max_new) * a.rep, r0 = tile * TR;
  if (r0 >= rows) return false;
  w.r0 = r0;
  w.r1 = min(r0 + TR - 1, rows - 1);
  const int len = length_of(b, s);
  const int lo = new_position(len, count, a.by_rep.quot(r0)), hi = new_position(len, count, a.by_rep.quot(w.r1));
  const int low = x.units ? n : 0, keys = max(0, min(hi + 1, max(b.cap, n)) - low);
  const int each = split_len(keys, a.n_splits, a.split_len);
  parts = split_count(keys, a.n_splits, a.split_len);
  if (z >= parts) return false;
  w.sp = {lo, hi, 0, low, keys};
  if constexpr (TR == kAttnRows) w.rows = {new_position(len, count, a.by_rep.quot(my_row<TR>(r0, w.r1))), lo, hi, false};
  else {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), w0 = min(r0 + wave * 32, w.r1), w1 = min(w0 + 31, w.r1);
    w.rows = {new_position(len, count, a.by_rep.quot(my_row<TR>(r0, w.r1))), new_position(len, count, a.by_rep.quot(w0)),
              new_position(len, count, a.by_rep.quot(w1)), false};
  }
  w.keys = {x.table + (long long)max(g, 0) * x.table_stride, b.table + (long long)s * b.table_stride, n};
  w.i0 = z * each;
  w.i1 = z == parts - 1 ? keys : w.i0 + each;
  if constexpr (F::have) first_entries<C, HD, TR>(c, w, first);
  w.first_token = first_token;
  w.row0 = first_token;
  w.head = head;
  const int before = x.units ? x.n_splits : 0;
  w.part = before + z;
  w.whole = parts == 1 && (n == 0 || !x.units);
  return true;
}

// PM, OM: tiles of 128 rows (many_unit) of the groups, of the sequences; else of 16 (split_unit).  Bounds and layouts: see there.
template <class T, class C, int HD, bool PM, bool OM>
struct ShareLds {
  static constexpr int SPLIT = kAttnWaves * SplitLds<C, HD>::AREA, RES = kAttnWaves * 16 * 8, MANY = OM ? Many<C, HD>::LDS : PM ? Many<C, HD, kAhead>::LDS : 0;
  static constexpr int BYTES = (PM && OM) || MANY > SPLIT + RES ? MANY : SPLIT + RES;
};
// Both kinds in one kernel take more than the 168 registers that leave three workgroups a CU at head size 64: two (24 sequences behind
// 131071 85 -> 75 us, without the 20 registers that were spilled).  What is still spilled: 11 registers of fp32 rows at head size 128, 3 of rows over half pages
// there, 11 of tiles with two numbers a probability, 5 or 6 of tiles at 64: in front of a pass or of the results, and in careful passes.
template <class T, class C, int HD, bool PM, bool OM, bool TWO>
__global__ __launch_bounds__(kAttnThreads, HD == 64 && !(PM && !OM) ? 3 : 2) void k_share(Cache c, Batch b, AttnArgs a, Prefixes x) {
  extern __shared__ __align__(1024) char lds[];
  constexpr int PR = PM ? Many<C, HD>::ROWS : kAttnRows, OR = OM ? Many<C, HD>::ROWS : kAttnRows;
  Share w;
  w.n_parts = (x.units ? x.n_splits : 0) + a.n_splits;
  int tile, s, z, head, parts;
  if constexpr (!OM) {                    // (sequences whose rows fill such tiles go through their prefixes themselves)
    First<FirstOf<C, HD, OR>::N> first;
    if (blockIdx.x < x.units) {
      // A tile's splits follow each other, so that the tiles that groups have fill all XCDs and the empty ones come last (four key heads, 2 sequences
      // behind 7479 and five that have no prefix: 22.9 us with the tiles innermost, 16.1)
      const unsigned u = blockIdx.x / c.n_kv_heads;
      if constexpr (PM) {
        First<FirstOf<C, HD, PR>::N> first;
        if (prefix_unit<C, HD, PR>(c, x, b, a, u / x.n_splits, u % x.n_splits, blockIdx.x % c.n_kv_heads, w, first))
          many_unit<T, C, HD, kAhead, TWO>(c, a, w, first, lds);
        return;
      } else if (!prefix_unit<C, HD, PR>(c, x, b, a, u / x.n_splits, u % x.n_splits, blockIdx.x % c.n_kv_heads, w, first)) return;
    } else {
      work_of(blockIdx.x - x.units, c, b, a, tile, s, z, head);
      if (!own_unit<C, HD, OR>(c, x, b, a, s, tile, z, head, w, first, parts)) return;
    }
    int early[2][Tile<C, HD>::KB];
#pragma unroll
    for (int j = 0; j < FirstOf<C, HD, OR>::N; ++j) early[j / Tile<C, HD>::KB][j % Tile<C, HD>::KB] = first.e[j];
    float v[RowPart<HD>::E];
    split_unit<T, C, HD>(c, a, w, lds, (float2(*)[16])(lds + ShareLds<T, C, HD, PM, OM>::SPLIT), true, early, v);
    if constexpr (!PM) {                  // (tickets: there are no prefixes' units)
      if (a.tickets && parts > 1) join_last<T, HD>(a, w, parts, (s * c.n_kv_heads + head) * a.tiles + tile);
    }
  } else {
    NoFirst first;
    work_of(blockIdx.x, c, b, a, tile, s, z, head);
    if (own_unit<C, HD, OR>(c, x, b, a, s, tile, z, head, w, first, parts)) many_unit<T, C, HD, 2, false>(c, a, w, first, lds);
  }
}

// Head h of new token i of sequence s, which has n positions of a prefix: parts of the prefix, parts of its own, its position.
__device__ __forceinline__ void parts_of(const Batch &b, const AttnArgs &a, const Prefixes &x, int s, int count, int i, int h, int n, int &common, int &own, int &p) {
  const int len = length_of(b, s), low = x.units ? n : 0;
  common = low ? split_count(n, x.n_splits, x.least) : 0;
  // (the last row of this one's tile: see own_unit)
  const int r = i * a.rep + h % a.rep, r1 = min(r - r % a.tile_rows + a.tile_rows, min(count, a.max_new) * a.rep) - 1;
  const int keys = max(0, min(new_position(len, count, a.by_rep.quot(r1)) + 1, max(b.cap, n)) - low);
  own = split_count(keys, a.n_splits, a.split_len);
  p = new_position(len, count, i);
}

// Few parts where prefixes have no units: bit for bit what a tile's last workgroup does where it has tickets.  Sixteen rows a workgroup, of any
// tokens.  Bound: latency.
template <class T, int HD>
__global__ __launch_bounds__(256) void k_share_join_few(Batch b, AttnArgs a, Prefixes x) {
  constexpr int E = RowPart<HD>::E, LANES = RowPart<HD>::LANES;
  const int w = blockIdx.x * 16 + threadIdx.x / LANES, t = w / a.nq, h = w - t * a.nq, e0 = threadIdx.x % LANES * E;
  if (t >= b.n_tokens) return;
  const int s = seq_of(b, t);
  if (s < 0) return;
  int first, count;
  seq_tokens(b, s, first, count);
  if (t - first >= min(count, a.max_new)) return;
  int n = 0;
  if (x.n_groups && s >= x.seq_start[0]) {
    int g = 0, hi = x.n_groups + 1;       // the last that begins at or before s
    while (g + 1 < hi) {
      const int mid = (g + hi) >> 1;
      if (x.seq_start[mid] <= s) g = mid; else hi = mid;
    }
    if (g < x.n_groups) n = cut_len(x, x.lens[g]);
  }
  int common, own, p;
  parts_of(b, a, x, s, count, t - first, h, n, common, own, p);
  if (own == 1) return;
  float v[E], sum;
  join_parts<HD, E>(a, (long long)w * a.n_splits, own, e0, v, sum);
  store_row<T, E>((T *)a.out + (long long)t * a.out_stride + (long long)h * HD + e0, v, sum);
}

// A row's parts, joined: those of its group's prefix, then its sequence's own.  A workgroup has RB heads of one token, and where a row has
// many parts G groups of lanes that take other parts each; their sums are added in their order.  Bound: latency; so the first parts are on
// their way before it is known which of them there are.
template <class T, int HD, int RB>
__global__ __launch_bounds__(256) void k_share_join(Batch b, AttnArgs a, Prefixes x, int chunks) {
  constexpr int LANES = HD / 4, G = 256 / (RB * LANES), AT_ONCE = 8;
  const int t = blockIdx.x / chunks, in = threadIdx.x / LANES % RB, group = threadIdx.x / (LANES * RB), e0 = threadIdx.x % LANES * 4;
  const int h = min(blockIdx.x % chunks * RB + in, a.nq - 1);
  const int before = x.units ? x.n_splits : 0, n_parts = before + a.n_splits;
  const long long row = ((long long)t * a.nq + h) * n_parts;
  float2 ml[AT_ONCE];
  f32x4 o[AT_ONCE];
  auto fetch = [&](int y0) {
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const long long part = row + min(y0 + k * G, n_parts - 1);
      ml[k] = a.part_ml[part];
      o[k] = *(const f32x4 *)(a.part_o + part * HD + e0);
    }
  };
  fetch(group);
  int s = t;
  if (b.q_start) {
    s = __builtin_amdgcn_readfirstlane(count_up_to(b.q_start, b.n_seq + 1, t)) - 1;
    if (s < 0 || s >= b.n_seq) return;
  }
  int first, count, g, n, common, own, p;
  seq_tokens(b, s, first, count);
  if (t - first >= min(count, a.max_new)) return;
  find_group(x, s, g, n);
  parts_of(b, a, x, s, count, t - first, h, n, common, own, p);
  float big = -INFINITY, sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int y0 = group;;) {
    float now = big;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int y = y0 + k * G;
      const bool there = y < common || (y >= before && y < before + own);
      if (y < common) ml[k].x += x.shift;
      if (!there) {
        ml[k] = make_float2(-INFINITY, 0.f);
        o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      now = fmaxf(now, ml[k].x);
    }
    const float off = now == -INFINITY ? 0.f : now, f = __builtin_amdgcn_exp2f(big - off);
    sum *= f;
    v *= f;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const float p = __builtin_amdgcn_exp2f(ml[k].x - off);
      sum += p * ml[k].y;
      v += p * o[k];
    }
    big = now;
    y0 += AT_ONCE * G;
    if (y0 - group >= before + own) break;
    fetch(y0);
  }
  if constexpr (G > 1) {
    __shared__ f32x4 part_v[G][RB][LANES];
    __shared__ float2 part_ml[G][RB];
    part_v[group][in][threadIdx.x % LANES] = v;
    if (e0 == 0) part_ml[group][in] = make_float2(big, sum);
    __syncthreads();
    if (group) return;
    float top = big;
#pragma unroll
    for (int k = 1; k < G; ++k) top = fmaxf(top, part_ml[k][in].x);
    const float off = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(big - off);
    sum *= f;
    v *= f;
#pragma unroll
    for (int k = 1; k < G; ++k) {
      const float2 m = part_ml[k][in];
      const float p = __builtin_amdgcn_exp2f(m.x - off);
      sum += p * m.y;
      v += p * part_v[k][in][threadIdx.x % LANES];
    }
  }
  if (common + own == 1 || blockIdx.x % chunks * RB + in >= a.nq) return;          // (it is done already, or no row)
  if (p < 0) sum = 0.f;                                          // (a token without a position sees nothing)
  const float out[4] = {v[0], v[1], v[2], v[3]};
  store_row<T, 4>((T *)a.out + (long long)t * a.out_stride + (long long)h * HD + e0, out, sum);
}

}  // namespace pg
}  // namespace river
