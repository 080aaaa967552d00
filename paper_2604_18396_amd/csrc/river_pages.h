// Device code of the paged key-value cache (gfx950): rotary positions with the store into the pages, attention over
// the pages, page copies.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace river {
namespace pg {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// n / d for 0 <= n < 2^31 and 1 <= d <= 2^16 as a product: with 2^s >= d and m = ceil(2^(31+s) / d) the error m d - 2^(31+s)
// is below d <= 2^s, so (n m) >> (31+s) is exact (Granlund and Montgomery, 1994).
struct Div {
  uint32_t d, m, s;
  __device__ __forceinline__ int quot(int n) const { return (int)(__umulhi(2u * (uint32_t)n, m) >> s); }
};

// One layer's pages.  Element types: the activations' T and the pages' C below.
struct Cache {
  void *k, *v;
  long long page_stride;                  // elements
  uint32_t page_pieces;                   // the same in pieces of 16 bytes
  int n_pages, page_size, n_kv_heads;
  Div by_page;
};

struct Batch {
  const int *table, *lens, *q_start;
  int n_seq, n_tokens, max_pages, table_stride;
  int cap;                                // max_pages * page_size: positions from here on have no page
};

// The new tokens of sequence s: the first, and how many (within the call's tokens, whatever q_start holds).
__device__ __forceinline__ void seq_tokens(const Batch &b, int s, int &first, int &count) {
  if (!b.q_start) { first = s; count = 1; return; }
  first = min(max(b.q_start[s], 0), b.n_tokens);
  count = min(max(b.q_start[s + 1], first), b.n_tokens) - first;
}

// The sequence that token t belongs to, or -1.
__device__ __forceinline__ int seq_of(const Batch &b, int t) {
  if (!b.q_start) return t;
  int lo = 0, hi = b.n_seq;               // the first s with t < q_start[s + 1]
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (t < b.q_start[mid + 1]) hi = mid; else lo = mid + 1;
  }
  return lo < b.n_seq && t >= b.q_start[lo] ? lo : -1;
}

// The position of token t of sequence s, negative if it has none.
__device__ __forceinline__ int position_of(const Batch &b, int s, int t) {
  int first, count;
  seq_tokens(b, s, first, count);
  const long long p = (long long)b.lens[s] - count + (t - first);
  return p < 0 ? -1 : (int)p;
}

// The same from the sequence's length (length_of) for its new token i of `count`: -1 if it has none, and no less, so that a window of up
// to 2^31 - 1 can be taken from it.
__device__ __forceinline__ int length_of(const Batch &b, int s) { return max(b.lens[s], 0); }
__device__ __forceinline__ int new_position(int len, int count, int i) { return max(len - count + i, -1); }

// The page of position p (0 <= p) and the slot in it; -1: there is none.
__device__ __forceinline__ int page_of(const Cache &c, const Batch &b, int s, int p, int &slot) {
  if (p >= b.cap) return -1;
  const int i = c.by_page.quot(p);
  slot = p - i * c.page_size;
  const int page = b.table[(long long)s * b.table_stride + i];
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}

// ------------------------------------------------------------------ rotary positions and the store
//
// (x, y) of a pair -> (x cos a - y sin a, x sin a + y cos a) times mscale, a = p f.  The angle is taken in 64 bits and reduced to
// turns before it is rounded (p f of a far position has its fraction in bits that fp32 does not keep); sine and
// cosine of the reduced angle, and the products, are fp32.  One workgroup per token: its angles are shared by all its heads.
// This kernel, element by element, takes what k_rope_store_wide cannot (odd strides, addresses, widths).
constexpr int kRopeThreads = 256;

__device__ __forceinline__ float2 turn(int p, double f, float mscale) {
  double t = (double)p * (f * 0.15915494309189533577);           // turns
  t -= rint(t);
  float s, c;
  sincospif((float)(2.0 * t), &s, &c);
  return make_float2(c * mscale, s * mscale);
}

struct RopeArgs {
  const double *inv_freq;
  int rot, interleaved;
  float mscale;
  int nq;
  const void *q, *k, *v;
  void *q_out;
  long long q_stride, k_stride, v_stride, q_out_stride;
};

template <class T, class C, int HD>
__global__ __launch_bounds__(kRopeThreads) void k_rope_store(Cache c, Batch b, RopeArgs a) {
  const int t = blockIdx.x;
  const int s = seq_of(b, t);
  if (s < 0) return;
  const int p = position_of(b, s, t);
  if (p < 0) return;
  __shared__ float2 cs[HD / 2];
  if ((int)threadIdx.x < a.rot / 2) cs[threadIdx.x] = turn(p, a.inv_freq[threadIdx.x], a.mscale);
  __syncthreads();
  int slot = 0;
  const int page = page_of(c, b, s, p, slot);
  const T *q = (const T *)a.q + t * a.q_stride, *k = (const T *)a.k + t * a.k_stride, *v = (const T *)a.v + t * a.v_stride;
  T *qo = (T *)a.q_out + t * a.q_out_stride;
  const long long row = (long long)page * c.page_stride + (long long)slot * HD, head = (long long)c.page_size * HD;
  C *ko = (C *)c.k + row, *vo = (C *)c.v + row;
  const int pairs = HD / 2, heads = a.nq + (page < 0 ? 0 : 2 * c.n_kv_heads);
  for (int i = threadIdx.x; i < heads * pairs; i += kRopeThreads) {
    const int h = i / pairs, j = i % pairs;
    // the two elements of pair j; behind the rotated part, neighbours
    const bool rot = 2 * j < a.rot;
    const int e0 = rot && !a.interleaved ? j : 2 * j, e1 = rot && !a.interleaved ? j + a.rot / 2 : 2 * j + 1;
    if (h >= a.nq + c.n_kv_heads) {
      const int g = h - a.nq - c.n_kv_heads;
      vo[g * head + e0] = (C)(float)v[g * HD + e0];
      vo[g * head + e1] = (C)(float)v[g * HD + e1];
      continue;
    }
    const bool key = h >= a.nq;
    const T *src = key ? k + (h - a.nq) * HD : q + h * HD;
    const float x = (float)src[e0], y = (float)src[e1];
    float2 w = rot ? cs[j] : make_float2(1.f, 0.f);
    const float u = rot ? x * w.x - y * w.y : x, z = rot ? y * w.x + x * w.y : y;
    if (key) {
      ko[(h - a.nq) * head + e0] = (C)u;
      ko[(h - a.nq) * head + e1] = (C)z;
    } else {
      qo[h * HD + e0] = (T)u;
      qo[h * HD + e1] = (T)z;
    }
  }
}

// The same by 16-byte pieces, where rows, strides and the rotated part allow it.  Bound: memory (a token's row in, its queries and
// cache rows out).  A unit is a piece, or the two pieces whose elements are pairs; a thread has kRopeUnits of them in flight (its loads
// stand in front of its stores, which the compiler may not move them past: the queries may be rotated in place).  8B shape: 4096
// tokens, 101 MB, 17 us (element by element 29), 5.9 TB/s; 32 tokens 4.5 us, one 2.7: start, the two or three loads that find its
// row, the angles.
constexpr int kRopeUnits = 2;
template <class T, class C, int HD>
__global__ __launch_bounds__(kRopeThreads) void k_rope_store_wide(Cache c, Batch b, RopeArgs a, Div by_units) {
  constexpr int PER = 16 / sizeof(T), P = HD / PER;
  const int t = blockIdx.x;
  const int s = seq_of(b, t);
  if (s < 0) return;
  const int p = position_of(b, s, t);
  if (p < 0) return;
  __shared__ float2 cs[HD / 2];
  const T *q = (const T *)a.q + t * a.q_stride, *k = (const T *)a.k + t * a.k_stride, *v = (const T *)a.v + t * a.v_stride;
  T *qo = (T *)a.q_out + t * a.q_out_stride;
  int slot = 0;
  const int page = page_of(c, b, s, p, slot);
  const long long row = (long long)page * c.page_stride + (long long)slot * HD, head = (long long)c.page_size * HD;
  C *ko = (C *)c.k + row, *vo = (C *)c.v + row;
  const int pairs = a.interleaved ? 0 : a.rot / (2 * PER);       // units of two pieces a head; the others are of one
  const int turned = (a.nq + c.n_kv_heads) * (int)by_units.d;    // units of queries and keys
  const int all = page < 0 ? a.nq * (int)by_units.d : turned + c.n_kv_heads * P;
  struct Unit { const T *from; int h, e; bool two, rot; };       // h: head, of the queries, the keys, then the values
  auto unit = [&](int i) {
    Unit u;
    if (i >= turned) {
      u.h = a.nq + c.n_kv_heads + (i - turned) / P;
      u.e = (i - turned) % P * PER;
      u.two = u.rot = false;
      u.from = v + (u.h - a.nq - c.n_kv_heads) * HD + u.e;
      return u;
    }
    u.h = by_units.quot(i);
    const int j = i - u.h * (int)by_units.d;
    u.two = j < pairs;
    u.e = (j < pairs ? j : j + pairs) * PER;
    u.rot = u.two || (a.interleaved && u.e < a.rot);
    u.from = (u.h < a.nq ? q + u.h * HD : k + (u.h - a.nq) * HD) + u.e;
    return u;
  };
  auto store = [&](const Unit &u, int e, const float (&x)[PER]) {
    if (u.h < a.nq) {
      T y[PER];
#pragma unroll
      for (int n = 0; n < PER; ++n) y[n] = (T)x[n];
      *(u32x4 *)(qo + u.h * HD + e) = *(const u32x4 *)y;
    } else {
      const bool key = u.h < a.nq + c.n_kv_heads;
      C y[PER];
#pragma unroll
      for (int n = 0; n < PER; ++n) y[n] = (C)x[n];
      *(u32x4 *)((key ? ko : vo) + (u.h - a.nq - (key ? 0 : c.n_kv_heads)) * head + e) = *(const u32x4 *)y;
    }
  };
  const int apart = a.rot / 2;
  bool first = true;
  for (int i = threadIdx.x; i < all || first; i += kRopeThreads * kRopeUnits) {
    Unit u[kRopeUnits];
    u32x4 w[kRopeUnits][2];
#pragma unroll
    for (int n = 0; n < kRopeUnits; ++n)
      if (i + n * kRopeThreads < all) {
        u[n] = unit(i + n * kRopeThreads);
        w[n][0] = *(const u32x4 *)u[n].from;
        if (u[n].two) w[n][1] = *(const u32x4 *)(u[n].from + apart);
      }
    if (first) {                                                 // (the angles, while the first rows are on their way)
      if ((int)threadIdx.x < apart) cs[threadIdx.x] = turn(p, a.inv_freq[threadIdx.x], a.mscale);
      __syncthreads();
      first = false;
    }
#pragma unroll
    for (int n = 0; n < kRopeUnits; ++n)
      if (i + n * kRopeThreads < all) {
        float x[PER], y[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) { x[e] = (float)((const T *)&w[n][0])[e]; }
        if (u[n].two) {
#pragma unroll
          for (int e = 0; e < PER; ++e) {
            const float z = (float)((const T *)&w[n][1])[e];
            const float2 f = cs[u[n].e + e];
            y[e] = z * f.x + x[e] * f.y;
            x[e] = x[e] * f.x - z * f.y;
          }
          store(u[n], u[n].e + apart, y);
        } else if (u[n].rot) {
#pragma unroll
          for (int e = 0; e < PER; e += 2) {
            const float2 f = cs[(u[n].e + e) / 2];
            const float z = x[e + 1];
            x[e + 1] = z * f.x + x[e] * f.y;
            x[e] = x[e] * f.x - z * f.y;
          }
        }
        store(u[n], u[n].e, x);
      }
  }
}

// ------------------------------------------------------------------ attention
//
// Rows.  The new tokens of a sequence and the rep query heads that share a key head make count * rep rows of one product:
// row R is head R % rep of new token R / rep.  Sixteen neighbouring rows are a tile.
// Keys.  What any row of a tile can see is [0, hs) and [low, end): its keys are counted through both, i = 0 .. hs + end - low - 1.

struct AttnArgs {
  const void *q;
  void *out;
  long long q_stride, out_stride;
  int nq, rep;                            // query heads, and how many of them share a key head
  Div by_rep;
  float scale2;                           // scale * log2 e
  int window, sinks;                      // (no window: sinks is 0)
  int n_splits, split_len, tiles, tile_rows;   // of the keys; tiles of rows per sequence and key head
  int turn_s, turn_z;                     // see work_of
  int max_new;                            // new tokens of a sequence beyond these are left out
  float *part_o;                          // [n_seq][max_new][nq][n_splits][HD], where a tile has several splits
  float2 *part_ml;                        // [n_seq][max_new][nq][n_splits] maximum (base 2) and sum
  unsigned int *tickets;                  // [sequences x key heads x tiles] workgroups that are done; zero between calls (null: a
                                          // launch of its own joins the splits)
};

struct Span {                             // the keys of a tile of rows
  int first, last;                        // positions of its first and its last row's token
  int hs, low, n;
  __device__ __forceinline__ int pos(int i) const { return i < hs ? i : i - hs + low; }
  // Index of position p >= low.
  __device__ __forceinline__ int at(int p) const { return p - low + hs; }
};
// What the row of a token at position p sees of a tile's keys, by index: those up to `to`, of these from `from` on and below
// `sinks` (the same for all rows).  As bits of the 32 keys from index `base` on:
struct Sight {
  int to, from, sinks;
  static __device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
  __device__ __forceinline__ uint32_t bits(int base) const { return below(to + 1 - base) & (~below(from - base) | below(sinks - base)); }
};
// rows r0 .. r1 of a sequence with `count` new tokens
__device__ __forceinline__ Span span_of(const Batch &b, const AttnArgs &a, int len, int count, int r0, int r1) {
  Span s;
  s.first = new_position(len, count, a.by_rep.quot(r0));
  s.last = new_position(len, count, a.by_rep.quot(r1));
  const int end = min(s.last + 1, b.cap);
  s.low = a.window ? max(0, s.first - a.window + 1) : 0;
  s.hs = max(0, min(min(a.sinks, s.low), end));
  s.n = s.hs + max(0, end - s.low);
  return s;
}
__device__ __forceinline__ Sight sight_of(const AttnArgs &a, const Span &s, int p) {
  return Sight{s.at(p), a.window ? max(0, s.at(max(p, -1) - a.window + 1)) : 0, max(s.hs, s.at(a.sinks))};
}
// Splits of a tile that have keys, at least one; the last split of a launch takes what is left.
__device__ __forceinline__ int splits_of(const AttnArgs &a, int n) { return min(a.n_splits, max(1, (n + a.split_len - 1) / a.split_len)); }

// Workgroup -> (tile, sequence, split, key head): the key heads next to each other (eight of them are the eight XCDs, so that the
// tiles of the same keys meet in one L2), then the splits, the sequences, and the tiles, the last, which sees most keys, first.
// Workgroups go to the XCDs in turn, within one to its four shader engines in turn, and one that has no place on its engine holds up all
// behind it.  So the order of the sequences, and of the splits in one, turns by one each time they come back to the same engines
// (2^turn rounds): else the longest of four sequences has one engine in four, and the empty tiles and splits of short ones leave the
// others idle (8B shape, us, without / with: prompts of 2048, 2015, 551 and 513 tokens 181 / 122, of eight of 366 .. 1024 81 / 64, single
// tokens of 32 sequences of 1024 .. 4096 82 / 77).
__device__ __forceinline__ void work_of(const Cache &c, const Batch &b, const AttnArgs &a, int &tile, int &s, int &z, int &head) {
  const unsigned u = blockIdx.x / c.n_kv_heads, v = u / a.n_splits, t = v / b.n_seq;
  head = blockIdx.x % c.n_kv_heads;
  z = (u + (v >> a.turn_z)) % a.n_splits;
  s = (v + (t >> a.turn_s)) % b.n_seq;
  tile = a.tiles - 1 - t;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));

// What a type of pages is multiplied with.  16-bit: D[16 x 16] += A[16 x 32] B[32 x 16], lane l has A's row l % 16 and B's
// column l % 16, in both the contraction's elements 8 (l / 16) .. + 7, and D's rows 4 (l / 16) .. + 3 of column l % 16.  fp32: four
// elements of the contraction, one in each quarter of the wavefront.
template <class C> struct Mat;
template <> struct Mat<__bf16> {
  static constexpr int kKeys = 32;        // keys of a step
  static constexpr float kBias = 0.f, kLazy = 8.f, kLazyBias = 0.f;
  static constexpr bool kSplitP = true;   // probabilities as a sum of two bf16 numbers (see Step)
  static __device__ __forceinline__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y}); }
  static __device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
  static __device__ __forceinline__ float add_pair(uint32_t w, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), bf16x2{(__bf16)1.f, (__bf16)1.f}, c, false);
  }
  static constexpr uint32_t kExp = 0x7f80u;
};
template <> struct Mat<_Float16> {
  static constexpr int kKeys = 32;
  // probabilities times 2^15: fp16's normal numbers then reach down to 2^-29 of the most likely key's
  static constexpr float kBias = 15.f;
  // (where the maximum may lag behind by kLazy)
  static constexpr float kLazy = 8.f, kLazyBias = 7.f;
  static constexpr bool kSplitP = false;  // (their 11 bits are eight times finer than the result's)
  static __device__ __forceinline__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) { return __builtin_bit_cast(uint32_t, half2v{(_Float16)x, (_Float16)y}); }
  static __device__ __forceinline__ float low(uint32_t w) { return (float)__builtin_bit_cast(half2v, w).x; }
  static __device__ __forceinline__ float high(uint32_t w) { return (float)__builtin_bit_cast(half2v, w).y; }
  static __device__ __forceinline__ float add_pair(uint32_t w, float c) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, w), half2v{(_Float16)1.f, (_Float16)1.f}, c, false);
  }
  static constexpr uint32_t kExp = 0x7c00u;
};
template <> struct Mat<float> {
  static constexpr int kKeys = 16;
  static constexpr float kBias = 0.f;
  static __device__ __forceinline__ f32x4 mul1(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
};

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
// a 32-bit word of the pages' type with its elements that are not finite as zeros
template <class C>
__device__ __forceinline__ uint32_t finite_only(uint32_t w) {
  if constexpr (sizeof(C) == 4) return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
  else {
    constexpr uint32_t e = Mat<C>::kExp;
    if ((w & e) == e) w &= 0xffff0000u;
    if ((w & (e << 16)) == (e << 16)) w &= 0xffffu;
    return w;
  }
}

struct False { static constexpr bool value = false; };
struct True { static constexpr bool value = true; };

// E neighbouring elements of a row that is divided by its sum, rounded once.  A sum of zero (nothing was seen, or only scores of
// -infinity) makes a row of zeros, also where a value that counts for nothing is not finite.
template <class T, int E>
__device__ __forceinline__ void store_row(T *to, const float (&v)[E], float sum) {
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  T x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = (T)(sum == 0.f ? 0.f : v[e] * f);
  if constexpr (sizeof(x) >= 16) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(x) / 16; ++i) ((u32x4 *)to)[i] = ((const u32x4 *)x)[i];
  } else {
    *(u32x2 *)to = *(const u32x2 *)x;
  }
}

// Attention of a tile of 16 rows over one split of its keys: one workgroup of four wavefronts, which take steps of
// Mat::kKeys keys in turn and join at the end.
//
// Bound: the stream of keys and values (a key head's are read once for the rows that share it).  A lane loads whole 16-byte pieces
// in the order in which the matrix instruction wants keys: row l % 16, pieces l / 16 + 4 j (the order of the contraction is free as
// long as the queries have the same), the next step's while this one is worked on; no barrier, each wavefront for itself.
// The product is S^T = K Q^T, so that a row's scores lie along a lane's registers: its running maximum moves seldom, and only then are the
// lanes of a row asked and O rescaled.  P^T is then in the order that O^T += V^T P^T wants its right operand in; V^T comes out of
// the wavefront's own LDS, whose transposing read gives a lane four keys of one element.
// LDS pieces lie in an order by row (swizzle), so that neither side meets in one bank.
// 8B shape: one sequence of 131071 positions, 537 MB, 93 us, 5.8 TB/s (a read alone reaches 6.8; two workgroups a CU, all 256 registers of a lane:
// steps of 16 keys and three workgroups are 1 % faster there and 18 % slower for 16 sequences of 1200); 32 sequences of up to 4096 76 us,
// 4.6 TB/s, what is missing there is that sequences differ; one of 512 8.1 us, of which the keys are 1: start, length, entries, rows,
// tickets, partial results one after the other.  fp32 prompts: 68 TFLOP/s of 135, the L2's rate for keys that every 16 rows read again.
template <class C, int HD>
struct Tile {
  typedef Mat<C> M;
  static constexpr int KB = M::kKeys / 16;               // blocks of 16 keys in a step
  static constexpr int ES = sizeof(C), PER = 16 / ES;    // elements of a 16-byte piece
  static constexpr int NP = HD / PER / 4;                // pieces of a lane in a row
  static constexpr int ROW = HD * ES;                    // bytes
  static constexpr int LDS = M::kKeys * ROW;             // of a wavefront
  static constexpr int ND = HD / 16;
  struct Data { u32x4 k[KB][NP], v[KB][NP]; };
  static __device__ __forceinline__ int swizzle(int row, int piece) {
    if constexpr (ES == 4) return piece ^ (((row >> 2) & 3) << 2);
    else if constexpr (HD == 128) return piece ^ (((row & 7) << 1) | ((row >> 3) & 1));
    else return piece ^ ((((row >> 1) & 3) << 1) | ((row >> 3) & 1));
  }
  static __device__ __forceinline__ int at(int row, int piece) { return row * ROW + swizzle(row, piece) * 16; }
};

constexpr int kAttnWaves = 4, kAttnThreads = 64 * kAttnWaves;
constexpr int kJoinAtOnce = 4;            // parts of a row that a thread fetches at once
// Eight bytes at agent scope
__device__ __forceinline__ void put_through(float *to, float x, float y) {
  __hip_atomic_store((unsigned long long *)to, __builtin_bit_cast(unsigned long long, make_float2(x, y)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_past(const float2 *from) {
  return __builtin_bit_cast(float2, __hip_atomic_load((const unsigned long long *)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// a wavefront's result in its LDS: 16 rows of HD fp32 numbers, 16-byte pieces in an order by row
template <int HD>
__device__ __forceinline__ int res_at(int row, int piece) { return row * HD + (piece ^ row) * 4; }

// E elements of a row from its parts, in their order
template <int HD, int E>
__device__ __forceinline__ void join_parts(const AttnArgs &a, long long first_part, int parts, int e0, float (&v)[E], float &sum) {
  float big = -INFINITY;
  sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = 0.f;
  for (int y0 = 0; y0 < parts; y0 += kJoinAtOnce) {              // (as many on their way at once)
    float2 ml[kJoinAtOnce], x[kJoinAtOnce][E / 2];
#pragma unroll
    for (int y = 0; y < kJoinAtOnce; ++y) {
      const long long part = first_part + min(y0 + y, parts - 1);
      ml[y] = get_past(a.part_ml + part);
#pragma unroll
      for (int e = 0; e < E; e += 2) x[y][e / 2] = get_past((const float2 *)(a.part_o + part * HD + e0 + e));
    }
    float now = big;
#pragma unroll
    for (int y = 0; y < kJoinAtOnce; ++y) now = fmaxf(now, ml[y].x);
    const float before = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(big - now);
    sum *= before;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= before;
    big = now;
#pragma unroll
    for (int y = 0; y < kJoinAtOnce; ++y)
      if (y0 + y < parts) {
        const float f = big == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[y].x - big);
        sum += f * ml[y].y;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          v[e] += f * x[y][e / 2].x;
          v[e + 1] += f * x[y][e / 2].y;
        }
      }
  }
}

template <class T, class C, int HD>
__global__ __launch_bounds__(kAttnThreads, HD == 64 ? 3 : 2) void k_attn_split(Cache c, Batch b, AttnArgs a) {
  typedef Tile<C, HD> W;
  typedef Mat<C> M;
  constexpr int KB = W::KB, NP = W::NP, ND = W::ND, PER = W::PER;
  constexpr int AREA = W::LDS > 64 * HD ? W::LDS : 64 * HD;     // of a wavefront: its values, then its result
  __shared__ __align__(16) char lds[kAttnWaves * AREA];
  __shared__ float2 res_ml[kAttnWaves][16];
  int tile, s, z, head;
  work_of(c, b, a, tile, s, z, head);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 16, g = lane / 16;
  // Without a window the first steps' keys do not depend on the length: their entries come with it, not behind it
  int early[2][KB];
#pragma unroll
  for (int it = 0; it < 2; ++it)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      early[it][kb] = b.table[(long long)s * b.table_stride +
                              min(c.by_page.quot(z * a.split_len + (it * kAttnWaves + wave) * M::kKeys + kb * 16 + col), b.max_pages - 1)];
  int first_token, count;
  seq_tokens(b, s, first_token, count);
  const int rows = min(count, a.max_new) * a.rep, r0 = tile * 16;
  if (r0 >= rows) return;
  const int r1 = min(r0 + 15, rows - 1);
  const Span sp = span_of(b, a, length_of(b, s), count, r0, r1);
  const int parts = splits_of(a, sp.n);
  if (z >= parts) return;
  const int i0 = z * a.split_len, i1 = z == parts - 1 ? sp.n : min(sp.n, i0 + a.split_len);

  // this lane's row: its query in the order of the contraction, its position
  const int r = min(r0 + col, r1), tok = a.by_rep.quot(r), qh = head * a.rep + (r - tok * a.rep);
  const int mypos = new_position(length_of(b, s), count, tok);
  const T *qrow = (const T *)a.q + (long long)(first_token + tok) * a.q_stride + (long long)qh * HD;
  u32x4 qf[NP];
  float sc = a.scale2;
  if constexpr (sizeof(T) == sizeof(C) && !(sizeof(C) == 2 && M::kBias != 0.f)) {
#pragma unroll
    for (int j = 0; j < NP; ++j) qf[j] = *(const u32x4 *)(qrow + (g + 4 * j) * PER);
  } else {
    // bf16 queries over fp16 pages: a row is divided by a power of two so that its largest element is below 2 (what
    // gets below fp16's numbers is below 2^-24 of that), which goes into the row's scale
    u32x4 w[NP];
    float big = 0.f;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      w[j] = *(const u32x4 *)(qrow + (g + 4 * j) * PER);
      for (int e = 0; e < 4; ++e)
        big = fmaxf(big, fmaxf(fabsf(Mat<__bf16>::low(w[j][e])), fabsf(Mat<__bf16>::high(w[j][e]))));
    }
    big = fmaxf(big, __shfl_xor(big, 16));
    big = fmaxf(big, __shfl_xor(big, 32));
    const int ex = big > 0.f && !not_finite(big) ? ilogbf(big) : 0;
    sc = ldexpf(sc, ex);
#pragma unroll
    for (int j = 0; j < NP; ++j)
      for (int e = 0; e < 4; ++e)
        qf[j][e] = M::pack(ldexpf(Mat<__bf16>::low(w[j][e]), -ex), ldexpf(Mat<__bf16>::high(w[j][e]), -ex));
  }

  const C *kp = (const C *)c.k + (long long)head * c.page_size * HD, *vp = (const C *)c.v + (long long)head * c.page_size * HD;
  char *mine = lds + wave * AREA;
  f32x4 o[ND];
  float m, l;

  // The entries of step `it`'s keys, a step ahead of the loads that need them
  const int steps = (i1 - i0 + kAttnWaves * M::kKeys - 1) / (kAttnWaves * M::kKeys);
  auto key_of = [&](int it, int kb) { return i0 + (it * kAttnWaves + wave) * M::kKeys + kb * 16 + col; };
  auto entries = [&](int it, int (&e)[KB]) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      e[kb] = b.table[(long long)s * b.table_stride + c.by_page.quot(sp.pos(min(key_of(it, kb), i1 - 1)))];
  };
  // Rows without a page, or behind the split's end, are page 0's first (any memory of the cache will do)
  auto fetch = [&](int it, const int (&e)[KB], typename W::Data &d, uint32_t &there) {
    there = 0;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int i = key_of(it, kb), p = sp.pos(min(i, i1 - 1));
      const bool ok = i < i1 && (unsigned)e[kb] < (unsigned)c.n_pages;
      const long long at = ok ? (long long)e[kb] * c.page_stride + (long long)(p - c.by_page.quot(p) * c.page_size) * HD : 0;
      there |= (uint32_t)(__ballot(ok) & 0xffffu) << (16 * kb);
#pragma unroll
      for (int j = 0; j < NP; ++j) d.k[kb][j] = *(const u32x4 *)(kp + at + (g + 4 * j) * PER);
#pragma unroll
      for (int j = 0; j < NP; ++j) d.v[kb][j] = *(const u32x4 *)(vp + at + (g + 4 * j) * PER);
    }
  };

  // CAREFUL: values that are not finite stand where some rows see them and others do not (0 times them would be NaN):
  // they are taken out of the product and added to the rows that see them.  Everything else has the same bits.
  auto work = [&](auto careful_, int it, typename W::Data &d, uint32_t there) {
    constexpr bool CAREFUL = decltype(careful_)::value;
    f32x4 sc_[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      sc_[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        if constexpr (W::ES == 2) sc_[kb] = M::mul(d.k[kb][j], qf[j], sc_[kb]);
        else {
#pragma unroll
          for (int e = 0; e < 4; ++e) sc_[kb] = M::mul1(__uint_as_float(d.k[kb][j][e]), __uint_as_float(qf[j][e]), sc_[kb]);
        }
      }
    }
    // does every row see every key of this step?
    const int base = i0 + (it * kAttnWaves + wave) * M::kKeys, lo = sp.pos(base), hi = sp.pos(min(base + M::kKeys, i1) - 1);
    const bool all = __popc(there) == M::kKeys && hi <= sp.first && (!a.window || lo > sp.last - a.window || hi < a.sinks);
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        float v = sc_[kb][n] * sc;
        if (!all) {
          const int key = kb * 16 + 4 * g + n, p = sp.pos(base + key);
          const bool ok = (there >> key & 1) && p <= mypos && (!a.window || p > mypos - a.window || p < a.sinks);
          v = ok ? v : -INFINITY;
        }
        sc_[kb][n] = v;
        top = fmaxf(top, v);
      }
    if (__any(top > m)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float now = fmaxf(m, top), f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= f;
#pragma unroll
      for (int t = 0; t < ND; ++t) o[t] *= f;
    }
    const float off = (m == -INFINITY ? 0.f : m) - M::kBias;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float p = __builtin_amdgcn_exp2f(sc_[kb][n] - off);
        sc_[kb][n] = p;
        l += p;
      }
    // values: rows that no row of the tile sees are zeros, whatever their bits
    if (!all) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const int p = sp.pos(base + kb * 16 + col);
        const bool some = (there >> (kb * 16 + col) & 1) && p <= sp.last && (!a.window || p > sp.first - a.window || p < a.sinks);
#pragma unroll
        for (int j = 0; j < NP; ++j) d.v[kb][j] = some ? d.v[kb][j] : u32x4{0, 0, 0, 0};
      }
    }
    auto put = [&] {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int j = 0; j < NP; ++j) *(u32x4 *)(mine + W::at(kb * 16 + col, g + 4 * j)) = d.v[kb][j];
      __builtin_amdgcn_wave_barrier();
    };
    put();
    if constexpr (CAREFUL) {
      for (int key = 0; key < M::kKeys; ++key) {
        const int p = sp.pos(base + key);
        const bool ok = (there >> key & 1) && p <= mypos && (!a.window || p > mypos - a.window || p < a.sinks);
        for (int t = 0; t < ND; ++t)
          for (int n = 0; n < 4; ++n) {
            const int e = t * 16 + 4 * g + n;
            const float v = (float)*(const C *)(mine + W::at(key, e / PER) + e % PER * W::ES);
            if (ok && not_finite(v)) o[t][n] += v;
          }
      }
      __builtin_amdgcn_wave_barrier();
      for (int kb = 0; kb < KB; ++kb)
        for (int j = 0; j < NP; ++j)
          for (int e = 0; e < 4; ++e) d.v[kb][j][e] = finite_only<C>(d.v[kb][j][e]);
      put();
    }
    if constexpr (W::ES == 2) {
      // P^T: the keys 4 g .. of both blocks.  A bf16 probability leaves out 2^-9 of itself, as much as the result's own rounding
      // does; what it leaves out is a second product, which costs nothing beside the stream
      u32x4 hi, rest;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float p0 = sc_[w / 2][2 * (w & 1)], p1 = sc_[w / 2][2 * (w & 1) + 1];
        hi[w] = M::pack(p0, p1);
        if constexpr (M::kSplitP) rest[w] = M::pack(p0 - M::low(hi[w]), p1 - M::high(hi[w]));
      }
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        u32x4 v;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const int row = kb * 16 + 4 * g + col / 4;
          const s16x4 four = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4 *)(mine + W::at(row, 2 * t + (col >> 1 & 1)) + (col & 1) * 8));
          const u32x2 w2 = __builtin_bit_cast(u32x2, four);
          v[2 * kb] = w2.x;
          v[2 * kb + 1] = w2.y;
        }
        o[t] = M::mul(v, hi, o[t]);
        if constexpr (M::kSplitP) o[t] = M::mul(v, rest, o[t]);
      }
    } else {
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int row = 4 * g + n, e = t * 16 + col;
          o[t] = M::mul1(*(const float *)(mine + W::at(row, e / 4) + e % 4 * 4), sc_[0][n], o[t]);
        }
    }
    __builtin_amdgcn_wave_barrier();
  };

  auto pass = [&](auto careful_) {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < ND; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (a wavefront whose keys are beyond the end works on none that any row sees)
    if (steps == 0) return;
    int e[KB], e1[KB];
    typename W::Data d, d1;
    uint32_t there, there1;
    if (a.window) {
      entries(0, e);
      entries(1, e1);
    } else {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) { e[kb] = early[0][kb]; e1[kb] = early[1][kb]; }
    }
    fetch(0, e, d, there);
    for (int it = 0; it + 1 < steps; ++it) {
      entries(it + 2, e);
      fetch(it + 1, e1, d1, there1);
      work(careful_, it, d, there);
      d = d1;
      there = there1;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) e1[kb] = e[kb];
    }
    work(careful_, steps - 1, d, there);
  };
  pass(False{});
  float sick = 0.f;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int n = 0; n < 4; ++n) sick += o[t][n] * 0.f;
  if (__any(sick != 0.f)) pass(True{});

  // the wavefronts' results, added in their order
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  float *res = (float *)lds;
  constexpr int LD = AREA / 4;
#pragma unroll
  for (int t = 0; t < ND; ++t) *(f32x4 *)(res + wave * LD + res_at<HD>(col, 4 * t + g)) = o[t];
  if (g == 0) res_ml[wave][col] = make_float2(m, l);
  __syncthreads();
  constexpr int E = HD * 16 / kAttnThreads > 4 ? HD * 16 / kAttnThreads : 4, LANES = HD / E;   // elements of a thread, threads of a row
  const int row = threadIdx.x / LANES, e0 = threadIdx.x % LANES * E;
  static_assert(16 * LANES == kAttnThreads, "every thread has a part of a row");
  const bool have = r0 + row <= r1;
  float big = -INFINITY, sum = 0.f, v[E];
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) big = fmaxf(big, res_ml[w][row].x);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = 0.f;
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) {
    const float2 ml = res_ml[w][row];
    const float f = big == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml.x - big);
    sum += f * ml.y;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const f32x4 x4 = *(const f32x4 *)(res + w * LD + res_at<HD>(row, (e0 + e) / 4));
#pragma unroll
      for (int n = 0; n < 4; ++n) v[e + n] += f * x4[n];
    }
  }
  const int to = a.by_rep.quot(min(r0 + row, r1)), oh = head * a.rep + (min(r0 + row, r1) - to * a.rep);
  const long long t = first_token + to;
  T *const out = (T *)a.out + t * a.out_stride + (long long)oh * HD + e0;
  if (parts == 1) {
    if (have) store_row<T, E>(out, v, sum);
    return;
  }
  // Parts cross XCDs, whose L2s are not coherent: they are written through and read past the L2, eight bytes at a time
  const long long first_part = (((long long)s * a.max_new + to) * a.nq + oh) * a.n_splits;
  if (have) {
#pragma unroll
    for (int e = 0; e < E; e += 2) put_through(a.part_o + (first_part + z) * HD + e0 + e, v[e], v[e + 1]);
    if (e0 == 0) put_through((float *)(a.part_ml + first_part + z), big, sum);
  }
  if (!a.tickets) return;
  // The last workgroup of the tile joins the parts, in their order
  __shared__ unsigned int order;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  unsigned int *const ticket = a.tickets + ((long long)s * c.n_kv_heads + head) * a.tiles + tile;
  if (threadIdx.x == 0) order = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (order != (unsigned)parts - 1) return;
  if (threadIdx.x == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (!have) return;
  join_parts<HD, E>(a, first_part, parts, e0, v, sum);
  store_row<T, E>(out, v, sum);
}

// ------------------------------------------------------------------ attention of many rows (16-bit pages)
//
// Bound: the matrix cores and the vector instructions (exponentials above all) about alike, 48 % and 49 % of a SIMD's cycles, neither of them
// full: its wavefronts wait for a quarter to a third of theirs.  The clock is 1.84 .. 2.07 GHz meanwhile (a decode call's 2.44 .. 2.57).  A wavefront holds 32 rows in fewer than 256 registers, all of them general ones,
// so that two workgroups of 128 rows are on a CU (three at head size 64, whose few spilled registers lie outside the steps: 4096
// tokens 114 / 98 us) and one's waits, beginning and end lie beside the other's products.  (64 rows a
// wavefront, one to a SIMD, read LDS half as often, but nothing runs beside their waits: us, 64 rows / 32 rows, 8B shape: 4096 tokens
// 163 / 148, 2048 behind 16384 640 / 615, five windows of 1024 223 / 171, prompts of 2048, 2015, 551 and 513 122 / 102; 1B shape 4096
// tokens 146 / 98.)
// What would wait for each other is taken from different steps of 32 keys: step n multiplies S(n+1) = K Q^T, takes the exponentials
// of S(n), and adds P(n-1) V, three things that do not depend on each other.
// O is therefore rescaled one step after the maximum has moved (pend); it moves when a score is 2^kLazy times as likely as
// what was the maximum (one of 32 rows has a new maximum in most steps, and rescaling takes half as long as the step).
// A probability is rounded once to the pages' type, and the sum is of what is multiplied: over bf16 pages that leaves out up to half a step of the
// result (4096 tokens: off by 2.1e-3 of the norm, 1.6e-3 with fp32 ones); a second product, as in k_attn_split, would cost a third of the time.
// Keys and values go from memory straight into LDS (no registers, AHEAD steps in flight), in rings, one barrier a step; where a key's
// row lies is looked up for CHUNK steps at once.
// 8B shape, 4096 tokens: 148 .. 158 us by the box, 870 .. 930 TFLOP/s; 2048 behind 16384 615 us, 950; the largest matrix products of the library reach 1250.
template <class C, int HD>
struct Many {
  typedef Mat<C> M;
  static constexpr int KEYS = 32, WROWS = 32, ROWS = 4 * WROWS;
  static constexpr int AHEAD = 2, KRING = 2, VRING = 4;  // in steps
  static constexpr int CHUNK = 16;                       // steps whose rows are looked up at once
  static constexpr int ROW = HD * 2, PIECES = HD / 8;    // bytes and 16-byte pieces of a row
  static constexpr int KS = HD / 16, DB = HD / 32;
  static constexpr int STAGE = KEYS * ROW;
  static constexpr int V = KRING * STAGE, PLACES = V + VRING * STAGE, THERE = PLACES + 2 * CHUNK * KEYS * 16, LDS = THERE + 2 * CHUNK * 4;
  static constexpr int PER = 64 / PIECES, NL = 8 / PER;  // a wavefront loads eight rows, PER of them at a time
  // Pieces of a row lie in an order by row: neighbouring rows of keys, and the four rows (of 64 bytes each) that half a wavefront's
  // transposing read of values takes, meet in different banks (conflicts: 1 % of LDS cycles; values in pairs of pieces 30 %)
  static __device__ __forceinline__ int k_swizzle(int row) { return HD == 128 ? row & 15 : row & 7; }
  static __device__ __forceinline__ int v_swizzle(int row) {
    return HD == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 3) << 1) | ((row >> 2) & 1);
  }
  static __device__ __forceinline__ int k_at(int row, int piece) { return row * ROW + (piece ^ k_swizzle(row)) * 16; }
  static __device__ __forceinline__ int v_at(int row, int piece) { return row * ROW + (piece ^ v_swizzle(row)) * 16; }
};
// 16 bytes a lane from memory to LDS, the lanes' one after the other from byte `lds` on.  Counts on vmcnt; no register is written but m0, which the
// compiler keeps nothing in (it is reserved: it sets it in front of each use of its own, and takes no clobber of it).
__device__ __forceinline__ void load_lds16(uint32_t lds, const void *from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from));
}
template <int N>
__device__ __forceinline__ void wait_and_meet() {        // all but the last N loads done, by every wavefront
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
__device__ const u32x4 g_zero_row[16] = {};
typedef float f32x16 __attribute__((ext_vector_type(16)));
template <class C>
__device__ __forceinline__ f32x16 mul32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (Mat<C>::kSplitP)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

template <class T, class C, int HD>
__global__ __launch_bounds__(256, HD == 64 ? 3 : 2) void k_attn_many(Cache c, Batch b, AttnArgs a) {
  typedef Many<C, HD> W;
  typedef Mat<C> M;
  constexpr int KS = W::KS, DB = W::DB, NL = W::NL, KEYS = W::KEYS;
  extern __shared__ __align__(1024) char lds[];
  char *const vlds = lds + W::V;
  typedef unsigned long long Place __attribute__((ext_vector_type(2)));
  Place *const places = (Place *)(lds + W::PLACES);
  uint32_t *const there_of = (uint32_t *)(lds + W::THERE);
  int tile, s, z, head;
  work_of(c, b, a, tile, s, z, head);
  int first_token, count;
  seq_tokens(b, s, first_token, count);
  const int rows = min(count, a.max_new) * a.rep, r0 = tile * W::ROWS;
  if (r0 >= rows) return;
  const int r1 = min(r0 + W::ROWS - 1, rows - 1), len = length_of(b, s);
  const Span sp = span_of(b, a, len, count, r0, r1);
  const int parts = splits_of(a, sp.n);
  if (z >= parts) return;
  const int i0 = z * a.split_len, i1 = z == parts - 1 ? sp.n : min(sp.n, i0 + a.split_len);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 32, h = lane / 32;
  const int steps = (i1 - i0 + KEYS - 1) / KEYS;

  // this wavefront's rows: rows behind the last repeat it
  const int w0 = min(r0 + wave * W::WROWS, r1), w1 = min(w0 + W::WROWS - 1, r1);
  const int first = len - count + a.by_rep.quot(w0), last = len - count + a.by_rep.quot(w1);
  const int my_slot = lane % W::PIECES;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  // Their queries in the operand's order.  (Through LDS, in whole rows of memory, they take as long: 4500 cycles, on the way with
  // the table's entries.)
  u32x4 qf[KS];
  float sc = a.scale2;
  const int r = min(r0 + wave * W::WROWS + col, r1), tok = a.by_rep.quot(r);
  const Sight sight = sight_of(a, sp, len - count + tok);
  const T *q = (const T *)a.q + (long long)(first_token + tok) * a.q_stride + (long long)(head * a.rep + r - tok * a.rep) * HD;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const u32x4 *)(q + (2 * ks + h) * 8);
  auto queries = [&] {
    if constexpr (!M::kSplitP) {                         // fp16 pages: see k_attn_split
      float big = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        for (int e = 0; e < 4; ++e)
          big = fmaxf(big, fmaxf(fabsf(Mat<__bf16>::low(qf[ks][e])), fabsf(Mat<__bf16>::high(qf[ks][e]))));
      big = fmaxf(big, __shfl_xor(big, 32));
      const int ex = big > 0.f && !not_finite(big) ? ilogbf(big) : 0;
      sc = ldexpf(sc, ex);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        for (int e = 0; e < 4; ++e)
          qf[ks][e] = M::pack(ldexpf(Mat<__bf16>::low(qf[ks][e]), -ex), ldexpf(Mat<__bf16>::high(qf[ks][e]), -ex));
    }
    sc = fmaxf(sc, 1e-37f);                              // (-infinity times it stays one)
  };

  const u32x4 *kp = (const u32x4 *)((const C *)c.k + (long long)head * c.page_size * HD), *vp = (const u32x4 *)((const C *)c.v + (long long)head * c.page_size * HD);
  const int *row_of_table = b.table + (long long)s * b.table_stride;
  constexpr int CK = W::CHUNK * KEYS;
  // Where the rows of CHUNK steps lie, and a bit a key.  What has no row (no page, behind the end): keys of page 0, which no
  // score counts, and values of zeros, whatever the bits of the cache there
  auto look_up = [&](int chunk) {
#pragma unroll
    for (int j = 0; j < CK / 256; ++j) {
      const int k = j * 256 + (int)threadIdx.x, i = chunk * CK + k, p = sp.pos(min(i0 + i, i1 - 1)), page = c.by_page.quot(p);
      const int e = row_of_table[page];
      const bool ok = i0 + i < i1 && (unsigned)e < (unsigned)c.n_pages;
      const unsigned long long at = (unsigned long long)(uint32_t)e * c.page_pieces + (uint32_t)((p - page * c.page_size) * W::PIECES);
      places[(chunk & 1) * CK + k] = Place{(uintptr_t)(kp + (ok ? at : 0)), (uintptr_t)(ok ? vp + at : g_zero_row)};
      const unsigned long long all = __ballot(ok);
      if (lane < 2) there_of[(chunk & 1) * W::CHUNK + (j * 256 + wave * 64) / KEYS + lane] = (uint32_t)(all >> (32 * lane));
    }
  };
  // a lane's piece of a row: in LDS it lies where the swizzle puts it
  const int my_row = wave * 8 + lane / W::PIECES;
  int k_piece[NL], v_piece[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    k_piece[j] = my_slot ^ W::k_swizzle(my_row + j * W::PER);
    v_piece[j] = my_slot ^ W::v_swizzle(my_row + j * W::PER);
  }
  const uint32_t lds0 = lds_base + wave * 8 * W::ROW;
  auto find = [&](int n, Place (&at)[NL]) {
#pragma unroll
    for (int j = 0; j < NL; ++j) at[j] = places[n % (2 * W::CHUNK) * KEYS + my_row + j * W::PER];
  };
  // (a step's keys, then its values: they are needed a step later, and a wait may leave the last of them in flight)
  auto fetch = [&](int n, const Place (&at)[NL]) {
#pragma unroll
    for (int j = 0; j < NL; ++j) load_lds16(lds0 + n % W::KRING * W::STAGE + j * W::PER * W::ROW, (const u32x4 *)at[j].x + k_piece[j]);
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      load_lds16(lds0 + W::V + n % W::VRING * W::STAGE + j * W::PER * W::ROW, (const u32x4 *)at[j].y + v_piece[j]);
    }
  };

  typedef float Scores[16];
  typedef u32x4 Probs[2];
  f32x16 o[DB];
  float m, lim, l, off, fac, top;
  bool pend;
  // Steps of which every row of this wavefront sees every key (where all pages are there): their last key is at most all_to,
  // and their first is at least all_from or their last below all_sinks, by index in the split
  const int all_to = sp.at(first) - i0, all_from = (a.window ? max(0, sp.at(max(last, -1) - a.window + 1)) : 0) - i0, all_sinks = sight.sinks - i0;

  // Step n's scores as they count: what a row does not see is -infinity.  The maximum, where that moves it.
  auto settle = [&](int n, Scores &sx, uint32_t there_) {
    const uint32_t there = __builtin_amdgcn_readfirstlane(there_);
    const int base = n * KEYS;
    if (there != 0xffffffffu || base + KEYS - 1 > all_to || (base < all_from && base + KEYS > all_sinks)) {
      const uint32_t see = (sight.bits(i0 + base) & there) >> (4 * h);
      top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sx[i] = (see >> (8 * (i / 4) + i % 4) & 1) ? sx[i] : -INFINITY;
        top = __builtin_elementwise_maximum(top, sx[i]);
      }
    }
    if (pend) {
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        o[d] *= fac;
        __builtin_amdgcn_sched_barrier(0);               // (one after the other: few registers)
      }
    }
    pend = __any(top > lim);
    if (pend) {
      // (each row by its own scores alone, whatever the others did)
      const float high = fmaxf(top, __shfl_xor(top, 32)), now = high > lim ? high : m;
      const float to = (now == -INFINITY ? 0.f : now * sc) - M::kLazyBias;
      fac = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(off - to);
      if (now == m) fac = 1.f;
      m = now;
      lim = now + M::kLazy / sc;
      off = to;
      l *= fac;
    }
  };

  // Careful: a value that is not finite stands where some rows see it and others do not (0 times it would be NaN).  Such
  // values are left out of what is multiplied and added to the rows that see them; everything else has the same bits.
  bool careful = false;
  for (;;) {
    m = lim = -INFINITY;
    l = 0.f;
    off = -M::kLazyBias;
    fac = 1.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x16{};
    pend = false;
    if (steps == 0) break;
    // (careful: this wavefront's own rows of step n, which have arrived)
    auto clean = [&](int n) {
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        uint32_t *at = (uint32_t *)(vlds + n % W::VRING * W::STAGE + (my_row + j * W::PER) * W::ROW + my_slot * 16);
#pragma unroll
        for (int w = 0; w < 4; ++w) at[w] = finite_only<C>(at[w]);
      }
    };
    look_up(0);
    // the values of step -1 are zeros
    for (int i = threadIdx.x; i < W::STAGE / 16; i += 256) *(u32x4 *)(vlds + (W::VRING - 1) * W::STAGE + i * 16) = u32x4{0, 0, 0, 0};
    wait_and_meet<0>();
#pragma unroll
    for (int n = 0; n < W::AHEAD; ++n) {
      Place at[NL];
      find(n, at);
      fetch(n, at);
    }
    if (careful) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      for (int n = 0; n < W::AHEAD; ++n) clean(n);
    } else {
      queries();
    }
    wait_and_meet<(W::AHEAD - 2) * 2 * NL + NL>();
    // The operands of a step, one after the other: keys of S(n + 1), then values of step n - 1.  The swizzle's part that
    // depends on the operand is an exclusive or with a constant, the rest is the lane's.
    const uint32_t k0 = lds_base + W::k_at(col, h);
    const uint32_t v0 = lds_base + W::V + W::v_at(4 * h + lane % 16 / 4, (lane % 32 / 16) * 2 + lane % 4 / 2) + lane % 2 * 8;
    auto operand = [&](int g, uint32_t k_step, uint32_t v_step) {
      if (g < KS) return *(__attribute__((address_space(3))) u32x4 *)(uintptr_t)(k_step ^ (uint32_t)(g * 32));
      // four keys 16 t + 8 u + 4 h .. of the element d * 32 + lane % 32
      const int t = (g - KS) / DB, d = (g - KS) % DB;
      u32x4 f;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t at = (v_step ^ (uint32_t)(d * 64 + (HD == 128 ? u * 32 : 0))) + (16 * t + 8 * u) * W::ROW;
        const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)at));
        f[2 * u] = w.x;
        f[2 * u + 1] = w.y;
      }
      return f;
    };
    // Step n with the scores s (of step n) and probabilities p (of step n - 1); leaves those of the next in s1 and p1.
    // In slots of one product, the operand of the third product after it, and a share of the vector instructions, each
    // from another stage of its chain (argument, exponential, rounding and sum), so that nothing waits.  The compiler must not mix
    // the slots: left alone it fetches each operand right in front of its products and waits for it, and takes the
    // exponentials past the branches that follow.
    auto step = [&](int n, Scores &s, Probs &p, Scores &s1, Probs &p1) {
      constexpr int SLOTS = KS + 2 * DB, PRE = 3, EACH = 16 / SLOTS;   // EACH: exponentials
      constexpr int FROM = KS + 2, PER_SLOT = (16 + SLOTS - FROM - 1) / (SLOTS - FROM);
      const uint32_t k_step = k0 + (n + 1) % W::KRING * W::STAGE, v_step = v0 + (n + W::VRING - 1) % W::VRING * W::STAGE;
      f32x16 sn;
      u32x4 f[PRE + 1];
      float x[2][2], y[2][2];                            // arguments and exponentials of a pair, by its parity
      const uint32_t there = there_of[(n + 1) % (2 * W::CHUNK)];
      Place at[NL];
      find(n + W::AHEAD, at);
#pragma unroll
      for (int g = 0; g < PRE; ++g) f[g] = operand(g, k_step, v_step);
      auto arguments = [&](int q) {
#pragma unroll
        for (int e = 0; e < 2; ++e) x[q % 2][e] = fmaf(s[2 * q + e], sc, -off);
      };
      auto round_and_add = [&](int q) {
        uint32_t w = M::pack(y[q % 2][0], y[q % 2][1]);
        l = M::add_pair(w, l);                                   // (the sum of what is multiplied: rounded alike)
        asm volatile("" : "+v"(w), "+v"(l));
        p1[q / 4][q % 4] = w;
      };
      arguments(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int slot = 0; slot < SLOTS; ++slot) {
        if (slot + PRE < SLOTS) f[(slot + PRE) % (PRE + 1)] = operand(slot + PRE, k_step, v_step);
        const u32x4 x0 = f[slot % (PRE + 1)];
        if (slot < KS) sn = mul32<C>(x0, qf[slot], slot ? sn : f32x16{});
        else o[(slot - KS) % DB] = mul32<C>(x0, p[(slot - KS) / DB], o[(slot - KS) % DB]);
#pragma unroll
        for (int e = slot * EACH; e < (slot + 1) * EACH; ++e) {
          const int q = e / 2;
          if (e % 2 == 0 && q + 1 < 8) arguments(q + 1);
          y[q % 2][e % 2] = __builtin_amdgcn_exp2f(x[q % 2][e % 2]);
          asm volatile("" : "+v"(y[q % 2][e % 2]));
          if (e % 2 == 0 && q > 0) round_and_add(q - 1);
        }
        if (slot == 4) fetch(n + W::AHEAD, at);
        // The new scores and their maxima (the one that is NaN where one of its arguments is: two of it are one instruction.  A
        // row with such a score is NaN anyway)
        if (slot >= FROM) {
#pragma unroll
          for (int e = (slot - FROM) * PER_SLOT; e < (slot - FROM + 1) * PER_SLOT && e < 16; ++e) {
            float v = sn[e];
            asm volatile("" : "+v"(v));
            s1[e] = v;
            top = e ? __builtin_elementwise_maximum(top, v) : v;
          }
          asm volatile("" : "+v"(top));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      round_and_add(7);
      settle(n + 1, s1, there);
      if ((n + W::AHEAD + 1) % W::CHUNK == 0) look_up((n + W::AHEAD + 1) / W::CHUNK);
      if (careful) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        clean(n + W::AHEAD);
      }
      wait_and_meet<(W::AHEAD - 2) * 2 * NL + NL>();
    };
    Scores s0, s1;
    Probs p0, p1;
    {
      f32x16 sn;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sn = mul32<C>(operand(ks, k0, 0), qf[ks], ks ? sn : f32x16{});
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float v = sn[i];
        asm volatile("" : "+v"(v));
        s0[i] = v;
        top = i ? __builtin_elementwise_maximum(top, v) : v;
      }
      p0[0] = p0[1] = u32x4{0, 0, 0, 0};
    }
    settle(0, s0, there_of[0]);
    wait_and_meet<(W::AHEAD - 2) * 2 * NL + NL>();               // (step 0 fetches over the keys of S(0))
    // step `steps` only adds what the last one left
    for (int n = 0; n <= steps; n += 2) {
      step(n, s0, p0, s1, p1);
      if (n == steps) break;
      step(n + 1, s1, p1, s0, p0);
    }
    wait_and_meet<0>();                                          // (nothing may land in LDS behind the end)
    if (careful) {
      // (a row whose scores here are all -infinity stays zero: see store_row)
      const bool counts = l + __shfl_xor(l, 32) != 0.f;
      for (int i = i0; i < i1; ++i) {
        int slot;
        const int page = page_of(c, b, s, sp.pos(i), slot);
        if (page < 0) continue;
        const C *row = (const C *)vp + (long long)page * c.page_stride + (long long)slot * HD + 4 * h;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e4 = 0; e4 < 16; ++e4) {
            const float v = (float)row[d * 32 + 8 * (e4 / 4) + e4 % 4];
            if (counts && (sight.bits(i) & 1) && not_finite(v)) o[d][e4] += v;
          }
      }
      break;
    }
    float sick = 0.f;                                            // (not finite if one of them is not)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) sick = __builtin_elementwise_maximum(sick, fabsf(o[d][i]));
    const bool any_sick = __any(not_finite(sick));
    if (lane == 0) there_of[wave] = any_sick;
    wait_and_meet<0>();
    if (!(there_of[0] | there_of[1] | there_of[2] | there_of[3])) break;
    wait_and_meet<0>();                                          // (read before it is written again)
    careful = true;
  }

  // Results.  A lane has four neighbouring elements of its row at a time: they go through this wavefront's part of LDS, pieces of 16 bytes in an order by row, so that memory gets whole rows.
  char *const mine = lds + wave * (W::STAGE * (parts == 1 ? 1 : 2));
  l += __shfl_xor(l, 32);
  const int from = r0 + wave * W::WROWS;                         // this wavefront's first row
  if (from <= r1) {
    // row `row` of them in memory
    int tok, qh;
    auto place = [&](int row) {
      const int r = min(from + row, r1);
      tok = a.by_rep.quot(r);
      qh = head * a.rep + r - tok * a.rep;
      return from + row <= r1;
    };
    if (parts == 1) {
      const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int piece = 4 * d + i / 4;
          *(u32x2 *)(mine + col * W::ROW + (piece ^ (col % W::PIECES)) * 16 + 8 * h) =
              u32x2{Mat<__bf16>::pack(o[d][i] * f, o[d][i + 1] * f), Mat<__bf16>::pack(o[d][i + 2] * f, o[d][i + 3] * f)};
        }
      __builtin_amdgcn_wave_barrier();
      u32x4 v[32 / W::PER];
#pragma unroll
      for (int j = 0; j < 32 / W::PER; ++j) {
        const int row = j * W::PER + lane / W::PIECES;
        v[j] = *(const u32x4 *)(mine + row * W::ROW + (my_slot ^ (row % W::PIECES)) * 16);
      }
#pragma unroll
      for (int j = 0; j < 32 / W::PER; ++j)
        if (place(j * W::PER + lane / W::PIECES))
          *(u32x4 *)((T *)a.out + (long long)(first_token + tok) * a.out_stride + (long long)qh * HD + my_slot * 8) = v[j];
    } else {
      constexpr int P = 2 * W::PIECES;                           // fp32: twice as many pieces
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int piece = 8 * d + i / 2 + h;
          *(f32x4 *)(mine + col * (2 * W::ROW) + (piece ^ (col % P)) * 16) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < 32 * P / 64; ++j) {
        const int row = j * (64 / P) + lane / P, piece = lane % P;
        const f32x4 v = *(const f32x4 *)(mine + row * (2 * W::ROW) + (piece ^ (row % P)) * 16);
        if (place(row)) *(f32x4 *)(a.part_o + ((((long long)s * a.max_new + tok) * a.nq + qh) * a.n_splits + z) * HD + piece * 4) = v;
      }
      // (maxima in base 2, as k_attn_split has them)
      if (h == 0 && place(col))
        a.part_ml[(((long long)s * a.max_new + tok) * a.nq + qh) * a.n_splits + z] = make_float2(m == -INFINITY ? -INFINITY : off + M::kLazyBias, l);
    }
  }
}

// Row w of the partial results: head h of new token i of sequence s.  Its number of splits (0: no row, 1: it is done already), and its
// place in the output.
__device__ __forceinline__ int parts_of(const Batch &b, const AttnArgs &a, long long w, int head_dim, long long &out) {
  const int h = (int)(w % a.nq), i = (int)(w / a.nq % a.max_new), s = (int)(w / a.nq / a.max_new);
  if (s >= b.n_seq) return 0;
  int first, count;
  seq_tokens(b, s, first, count);
  if (i >= count) return 0;
  const int r = i * a.rep + h % a.rep, r0 = r - r % a.tile_rows;
  out = (long long)(first + i) * a.out_stride + (long long)h * head_dim;
  return splits_of(a, span_of(b, a, length_of(b, s), count, r0, min(r0 + a.tile_rows, min(count, a.max_new) * a.rep) - 1).n);
}

// Few splits joined in a launch of their own: bit for bit what the last workgroup of k_attn_split does.  Bound: latency (4 us).
template <class T, int HD>
__global__ __launch_bounds__(256) void k_attn_join_few(Batch b, AttnArgs a) {
  constexpr int E = HD * 16 / kAttnThreads > 4 ? HD * 16 / kAttnThreads : 4, LANES = HD / E;
  const long long w = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const int e0 = threadIdx.x % LANES * E;
  long long out;
  const int parts = parts_of(b, a, w, HD, out);
  if (parts <= 1) return;
  float v[E], sum;
  join_parts<HD, E>(a, w * a.n_splits, parts, e0, v, sum);
  store_row<T, E>((T *)a.out + out + e0, v, sum);
}

// Many splits joined, a workgroup a row: HD / 4 lanes have a row's elements, the others take other splits; the wavefronts' sums are added
// in their order.  Bound: latency (8B shape, 64 splits of one token 6 us: start, length, maxima, 32 partial results a lane group).
template <class T, int HD>
__global__ __launch_bounds__(256) void k_attn_join_many(Batch b, AttnArgs a) {
  constexpr int LANES = HD / 4, GROUPS = 256 / LANES;
  const long long w = blockIdx.x;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, e0 = lane % LANES * 4;
  long long out;
  const int parts = parts_of(b, a, w, HD, out);
  if (parts <= 1) return;
  const float2 *ml = a.part_ml + w * a.n_splits;
  const float *po = a.part_o + w * a.n_splits * HD + e0;
  float big = -INFINITY, sum = 0.f;
  for (int z = lane; z < parts; z += 64) big = fmaxf(big, ml[z].x);
#pragma unroll
  for (int d = 32; d; d >>= 1) big = fmaxf(big, __shfl_xor(big, d));
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int z = threadIdx.x / LANES; z < parts; z += GROUPS) {
    const float f = big == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[z].x - big);
    sum += f * ml[z].y;
    v += f * *(const f32x4 *)(po + (long long)z * HD);
  }
#pragma unroll
  for (int d = LANES; d < 64; d <<= 1) {
    sum += __shfl_xor(sum, d);
#pragma unroll
    for (int n = 0; n < 4; ++n) v[n] += __shfl_xor(v[n], d);
  }
  __shared__ f32x4 part[4][LANES];
  __shared__ float part_sum[4];
  if (lane < LANES) part[wave][lane] = v;
  if (lane == 0) part_sum[wave] = sum;
  __syncthreads();
  if (wave || lane >= LANES) return;
#pragma unroll
  for (int i = 1; i < 4; ++i) { v += part[i][lane]; sum += part_sum[i]; }
  const float x[4] = {v[0], v[1], v[2], v[3]};
  store_row<T, 4>((T *)a.out + out + e0, x, sum);
}

// ------------------------------------------------------------------ copies

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
