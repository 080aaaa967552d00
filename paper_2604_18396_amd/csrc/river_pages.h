// Device code of the paged key-value cache (gfx950): rotary positions with the store into the pages, attention over
// the pages, page copies.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace river {
namespace pg {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

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

// ------------------------------------------------------------------ attention

struct AttnArgs {
  const void *q;
  void *out;
  long long q_stride, out_stride;
  int nq, rep;                            // query heads, and how many of them share a key head
  float scale2;                           // scale * log2 e
  int window, sinks;
};

// One wavefront per (token, query head), one position after the other.
template <class T, class C, int HD>
__global__ __launch_bounds__(256) void k_attn_rows(Cache c, Batch b, AttnArgs a) {
  constexpr int E = HD / 64;
  const long long w = (long long)blockIdx.x * 4 + threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  if (w >= (long long)b.n_tokens * a.nq) return;
  const int t = (int)(w / a.nq), h = (int)(w % a.nq);
  const int s = seq_of(b, t);
  if (s < 0) return;
  const int p = position_of(b, s, t);
  float q[E], o[E];
  for (int e = 0; e < E; ++e) { q[e] = (float)((const T *)a.q)[t * a.q_stride + h * HD + lane * E + e]; o[e] = 0.f; }
  float m = -INFINITY, l = 0.f;
  const int low = a.window ? max(0, p - a.window + 1) : 0;
  const int end = min(p + 1, b.cap);
  for (int j = a.window && a.sinks ? 0 : low; j < end; ++j) {
    if (j < low && j >= a.sinks) { j = low - 1; continue; }
    int slot;
    const int page = page_of(c, b, s, j, slot);
    if (page < 0) continue;
    const long long at = (long long)page * c.page_stride + ((long long)(h / a.rep) * c.page_size + slot) * HD + lane * E;
    float x = 0.f;
    for (int e = 0; e < E; ++e) x += q[e] * (float)((const C *)c.k)[at + e];
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    x *= a.scale2;
    const float n = fmaxf(m, x), mm = n == -INFINITY ? 0.f : n;
    const float r = exp2f(m - mm), pr = exp2f(x - mm);
    l = l * r + pr;
    for (int e = 0; e < E; ++e) o[e] = o[e] * r + pr * (float)((const C *)c.v)[at + e];
    m = n;
  }
  for (int e = 0; e < E; ++e)
    ((T *)a.out)[t * a.out_stride + h * HD + lane * E + e] = (T)(l == 0.f ? 0.f : o[e] / l);
}

// ------------------------------------------------------------------ copies

constexpr int kPairs = 448;               // of a launch: they travel as kernel arguments (below 4 KiB)
struct Pairs { int src[kPairs], dst[kPairs]; };

// One workgroup per 16 KiB of a page; grid (pieces, pairs, layers x {k, v}).
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
