// Device code that lays a step out (gfx950): pages from a free list on the device, slot maps, keys and values stored by them.
#pragma once
#include "river_pages.h"

namespace river {
namespace pg {

// ------------------------------------------------------------------ a step from the requests' lengths
//
// Sequence s has lens[s] positions and asks for n_new[s] more (gives back -n_new[s] where that is negative).  Everything follows from
// running sums over the sequences in their order, tokens and pages asked for so far: who is served, where each one's tokens begin, which
// pages of the free list it gets.  One workgroup keeps them in LDS (12 bytes a sequence); a thread has neighbouring sequences.

constexpr int kBuildThreads = 1024, kBuildSeqs = 4096, kBuildEach = kBuildSeqs / kBuildThreads;

struct BuildArgs {
  int *table;
  const int *lens, *n_new, *n_free, *n_shared;
  int *lens_out, *free_pages, *n_free_out;
  int n_seq, max_pages, table_stride, n_pages, page_size, n_tokens;
  int cap;                                // positions that a row has entries for
  Div by_page;
  int *q_start;
  long long *slots;
  int *positions, *refused;
};

// Pages of n positions
__device__ __forceinline__ int pages_of(const BuildArgs &a, int n) { return n > 0 ? a.by_page.quot(n - 1) + 1 : 0; }

// Sums that stop at kMuch (more than there are tokens in a call, or pages): in any order the same, and no overflow.
constexpr uint32_t kMuch = 1u << 30;
struct Two { uint32_t x, y; };
__device__ __forceinline__ Two add(Two a, Two b) { return {min(a.x + b.x, kMuch), min(a.y + b.y, kMuch)}; }
// What the lanes before this one have, and all of the wavefront
__device__ __forceinline__ Two lanes_before(Two mine, Two &all) {
  const int lane = threadIdx.x % 64;
  Two t = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Two o = {__shfl_up(t.x, d), __shfl_up(t.y, d)};
    if (lane >= d) t = add(t, o);
  }
  all = {(uint32_t)__builtin_amdgcn_readlane(t.x, 63), (uint32_t)__builtin_amdgcn_readlane(t.y, 63)};
  const Two before = {__shfl_up(t.x, 1), __shfl_up(t.y, 1)};
  return lane ? before : Two{0, 0};
}
// The same over the workgroup; two barriers.
__device__ __forceinline__ Two threads_before(Two mine, Two *waves, Two &all) {
  const int wave = threadIdx.x / 64, n = blockDim.x / 64;
  Two sum, before = lanes_before(mine, sum);
  __syncthreads();
  if (threadIdx.x % 64 == 0) waves[wave] = sum;
  __syncthreads();
  Two of[kBuildThreads / 64];             // (all at once: a read behind the other takes as long as the rest)
#pragma unroll
  for (int w = 0; w < kBuildThreads / 64; ++w) of[w] = waves[w];
  all = {0, 0};
  Two here = {0, 0};
#pragma unroll
  for (int w = 0; w < kBuildThreads / 64; ++w) {
    if (w == wave) here = all;
    if (w < n) all = add(all, of[w]);
  }
  return add(here, before);
}

// The first i of n with v[i] > x (v ascends).
__device__ __forceinline__ int first_above(const int *v, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (v[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// The same where a lane has one of the n numbers (at most 64) and they lie in LDS too: x is x0 and the lane, so that most wavefronts meet one or
// two of them and need not search.
__device__ __forceinline__ int first_above(const int *v, int mine, int n, int x0) {
  const int lane = threadIdx.x % 64;
  const int lo = __popcll(__ballot(lane < n && mine <= x0)), hi = __popcll(__ballot(lane < n && mine <= x0 + 63));
  return lo + first_above(v + lo, hi - lo, x0 + lane);
}

// slots and positions of token t, which is at position p and has page `page`; p < 0: no token
__device__ __forceinline__ void put_token(const BuildArgs &a, int t, int p, int page, int in_page) {
  if (a.slots) a.slots[t] = p >= 0 && (unsigned)page < (unsigned)a.n_pages ? (long long)page * a.page_size + in_page : -1;
  if (a.positions) a.positions[t] = max(p, 0);
}

// FEW: at most 64 sequences, a lane each, and every wavefront has all of them: its sums are its own, what it writes to LDS every other
// writes too, and no barrier stands between.  Else a thread has EACH neighbouring ones at most (one, or four of more than 1024: next
// tokens of 256 sequences 8.2 us with room for four, 7.2 with one), and the sums go through LDS.
// Bound: latency, of the loads that need what others brought (lengths, the free list, the rows), and of the barriers.
template <bool TOKENS, bool FEW, int EACH>
__global__ __launch_bounds__(kBuildThreads) void k_build(BuildArgs a) {
  extern __shared__ int sums[];
  const int n = a.n_seq, nt = blockDim.x, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  int *const len = sums, *const page_sum = sums + n, *const start = sums + 2 * n;     // [n], [n], [n + 1]
  __shared__ Two waves[kBuildThreads / 64];
  __shared__ int gone[2][kBuildThreads / 64];
  __shared__ int taken_;
  auto sum_before = [&](Two mine, Two &all) { return FEW ? lanes_before(mine, all) : threads_before(mine, waves, all); };
  const int each = FEW ? 1 : (n + nt - 1) / nt, s0 = FEW ? lane : tid * each;
  auto mine = [&](int i) { return i < each && s0 + i < n; };      // is sequence s0 + i this thread's?
  int free = min(max(*a.n_free, 0), a.n_pages);
  int old[EACH], d[EACH], kept[EACH], shared[EACH];
  bool back = false;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    old[i] = d[i] = kept[i] = shared[i] = 0;
    if (!mine(i)) continue;
    kept[i] = a.lens[s0 + i];
    d[i] = a.n_new[s0 + i];
    if (a.n_shared) shared[i] = a.n_shared[s0 + i];
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    old[i] = max(kept[i], 0);
    if (d[i] < 0) kept[i] = (int)max(0ll, (long long)old[i] + d[i]);
    back |= d[i] < 0;
  }
  if (tid == 0) taken_ = 0;
  if (__syncthreads_or(back)) {           // (and everything has been read that may be written over)
    // Given back: entries of a row that name pages, from the last one on down to what is kept or shared, the last sequence's first, so that pages
    // that a call has given out come to lie in the free list as they lay before it.  A thread an entry, in that order: sequence n - 1 - r has
    // those below page_sum[r].
    uint32_t to[EACH];
    Two go[EACH], sum = {0, 0}, all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      to[i] = min(pages_of(a, old[i]), a.max_pages);
      go[i] = {(uint32_t)(d[i] < 0 ? max(0, (int)to[i] - max(pages_of(a, max(kept[i], 0)), shared[i])) : 0), 0};
      sum = add(sum, go[i]);
    }
    Two before = sum_before(sum, all);
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (mine(i)) {
        page_sum[n - 1 - s0 - i] = (int)(all.x - before.x);
        before = add(before, go[i]);
        start[s0 + i] = (int)to[i];
      }
    if (!FEW) __syncthreads();
    int done = 0;
    for (int j0 = 0, buf = 0; j0 < (int)all.x; j0 += nt, buf ^= 1) {
      const int j = j0 + tid;
      int *entry = nullptr, page = -1;
      if (j < (int)all.x) {
        const int r = first_above(page_sum, n, j), s = n - 1 - r;
        entry = a.table + (long long)s * a.table_stride + start[s] - 1 - (j - (r ? page_sum[r - 1] : 0));
        page = *entry;
      }
      const bool ok = (unsigned)page < (unsigned)a.n_pages;
      const unsigned long long oks = __ballot(ok);
      if (lane == 0) gone[buf][wave] = __popcll(oks);
      __syncthreads();
      int at = free + done + __popcll(oks & ((1ull << lane) - 1));
      for (int w = 0; w < nt / 64; ++w) {
        if (w < wave) at += gone[buf][w];
        done += gone[buf][w];
      }
      if (ok && at < a.n_pages) a.free_pages[at] = page;
      if (entry) *entry = -1;
    }
    free = min(a.n_pages, free + done);
    __syncthreads();
  }
  // Asked for: tokens and pages, one after the other.  Who has no room in its row takes no part.
  Two ask[EACH], all;
  Two sum = {0, 0};
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const bool fits = d[i] > 0 && (long long)old[i] + d[i] <= a.cap;
    ask[i].x = fits ? d[i] : 0;
    ask[i].y = fits ? pages_of(a, old[i] + d[i]) - pages_of(a, old[i]) : 0;
    sum = add(sum, ask[i]);
  }
  Two so_far = sum_before(sum, all), given = {0, 0};
  int taken = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    so_far = add(so_far, ask[i]);
    const bool yes = so_far.x <= (uint32_t)a.n_tokens && (ask[i].y == 0 || so_far.y <= (uint32_t)free);
    if (!yes) ask[i].x = 0;
    else if (ask[i].y) taken = (int)so_far.y;
    if (mine(i)) page_sum[s0 + i] = (int)so_far.y;
    given.x += ask[i].x;
    given.y += d[i] > 0 && ask[i].x == 0;
  }
  if constexpr (FEW) {                    // (the sums ascend: the last that took any has the most)
    const unsigned long long took = __ballot(taken > 0);
    taken = took ? __builtin_amdgcn_readlane(taken, 63 - __clzll(took)) : 0;
  } else if (taken) atomicMax(&taken_, taken);
  Two before = sum_before(given, all);
  const bool writes = !FEW || wave == 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int s = s0 + i;
    if (!mine(i)) continue;
    len[s] = old[i];
    start[s] = (int)before.x;
    if (writes) {
      a.q_start[s] = (int)before.x;
      a.lens_out[s] = ask[i].x ? old[i] + (int)ask[i].x : kept[i];
    }
    before.x += ask[i].x;
  }
  if (!FEW) taken = taken_;
  if (FEW ? lane == 0 : tid == 0) start[n] = (int)all.x;
  if (tid == 0) {
    a.q_start[n] = (int)all.x;
    *a.n_free_out = free - taken;
    if (a.refused) *a.refused = (int)all.y;
  }
  if (FEW) __builtin_amdgcn_wave_barrier();
  else __syncthreads();
  // Page j of those that are taken is the one that lies j below the top
  for (int j0 = wave * 64; j0 < taken; j0 += nt) {
    const int j = j0 + lane, s = FEW ? first_above(page_sum, (int)so_far.y, n, j0) : first_above(page_sum, n, j);
    if (j < taken) a.table[(long long)s * a.table_stride + pages_of(a, len[s]) + j - (s ? page_sum[s - 1] : 0)] = a.free_pages[free - 1 - j];
  }
  if constexpr (TOKENS) {
    for (int t0 = wave * 64; t0 < a.n_tokens; t0 += nt) {
      const int t = t0 + lane, s = FEW ? first_above(start + 1, (int)before.x, n, t0) : first_above(start + 1, n, t);
      if (t >= a.n_tokens) break;
      int p = -1, page = -1, in_page = 0;
      if (t < start[n]) {
        p = len[s] + t - start[s];
        const int i = a.by_page.quot(p), fresh = i - pages_of(a, len[s]);
        in_page = p - i * a.page_size;
        page = fresh < 0 ? a.table[(long long)s * a.table_stride + i] : a.free_pages[free - 1 - (s ? page_sum[s - 1] : 0) - fresh];
      }
      put_token(a, t, p, page, in_page);
    }
  }
}

// The tokens' slots and positions in a launch of their own, from what k_build has left: where there are more than a workgroup does
// quickly.  A wavefront has 256 tokens.
constexpr int kSlotsEach = 4;
__global__ __launch_bounds__(256) void k_slots(BuildArgs a) {
  const int lane = threadIdx.x % 64, t0 = (blockIdx.x * 4 + threadIdx.x / 64) * 64 * kSlotsEach, n = a.n_seq;
  if (t0 >= a.n_tokens) return;
  const int total = a.q_start[n];
  // the sequences of the first token and of the last one (the last of those that begin there: for tokens below `total`, their own)
  const int from = count_up_to(a.q_start, n, t0) - 1, upto = count_up_to(a.q_start, n, t0 + 64 * kSlotsEach - 1) - 1;
#pragma unroll
  for (int j = 0; j < kSlotsEach; ++j) {
    const int t = t0 + j * 64 + lane;
    if (t >= a.n_tokens) return;
    int p = -1, page = -1, in_page = 0;
    if (t < total) {
      int s = from, hi = upto + 1;
      while (s + 1 < hi) {
        const int mid = (s + hi) >> 1;
        if (a.q_start[mid] <= t) s = mid; else hi = mid;
      }
      p = a.lens_out[s] + t - a.q_start[s + 1];
      const int i = a.by_page.quot(p);
      page = a.table[(long long)s * a.table_stride + i];
      in_page = p - i * a.page_size;
    }
    put_token(a, t, p, page, in_page);
  }
}

// ------------------------------------------------------------------ keys and values by a slot map
//
// Row t of keys and values goes to slot slots[t] = page * page_size + place in the page, rounded once to the pages' type; a slot that
// no page has is left out.  Bound: memory.  A workgroup has a few whole tokens, a thread kStoreEach pieces (what makes 16 bytes in the
// pages or, wider, in the rows) on their way at once.
constexpr int kStoreThreads = 256, kStoreEach = 4;

struct StoreArgs {
  const long long *slots;
  const void *k, *v;
  long long k_stride, v_stride;
  double by_page;                         // 1 / page_size
  long long n_slots;                      // of the pages
  int n_tokens, tokens;                   // of the call, of a workgroup
  Div by_row;                             // pieces of a token: its keys, then its values
};

template <class T, class C, int HD, bool WIDE>
__global__ __launch_bounds__(kStoreThreads) void k_store_slots(Cache c, StoreArgs a) {
  constexpr int PER = 16 / sizeof(T), P = HD / PER;
  const int first = blockIdx.x * a.tokens, pieces = min(a.tokens, a.n_tokens - first) * (int)a.by_row.d, half = a.by_row.d / 2;
  for (int at = threadIdx.x; at < pieces; at += kStoreThreads * kStoreEach) {
    u32x4 w[kStoreEach];
    long long slot[kStoreEach];
#pragma unroll
    for (int n = 0; n < kStoreEach; ++n) {
      const int i = at + n * kStoreThreads;
      if (i >= pieces) continue;
      const int t = a.by_row.quot(i), j = i - t * (int)a.by_row.d;
      slot[n] = a.slots[first + t];
      const T *from = j < half ? (const T *)a.k + (first + t) * a.k_stride + j * PER : (const T *)a.v + (first + t) * a.v_stride + (j - half) * PER;
      if constexpr (WIDE) w[n] = *(const u32x4 *)from;
      else {
        T x[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) x[e] = from[e];
        w[n] = *(const u32x4 *)x;
      }
    }
#pragma unroll
    for (int n = 0; n < kStoreEach; ++n) {
      const int i = at + n * kStoreThreads;
      if (i >= pieces || slot[n] < 0 || slot[n] >= a.n_slots) continue;
      const int t = a.by_row.quot(i), j = i - t * (int)a.by_row.d, jj = j < half ? j : j - half, h = jj / P, e = jj % P * PER;
      // (slots are below 2^47: their product with 1 / page_size is off by less than one)
      long long page = (long long)((double)slot[n] * a.by_page);
      int place = (int)(slot[n] - page * c.page_size);
      if (place < 0) { --page; place += c.page_size; }
      if (place >= c.page_size) { ++page; place -= c.page_size; }
      C *to = (C *)(j < half ? c.k : c.v) + page * c.page_stride + ((long long)h * c.page_size + place) * HD + e;
      if constexpr (__is_same(T, C)) *(u32x4 *)to = w[n];
      else {
        C y[PER];
#pragma unroll
        for (int x = 0; x < PER; ++x) y[x] = (C)(float)((const T *)&w[n])[x];
        *(u32x4 *)to = *(const u32x4 *)y;
      }
    }
  }
}

}  // namespace pg
}  // namespace river
