// Bookkeeping of a paged cache: which sequence has which pages, how many sequences share one, which are free.
// Host only; the device's copy of lengths and table is brought up to date by river_pool_flush (river_pages.hip).
#pragma once
#include <algorithm>
#include <functional>
#include <utility>
#include <vector>

#include "river.h"

struct river_pool {
  int n_pages, page_size, max_seqs, max_pages;
  std::vector<int> refs;                         // sequences that have a page
  std::vector<int> free_heap;                    // free pages, least first (a min-heap)
  std::vector<int> len;                          // [max_seqs]
  std::vector<int> table;                        // [max_seqs][max_pages], -1 where there is no page
  std::vector<std::pair<int, int>> copies;       // queued page copies (from, to), in order
  std::vector<int> dirty;                        // changed words of the device's state: lengths, then the table
  std::vector<char> is_dirty;
  bool on_device = false;                        // the device's state has been written once

  river_pool(int pages, int size, int seqs, int per_seq)
      : n_pages(pages), page_size(size), max_seqs(seqs), max_pages(per_seq), refs(pages, 0), free_heap(pages), len(seqs, 0),
        table((size_t)seqs * per_seq, -1), is_dirty((size_t)seqs * (per_seq + 1), 0) {
    for (int i = 0; i < pages; ++i) free_heap[i] = i;            // (ascending: a heap)
    // nothing below allocates: a queue that has no room is an error before anything changes (extend, compact)
    dirty.reserve(is_dirty.size());
  }
  int *row(int s) { return table.data() + (size_t)s * max_pages; }
  const int *row(int s) const { return table.data() + (size_t)s * max_pages; }
  int pages_of(int n) const { return (int)(((long long)n + page_size - 1) / page_size); }
  void touch(size_t word) {
    if (!is_dirty[word]) { is_dirty[word] = 1; dirty.push_back((int)word); }
  }
  void set_len(int s, int n) { len[s] = n; touch(s); }
  void set_entry(int s, int i, int page) {
    row(s)[i] = page;
    touch((size_t)max_seqs + (size_t)s * max_pages + i);
  }
  int take() {
    std::pop_heap(free_heap.begin(), free_heap.end(), std::greater<int>());
    const int p = free_heap.back();
    free_heap.pop_back();
    refs[p] = 1;
    return p;
  }
  void drop(int p) {
    if (p < 0 || --refs[p]) return;
    free_heap.push_back(p);                      // (never more than n_pages: its capacity)
    std::push_heap(free_heap.begin(), free_heap.end(), std::greater<int>());
  }
  bool has(int s) const { return s >= 0 && s < max_seqs; }

  int extend(int s, int n, const char **why) {
    const long long to = (long long)len[s] + n;
    if (to > (long long)max_pages * page_size) { *why = "the sequence's row of the table is full"; return RIVER_ENOSPC; }
    const int have = pages_of(len[s]), need = pages_of((int)to) - have;
    // the last page is written next: where another sequence has it too, this one goes on in a copy
    const int last = len[s] % page_size ? row(s)[have - 1] : -1;
    const bool own = n > 0 && last >= 0 && refs[last] > 1;
    if (need + (own ? 1 : 0) > (int)free_heap.size()) { *why = "no free pages"; return RIVER_ENOSPC; }
    if (own) {
      if (copies.size() == copies.capacity()) copies.reserve(2 * copies.size() + 16);
      const int p = take();
      copies.emplace_back(last, p);
      drop(last);
      set_entry(s, have - 1, p);
    }
    for (int i = 0; i < need; ++i) set_entry(s, have + i, take());
    if (n > 0) set_len(s, (int)to);
    return RIVER_OK;
  }
  void fork(int from, int to) {
    for (int i = 0, n = pages_of(len[from]); i < n; ++i) {
      const int p = row(from)[i];
      if (p >= 0) ++refs[p];
      set_entry(to, i, p);
    }
    set_len(to, len[from]);
  }
  void rewind(int s, int n) {
    for (int i = pages_of(n), e = pages_of(len[s]); i < e; ++i) {
      drop(row(s)[i]);
      set_entry(s, i, -1);
    }
    set_len(s, n);
  }
  // A later position p >= len - 1 sees j > p - window and j < sinks: pages between them are seen by none.
  void trim(int s, int window, int sinks) {
    const long long gone = (long long)len[s] - window;           // positions below this are behind the window
    for (long long i = ((long long)sinks + page_size - 1) / page_size; (i + 1) * page_size <= gone; ++i)    // (sinks: up to 2^31 - 1)
      if (row(s)[i] >= 0) {
        drop(row(s)[i]);
        set_entry(s, (int)i, -1);
      }
  }
  // Pages from `used` on move to the free ones below it.
  int compact() {
    const int used = n_pages - (int)free_heap.size();
    std::vector<int> to(n_pages, -1), holes;
    for (int p = 0; p < used; ++p)
      if (!refs[p]) holes.push_back(p);
    copies.reserve(copies.size() + holes.size());
    int moves = 0;
    for (int p = used; p < n_pages; ++p)
      if (refs[p]) {
        const int q = holes[moves++];
        to[p] = q;
        refs[q] = refs[p];
        refs[p] = 0;
        copies.emplace_back(p, q);
      }
    if (!moves) return 0;
    for (int s = 0; s < max_seqs; ++s)
      for (int i = 0, n = pages_of(len[s]); i < n; ++i)
        if (row(s)[i] >= 0 && to[row(s)[i]] >= 0) set_entry(s, i, to[row(s)[i]]);
    free_heap.clear();
    for (int p = used; p < n_pages; ++p) free_heap.push_back(p);
    return moves;
  }
};
