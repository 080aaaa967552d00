// What the library's translation units share on the host side.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

#include "river.h"

namespace river {

// text of the last error of a call without a context, per host thread (river_last_error(NULL))
std::string &call_error();

// Rows between a context's cache and pages (river_save_pages, river_load_pages): positions first .. first + n - 1 of
// all layers.  kc, vc: the sequence's first row in layer 0, layers max_seq rows apart, a row n_kv_heads * head_dim wide.
hipError_t move_rows(const river_pages &p, const int32_t *row, int max_pages, void *kc, void *vc, int max_seq, int first, int n,
                     bool to_pages, hipStream_t stream);
hipError_t set_word(int *at, int value, hipStream_t stream);     // *at = value (DEVICE)
// RIVER_OK, or an error with its text: is this a cache that the operators take?
int check_pages(const river_pages *p, std::string *why);

}  // namespace river
