// What the entry points of the paged cache share.
#pragma once

#include <initializer_list>

#include "zc_common.hpp"

// Page pools that belong together, and rows of new tokens [1, any number of heads, T, D] beside them (defined in paged_cache.hip).
int zc_validate_pages(const zc_tensor4* k, const zc_tensor4* v);
int zc_validate_heads(const zc_tensor4* x, const zc_tensor4* pages);
// Whether no element of a tensor that is written lies in memory of another: of its axes' strides, those of one element left out, each
// is at least what the smaller ones span (defined in paged_cache.hip).
bool zc_rows_apart(const zc_tensor4* x);
