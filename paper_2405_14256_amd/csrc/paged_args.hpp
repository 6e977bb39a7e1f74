// What the entry points of the paged cache share.
#pragma once

#include <initializer_list>

#include "zc_common.hpp"

// Page pools that belong together, and rows of new tokens [1, any number of heads, T, D] beside them (defined in paged_cache.hip).
int zc_validate_pages(const zc_tensor4* k, const zc_tensor4* v);
int zc_validate_heads(const zc_tensor4* x, const zc_tensor4* pages);
