// What the calls on a paged cache share.
#pragma once

#include <type_traits>

#include "a3_internal.cuh"

namespace a3 {

// The checks of a cache that every call on it makes; also that the handle's device is the current one.
int paged_cache_check(const a3_handle* h, const a3_paged_cache* c);

}  // namespace a3
