// kia_cache.hpp -- the layout of the 4-bit key/value cache (documented in kia.h).
#pragma once

#include "kia_around.hpp"

namespace kia {

// Byte offset of one head's block of a page: which = 0 its keys, 1 its values.
// A block is codes (D / 2 bytes a token), then scale bytes (D / 32 a token).
template <int D>
__device__ __forceinline__ int64_t cache_block(int page, int which, int h, int Hkv, int lpage) {
  return (((int64_t)page * 2 + which) * Hkv + h) * (int64_t)((D / 2 + D / 32) << lpage);
}

}  // namespace kia
