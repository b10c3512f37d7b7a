// What the kernels of the paged 8-bit cache share.
#pragma once
#include "common.h"

namespace repq {
namespace cache {

// Argument checks of a cache.
repq_status check(const repq_cache& c, const char* who);

inline int log2_block(int block_size) { return block_size == 16 ? 4 : block_size == 32 ? 5 : block_size == 64 ? 6 : 7; }

}  // namespace cache
}  // namespace repq
