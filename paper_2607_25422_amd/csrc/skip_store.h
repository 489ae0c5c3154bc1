// Shapes of the 4-bit passage store shared by its kernels (internal to
// libskip.so; the record's layout is at the top of store.hip).
#pragma once

#include "skip_common.h"

namespace skip {

constexpr int kStoreBlock = 32;               // tokens of a record
template <int D>
constexpr int kStoreRecord = 34 * D;          // bytes of a record

// A batch of passages and where the store holds them.
struct StoreShape {
  const int32_t* passage_offsets;
  const int32_t* passage_blocks;
  long long n_blocks;
  int total_tokens, heads, head_groups, blocks_max;
};

}  // namespace skip
