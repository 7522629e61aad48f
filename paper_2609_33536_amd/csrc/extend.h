// The table-extension launch (internal header).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ekv {

constexpr int kExtendBatch = 4096;   // most sequences of one call

// why a call took nothing (status[0])
enum { kExtendRow = 1, kExtendTokens = 2, kExtendBlocks = 4, kExtendBase = 8 };

struct ExtendArgs {
  const int32_t* ids;        // [capacity], a ring
  const int32_t* cursor;     // {head, count}
  int32_t* cursor_out;       // may be cursor
  const int32_t* lens;       // [batch]
  const int32_t* new_lens;   // [batch] or null (one each)
  const int32_t* start;      // [batch] or null (0): added to positions
  int32_t* bt;               // [batch][max_blocks]
  uint8_t* tags;             // [batch][max_blocks] or null
  int32_t* lens_out;         // [batch], may be lens
  int32_t* cu;               // [batch + 1]
  int32_t* slots;            // [max_tokens]
  int32_t* positions;        // [max_tokens] or null
  int32_t* status;           // [4]
  int32_t capacity, num_blocks, batch, max_blocks, max_tokens;
  int32_t commit, commit_only;   // set by the launcher: this launch updates lengths and cursor; and does only that
};

hipError_t launch_extend(const ExtendArgs& a, hipStream_t st);

}  // namespace ekv
