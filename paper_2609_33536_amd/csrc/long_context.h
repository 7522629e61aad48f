// Launches of the long-context decode step: key bounds, block selection and
// decode over selected blocks (internal header).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ekv {

// The sequences' blocks as the kernels below read them.
struct BlockRows {
  const uint16_t* pool;      // [NB][2][Hkv][16][128]
  const int32_t* lens;       // [B]
  const int32_t* bt;         // [B][max_blocks]
  const uint8_t* tags;       // [B][max_blocks] or null
  const int32_t* base;       // [B][2]: pair range that is BASE (-1: by tags), or null
  int32_t batch, num_kv_heads, max_blocks;
  int32_t num_blocks;        // pool size: table entries are clamped into it
  int32_t len_cap;           // sequence lengths are clamped to this
};

struct BoundsArgs {
  BlockRows rows;
  const int32_t* known;      // [B]: tokens whose bounds are there, or null (0)
  void* bounds;              // [B][Hkv][max_blocks][2][128] of the pool's element type
};
hipError_t launch_key_bounds(const BoundsArgs& a, int dtype, bool elastic, hipStream_t st);

struct SelectArgs {
  const int32_t* lens;       // [B]
  const uint16_t* q;         // [B][Hq][128]
  const void* bounds;        // as above
  int32_t* selected;         // [B][Hkv][budget]
  int32_t* counts;           // [B][Hkv]
  int32_t batch, num_kv_heads, group, max_blocks, len_cap;
  int32_t budget, sink, recent;
  // A row is scored in chunks; with more than one, each keeps its `kept` best, as
  // scores' keys and block numbers (set by plan_select):
  int32_t chunk, chunks, kept;
  uint64_t* keys;            // [B Hkv][chunks][kept] scratch
  int32_t* blocks;           // the same shape
};
// Fills in the chunks for rows of at most `blocks` blocks.
void plan_select(SelectArgs* a, int blocks);
// The most that chunks * kept of a plan with several chunks can be, for any number of rows of at most `blocks` blocks and
// any budget up to this one: it grows with both.
size_t most_kept(int blocks, int budget);
hipError_t launch_select(const SelectArgs& a, int dtype, hipStream_t st);

struct SelectedArgs {
  BlockRows rows;
  const uint16_t* q;         // [B][Hq][128]
  const int32_t* selected;   // [B][Hkv][budget]
  const int32_t* counts;     // [B][Hkv] or null (budget)
  float* ws_o;               // [B Hkv][pieces][G][128] partial outputs
  float* ws_ml;              // [B Hkv][pieces][G][2]   partial (max, sum)
  uint32_t* counters;        // [B Hkv], zero between calls
  void* out;                 // [B][Hq][128]
  int32_t num_q_heads, budget, pieces, out_fp32;
  float scale_log2;          // softmax scale * log2(e)
};
// Workgroups that share the list of a (sequence, KV head), of up to `blocks` blocks.
int selected_pieces(int64_t rows, int blocks);
hipError_t launch_selected(const SelectedArgs& a, int dtype, int group, bool elastic, hipStream_t st);

}  // namespace ekv
