// The rotary-position launch (internal header).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ekv {

struct RopeArgs {
  const int32_t* positions;  // [n]
  const int32_t* slots;      // [n]
  const uint16_t* q;         // rows of heads x 128 values, `*_stride` values apart
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  void* pool;                // [NB][2][Hkv][16][128]
  const uint64_t* turns;     // [rotary_dim / 2]: turns a position, in units of 2^-64
  int64_t q_stride, k_stride, v_stride, out_stride;
  int32_t n, num_q_heads, num_kv_heads, num_blocks;
  int32_t rotary_dim;        // a multiple of 16
  int32_t pairs;             // pair i: elements (2i, 2i + 1) rather than (i, i + rotary_dim / 2)
  float magnitude;
  int32_t rows_per_wave;     // set by the launcher
  // The norm of each query and key head (norm = 0: none, the rest is not read)
  int32_t norm;
  const uint16_t* q_weight;  // [128] a head, `*_weight_stride` values apart (0: one for all heads), or null (ones)
  const uint16_t* k_weight;
  int32_t q_weight_stride, k_weight_stride;
  float eps, offset;         // inside the root; added to the weights
};

// dtype: of the pool (0 bf16, 1 fp16, 3 8-bit with FP16 inputs)
hipError_t launch_rope(const RopeArgs& a, int dtype, hipStream_t st);

}  // namespace ekv
