// Argument checks shared by the C entry points (internal header; defined in
// api.hip).  Each returns EKV_OK or records a message and returns the error.
#pragma once

#include <hip/hip_runtime_api.h>

#include "ekv.h"

namespace ekv {

ekv_status hip_status(hipError_t e, const char* what);
ekv_status check_pool(const ekv_pool* p);
ekv_status check_attention_batch(const ekv_pool* p, const ekv_batch* b, int* group);
int max_seq_blocks(const ekv_batch* b);   // blocks of the longest sequence that the batch states
float log2e_scale(float scale);

// EKV_DEBUG=1: the device checks of a batch, synchronised
bool debug_mode();
ekv_status debug_check_batch(const ekv_pool* pool, const ekv_batch* batch, hipStream_t stream, const char* call);

}  // namespace ekv
