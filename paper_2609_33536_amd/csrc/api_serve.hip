// C entry points of the serving step around the cache: table extension, rotary
// append and decode over shared prefixes.  Declarations and contracts: include/ekv.h.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <vector>

#include "common.h"
#include "ekv.h"
#include "extend.h"
#include "host_checks.h"
#include "host_status.h"
#include "rope.h"
#include "shared_plan.h"

namespace {

using namespace ekv;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// ---- shared-prefix decode -------------------------------------------------

// Scratch of a call: [12 ints a sequence for the merge | (m, l) and o of 32-column slots | of G-column slots],
// 256-B aligned parts.
struct SharedLayout : SharedSize {
  size_t ml_wide, o_wide, ml_own, o_own, total;
};

ekv_status plan_shared(const ekv_pool* p, const ekv_batch* prefixes, const ekv_batch* b, int group, SharedLayout* l) {
  const int64_t units_p = (max_seq_blocks(prefixes) + 1) / 2, units_s = (max_seq_blocks(b) + 1) / 2;
  if (!size_shared(prefixes->batch, b->batch, units_p, units_s, p->num_kv_heads, group, l))
    return fail(EKV_ERR_UNSUPPORTED, "batch too large for one shared-prefix decode call");
  if (b->batch > 64 * l->grid)   // (each workgroup describes 64 sequences to the merge)
    return fail(EKV_ERR_UNSUPPORTED, "at most %d sequences in one shared-prefix decode call", 64 * kMaxSharedGrid);
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  l->ml_wide = align(sizeof(Describe) * (size_t)b->batch);
  l->o_wide = align(l->ml_wide + (size_t)l->wide_slots * 32 * 8);
  l->ml_own = align(l->o_wide + (size_t)l->wide_slots * 32 * kHeadDim * 4);
  l->o_own = align(l->ml_own + (size_t)l->own_slots * group * 8);
  l->total = l->o_own + (size_t)l->own_slots * group * kHeadDim * 4;
  return EKV_OK;
}

ekv_status check_shared(const ekv_pool* pool, const ekv_batch* prefixes, const ekv_batch* batch, int* group) {
  ekv_status st = check_pool(pool);
  if (st != EKV_OK) return st;
  if ((st = check_attention_batch(pool, batch, group)) != EKV_OK) return st;
  if (!prefixes) return fail(EKV_ERR_INVALID, "prefixes is NULL");
  int prefix_group = 0;
  ekv_batch p = *prefixes;
  if (p.batch == 0) p.mode = EKV_MODE_NATIVE;   // (no rows: no tags or boundaries either)
  if ((st = check_attention_batch(pool, &p, &prefix_group)) != EKV_OK) return st;
  if (prefixes->max_blocks >= (1 << 26) || batch->max_blocks >= (1 << 26))
    return fail(EKV_ERR_UNSUPPORTED, "max_blocks must be below 2^26");
  if (prefix_group != *group) return fail(EKV_ERR_INVALID, "prefixes and batch must have the same num_q_heads");
  return EKV_OK;
}

SharedPart shared_part(const ekv_pool* pool, const ekv_batch* b) {
  SharedPart p{};
  p.pool = static_cast<const uint16_t*>(pool->kv);
  p.lens = b->seq_lens;
  p.bt = b->block_table;
  p.tags = b->mode == EKV_MODE_NATIVE ? nullptr : b->tags;
  p.bounds = b->mode == EKV_MODE_NATIVE ? nullptr : b->boundaries;
  p.rows = b->batch;
  p.max_blocks = b->max_blocks;
  p.num_blocks = pool->num_blocks;
  p.num_kv_heads = pool->num_kv_heads;
  p.len_cap = b->max_seq_len > 0 ? b->max_seq_len : b->max_blocks * kPage;
  return p;
}

// ---- EKV_DEBUG: what the arrays of a call must not hold twice ------------

// An array of the device, once the stream has reached it.
ekv_status debug_read(const int32_t* from, size_t n, std::vector<int32_t>* to, hipStream_t stream, const char* call) {
  to->resize(n);
  hipError_t e = n ? hipMemcpyAsync(to->data(), from, n * sizeof(int32_t), hipMemcpyDeviceToHost, stream) : hipSuccess;
  if (e == hipSuccess) e = hipStreamSynchronize(stream);
  return e == hipSuccess ? EKV_OK : hip_status(e, call);
}

// Two rows that would write one token's K and V.
ekv_status debug_check_slots(const ekv_pool* pool, int32_t n, const int32_t* slots, hipStream_t stream, const char* call) {
  std::vector<int32_t> at;
  const ekv_status st = debug_read(slots, (size_t)n, &at, stream, call);
  if (st != EKV_OK) return st;
  at.erase(std::remove_if(at.begin(), at.end(), [&](int32_t s) { return s < 0 || s / kPage >= pool->num_blocks; }), at.end());
  std::sort(at.begin(), at.end());
  const auto twice = std::adjacent_find(at.begin(), at.end());
  if (twice != at.end()) return fail(EKV_ERR_INVALID, "%s (EKV_DEBUG): token slot %d for two rows", call, *twice);
  return EKV_OK;
}

// A free block that is listed twice, or that a sequence still holds.
ekv_status debug_check_free(const ExtendArgs& a, hipStream_t stream, const char* call) {
  if ((long long)a.batch * a.max_blocks >= (1LL << 31))
    return fail(EKV_ERR_UNSUPPORTED, "%s (EKV_DEBUG): batch * max_blocks must be below 2^31", call);
  std::vector<int32_t> cursor, ids, lens, table;
  ekv_status st;
  if ((st = debug_read(a.cursor, 2, &cursor, stream, call)) != EKV_OK ||
      (st = debug_read(a.ids, (size_t)a.capacity, &ids, stream, call)) != EKV_OK ||
      (st = debug_read(a.lens, (size_t)a.batch, &lens, stream, call)) != EKV_OK ||
      (st = debug_read(a.bt, (size_t)a.batch * a.max_blocks, &table, stream, call)) != EKV_OK)
    return st;
  const int count = std::min(std::max(cursor[1], 0), a.capacity);
  int head = cursor[0] % a.capacity;
  if (head < 0) head += a.capacity;
  std::vector<int32_t> open;
  for (int k = 0; k < count; ++k) {
    const int32_t id = ids[((size_t)head + k) % a.capacity];
    if (id >= 0 && id < a.num_blocks) open.push_back(id);   // (outside the pool: no slot)
  }
  std::sort(open.begin(), open.end());
  const auto twice = std::adjacent_find(open.begin(), open.end());
  if (twice != open.end()) return fail(EKV_ERR_INVALID, "%s (EKV_DEBUG): block %d is in the free list twice", call, *twice);
  for (int s = 0; s < a.batch; ++s) {
    if (lens[s] < 0 || lens[s] > (int64_t)a.max_blocks * kPage) continue;   // (the call's status says so)
    for (int b = 0; b < (lens[s] + kPage - 1) / kPage; ++b) {
      const int32_t id = table[(size_t)s * a.max_blocks + b];
      if (std::binary_search(open.begin(), open.end(), id))
        return fail(EKV_ERR_INVALID, "%s (EKV_DEBUG): block %d is free and held by sequence %d", call, id, s);
    }
  }
  return EKV_OK;
}

}  // namespace

extern "C" {

ekv_status ekv_extend(const ekv_free_list* free_list, int32_t batch, int32_t max_blocks, const int32_t* seq_lens,
                      const int32_t* new_lens, const int32_t* start, int32_t* block_table, uint8_t* tags,
                      int32_t* seq_lens_out, int32_t* cu_q, int32_t max_tokens, int32_t* slots, int32_t* positions,
                      int32_t* status, hipStream_t stream) {
  return ekv::guard("ekv_extend", [&]() -> ekv_status {
    if (!free_list || !free_list->ids || !free_list->cursor || !free_list->cursor_out)
      return fail(EKV_ERR_INVALID, "ekv_extend: the free list's ids, cursor and cursor_out are required");
    if (free_list->capacity <= 0 || free_list->num_blocks <= 0 || batch < 0 || max_blocks <= 0 || max_tokens < 0)
      return fail(EKV_ERR_INVALID, "ekv_extend: bad sizes");
    if (batch > 0 && (!seq_lens || !block_table || !seq_lens_out))
      return fail(EKV_ERR_INVALID, "ekv_extend: seq_lens, block_table and seq_lens_out are required");
    if (!cu_q || !status || (max_tokens > 0 && !slots))
      return fail(EKV_ERR_INVALID, "ekv_extend: cu_q, slots and status are required");
    if (batch > kExtendBatch) return fail(EKV_ERR_UNSUPPORTED, "ekv_extend: at most %d sequences", kExtendBatch);
    if (free_list->num_blocks >= (1 << 27) || max_blocks >= (1 << 26) || max_tokens >= (1 << 30) ||
        free_list->capacity >= (1 << 30))
      return fail(EKV_ERR_UNSUPPORTED, "ekv_extend: slots must fit 32 bits");
    ExtendArgs a{};
    a.ids = free_list->ids;
    a.cursor = free_list->cursor;
    a.cursor_out = free_list->cursor_out;
    a.lens = seq_lens;
    a.new_lens = new_lens;
    a.start = start;
    a.bt = block_table;
    a.tags = tags;
    a.lens_out = seq_lens_out;
    a.cu = cu_q;
    a.slots = slots;
    a.positions = positions;
    a.status = status;
    a.capacity = free_list->capacity;
    a.num_blocks = free_list->num_blocks;
    a.batch = batch;
    a.max_blocks = max_blocks;
    a.max_tokens = max_tokens;
    const ekv_status st = debug_mode() ? debug_check_free(a, stream, "ekv_extend") : EKV_OK;
    if (st != EKV_OK) return st;
    return hip_status(launch_extend(a, stream), "ekv_extend launch");
  });
}

ekv_status ekv_rope_freqs(int32_t rotary_dim, double base, int32_t scaling, double factor, double context, double low,
                          double high, uint64_t* h_turns_out) {
  return ekv::guard("ekv_rope_freqs", [&]() -> ekv_status {
    if (rotary_dim <= 0 || rotary_dim % 16 || rotary_dim > kHeadDim)
      return fail(EKV_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16, at most 128");
    if (!h_turns_out) return fail(EKV_ERR_INVALID, "h_turns_out is NULL");
    if (!(base >= 1.0) || !std::isfinite(base)) return fail(EKV_ERR_INVALID, "base must be at least 1");
    if (scaling < EKV_ROPE_PLAIN || scaling > EKV_ROPE_PARTS) return fail(EKV_ERR_INVALID, "unknown scaling %d", scaling);
    if (scaling != EKV_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
      return fail(EKV_ERR_INVALID, "factor must be at least 1");
    if (scaling == EKV_ROPE_PARTS &&
        (!(context > 0.0) || !std::isfinite(context) || !(low >= 0.0) || !(high > low) || !std::isfinite(high)))
      return fail(EKV_ERR_INVALID, "scaling by parts needs a context and 0 <= low < high");
    constexpr double kTwoPi = 6.283185307179586476925286766559;
    const double b = scaling == EKV_ROPE_BASE ? base * std::pow(factor, rotary_dim / (rotary_dim - 2.0)) : base;
    for (int i = 0; i < rotary_dim / 2; ++i) {
      double theta = std::pow(b, -2.0 * i / rotary_dim);
      if (scaling == EKV_ROPE_LINEAR) theta /= factor;
      if (scaling == EKV_ROPE_PARTS) {
        const double keep = std::min(1.0, std::max(0.0, (context * theta / kTwoPi - low) / (high - low)));
        theta = theta / factor * (1.0 - keep) + theta * keep;
      }
      h_turns_out[i] = (uint64_t)std::ldexp(theta / kTwoPi, 64);   // (theta <= 1: below a sixth of a turn)
    }
    return EKV_OK;
  });
}

ekv_status ekv_rope_append(const ekv_pool* pool, const ekv_rope* rope, int32_t n, const int32_t* positions,
                           const int32_t* slots, const void* q, int64_t q_stride, int32_t num_q_heads, const void* k,
                           int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride,
                           hipStream_t stream) {
  return ekv::guard("ekv_rope_append", [&]() -> ekv_status {
    ekv_status st = check_pool(pool);
    if (st != EKV_OK) return st;
    if (!rope || !rope->turns) return fail(EKV_ERR_INVALID, "rope and its turns are required");
    if (rope->rotary_dim <= 0 || rope->rotary_dim % 16 || rope->rotary_dim > kHeadDim)
      return fail(EKV_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16, at most 128");
    if (rope->layout != EKV_ROPE_HALF && rope->layout != EKV_ROPE_PAIRS)
      return fail(EKV_ERR_INVALID, "unknown rotary layout %d", rope->layout);
    if (!std::isfinite(rope->magnitude)) return fail(EKV_ERR_INVALID, "magnitude must be finite");
    if (n < 0 || num_q_heads <= 0) return fail(EKV_ERR_INVALID, "bad sizes");
    if (n >= (1 << 26) || num_q_heads > 1024) return fail(EKV_ERR_UNSUPPORTED, "at most 2^26 tokens and 1024 query heads");
    if (n == 0) return EKV_OK;
    if (!positions || !slots || !q || !k || !v || !q_out)
      return fail(EKV_ERR_INVALID, "positions, slots, q, k, v and q_out are required");
    const int64_t q_row = (int64_t)num_q_heads * kHeadDim, kv_row = (int64_t)pool->num_kv_heads * kHeadDim;
    if (q_stride < q_row || q_out_stride < q_row || k_stride < kv_row || v_stride < kv_row)
      return fail(EKV_ERR_INVALID, "a row stride is shorter than its heads");
    if ((q_stride | q_out_stride | k_stride | v_stride) % 8 || !aligned16(q) || !aligned16(k) || !aligned16(v) ||
        !aligned16(q_out) || !aligned16(pool->kv))
      return fail(EKV_ERR_INVALID, "rows must be 16-byte aligned");
    if (debug_mode() && (st = debug_check_slots(pool, n, slots, stream, "ekv_rope_append")) != EKV_OK) return st;
    RopeArgs a{};
    a.positions = positions;
    a.slots = slots;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.pool = pool->kv;
    a.turns = rope->turns;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.out_stride = q_out_stride;
    a.n = n;
    a.num_q_heads = num_q_heads;
    a.num_kv_heads = pool->num_kv_heads;
    a.num_blocks = pool->num_blocks;
    a.rotary_dim = rope->rotary_dim;
    a.pairs = rope->layout == EKV_ROPE_PAIRS;
    a.magnitude = rope->magnitude;
    return hip_status(launch_rope(a, pool->dtype, stream), "ekv_rope_append launch");
  });
}

size_t ekv_decode_shared_workspace_bytes(const ekv_pool* pool, const ekv_batch* prefixes, const ekv_batch* batch) {
  int group = 0;   // (no allocation or exception on this path)
  SharedLayout l{};
  if (check_shared(pool, prefixes, batch, &group) != EKV_OK || plan_shared(pool, prefixes, batch, group, &l) != EKV_OK)
    return 0;
  return l.total;
}

ekv_status ekv_attn_decode_shared(const ekv_pool* pool, const ekv_batch* prefixes, const int32_t* group_start,
                                  const ekv_batch* batch, const void* q, void* out, int32_t out_dtype, float scale,
                                  void* ws, size_t ws_bytes, hipStream_t stream) {
  return ekv::guard("ekv_attn_decode_shared", [&]() -> ekv_status {
    int group = 0;
    ekv_status st = check_shared(pool, prefixes, batch, &group);
    if (st != EKV_OK) return st;
    if (batch->batch == 0) return EKV_OK;
    if (!q || !out) return fail(EKV_ERR_INVALID, "q and out are required");
    if (prefixes->batch > 0 && !group_start) return fail(EKV_ERR_INVALID, "group_start is required");
    const int q_dtype = pool->dtype == EKV_DTYPE_E5M2 ? EKV_DTYPE_FP16 : pool->dtype;   // 8-bit pools: FP16 queries
    if (out_dtype != q_dtype && out_dtype != EKV_DTYPE_FP32)
      return fail(EKV_ERR_INVALID, "out_dtype must be the query dtype or fp32");
    if (!std::isfinite(scale)) return fail(EKV_ERR_INVALID, "scale must be finite");
    SharedLayout l{};
    if ((st = plan_shared(pool, prefixes, batch, group, &l)) != EKV_OK) return st;
    if (!ws || ws_bytes < l.total)
      return fail(EKV_ERR_INVALID, "workspace of %zu bytes needed, %zu given", l.total, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws) || !aligned16(q) || !aligned16(out) || !aligned16(pool->kv))
      return fail(EKV_ERR_INVALID, "ws, q, out and the pool must be 16-byte aligned");
    if (debug_mode() && ((prefixes->batch > 0 && (st = debug_check_batch(pool, prefixes, stream, "ekv_attn_decode_shared")) != EKV_OK) ||
                         (st = debug_check_batch(pool, batch, stream, "ekv_attn_decode_shared")) != EKV_OK))
      return st;
    int resident = 0;
    if ((st = hip_status(shared_resident(&resident), "ekv_attn_decode_shared device")) != EKV_OK) return st;
    SharedArgs a{};
    a.prefix = shared_part(pool, prefixes);
    a.own = shared_part(pool, batch);
    a.starts = group_start;
    a.q = static_cast<const uint16_t*>(q);
    a.out = out;
    char* at = static_cast<char*>(ws);
    a.plan = reinterpret_cast<int32_t*>(at);
    a.ml_wide = reinterpret_cast<float*>(at + l.ml_wide);
    a.o_wide = reinterpret_cast<float*>(at + l.o_wide);
    a.ml_own = reinterpret_cast<float*>(at + l.ml_own);
    a.o_own = reinterpret_cast<float*>(at + l.o_own);
    a.wide_slots = (int32_t)l.wide_slots;
    a.own_slots = (int32_t)l.own_slots;
    a.num_kv_heads = pool->num_kv_heads;
    a.num_q_heads = batch->num_q_heads;
    a.log2_group = __builtin_ctz((unsigned)group);
    a.out_fp32 = out_dtype == EKV_DTYPE_FP32;
    a.grid = std::max(4, std::min(l.grid, resident));
    if (batch->batch > 64 * a.grid)
      return fail(EKV_ERR_UNSUPPORTED, "at most %d sequences in one shared-prefix decode call on this device", 64 * a.grid);
    a.min_units = l.min_units;
    a.merge_ways = l.merge_ways;
    a.scale_log2 = log2e_scale(scale);
    const bool elastic = (prefixes->batch > 0 && prefixes->mode != EKV_MODE_NATIVE) || batch->mode != EKV_MODE_NATIVE;
    return hip_status(launch_shared(a, pool->dtype, elastic, stream), "ekv_attn_decode_shared launch");
  });
}

}  // extern "C"
