// C entry points of the long-context decode step: key bounds, block selection and
// decode over selected blocks.  Declarations and contracts: include/ekv.h.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <vector>

#include "common.h"
#include "ekv.h"
#include "host_checks.h"
#include "host_status.h"
#include "launch.h"
#include "long_context.h"

namespace {

using namespace ekv;

constexpr int kMostRows = 1 << 22;   // (sequence, KV head)s of a call: grids stay within 2^32 threads
// Counters at the start of a decode workspace, whatever the batch: as many as ekv_attn_decode keeps there, so that neither
// call finds the other's partial results where it expects zeros.
constexpr int kCounters = 2 * kMaxDecodeGrid;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The checks that the three calls share.
ekv_status check_rows(const ekv_pool* pool, const ekv_batch* batch, int* group) {
  ekv_status st = check_pool(pool);
  if (st != EKV_OK) return st;
  if ((st = check_attention_batch(pool, batch, group)) != EKV_OK) return st;
  if (batch->max_blocks >= (1 << 26)) return fail(EKV_ERR_UNSUPPORTED, "max_blocks must be below 2^26");
  if ((int64_t)batch->batch * pool->num_kv_heads > kMostRows)
    return fail(EKV_ERR_UNSUPPORTED, "batch * num_kv_heads must be at most 2^22");
  return EKV_OK;
}

BlockRows block_rows(const ekv_pool* pool, const ekv_batch* b) {
  BlockRows r{};
  r.pool = static_cast<const uint16_t*>(pool->kv);
  r.lens = b->seq_lens;
  r.bt = b->block_table;
  r.tags = b->mode == EKV_MODE_NATIVE ? nullptr : b->tags;
  r.base = b->mode == EKV_MODE_NATIVE ? nullptr : b->boundaries;
  r.batch = b->batch;
  r.num_kv_heads = pool->num_kv_heads;
  r.max_blocks = b->max_blocks;
  r.num_blocks = pool->num_blocks;
  r.len_cap = b->max_seq_len > 0 ? b->max_seq_len : b->max_blocks * kPage;
  return r;
}

ekv_status check_budget(int32_t budget) {
  if (budget <= 0) return fail(EKV_ERR_INVALID, "budget must be positive");
  if (budget >= (1 << 20)) return fail(EKV_ERR_UNSUPPORTED, "budget must be below 2^20");
  return EKV_OK;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Scratch of a selection whose rows take several chunks: [keys u64 | block numbers], 256-B aligned parts, for `kept` of both.
struct SelectLayout {
  size_t blocks, total;
};
SelectLayout select_layout(size_t kept) {
  SelectLayout l{};
  l.blocks = align256(kept * sizeof(uint64_t));
  l.total = std::max<size_t>(256, l.blocks + align256(kept * sizeof(int32_t)));
  return l;
}
SelectArgs select_args(const ekv_pool* pool, const ekv_batch* b, int group, int32_t budget, int32_t sink, int32_t recent) {
  const BlockRows rows = block_rows(pool, b);
  SelectArgs a{};
  a.lens = rows.lens;
  a.batch = rows.batch;
  a.num_kv_heads = rows.num_kv_heads;
  a.group = group;
  a.max_blocks = rows.max_blocks;
  a.len_cap = rows.len_cap;
  a.budget = budget;
  a.sink = sink;
  a.recent = recent;
  plan_select(&a, max_seq_blocks(b));
  return a;
}

// Scratch of a decode over selected blocks whose lists are cut into `pieces`: [merge counters | (m, l) | o], 256-B aligned
// parts.  The size does not grow with the batch (many lists are not cut), so a call takes any workspace that holds the
// counters and cuts its lists into no more pieces than there is room for.
struct SelectedLayout {
  size_t ml, o, total;
};
SelectedLayout selected_layout(int64_t rows, int pieces, int group) {
  SelectedLayout l{};
  const size_t slots = pieces > 1 ? (size_t)rows * pieces * group : 0;
  l.ml = align256(kCounters * sizeof(uint32_t));
  l.o = align256(l.ml + slots * 2 * sizeof(float));
  l.total = align256(l.o + slots * kHeadDim * sizeof(float));
  return l;
}

// EKV_DEBUG: a block of its sequence that a list names twice.
ekv_status debug_check_lists(const ekv_pool* pool, const ekv_batch* b, const int32_t* selected, const int32_t* counts,
                             int32_t budget, hipStream_t stream) {
  const size_t rows = (size_t)b->batch * pool->num_kv_heads;
  std::vector<int32_t> list(rows * budget), n(rows, budget), lens(b->batch);
  auto read = [&](std::vector<int32_t>& to, const int32_t* from) {
    return hipMemcpyAsync(to.data(), from, to.size() * sizeof(int32_t), hipMemcpyDeviceToHost, stream);
  };
  hipError_t e = read(list, selected);
  if (e == hipSuccess) e = read(lens, b->seq_lens);
  if (e == hipSuccess && counts) e = read(n, counts);
  if (e == hipSuccess) e = hipStreamSynchronize(stream);
  if (e != hipSuccess) return hip_status(e, "ekv_attn_decode_selected (EKV_DEBUG)");
  for (size_t r = 0; r < rows; ++r) {
    const int s = (int)(r / pool->num_kv_heads), blocks = (lens[s] + kPage - 1) / kPage;   // (lengths are checked before)
    const auto begin = list.begin() + r * budget;
    const auto end = std::remove_if(begin, begin + std::min(std::max(n[r], 0), budget), [&](int32_t i) { return i < 0 || i >= blocks; });
    std::sort(begin, end);
    const auto twice = std::adjacent_find(begin, end);
    if (twice != end)
      return fail(EKV_ERR_INVALID, "ekv_attn_decode_selected (EKV_DEBUG): block %d is listed twice for sequence %d, KV head %d",
                  *twice, s, (int)(r % pool->num_kv_heads));
  }
  return EKV_OK;
}

}  // namespace

extern "C" {

ekv_status ekv_key_bounds(const ekv_pool* pool, const ekv_batch* batch, const int32_t* known, void* bounds,
                          hipStream_t stream) {
  return ekv::guard("ekv_key_bounds", [&]() -> ekv_status {
    int group = 0;
    ekv_status st = check_rows(pool, batch, &group);
    if (st != EKV_OK) return st;
    if ((int64_t)batch->batch * pool->num_kv_heads * ((max_seq_blocks(batch) + 1) / 2) >= (1LL << 31))
      return fail(EKV_ERR_UNSUPPORTED, "ekv_key_bounds: the batch has too many blocks for one call");
    if (batch->batch == 0) return EKV_OK;
    if (!bounds) return fail(EKV_ERR_INVALID, "bounds is NULL");
    if (!aligned16(bounds) || !aligned16(pool->kv)) return fail(EKV_ERR_INVALID, "bounds and the pool must be 16-byte aligned");
    if (debug_mode() && (st = debug_check_batch(pool, batch, stream, "ekv_key_bounds")) != EKV_OK) return st;
    BoundsArgs a{};
    a.rows = block_rows(pool, batch);
    a.known = known;
    a.bounds = bounds;
    return hip_status(launch_key_bounds(a, pool->dtype, batch->mode != EKV_MODE_NATIVE, stream), "ekv_key_bounds launch");
  });
}

size_t ekv_select_workspace_bytes(const ekv_pool* pool, const ekv_batch* batch, int32_t budget) {
  int group = 0;
  if (check_rows(pool, batch, &group) != EKV_OK || check_budget(budget) != EKV_OK) return 0;
  return select_layout((size_t)batch->batch * pool->num_kv_heads * most_kept(max_seq_blocks(batch), budget)).total;
}

ekv_status ekv_select_blocks(const ekv_pool* pool, const ekv_batch* batch, const void* q, const void* bounds, int32_t budget,
                             int32_t sink, int32_t recent, int32_t* selected, int32_t* counts, void* ws, size_t ws_bytes,
                             hipStream_t stream) {
  return ekv::guard("ekv_select_blocks", [&]() -> ekv_status {
    int group = 0;
    ekv_status st = check_rows(pool, batch, &group);
    if (st != EKV_OK) return st;
    if ((st = check_budget(budget)) != EKV_OK) return st;
    if (sink < 0 || recent < 0 || (int64_t)sink + recent > budget)
      return fail(EKV_ERR_INVALID, "sink and recent must not be negative, nor their sum exceed the budget");
    if ((int64_t)batch->batch * pool->num_kv_heads * ((max_seq_blocks(batch) + 511) / 512) > kMostRows)
      return fail(EKV_ERR_UNSUPPORTED, "ekv_select_blocks: the batch has too many blocks for one call");
    if (batch->batch == 0) return EKV_OK;
    if (!q || !bounds || !selected || !counts) return fail(EKV_ERR_INVALID, "q, bounds, selected and counts are required");
    SelectArgs a = select_args(pool, batch, group, budget, sink, recent);
    const SelectLayout l = select_layout(a.chunks > 1 ? (size_t)a.batch * a.num_kv_heads * a.chunks * a.kept : 0);
    const size_t need = l.total;
    if (!ws || ws_bytes < need)
      return fail(EKV_ERR_INVALID, "workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(q) || !aligned16(bounds) || !aligned16(ws))
      return fail(EKV_ERR_INVALID, "q, bounds and ws must be 16-byte aligned");
    if (debug_mode() && (st = debug_check_batch(pool, batch, stream, "ekv_select_blocks")) != EKV_OK) return st;
    a.q = static_cast<const uint16_t*>(q);
    a.bounds = bounds;
    a.selected = selected;
    a.counts = counts;
    a.keys = static_cast<uint64_t*>(ws);
    a.blocks = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + l.blocks);
    return hip_status(launch_select(a, pool->dtype, stream), "ekv_select_blocks launch");
  });
}

size_t ekv_decode_selected_workspace_bytes(const ekv_pool* pool, const ekv_batch* batch, int32_t budget) {
  int group = 0;
  if (check_rows(pool, batch, &group) != EKV_OK || check_budget(budget) != EKV_OK) return 0;
  const int64_t rows = (int64_t)batch->batch * pool->num_kv_heads;
  return selected_layout(rows, selected_pieces(rows, budget), group).total;   // (no fewer pieces for a larger budget)
}

ekv_status ekv_attn_decode_selected(const ekv_pool* pool, const ekv_batch* batch, const int32_t* selected,
                                    const int32_t* counts, int32_t budget, const void* q, void* out, int32_t out_dtype,
                                    float scale, void* ws, size_t ws_bytes, hipStream_t stream) {
  return ekv::guard("ekv_attn_decode_selected", [&]() -> ekv_status {
    int group = 0;
    ekv_status st = check_rows(pool, batch, &group);
    if (st != EKV_OK) return st;
    if ((st = check_budget(budget)) != EKV_OK) return st;
    if (batch->batch == 0) return EKV_OK;
    if (!selected || !q || !out) return fail(EKV_ERR_INVALID, "selected, q and out are required");
    const int q_dtype = pool->dtype == EKV_DTYPE_E5M2 ? EKV_DTYPE_FP16 : pool->dtype;   // 8-bit pools: FP16 queries
    if (out_dtype != q_dtype && out_dtype != EKV_DTYPE_FP32)
      return fail(EKV_ERR_INVALID, "out_dtype must be the query dtype or fp32");
    if (!std::isfinite(scale)) return fail(EKV_ERR_INVALID, "scale must be finite");
    const int64_t rows = (int64_t)batch->batch * pool->num_kv_heads;
    // (no list needs more than its sequence's blocks; the reported size is that of the budget whatever the lengths)
    int pieces = selected_pieces(rows, std::min(budget, max_seq_blocks(batch)));
    SelectedLayout l = selected_layout(rows, pieces, group);
    while (pieces > 1 && l.total > ws_bytes) l = selected_layout(rows, --pieces, group);
    if (!ws || ws_bytes < l.total)
      return fail(EKV_ERR_INVALID, "workspace of %zu bytes needed, %zu given", l.total, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws) || !aligned16(q) || !aligned16(out) || !aligned16(pool->kv))
      return fail(EKV_ERR_INVALID, "ws, q, out and the pool must be 16-byte aligned");
    if (debug_mode() && ((st = debug_check_batch(pool, batch, stream, "ekv_attn_decode_selected")) != EKV_OK ||
                         (st = debug_check_lists(pool, batch, selected, counts, budget, stream)) != EKV_OK))
      return st;
    char* at = static_cast<char*>(ws);
    SelectedArgs a{};
    a.rows = block_rows(pool, batch);
    a.q = static_cast<const uint16_t*>(q);
    a.selected = selected;
    a.counts = counts;
    a.counters = reinterpret_cast<uint32_t*>(at);
    a.ws_ml = reinterpret_cast<float*>(at + l.ml);
    a.ws_o = reinterpret_cast<float*>(at + l.o);
    a.out = out;
    a.num_q_heads = batch->num_q_heads;
    a.budget = budget;
    a.pieces = pieces;
    a.out_fp32 = out_dtype == EKV_DTYPE_FP32;
    a.scale_log2 = log2e_scale(scale);
    return hip_status(launch_selected(a, pool->dtype, group, batch->mode != EKV_MODE_NATIVE, stream),
                      "ekv_attn_decode_selected launch");
  });
}

}  // extern "C"
