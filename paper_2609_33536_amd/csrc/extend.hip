// Block tables and slot maps built on the GPU from request lengths.
//
// For sequences s with len[s] cached and n[s] new tokens, in order:
//   old[s]  = ceil(len[s] / 16), need[s] = ceil((len[s] + n[s]) / 16) - old[s]
//   entry (s, old[s] + k) = free block number sum(need[0 .. s-1]) + k, k < need[s], tag TARGET
//   token i of s: position p = len[s] + i, slot = block(p / 16) 16 + p % 16,
//   at row cu[s] + i, cu the exclusive sums of n.
// All of it or nothing: what does not fit (table row, token rows, free blocks) leaves
// tables, lengths and the free list as they were and every slot -1.
//
// Every workgroup scans all lengths (their sums lie in LDS: at most kExtendBatch
// sequences) and then writes its part of the tokens and of the new entries, found by
// binary search in the sums.  Nothing is passed between workgroups.  Lengths and
// cursor may be updated in place: one workgroup does so behind a barrier; of
// several, all of which read them, none may, and a second launch of one does.
#include "common.h"
#include "extend.h"
#include "wave_scan.h"

namespace ekv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kFull = 1 << 30;   // sums saturate here, above any capacity (twice it fits 32 bits unsigned)

__device__ __forceinline__ int add(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)kFull); }

// the last index i < n with start[i] <= x (start[0] <= x)
__device__ __forceinline__ int holder(const int* start, int n, int x) {
  int lo = 0, hi = n;   // start[lo] <= x, start[hi] > x (hi = n: beyond)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kThreads) void extend_kernel(ExtendArgs a) {
  __shared__ int token0[kExtendBatch], block0[kExtendBatch], lens[kExtendBatch];
  __shared__ int sums[kWaves][2];
  __shared__ int refused_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) refused_s = 0;
  __syncthreads();

  // ---- sums: thread t scans sequences [t each, (t + 1) each)
  const int each = (a.batch + kThreads - 1) / kThreads;
  int tokens = 0, blocks = 0, refused = 0;
  for (int k = 0; k < each; ++k) {
    const int s = tid * each + k;
    if (s >= a.batch) break;
    const int len = a.lens[s], n = a.new_lens ? a.new_lens[s] : 1;
    const bool fits = len >= 0 && n >= 0 && (int64_t)len + n <= (int64_t)a.max_blocks * kPage;
    if (!fits) refused |= kExtendRow;
    lens[s] = fits ? len : 0;
    token0[s] = tokens;   // (relative to this thread's first; below made absolute)
    block0[s] = blocks;
    if (fits) {
      tokens = add(tokens, n);
      blocks = add(blocks, (len + n + kPage - 1) / kPage - (len + kPage - 1) / kPage);
      if (n > 0 && len % kPage && a.tags && a.tags[(size_t)s * a.max_blocks + len / kPage]) refused |= kExtendBase;
    }
  }
  const int it = wave_scan(tokens, add), ib = wave_scan(blocks, add);
  if (lane == 63) {
    sums[wave][0] = it;
    sums[wave][1] = ib;
  }
  if (refused) atomicOr(&refused_s, refused);
  __syncthreads();
  int before_t = __shfl_up(it, 1), before_b = __shfl_up(ib, 1);   // exclusive
  if (lane == 0) before_t = before_b = 0;
  int all_t = 0, all_b = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) {
      before_t = add(before_t, all_t);
      before_b = add(before_b, all_b);
    }
    all_t = add(all_t, sums[w][0]);
    all_b = add(all_b, sums[w][1]);
  }
  for (int k = 0; k < each; ++k) {
    const int s = tid * each + k;
    if (s >= a.batch) break;
    token0[s] = add(token0[s], before_t);
    block0[s] = add(block0[s], before_b);
  }
  const int free0 = min(max(a.cursor[1], 0), a.capacity);
  int head = a.cursor[0] % a.capacity;
  if (head < 0) head += a.capacity;
  refused = refused_s;
  if (all_t > a.max_tokens) refused |= kExtendTokens;
  if (all_b > free0) refused |= kExtendBlocks;
  const bool ok = refused == 0;
  __syncthreads();

  auto taken = [&](int k) -> int {   // free block number k (< all_b <= capacity)
    const int i = head + k;
    return a.ids[i >= a.capacity ? i - a.capacity : i];
  };
  const int first = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  if (!a.commit_only) {
    // ---- new entries
    if (ok) {
      for (int k = first; k < all_b; k += step) {
        const int s = holder(block0, a.batch, k);
        const size_t at = (size_t)s * a.max_blocks + (lens[s] + kPage - 1) / kPage + (k - block0[s]);
        a.bt[at] = taken(k);
        if (a.tags) a.tags[at] = 0;
      }
    }
    // ---- tokens
    for (int t = first; t < a.max_tokens; t += step) {
      int slot = -1, pos = 0;
      if (ok && t < all_t) {
        const int s = holder(token0, a.batch, t);
        const int p = lens[s] + (t - token0[s]), old = (lens[s] + kPage - 1) / kPage, b = p / kPage;
        const int block = b < old ? a.bt[(size_t)s * a.max_blocks + b] : taken(block0[s] + b - old);
        if ((unsigned)block < (unsigned)a.num_blocks) slot = block * kPage + p % kPage;
        pos = p + (a.start ? a.start[s] : 0);
      }
      a.slots[t] = slot;
      if (a.positions) a.positions[t] = pos;
    }
    for (int s = first; s < a.batch; s += step) a.cu[s] = ok ? token0[s] : 0;
    if (first == 0) {
      a.cu[a.batch] = ok ? all_t : 0;
      a.status[0] = refused;
      a.status[1] = all_t;
      a.status[2] = all_b;
      a.status[3] = ok ? free0 - all_b : free0;
    }
  }
  if (a.commit || a.commit_only) {
    for (int s = first; s < a.batch; s += step) {
      const int n = s + 1 < a.batch ? token0[s + 1] - token0[s] : all_t - token0[s];
      if (ok) a.lens_out[s] = lens[s] + n;
      else if (a.lens_out != a.lens) a.lens_out[s] = a.lens[s];
    }
    if (first == 0) {
      const int left = ok ? free0 - all_b : free0, at = ok ? head + all_b : head;
      a.cursor_out[0] = at >= a.capacity ? at - a.capacity : at;
      a.cursor_out[1] = left;
    }
  }
}

}  // namespace

hipError_t launch_extend(const ExtendArgs& a, hipStream_t st) {
  const int64_t work = a.max_tokens > a.batch ? a.max_tokens : a.batch;
  int64_t grid = (work + 8 * kThreads - 1) / (8 * kThreads);
  grid = grid < 1 ? 1 : (grid > 256 ? 256 : grid);
  ExtendArgs b = a;
  const bool in_place = a.lens_out == a.lens || a.cursor_out == a.cursor;
  b.commit = grid == 1 || !in_place;
  b.commit_only = 0;
  hipLaunchKernelGGL(extend_kernel, dim3((unsigned)grid), dim3(kThreads), 0, st, b);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || b.commit) return e;
  b.commit_only = 1;
  hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(kThreads), 0, st, b);
  return hipGetLastError();
}

}  // namespace ekv
