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
// Bound by latency: 64 single tokens 4.1 us (an empty launch takes as long back to back),
// 192 sequences with 24 thousand tokens 4.8, 512 prompts with 538 thousand 7.2; in place
// 3.7, 7.4 and 10.2.
#include "common.h"
#include "extend.h"
#include "wave_scan.h"

namespace ekv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTokens = 4;       // neighbouring tokens of a thread
constexpr int kDeep = 4;         // chunks of 64 sequences that a wave loads together
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

  // ---- sums: a wave scans a quarter of the sequences, 64 at a time, the loads of kDeep such chunks in flight together
  const int quarter = (a.batch + kThreads - 1) / kThreads * 64, s_end = min(a.batch, (wave + 1) * quarter);
  int tokens = 0, blocks = 0, refused = 0;
#pragma unroll 1
  for (int s0 = wave * quarter; s0 < s_end; s0 += 64 * kDeep) {
    int len[kDeep], n[kDeep], tag[kDeep];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int s = s0 + 64 * u + lane;
      len[u] = n[u] = tag[u] = 0;
      if (s0 + 64 * u >= s_end) break;
      if (s >= s_end) continue;
      len[u] = a.lens[s];
      n[u] = a.new_lens ? a.new_lens[s] : 1;
    }
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int s = s0 + 64 * u + lane;
      if (s0 + 64 * u >= s_end) break;
      if (len[u] < 0 || n[u] < 0 || (int64_t)len[u] + n[u] > (int64_t)a.max_blocks * kPage) {
        refused |= kExtendRow;
        len[u] = n[u] = 0;
      }
      if (n[u] > 0 && len[u] % kPage && a.tags) tag[u] = a.tags[(size_t)s * a.max_blocks + len[u] / kPage];
    }
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int s = s0 + 64 * u + lane;
      if (s0 + 64 * u >= s_end) break;
      const int need = (len[u] + n[u] + kPage - 1) / kPage - (len[u] + kPage - 1) / kPage;
      const int it = wave_scan(n[u], add), ib = wave_scan(need, add);
      if (s < s_end) {
        lens[s] = len[u];
        token0[s] = add(tokens, it) - n[u];   // (relative to this wave's first; below made absolute)
        block0[s] = add(blocks, ib) - need;
      }
      tokens = add(tokens, last_lane(it));
      blocks = add(blocks, last_lane(ib));
      if (tag[u]) refused |= kExtendBase;
    }
  }
  if (lane == 0) {
    sums[wave][0] = tokens;
    sums[wave][1] = blocks;
  }
  if (refused) atomicOr(&refused_s, refused);
  __syncthreads();
  int before_t = 0, before_b = 0, all_t = 0, all_b = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) {
      before_t = all_t;
      before_b = all_b;
    }
    all_t = add(all_t, sums[w][0]);
    all_b = add(all_b, sums[w][1]);
  }
  if (wave > 0) {
    for (int s = wave * quarter + lane; s < s_end; s += 64) {
      token0[s] += before_t;   // (sums that saturate are refused: nothing follows them)
      block0[s] += before_b;
    }
  }
  const int free0 = min(max(a.cursor[1], 0), a.capacity);
  int head = a.cursor[0] % a.capacity;
  if (head < 0) head += a.capacity;
  refused = refused_s;
  if (all_t > a.max_tokens) refused |= kExtendTokens;
  if (all_b > free0) refused |= kExtendBlocks;
  const bool ok = refused == 0;
  __syncthreads();

  auto taken = [&](int k) -> const int32_t* {   // free block number k (< all_b <= capacity)
    const int i = head + k;
    return a.ids + (i >= a.capacity ? i - a.capacity : i);
  };
  const int first = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  if (!a.commit_only) {
    // ---- new entries
    if (ok) {
      for (int k = first; k < all_b; k += step) {
        const int s = holder(block0, a.batch, k);
        const size_t at = (size_t)s * a.max_blocks + (lens[s] + kPage - 1) / kPage + (k - block0[s]);
        a.bt[at] = *taken(k);
        if (a.tags) a.tags[at] = 0;
      }
    }
    // ---- tokens: one a thread where there are threads for all of them (4096 sequences of one
    // token: 11.9 us, four neighbours a thread 15.4)
    if (a.max_tokens <= step) {
      if (first < a.max_tokens) {
        int slot = -1, pos = 0;
        if (ok && first < all_t) {
          const int s = holder(token0, a.batch, first);
          const int p = lens[s] + (first - token0[s]), old = (lens[s] + kPage - 1) / kPage, b = p / kPage;
          const int block = *(b < old ? a.bt + (size_t)s * a.max_blocks + b : taken(block0[s] + b - old));
          if ((unsigned)block < (unsigned)a.num_blocks) slot = block * kPage + p % kPage;
          pos = p + (a.start ? a.start[s] : 0);
        }
        a.slots[first] = slot;
        if (a.positions) a.positions[first] = pos;
      }
    } else {
      // (kTokens neighbours a thread: one search, and one for each sequence that begins among
      // them, then the blocks' numbers, all on their way at once)
      const bool wide = ((reinterpret_cast<uintptr_t>(a.slots) | reinterpret_cast<uintptr_t>(a.positions)) & 15) == 0;
      for (int64_t t0 = (int64_t)first * kTokens; t0 < a.max_tokens; t0 += (int64_t)step * kTokens) {
        const int t = (int)t0, here = ok ? min(all_t - t, kTokens) : 0;   // (tokens of sequences among them)
        const int32_t* at[kTokens];
        int in_block[kTokens], pos[kTokens], block[kTokens];
        int s = 0, end = 0, len = 0, old = 0, shift = 0;
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
          at[i] = nullptr;
          in_block[i] = pos[i] = 0;
          if (i >= here) continue;
          if (t + i >= end) {
            s = holder(token0, a.batch, t + i);
            end = s + 1 < a.batch ? token0[s + 1] : all_t;
            len = lens[s];
            old = (len + kPage - 1) / kPage;
            shift = a.start ? a.start[s] : 0;
          }
          const int p = len + (t + i - token0[s]), b = p / kPage;
          at[i] = b < old ? a.bt + (size_t)s * a.max_blocks + b : taken(block0[s] + b - old);
          in_block[i] = p % kPage;
          pos[i] = p + shift;
        }
#pragma unroll
        for (int i = 0; i < kTokens; ++i) block[i] = at[i] ? *at[i] : -1;
        int slot[kTokens];
#pragma unroll
        for (int i = 0; i < kTokens; ++i) slot[i] = (unsigned)block[i] < (unsigned)a.num_blocks ? block[i] * kPage + in_block[i] : -1;
        if (wide && t + kTokens <= a.max_tokens) {
          *reinterpret_cast<int4*>(a.slots + t) = int4{slot[0], slot[1], slot[2], slot[3]};
          if (a.positions) *reinterpret_cast<int4*>(a.positions + t) = int4{pos[0], pos[1], pos[2], pos[3]};
        } else {
#pragma unroll
          for (int i = 0; i < kTokens; ++i) {
            if (t + i >= a.max_tokens) continue;
            a.slots[t + i] = slot[i];
            if (a.positions) a.positions[t + i] = pos[i];
          }
        }
      }
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
  // One token a thread up to three workgroups a CU (48 KB of LDS each; 538 thousand tokens: 7.2 us,
  // with 512 and 256 workgroups 9.0 and 11.1).  In place, one workgroup does for 2048
  // tokens: 4.8 us, where 8 and the second launch take 5.6 (512 tokens: 3.7 and 5.1).
  const bool in_place = a.lens_out == a.lens || a.cursor_out == a.cursor;
  const int64_t work = a.max_tokens > a.batch ? a.max_tokens : a.batch;
  int64_t grid = (work + kThreads - 1) / kThreads;
  if (grid < 1 || (in_place && grid <= 8)) grid = 1;
  if (grid > 768) grid = 768;
  ExtendArgs b = a;
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
