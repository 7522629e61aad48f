// Selection of blocks by the largest scores that their key bounds allow.
//
// For query heads g of a KV head and a block with bounds lo, hi (per channel c)
//   score = sum_c (sum_g max(q_gc, 0)) hi_c + (sum_g min(q_gc, 0)) lo_c  >=  sum_g q_g . k
// for every key k of the block: one product of 256 terms a block, whatever the number of
// heads.  Scores are summed in 64 bits: products of 16-bit values are exact there and so are, as a rule, their
// sums, so that the order of near neighbours does not depend on the order of the sum.
//
// score_kernel: a wave takes 64 blocks, a lane 8 channels (16 of 8-bit bounds) of one bound,
// fixed for all of its loads, so that its share of the query stays in registers.  The partial sums
// of 32 (16) loads are summed over the lanes and dealt out to them in one go, half of them a step,
// and lane l ends up with the score of block l.  It is bound by HBM: 512 bytes of bounds a block.
// select_kernel: one workgroup a row finds the budget's last score by histograms of what is still
// in question, and lists the blocks above it in order.
#include <algorithm>

#include "common.h"
#include "long_context.h"
#include "wave_scan.h"

namespace ekv {
namespace {

constexpr int kTileBlocks = 64;

// A score as an integer that orders as it does: 0 below all scores, kForced above them, what is not a number next to that.
constexpr uint64_t kForced = ~0ull, kNotNumber = ~1ull;
__device__ __forceinline__ uint64_t score_key(double x) {
  if (x != x) return kNotNumber;
  const uint64_t w = __builtin_bit_cast(uint64_t, x + 0.0);   // (-0 is 0)
  return w >> 63 ? ~w : w | 1ull << 63;
}

template <int CTRL>
__device__ __forceinline__ double moved(double x) {
  const uint64_t w = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(w >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Two partial sums, each over pairs of lanes that differ in bit B: lanes with bit B = 0 get a's sums, the others b's.
// (For bit 2 the pairs are mirrored in 8 lanes, which serves the same.)  The additions
// form one tree over the lanes for every block: equal bounds give equal scores.
template <int B>
__device__ __forceinline__ double halved(double a, double b, int lane) {
  if constexpr (B == 4) {
    const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
    const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)y, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
    return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
  } else {
    const bool upper = lane >> B & 1;
    const double keep = upper ? b : a, give = upper ? a : b;
    if constexpr (B == 3) return keep + moved<0x128>(give);        // row_ror:8
    else if constexpr (B == 2) return keep + moved<0x141>(give);   // row_half_mirror
    else if constexpr (B == 1) return keep + moved<0x4E>(give);    // quad_perm 2,3,0,1
    else return keep + moved<0xB1>(give);                          // quad_perm 1,0,3,2
  }
}

// 16 bytes of bounds times the lane's part of the query
template <typename T, bool F8, int C>
__device__ __forceinline__ double dot(u32x4 w, const double (&q)[C]) {
  double s = 0.0;
  if constexpr (F8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = base_words_lo(w[i]), hi = base_words_hi(w[i]);
      s = fma((double)Mma<Fp16>::widen((uint16_t)lo), q[4 * i], s);
      s = fma((double)Mma<Fp16>::widen((uint16_t)(lo >> 16)), q[4 * i + 1], s);
      s = fma((double)Mma<Fp16>::widen((uint16_t)hi), q[4 * i + 2], s);
      s = fma((double)Mma<Fp16>::widen((uint16_t)(hi >> 16)), q[4 * i + 3], s);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s = fma((double)Mma<T>::widen((uint16_t)w[i]), q[2 * i], s);
      s = fma((double)Mma<T>::widen((uint16_t)(w[i] >> 16)), q[2 * i + 1], s);
    }
  }
  return s;
}

// The sums of loads u, u + 2^B, .. (all that share the bits below B with u), dealt out to lane bits B and up.
// w holds a batch's loads in the order of their bits from B0 on.
template <typename T, bool F8, int TOP, int B0, int B, int U, int C>
__device__ __forceinline__ double node(const u32x4* w, const double (&q)[C], int lane) {
  if constexpr (B == TOP) return dot<T, F8>(w[U], q);
  else {
    const double a = node<T, F8, TOP, B0, B + 1, U>(w, q, lane);
    const double b = node<T, F8, TOP, B0, B + 1, (U | 1 << (B - B0))>(w, q, lane);
    return halved<B>(a, b, lane);
  }
}

// Scores of blocks t0 .. t0 + 63 of a row of bounds, one a lane (blocks from n on: of no meaning).
template <typename T, bool F8>
struct Scorer {
  static constexpr int kLoads = F8 ? 16 : 32, kTop = F8 ? 4 : 5, kChannels = F8 ? 16 : 8;
  static constexpr int kRowBytes = F8 ? 2 * kHeadDim : 4 * kHeadDim;   // of one block
  double q[kChannels];
  int lane;

  // queries [group][128] of the KV head
  __device__ __forceinline__ void queries(const uint16_t* src, int group) {
    const int c0 = kChannels * (lane % (kLoads / 2));
    const bool high = lane % kLoads >= kLoads / 2;   // the lane holds upper bounds
#pragma unroll
    for (int i = 0; i < kChannels; ++i) q[i] = 0.0;
#pragma unroll 1
    for (int g = 0; g < group; ++g) {
#pragma unroll
      for (int h = 0; h < kChannels / 8; ++h) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(src + g * kHeadDim + c0 + 8 * h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = Mma<T>::widen((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
          q[8 * h + i] += (double)(high ? (x > 0.f ? x : 0.f) : (x < 0.f ? x : 0.f));
        }
      }
    }
  }

  __device__ __forceinline__ double score(const char* row, int t0, int n) const {
    // 8 loads (bits 2 and up of their number) at a time, 2 batches in flight
    constexpr int kBatches = kLoads / 8, kB0 = kTop - 3;
    const uint32_t at = (lane % kLoads) * 16;
    const int mine = t0 + (lane / kLoads) * kLoads;
    auto load = [&](u32x4 (&w)[8], int batch) {
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int block = min(mine + batch + u * kBatches, n - 1);
        w[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + (size_t)block * kRowBytes + at));
      }
    };
    u32x4 w[2][8];
    double part[kBatches];
    load(w[0], 0);
#pragma unroll
    for (int k = 0; k < kBatches; ++k) {
      if (k + 1 < kBatches) load(w[(k + 1) & 1], k + 1);
      part[k] = node<T, F8, kTop, kB0, kB0, 0>(w[k & 1], q, lane);
    }
    if constexpr (F8) return halved<0>(part[0], part[1], lane);
    else return halved<0>(halved<1>(part[0], part[2], lane), halved<1>(part[1], part[3], lane), lane);
  }
};

__device__ __forceinline__ int blocks_of(const SelectArgs& a, int s) {
  return (min(max(a.lens[s], 0), a.len_cap) + kPage - 1) / kPage;
}

constexpr int kScoreWaves = 4;

// Workgroup (row, part): 4 waves, 64 blocks each.  Rows that fit the budget need no scores.
template <typename T, bool F8>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(SelectArgs a, int parts) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x / (unsigned)parts, part = blockIdx.x - row * parts, s = row / (unsigned)a.num_kv_heads;
  const int n = blocks_of(a, s), t0 = (part * kScoreWaves + wave) * kTileBlocks;
  if (n <= a.budget || t0 >= n) return;
  Scorer<T, F8> sc;
  sc.lane = lane;
  sc.queries(a.q + (size_t)row * a.group * kHeadDim, a.group);
  const char* bounds = static_cast<const char*>(a.bounds) + (size_t)row * a.max_blocks * Scorer<T, F8>::kRowBytes;
  const double x = sc.score(bounds, t0, n);
  const int i = t0 + lane;
  if (i < n) a.keys[(size_t)row * a.key_stride + i] = i < a.sink || i >= n - a.recent ? kForced : score_key(x);
}

constexpr int kSelectWaves = 8, kBins = 1024;

struct SelectShared {
  uint32_t bins[kBins];
  uint64_t low[kSelectWaves], high[kSelectWaves];
  uint64_t list[64];
  int above[kSelectWaves], equal[kSelectWaves];
  int listed, bin, over;      // the list's length; the bin in question and how many lie above it
  uint64_t last;              // the last score that is taken, and how many equal to it are
  int ties;
};

// (of one type: mixed 64-bit types would be compared as doubles)
__device__ __forceinline__ uint64_t lower(uint64_t a, uint64_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint64_t higher(uint64_t a, uint64_t b) { return a < b ? b : a; }

__device__ __forceinline__ uint64_t wave_min(uint64_t x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = lower(x, __shfl_xor((unsigned long long)x, d));
  return x;
}
__device__ __forceinline__ uint64_t wave_max(uint64_t x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = higher(x, __shfl_xor((unsigned long long)x, d));
  return x;
}

// Finds sm.last and sm.ties such that the keys of [lo, hi) above `last` and the first `ties` equal to it are
// `need` in all (0 < need < hi - lo).  Every thread of the workgroup.
__device__ void find_last(const uint64_t* keys, int lo, int hi, int need, SelectShared& sm) {
  constexpr int kThreads = 64 * kSelectWaves;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t from = ~0ull, to = 0;
  for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
    const uint64_t k = keys[i];
    from = lower(from, k);
    to = higher(to, k);
  }
  from = wave_min(from);
  to = wave_max(to);
  if (lane == 0) {
    sm.low[wave] = from;
    sm.high[wave] = to;
  }
  __syncthreads();
  from = sm.low[0];
  to = sm.high[0];
#pragma unroll
  for (int w = 1; w < kSelectWaves; ++w) {
    from = lower(from, sm.low[w]);
    to = higher(to, sm.high[w]);
  }
  while (true) {   // the last key lies in [from, to], `need` of those from the top; each pass divides the range by 512 or more
    if (from == to) {
      if (threadIdx.x == 0) {
        sm.last = from;
        sm.ties = need;
      }
      break;
    }
    const int shift = max(0, 54 - __builtin_clzll(to - from));   // (to - from) >> shift < 1024
    for (int i = threadIdx.x; i < kBins; i += kThreads) sm.bins[i] = 0;
    if (threadIdx.x == 0) sm.listed = 0;
    __syncthreads();
    for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
      const uint64_t k = keys[i];
      if (k >= from && k <= to) atomicAdd(&sm.bins[(k - from) >> shift], 1u);
    }
    __syncthreads();
    if (wave == 0) {   // bins from the top, 16 a lane: the one in which the count reaches `need`
      int mine = 0;
#pragma unroll
      for (int b = 0; b < kBins / 64; ++b) mine += sm.bins[kBins - 1 - (lane * (kBins / 64) + b)];
      const int incl = sum_scan(mine);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(incl >= need);
      if (lane == (hit ? __builtin_ctzll(hit) : 63)) {
        int over = incl - mine, b = kBins - 1 - lane * (kBins / 64);
        while (b > 0 && over + (int)sm.bins[b] < need) over += sm.bins[b--];
        sm.bin = b;
        sm.over = over;
      }
    }
    __syncthreads();
    const uint64_t bottom = from + ((uint64_t)sm.bin << shift);
    const int count = sm.bins[sm.bin];
    need -= sm.over;
    from = bottom;
    to = lower(to, bottom + ((1ull << shift) - 1));
    if (need == count) {   // all of the bin (keys are never 0: nothing equals `bottom - 1` that is not below the bin)
      if (threadIdx.x == 0) {
        sm.last = bottom - 1;
        sm.ties = 0;
      }
      break;
    }
    if (count <= 64 && from != to) {   // few: ranked among themselves
      for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
        const uint64_t k = keys[i];
        if (k >= from && k <= to) sm.list[atomicAdd(&sm.listed, 1) & 63] = k;
      }
      __syncthreads();
      if (wave == 0) {
        const uint64_t k = lane < count ? sm.list[lane] : 0;
        int above = 0, equal = 0;
        for (int j = 0; j < count; ++j) {
          const uint64_t o = sm.list[j];
          above += o > k;
          equal += o == k;
        }
        if (lane < count && above < need && above + equal >= need) {   // (equal keys write the same)
          sm.last = k;
          sm.ties = need - above;
        }
      }
      break;
    }
    __syncthreads();   // (the bins are cleared next)
  }
  __syncthreads();
}

__global__ __launch_bounds__(64 * kSelectWaves) void select_kernel(SelectArgs a) {
  __shared__ SelectShared sm;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x, n = blocks_of(a, row / (unsigned)a.num_kv_heads), taken = min(n, a.budget);
  int32_t* out = a.selected + (size_t)row * a.budget;
  if (threadIdx.x == 0) a.counts[row] = taken;
  for (int i = taken + threadIdx.x; i < a.budget; i += 64 * kSelectWaves) out[i] = -1;
  if (n <= a.budget) {
    for (int i = threadIdx.x; i < n; i += 64 * kSelectWaves) out[i] = i;
    return;
  }
  const uint64_t* keys = a.keys + (size_t)row * a.key_stride;
  const int need = a.budget - a.sink - a.recent;
  uint64_t last = kNotNumber;   // (none beyond the first and newest blocks)
  int ties = 0;
  if (need > 0) {
    find_last(keys, a.sink, n - a.recent, need, sm);
    last = sm.last;
    ties = sm.ties;
  }
  // a wave's run of blocks: how many it takes, then its places, then its blocks in order
  const int run = ((n + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64, begin = min(n, wave * run), end = min(n, begin + run);
  int above = 0, equal = 0;
  for (int i0 = begin; i0 < end; i0 += 64) {
    const uint64_t k = i0 + lane < end ? keys[i0 + lane] : 0;
    above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k > last));
    equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k == last));
  }
  if (lane == 0) {
    sm.above[wave] = above;
    sm.equal[wave] = equal;
  }
  __syncthreads();
  int place = 0, seen = 0;   // blocks taken, and blocks equal to the last, before this wave's run
  for (int w = 0; w < wave; ++w) {
    place += sm.above[w] + min(sm.equal[w], max(0, ties - seen));
    seen += sm.equal[w];
  }
  const uint64_t below = (1ull << lane) - 1;
  for (int i0 = begin; i0 < end; i0 += 64) {
    const uint64_t k = i0 + lane < end ? keys[i0 + lane] : 0;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(k == last);
    const bool take = k > last || (k == last && seen + __builtin_popcountll(eq & below) < ties);
    const uint64_t all = __builtin_amdgcn_ballot_w64(take);
    const int at = place + __builtin_popcountll(all & below);
    if (take && at < taken) out[at] = i0 + lane;   // (always, unless another call writes this workspace meanwhile)
    place += __builtin_popcountll(all);
    seen += __builtin_popcountll(eq);
  }
}

template <typename T, bool F8>
void run_scores(const SelectArgs& a, hipStream_t st) {
  const int parts = (a.key_stride + kScoreWaves * kTileBlocks - 1) / (kScoreWaves * kTileBlocks);
  hipLaunchKernelGGL((score_kernel<T, F8>), dim3((unsigned)(a.batch * a.num_kv_heads * parts)), dim3(64 * kScoreWaves), 0, st, a, parts);
}

}  // namespace

hipError_t launch_select(const SelectArgs& a, int dtype, hipStream_t st) {
  if (a.batch == 0) return hipSuccess;
  if (a.key_stride > a.budget) {   // (else every row fits the budget)
    switch (dtype) {
      case 0: run_scores<Bf16, false>(a, st); break;
      case 1: run_scores<Fp16, false>(a, st); break;
      case 3: run_scores<Fp16, true>(a, st); break;
      default: return hipErrorInvalidValue;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)(a.batch * a.num_kv_heads)), dim3(64 * kSelectWaves), 0, st, a);
  return hipGetLastError();
}

}  // namespace ekv
