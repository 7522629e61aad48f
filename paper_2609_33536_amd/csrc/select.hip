// Selection of blocks by the largest scores that their key bounds allow.
//
// For query heads g of a KV head and a block with bounds lo, hi (per channel c)
//   score = sum_c (sum_g max(q_gc, 0)) hi_c + (sum_g min(q_gc, 0)) lo_c  >=  sum_g q_g . k
// for every key k of the block: one product of 256 terms a block, whatever the number of
// heads.  Scores are summed in 64 bits: products of 16-bit values are exact there and so are, as a rule, their
// sums, so that the order of near neighbours does not depend on the order of the sum.
//
// A wave takes 16 blocks (32 of 8-bit bounds) at a time in 8 loads, a lane 8 (16) channels of one
// bound, fixed for all of its loads, so that its share of the query stays in registers.  The partial
// sums of the 8 loads are summed over the lanes and dealt out to them in one go, half of them a
// step.  This is bound by HBM: 512 (256) bytes of bounds a block.  32 sequences of 16384 to 32768 16-bit tokens, 8 KV heads:
// 37.3 us (199 MB, 5.3 TB/s); one of a million 43.0 (256 MB, 6.0 TB/s) and 12.0 for the join; 12 blocks
// 5.6: a launch and four round trips (lengths, queries and bounds, the pick, the list).
//
// scan_kernel: a workgroup scores a chunk of a row's blocks into LDS, finds the budget's last score
// by histograms of what is still in question, and lists the blocks above it in order.  Where a
// row is one chunk, that is the result.  Else the chunk's own best, as many as the budget could
// take of it, go to the workspace, and join_kernel picks among those of all chunks the same way.
#include <algorithm>
#include <cstdint>

#include "common.h"
#include "key_bins.h"
#include "long_context.h"
#include "wave_scan.h"

namespace ekv {
namespace {

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

// The sums d[U], d[U + 2^(B - B0)], .. dealt out to lane bits B0 (the last bit of a load's number) to TOP.
template <int TOP, int B, int U>
__device__ __forceinline__ double node(const double (&d)[8], int lane) {
  if constexpr (B > TOP) return d[U];
  else {
    const double a = node<TOP, B + 1, U>(d, lane);
    const double b = node<TOP, B + 1, (U | 1 << (B - TOP + 2))>(d, lane);
    return halved<B>(a, b, lane);
  }
}

// The sums over a KV head's query heads of what is above and below zero, for each channel: [below | above], in runs of
// C channels (a lane's) with two unused places behind each: lanes that read runs side by side meet no bank twice.
template <int C>
struct Query {
  double part[4][2 * kHeadDim];
  double sum[2 * kHeadDim / C * (C + 2)];
};
// queries [group][128] of the KV head.  Every thread of the workgroup; ends with a barrier.  meanwhile() is called with the
// loads on their way.
template <typename T, int C, typename F>
__device__ __forceinline__ void sum_queries(const uint16_t* src, int group, Query<C>& sm, F meanwhile) {
  const int c = threadIdx.x % kHeadDim, share = threadIdx.x / kHeadDim;   // heads share, share + 4, ..
  uint16_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = src[min(share + 4 * k, group - 1) * kHeadDim + c];
  __builtin_amdgcn_sched_barrier(0);   // (in this order: what is loaded meanwhile is not waited for)
  meanwhile();
  double below = 0.0, above = 0.0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float x = share + 4 * k < group ? Mma<T>::widen(w[k]) : 0.f;
    below += (double)(x > 0.f ? 0.f : x);   // (a NaN is on both sides: no score of the KV head is a number then)
    above += (double)(x < 0.f ? 0.f : x);
  }
  sm.part[share][c] = below;
  sm.part[share][kHeadDim + c] = above;
  __syncthreads();
  const int i = threadIdx.x;
  if (i < 2 * kHeadDim) sm.sum[i + i / C * 2] = (sm.part[0][i] + sm.part[1][i]) + (sm.part[2][i] + sm.part[3][i]);
  __syncthreads();
}

// The non-temporal bit of the cache-policy operand: 41.5 us for those 32 sequences, 46.7 without (an earlier form).
constexpr int kOnce = 2;

// Scores of the blocks of a row of bounds.
template <typename T, bool F8>
struct Scorer {
  static constexpr int kSpan = F8 ? 16 : 32, kTop = F8 ? 3 : 4, kChannels = F8 ? 16 : 8;   // lanes of a block; their number's last bit
  static constexpr int kTile = 8 * 64 / kSpan;                                             // blocks of 8 loads
  static constexpr int kRowBytes = F8 ? 2 * kHeadDim : 4 * kHeadDim;                       // of one block
  __amdgpu_buffer_rsrc_t row;   // n blocks
  int lane, n;
  double q[kChannels];
  u32x4 w[8];

  // Load u of a tile; from block n on the descriptor's bound keeps it from memory.
  __device__ __forceinline__ void load(int t, int u) {
    const uint32_t at = (t + lane / kSpan * 8) * kRowBytes + (lane % kSpan) * 16;
    w[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(row, at + u * kRowBytes, 0, kOnce));
  }
  __device__ __forceinline__ void load(int t) {
#pragma unroll
    for (int u = 0; u < 8; ++u) load(t, u);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void queries(const Query<kChannels>& sm) {
    const double* run = sm.sum + lane % kSpan * (kChannels + 2);   // (lower bounds, then upper ones)
#pragma unroll
    for (int i = 0; i < kChannels; ++i) q[i] = run[i];
  }

  // put(i, score of block i) for the blocks of tiles first, first + stride, .. below n, each by one lane; tile `first` is
  // loaded already.  Each load is followed by that of the next tile as soon as it is used: 8 in flight, from one copy
  // of the code, which is fetched anew by each launch.
  template <typename F>
  __device__ __forceinline__ void scores(int first, int stride, F put) {
    const int at = lane / kSpan * 8 + (lane >> (kTop - 2)) % 8;   // the lane's block of a tile
    const bool mine = lane % (1 << (kTop - 2)) == 0;
#pragma unroll 1
    for (int t = first; t < n; t += stride) {
      double d[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        d[u] = dot<T, F8>(w[u], q);
        load(t + stride, u);
        asm volatile("" ::: "memory");   // (else each load is moved to its use)
        __builtin_amdgcn_sched_barrier(0);
      }
      double x = node<kTop, kTop - 2, 0>(d, lane);
      if constexpr (!F8) x += moved<0x4E>(x);   // (lanes l ^ 2)
      x += moved<0xB1>(x);                      // (lanes l ^ 1)
      if (mine && t + at < n) put(t + at, x);
    }
  }
};

__device__ __forceinline__ int blocks_of(const SelectArgs& a, int s) {
  return (min(max(a.lens[s], 0), a.len_cap) + kPage - 1) / kPage;
}

constexpr int kBins = 1024, kRanked = 64;

// (of one type: mixed 64-bit types would be compared as doubles)
__device__ __forceinline__ uint64_t lower(uint64_t a, uint64_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint64_t higher(uint64_t a, uint64_t b) { return a < b ? b : a; }

// Smallest and largest key seen; key 0 is none.
struct Range {
  uint64_t from = ~0ull, to = 0;
  __device__ __forceinline__ void add(uint64_t k) {
    if (k != 0) from = lower(from, k);
    to = higher(to, k);
  }
  template <int CTRL>
  __device__ __forceinline__ void step() {
    from = lower(from, __builtin_bit_cast(uint64_t, moved<CTRL>(__builtin_bit_cast(double, from))));
    to = higher(to, __builtin_bit_cast(uint64_t, moved<CTRL>(__builtin_bit_cast(double, to))));
  }
  __device__ __forceinline__ void over_row() {   // of 16 lanes
    step<0xB1>();    // quad_perm 1,0,3,2
    step<0x4E>();    // quad_perm 2,3,0,1
    step<0x141>();   // row_half_mirror
    step<0x140>();   // row_mirror
  }
};

// A pick among up to 2^31 keys by WAVES waves, AHEAD loads of keys in flight.
template <int WAVES, int AHEAD>
struct Picker {
  static constexpr int kThreads = 64 * WAVES;
  struct Shared {
    uint32_t bins[kBins];
    uint64_t low[4 * WAVES], high[4 * WAVES];
    uint64_t list[kRanked];
    int above[WAVES], equal[WAVES];
    int listed, bin, over;      // the list's length; the bin in question and how many lie above it
    uint64_t last;              // the last key that is taken, and how many equal to it are
    int ties;
  };

  static __device__ __forceinline__ uint64_t lane_key(uint64_t x, int l) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, l);
  }

  // f(key) for this thread's share of keys [lo, hi).
  template <typename F>
  static __device__ __forceinline__ void each_key(const uint64_t* keys, int lo, int hi, F f) {
    int i = lo + (int)threadIdx.x;
    if constexpr (AHEAD > 1) {
#pragma unroll 1
      for (; i + (AHEAD - 1) * kThreads < hi; i += AHEAD * kThreads) {
        uint64_t k[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) k[u] = keys[i + u * kThreads];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) f(k[u]);
      }
    }
#pragma unroll 1
    for (; i < hi; i += kThreads) f(keys[i]);
  }

  // Lane l's key of count <= 64 (0: none) ranked among them: sm.last and sm.ties for the largest `need`.
  static __device__ __forceinline__ void rank(uint64_t k, int count, int need, Shared& sm) {
    int above = 0, equal = 0;
    for (int j0 = 0; j0 < count; j0 += 4) {   // (lanes from count on hold 0, which is above nothing)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t o = lane_key(k, j0 + j);
        above += o > k;
        equal += o == k;
      }
    }
    if (k != 0 && above < need && above + equal >= need) {   // (equal keys write the same)
      sm.last = k;
      sm.ties = need - above;
    }
  }

  // Finds sm.last and sm.ties such that the keys of [lo, hi) above `last` and the first `ties` equal to it are
  // `need` in all (0 < need < the number of keys there).  Every thread of the workgroup, each with the range of the keys
  // that it has seen; the keys are as written before the call.
  static __device__ __forceinline__ void find_last(const uint64_t* keys, int lo, int hi, int need, Range seen, Shared& sm) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (hi - lo <= kRanked) {
      __syncthreads();
      if (wave == 0) rank(lo + lane < hi ? keys[lo + lane] : 0, hi - lo, need, sm);
      __syncthreads();
      return;
    }
    seen.over_row();
    if (lane % 16 == 0) {
      sm.low[threadIdx.x / 16] = seen.from;
      sm.high[threadIdx.x / 16] = seen.to;
    }
    for (int i = threadIdx.x; i < kBins; i += kThreads) sm.bins[i] = 0;
    if (threadIdx.x == 0) sm.listed = 0;
    __syncthreads();
    Range all;   // (each row of 16 lanes: 16 of the 4 * WAVES ranges)
    all.from = sm.low[lane % (4 * WAVES)];
    all.to = sm.high[lane % (4 * WAVES)];
    all.over_row();
    KeyBins in{~0ull, 0};   // the last key lies here, `need` of these from the top; a pass divides the range by 512 or more
#pragma unroll
    for (int r = 0; r < WAVES / 4; ++r) {
      in.from = lower(in.from, lane_key(all.from, 16 * r));
      in.to = higher(in.to, lane_key(all.to, 16 * r));
    }
    while (in.from < in.to) {
      const int shift = in.shift();
      each_key(keys, lo, hi, [&](uint64_t k) {
        if (in.holds(k)) atomicAdd(&sm.bins[in.bin(k, shift)], 1u);
      });
      __syncthreads();
      if (wave == 0) {   // bins from the top, 16 a lane: the one in which the count reaches `need`
        constexpr int kEach = kBins / 64;
        int mine = 0;
#pragma unroll
        for (int b = 0; b < kEach; ++b) mine += sm.bins[kBins - 1 - (lane * kEach + b)];
        const int incl = sum_scan(mine);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(incl >= need);
        if (lane == (hit ? __builtin_ctzll(hit) : 63)) {
          int over = incl - mine, b = kBins - 1 - lane * kEach;
          while (b > 0 && over + (int)sm.bins[b] < need) over += sm.bins[b--];
          sm.bin = b;
          sm.over = over;
        }
      }
      __syncthreads();
      const int bin = __builtin_amdgcn_readfirstlane(sm.bin), count = __builtin_amdgcn_readfirstlane(sm.bins[bin]);
      need -= __builtin_amdgcn_readfirstlane(sm.over);
      in.enter(bin, shift);
      if (need == count) {   // all of the bin (no key is 0 or 1: none is taken for the one below it)
        --in.from;
        need = 0;
        break;
      }
      if (count <= kRanked && in.from < in.to) {   // few: ranked among themselves
        each_key(keys, lo, hi, [&](uint64_t k) {
          if (in.holds(k)) sm.list[atomicAdd(&sm.listed, 1) % kRanked] = k;
        });
        __syncthreads();
        if (wave == 0) rank(lane < count ? sm.list[lane] : 0, count, need, sm);
        __syncthreads();
        return;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < kBins; i += kThreads) sm.bins[i] = 0;
      __syncthreads();
    }
    if (threadIdx.x == 0) {
      sm.last = in.from;
      sm.ties = need;
    }
    __syncthreads();
  }

  // put(place, i) for the keys i of [lo, hi) above `last` and the first `ties` equal to it, places 0, 1, .. in
  // order.  Every thread of the workgroup.
  template <typename F>
  static __device__ __forceinline__ void list_above(const uint64_t* keys, int lo, int hi, uint64_t last, int ties, Shared& sm, F put) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a wave's run of keys: how many it takes, then its places, then its keys in order
    const int run = ((hi - lo + WAVES - 1) / WAVES + 63) / 64 * 64, begin = min(hi, lo + wave * run), end = min(hi, begin + run);
    constexpr int kEach = AHEAD;
    auto load = [&](int i0, uint64_t (&k)[kEach]) {
#pragma unroll
      for (int u = 0; u < kEach; ++u) k[u] = i0 + 64 * u + lane < end ? keys[i0 + 64 * u + lane] : 0;
    };
    int above = 0, equal = 0;
#pragma unroll 1
    for (int i0 = begin; i0 < end; i0 += 64 * kEach) {
      uint64_t k[kEach];
      load(i0, k);
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k[u] > last));
        equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k[u] == last));
      }
    }
    if (lane == 0) {
      sm.above[wave] = above;
      sm.equal[wave] = equal;
    }
    __syncthreads();
    int place = 0, seen = 0;   // keys taken, and keys equal to the last, before this wave's run
    for (int w = 0; w < wave; ++w) {
      place += sm.above[w] + min(sm.equal[w], max(0, ties - seen));
      seen += sm.equal[w];
    }
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll 1
    for (int i0 = begin; i0 < end; i0 += 64 * kEach) {
      uint64_t k[kEach];
      load(i0, k);
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const uint64_t eq = __builtin_amdgcn_ballot_w64(k[u] == last);
        const bool take = k[u] > last || (k[u] == last && seen + __builtin_popcountll(eq & below) < ties);
        const uint64_t all = __builtin_amdgcn_ballot_w64(take);
        if (take) put(place + __builtin_popcountll(all & below), i0 + 64 * u + lane);
        place += __builtin_popcountll(all);
        seen += __builtin_popcountll(eq);
      }
    }
  }
};

// A row's list but for the blocks picked by score: the first and newest blocks around them and -1 behind, or all
// blocks if they fit the budget.  Returns whether a pick is to be made.
template <int THREADS>
__device__ __forceinline__ bool frame(const SelectArgs& a, int row, int n) {
  int32_t* out = a.selected + (size_t)row * a.budget;
  const bool all = n <= a.budget;
  const int taken = all ? n : a.budget, first = all ? n : a.sink, newest = all ? 0 : a.recent;
  if (threadIdx.x == 0) a.counts[row] = taken;
  for (int i = threadIdx.x; i < first; i += THREADS) out[i] = i;
  for (int i = threadIdx.x; i < newest; i += THREADS) out[taken - newest + i] = n - newest + i;
  for (int i = taken + threadIdx.x; i < a.budget; i += THREADS) out[i] = -1;
  return !all && a.sink + a.recent < a.budget;
}

constexpr int kScanWaves = 8;

// Workgroup (row, chunk of a.chunk blocks)
template <typename T, bool F8>
__global__ __launch_bounds__(64 * kScanWaves, 4) void scan_kernel(SelectArgs a) {
  typedef Picker<kScanWaves, 1> P;
  extern __shared__ uint64_t keys[];   // [a.chunk]
  __shared__ typename P::Shared sm;
  __shared__ Query<Scorer<T, F8>::kChannels> query;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x / (unsigned)a.chunks, part = blockIdx.x - row * a.chunks, s = row / (unsigned)a.num_kv_heads;
  const int n = blocks_of(a, s), c0 = part * a.chunk, need = a.budget - a.sink - a.recent;
  if (a.chunks == 1) {
    if (!frame<P::kThreads>(a, row, n)) return;
  } else if (n <= a.budget || need == 0 || c0 >= n) {   // (the join sees to it)
    return;
  }
  const int c1 = min(n, c0 + a.chunk);
  const int lo = max(a.sink, c0) - c0, hi = min(n - a.recent, c1) - c0;   // the chunk's blocks that are picked by score
  Scorer<T, F8> sc;
  sc.lane = lane;
  sc.n = c1 - c0;   // (offsets in a chunk fit 32 bits)
  sc.row = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<char*>(static_cast<const char*>(a.bounds)) + ((size_t)row * a.max_blocks + c0) * Scorer<T, F8>::kRowBytes, 0,
      sc.n * Scorer<T, F8>::kRowBytes, 0x00020000);
  const int first = wave * Scorer<T, F8>::kTile;
  static_assert(kScanWaves * 64 == 4 * kHeadDim, "a thread a channel and share of the heads");
  sum_queries<T>(a.q + (size_t)row * a.group * kHeadDim, a.group, query, [&]() { sc.load(first); });
  Range seen;
  if (first < sc.n) {
    sc.queries(query);
    sc.scores(first, kScanWaves * Scorer<T, F8>::kTile, [&](int i, double x) {
      const uint64_t k = score_key(x);
      keys[i] = k;
      if (i >= lo && i < hi) seen.add(k);
    });
  }
  uint64_t last = 0;   // (all)
  int ties = 0;
  if (hi - lo > need) {
    P::find_last(keys, lo, hi, need, seen, sm);
    last = sm.last;
    ties = sm.ties;
  } else {
    __syncthreads();
  }
  if (a.chunks == 1) {
    int32_t* out = a.selected + (size_t)row * a.budget + a.sink;
    P::list_above(keys, lo, hi, last, ties, sm, [&](int place, int i) {
      if (place < need) out[place] = i;   // (never more: the list's end does not hang on the pick)
    });
  } else {
    const size_t at = ((size_t)row * a.chunks + part) * a.kept;
    P::list_above(keys, lo, max(lo, hi), last, ties, sm, [&](int place, int i) {
      if (place >= a.kept) return;   // (nor the chunk's)
      a.keys[at + place] = keys[i];
      a.blocks[at + place] = c0 + i;
    });
    for (int i = max(0, min(need, hi - lo)) + threadIdx.x; i < a.kept; i += P::kThreads) a.keys[at + i] = 0;
  }
}

// Workgroup (row): picks among what the chunks kept, copied to LDS if it has room for it (LOCAL keys, or 0).
template <int WAVES, int LOCAL>
__global__ __launch_bounds__(64 * WAVES) void join_kernel(SelectArgs a) {
  typedef Picker<WAVES, (LOCAL > 0 ? 2 : 8)> P;
  __shared__ uint64_t local[LOCAL > 0 ? LOCAL : 1];
  __shared__ int32_t local_blocks[LOCAL > 0 ? LOCAL : 1];
  __shared__ typename P::Shared sm;
  const int row = blockIdx.x, n = blocks_of(a, row / (unsigned)a.num_kv_heads);
  if (!frame<P::kThreads>(a, row, n)) return;
  const int kept = (n + a.chunk - 1) / a.chunk * a.kept, need = a.budget - a.sink - a.recent;
  const size_t at = (size_t)row * a.chunks * a.kept;
  const uint64_t* keys = a.keys + at;
  const int32_t* blocks = a.blocks + at;
  Range seen;
  if constexpr (LOCAL > 0) {
#pragma unroll 4
    for (int i = threadIdx.x; i < kept; i += P::kThreads) {
      const uint64_t k = keys[i];
      local[i] = k;
      local_blocks[i] = blocks[i];
      seen.add(k);
    }
    keys = local;
    blocks = local_blocks;
  } else {
    P::each_key(keys, 0, kept, [&](uint64_t k) { seen.add(k); });
  }
  P::find_last(keys, 0, kept, need, seen, sm);   // (a row that fits the budget has ended above)
  int32_t* out = a.selected + (size_t)row * a.budget + a.sink;
  // (a place beyond `need` only if another call writes this workspace meanwhile)
  P::list_above(keys, 0, kept, sm.last, sm.ties, sm, [&](int place, int i) {
    if (place < need) out[place] = blocks[i];
  });
}

// 48 and 144 KiB of LDS.  Keys in LDS are read from there by every step of the pick, which else goes to
// memory each time; 8 waves are enough for few of them (19 rows of 4 chunks 5.1 us), 16 scan many (one million tokens' 31 chunks 12.0).
constexpr int kFewKept = 4096, kManyKept = 12288;

template <typename T, bool F8>
hipError_t run_typed(const SelectArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((scan_kernel<T, F8>), dim3((unsigned)(a.batch * a.num_kv_heads * a.chunks)), dim3(64 * kScanWaves),
                     a.chunk * sizeof(uint64_t), st, a);
  if (a.chunks > 1) {
    const int64_t most = (int64_t)a.chunks * a.kept;
    const dim3 grid((unsigned)(a.batch * a.num_kv_heads));
    if (most <= kFewKept) hipLaunchKernelGGL((join_kernel<8, kFewKept>), grid, dim3(512), 0, st, a);
    else if (most <= kManyKept) hipLaunchKernelGGL((join_kernel<16, kManyKept>), grid, dim3(1024), 0, st, a);
    else hipLaunchKernelGGL((join_kernel<16, 0>), grid, dim3(1024), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace

// Chunks of 4096 (32 KiB of LDS) to 256 blocks.  A compute unit takes some 9 ns a block, 128 blocks' time more for a chunk's
// queries and pick; a join costs 550 blocks' time and one for each 8 keys that the chunks keep.  (Not a
// matter of `sink` and `recent`: a workspace serves all of them.)  us by chunk, the one that this takes in brackets:
//   KV heads and blocks     4096     2048     1024      512      256
//      256 x  2048                  [37.0]    42.9     42.7     49.2
//      320 x  2048                   55.1     58.8    [51.9]    59.8
//      152 x   880                           [17.4]    25.6     23.9
//       72 x  6368, 8 bits   47.4    46.4    [33.4]    38.2     44.4
//       64 x  8192, 8 bits   48.0   [32.9]    35.9     41.9     50.9
//       24 x  8192           54.7    36.2    [29.9]    30.6     32.3
//       32 x  2048                   26.3     22.7     18.4    [17.0]
//        8 x 62501           64.4   [54.9]    64.7     76.0     96.5
constexpr int kMostChunk = 4096, kLeastChunk = 256;
void plan_select(SelectArgs* a, int blocks) {
  constexpr int kUnits = 256;
  const int64_t rows = (int64_t)a->batch * a->num_kv_heads;
  int64_t least = INT64_MAX;
  for (int most = kMostChunk; most >= kLeastChunk; most /= 2) {
    const int chunk = std::max(64, std::min(most, (blocks + 63) / 64 * 64));
    const int64_t chunks = std::max(1, (blocks + chunk - 1) / chunk);
    int64_t cost = (rows * chunks + kUnits - 1) / kUnits * (chunk + 128);
    if (chunks > 1) cost += 550 + chunks * std::min(chunk, a->budget) / 8;
    if (cost >= least) continue;
    least = cost;
    a->chunk = chunk;
    a->chunks = (int)chunks;
  }
  a->kept = std::min(a->chunk, a->budget - a->sink - a->recent);
}

// (Of every chunk that the loop above may take, whichever it takes: fewer rows may need more of it than many, and a workspace
// for the most serves all.  A row keeps less than a chunk more than its blocks, 12 bytes each, where their bounds have 512 or 256.)
size_t most_kept(int blocks, int budget) {
  size_t most = 0;
  for (int chunk = kMostChunk; chunk >= kLeastChunk; chunk /= 2)
    if (blocks > chunk) most = std::max(most, (size_t)((blocks + chunk - 1) / chunk) * std::min(chunk, budget));
  return most;
}

hipError_t launch_select(const SelectArgs& a, int dtype, hipStream_t st) {
  if (a.batch == 0) return hipSuccess;
  switch (dtype) {
    case 0: return run_typed<Bf16, false>(a, st);
    case 1: return run_typed<Fp16, false>(a, st);
    case 3: return run_typed<Fp16, true>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ekv
